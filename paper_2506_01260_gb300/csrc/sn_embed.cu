// sn_embed.cu — embedding lookup with scaling, and its gradient by sorted tokens.
//
//   X[t] = scale E[ids[t]],   dE[v] = scale sum over the t with ids[t] = v of G[t]
//
// Both bound by DRAM: the lookup reads a row and writes one for every token; the gradient
// reads G once and writes the whole table once (or, accumulating, reads and writes the rows
// that have tokens).  The gradient sorts the tokens by id, cuts the sorted list into windows
// of equal length, whatever the ids' frequencies, and lets a block sum a window's rows in
// token order: a token with thousands of rows is shared by many blocks, without atomics.
#include <algorithm>

#include "sn_vec.cuh"

namespace sn {
namespace {

constexpr int kThreads = 256;

// ---- lookup ------------------------------------------------------------------------------

struct LookupArgs {
    const void *table;
    int64_t vocab;
    int d;
    const int32_t *ids;
    int64_t T;
    float scale;
    void *X;
    unsigned int *err;      // null: out-of-range ids are not reported
};

// 2^lx lanes walk a row's pieces of 8 elements; a block takes 256 >> lx rows.
template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) k_lookup(const LookupArgs a, int lx)
{
    griddep_start();
    constexpr int N = 8, U = 2;
    const int lane = threadIdx.x & ((1 << lx) - 1), per = kThreads >> lx;
    const int nv = a.d / N;
    for (int64_t t = (int64_t)blockIdx.x * per + (threadIdx.x >> lx); t < a.T; t += (int64_t)gridDim.x * per) {
        const int id = a.ids[t];
        const bool good = (uint32_t)id < (uint64_t)a.vocab;
        if (!good && a.err && lane == 0)
            atomicOr(a.err, SN_EBIT_BAD_ID);
        const S *src = (const S *)a.table + (good ? (int64_t)id * a.d : 0);
        D *dst = (D *)a.X + t * a.d;
        for (int j0 = lane; j0 < nv; j0 += U << lx) {
            float f[U][N];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + (u << lx);
                if (j < nv)
                    load_floats(src + j * N, f[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + (u << lx);
                if (j >= nv)
                    continue;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    f[u][k] = good ? f[u][k] * a.scale : 0.f;
#pragma unroll
                for (int k = 0; k < N; k += Vec<D>::N)
                    *(uint4 *)(dst + j * N + k) = Vec<D>::pack(*(const float(*)[Vec<D>::N])(f[u] + k));
            }
        }
    }
}

// Widths that are no multiple of 8: single elements
template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) k_lookup_any(const LookupArgs a)
{
    griddep_start();
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int id = a.ids[t];
        const bool good = (uint32_t)id < (uint64_t)a.vocab;
        if (!good && a.err && threadIdx.x == 0)
            atomicOr(a.err, SN_EBIT_BAD_ID);
        const S *src = (const S *)a.table + (good ? (int64_t)id * a.d : 0);
        for (int j = threadIdx.x; j < a.d; j += kThreads)
            ((D *)a.X)[t * a.d + j] = Vec<D>::round(good ? Vec<S>::one(src[j]) * a.scale : 0.f);
    }
}

// ---- gradient: tokens sorted by id -----------------------------------------------------------
// The vocabulary is cut into ranges of `width` ids.  The block that has a range reads all ids
// twice (from L2): once to count the valid ids below its range, which is where its tokens
// start in the sorted list, and each of its own ids; once more to place its tokens, in token
// order.  No block waits for another.

constexpr int kSortThreads = 1024;
constexpr int kMaxWidth = 8192;                // ids of a range, one counter each

struct SortArgs {
    const int32_t *ids;
    int64_t T, vocab;
    int width, ranges;
    int32_t *order, *sorted;    // [T] token and id at each place of the sorted list
    int32_t *places;            // valid tokens
    uint32_t *used;             // a bit per id: has tokens
    unsigned int *err;
};

// The exclusive prefix sum of `n` over the block and its total; `warps`: 33 ints
__device__ __forceinline__ int block_scan(int n, int *warps, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        incl += lane >= o ? y : 0;
    }
    __syncthreads();
    if (lane == 31)
        warps[warp] = incl;
    __syncthreads();
    int mine = lane < kSortThreads / 32 ? warps[lane] : 0;
    int s = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        s += lane >= o ? y : 0;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    return __shfl_sync(0xffffffffu, s - mine, warp) + incl - n;
}

__global__ void __launch_bounds__(kSortThreads) k_sort_tokens(const SortArgs a)
{
    griddep_start();
    extern __shared__ int smem[];
    int *count = smem;                              // [width]: tokens of an id, then its next place
    int2 *list = (int2 *)(smem + a.width);          // [4 * kSortThreads]: id in the range, token
    __shared__ int warps[33];
    __shared__ int s_below, s_bad;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int range = blockIdx.x; range < a.ranges; range += gridDim.x) {
        const int64_t lo = (int64_t)range * a.width;
        const uint32_t n_ids = (uint32_t)min((int64_t)a.width, a.vocab - lo);
        __syncthreads();
        for (int i = threadIdx.x; i < a.width; i += kSortThreads)
            count[i] = 0;
        if (threadIdx.x == 0)
            s_below = s_bad = 0;
        __syncthreads();
        int below = 0, bad = 0;
        for (int64_t t = threadIdx.x; t < a.T; t += kSortThreads) {
            const int id = a.ids[t];
            const uint32_t local = (uint32_t)id - (uint32_t)lo;
            below += (uint32_t)id < (uint32_t)lo;
            bad |= (uint32_t)id >= (uint64_t)a.vocab;
            if (local < n_ids)
                atomicAdd(count + local, 1);
        }
        below = warp_sum(below);
        if (lane == 0 && below)
            atomicAdd(&s_below, below);
        if (bad)
            s_bad = 1;
        __syncthreads();
        // the bits of the ids that have tokens, and each id's first place
        int place = s_below;
        for (int i0 = 0; i0 < a.width; i0 += kSortThreads) {
            const int i = i0 + threadIdx.x;
            const int n = i < a.width ? count[i] : 0;
            const uint32_t bits = __ballot_sync(0xffffffffu, n > 0);
            if (lane == 0 && (uint32_t)i < n_ids)
                a.used[(lo + i) / 32] = bits;
            int total;
            const int at = block_scan(n, warps, total);
            if (i < a.width)
                count[i] = place + at;
            place += total;
        }
        if (threadIdx.x == 0) {
            if (range == a.ranges - 1)
                *a.places = place;
            if (range == 0 && s_bad && a.err)
                atomicOr(a.err, SN_EBIT_BAD_ID);
        }
        const int mine = place - s_below;
        if (mine == 0)
            continue;
        // place the tokens: 4 consecutive ones a thread, packed in token order, then ranked
        // by one warp, 32 at a time
        for (int64_t t0 = 0; t0 < a.T; t0 += 4 * kSortThreads) {
            const int64_t t = t0 + 4 * threadIdx.x;
            uint32_t local[4];
            int n = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                local[k] = t + k < a.T ? (uint32_t)a.ids[t + k] - (uint32_t)lo : 0xffffffffu;
                n += local[k] < n_ids;
            }
            int total;
            int at = block_scan(n, warps, total);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (local[k] < n_ids)
                    list[at++] = make_int2((int)local[k], (int)(t + k));
            __syncthreads();
            if (warp == 0)
                for (int i0 = 0; i0 < total; i0 += 32) {
                    const int i = i0 + lane;
                    const int2 e = i < total ? list[i] : make_int2(-1, 0);
                    const uint32_t same = __match_any_sync(0xffffffffu, e.x);
                    if (i < total) {
                        const int p = count[e.x] + __popc(same & ((1u << lane) - 1u));
                        a.order[p] = e.y;
                        a.sorted[p] = (int)lo + e.x;
                    }
                    __syncwarp();
                    if (i < total && (same >> lane) == 1u)      // the last lane of its id
                        count[e.x] += __popc(same);
                    __syncwarp();
                }
            __syncthreads();
        }
    }
}

// ---- gradient: sums --------------------------------------------------------------------------

struct SumArgs {
    const void *G;
    int64_t ldg, T, vocab;
    int d;
    float scale;
    void *dE;
    int accumulate;
    const int32_t *order, *sorted, *places;
    const uint32_t *used;
    int window, windows, slices;   // places of a window; blocks along a row
    float *part;                   // [windows][2][d]: sums of a first and a last id that go on in other windows
};

constexpr int kMaxWindow = 128;

// 8 columns of a row of dE: the sum times the scale, in addition to what is there
template <typename D>
__device__ __forceinline__ void write_piece(D *dst, const float (&acc)[8], float scale, bool accumulate)
{
    float f[8];
    if (accumulate) {
        load_floats(dst, f);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            f[k] = fmaf(acc[k], scale, f[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            f[k] = acc[k] * scale;
    }
#pragma unroll
    for (int k = 0; k < 8; k += Vec<D>::N)
        *(uint4 *)(dst + k) = Vec<D>::pack(*(const float(*)[Vec<D>::N])(f + k));
}

__device__ __forceinline__ void write_part(float *dst, const float (&acc)[8])
{
    *(float4 *)dst = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *(float4 *)(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// Blocks [0, windows * slices) sum; the others, 32 ids each, write the rows without tokens.
template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) k_sum_rows(const SumArgs a)
{
    griddep_start();
    const int nv = a.d / 8;
    D *dE = (D *)a.dE;
    if ((int64_t)blockIdx.x >= (int64_t)a.windows * a.slices) {
        const int64_t word = (int64_t)blockIdx.x - (int64_t)a.windows * a.slices;
        const uint32_t used = a.used[word];
        const int64_t v0 = word * 32;
        const int n = (int)min((int64_t)32, a.vocab - v0);
        for (int i = 0; i < n; ++i)
            if (!((used >> i) & 1u)) {
                uint4 *row = (uint4 *)(dE + (v0 + i) * a.d);
                for (int j = threadIdx.x; j < a.d / Vec<D>::N; j += kThreads)
                    row[j] = make_uint4(0, 0, 0, 0);
            }
        return;
    }
    const int w = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const int places = *a.places;
    const int p0 = w * a.window, p1 = min(places, p0 + a.window);
    if (p0 >= p1)
        return;
    // ids and tokens of the window, and the id before and after it
    __shared__ int ids[kMaxWindow + 2], tokens[kMaxWindow];
    for (int i = threadIdx.x; i < p1 - p0 + 2; i += kThreads) {
        const int p = p0 + i - 1;
        ids[i] = p < 0 || p >= places ? -1 : a.sorted[p];
        if (p >= p0 && p < p1)
            tokens[p - p0] = a.order[p];
    }
    __syncthreads();
    const int n = p1 - p0;
    const S *G = (const S *)a.G;
    constexpr int U = 4;
    for (int j = slice * kThreads + threadIdx.x; j < nv; j += a.slices * kThreads) {
        float acc[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            acc[k] = 0.f;
        bool first = ids[0] == ids[1];             // the run goes on from the window before
        for (int i0 = 0; i0 < n; i0 += U) {
            float g[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < n)
                    load_floats(G + (int64_t)tokens[i0 + u] * a.ldg + j * 8, g[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u >= n)
                    break;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    acc[k] += g[u][k];
                const int id = ids[i0 + u + 1];
                const bool ends = ids[i0 + u + 2] != id;
                if (!ends && i0 + u + 1 < n)
                    continue;
                if (first)
                    write_part(a.part + ((int64_t)w * 2) * a.d + j * 8, acc);
                else if (!ends)
                    write_part(a.part + ((int64_t)w * 2 + 1) * a.d + j * 8, acc);
                else
                    write_piece(dE + (int64_t)id * a.d + j * 8, acc, a.scale, a.accumulate);
                first = false;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    acc[k] = 0.f;
            }
        }
    }
}

// An id whose tokens go on from window to window is finished by the window where they start:
// its parts are added in the windows' order.
template <typename D>
__global__ void __launch_bounds__(kThreads) k_join_rows(const SumArgs a)
{
    griddep_start();
    const int w = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const int places = *a.places;
    const int p1 = (w + 1) * a.window;
    if (p1 >= places)
        return;
    const int id = a.sorted[p1 - 1];
    if (a.sorted[p1] != id)
        return;                                              // it ends here
    const int p0 = w * a.window;
    if (p0 > 0 && a.sorted[p0] == id && a.sorted[p0 - 1] == id)
        return;                                              // it started before
    int last = w + 1;                                        // the window where it ends
    while ((int64_t)(last + 1) * a.window < places && a.sorted[(last + 1) * a.window - 1] == id &&
           a.sorted[(last + 1) * a.window] == id)
        ++last;
    for (int j = slice * kThreads + threadIdx.x; j < a.d / 8; j += a.slices * kThreads) {
        float acc[8];
        load_floats(a.part + ((int64_t)w * 2 + 1) * a.d + j * 8, acc);
        for (int v = w + 1; v <= last; ++v) {
            float f[8];
            load_floats(a.part + ((int64_t)v * 2) * a.d + j * 8, f);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                acc[k] += f[k];
        }
        write_piece((D *)a.dE + (int64_t)id * a.d + j * 8, acc, a.scale, a.accumulate);
    }
}

// Widths that are no multiple of 8, gradients off the alignment: a block sums the runs that
// start in its window by single elements, to their ends.
template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) k_sum_rows_any(const SumArgs a)
{
    griddep_start();
    D *dE = (D *)a.dE;
    const S *G = (const S *)a.G;
    if ((int64_t)blockIdx.x >= a.windows) {
        const int64_t v0 = ((int64_t)blockIdx.x - a.windows) * 32;
        const uint32_t used = a.used[v0 / 32];
        const int n = (int)min((int64_t)32, a.vocab - v0);
        for (int i = 0; i < n; ++i)
            if (!((used >> i) & 1u))
                for (int j = threadIdx.x; j < a.d; j += kThreads)
                    dE[(v0 + i) * a.d + j] = Vec<D>::round(0.f);
        return;
    }
    const int places = *a.places;
    const int p0 = blockIdx.x * a.window, p1 = min(places, p0 + a.window);
    int p = p0;
    while (p < p1 && p > 0 && a.sorted[p] == a.sorted[p - 1])
        ++p;
    while (p < p1) {
        const int id = a.sorted[p];
        int end = p + 1;
        while (end < places && a.sorted[end] == id)
            ++end;
        for (int j = threadIdx.x; j < a.d; j += kThreads) {
            float acc = 0.f;
            for (int q = p; q < end; ++q)
                acc += Vec<S>::one(G[(int64_t)a.order[q] * a.ldg + j]);
            D *dst = dE + (int64_t)id * a.d + j;
            *dst = Vec<D>::round(a.accumulate ? fmaf(acc, a.scale, Vec<D>::one(*dst)) : acc * a.scale);
        }
        p = end;
    }
}

// ---- launches ----------------------------------------------------------------------------------

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), int64_t grid, int threads, size_t smem, cudaStream_t s,
                   const Args &...args)
{
    count_launch();
    const cudaError_t e = launch_dependent(kernel, dim3((unsigned)grid), dim3(threads), smem, s, args...);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename S, typename D>
cudaError_t lookup(const LookupArgs &a, cudaStream_t s)
{
    const int64_t most = (int64_t)1 << 30;
    if (a.d % 8 != 0)
        return launch(k_lookup_any<S, D>, std::min(a.T, most), kThreads, 0, s, a);
    int lx = 0;
    while (lx < 8 && (1 << lx) < a.d / 8)
        ++lx;
    const int per = kThreads >> lx;
    return launch(k_lookup<S, D>, std::min((a.T + per - 1) / per, most), kThreads, 0, s, a, lx);
}

// Where the sort's and the sums' buffers lie in the workspace
struct Layout {
    size_t order, sorted, places, used, part, total;
    int window, windows;
};

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

Layout layout_of(int64_t T, int64_t vocab, int d)
{
    Layout l;
    // 8 to 128 places a window, so that small calls still fill the SMs
    const int64_t sms = device_sms();
    int64_t w = 8;
    while (w < kMaxWindow && T / w * ((d + 2047) / 2048) > 8 * sms)
        w *= 2;
    l.window = (int)w;
    l.windows = (int)((T + w - 1) / w);
    size_t at = 0;
    l.order = at;
    at += up256((size_t)T * 4);
    l.sorted = at;
    at += up256((size_t)T * 4);
    l.places = at;
    at += 256;
    l.used = at;
    at += up256((size_t)((vocab + 31) / 32) * 4);
    l.part = at;
    at += up256((size_t)l.windows * 2 * d * sizeof(float));
    l.total = at;
    return l;
}

template <typename S, typename D>
cudaError_t sum_rows(const SumArgs &a, cudaStream_t s)
{
    const int64_t fill = a.accumulate ? 0 : (a.vocab + 31) / 32;
    if (a.d % 8 != 0 || a.ldg % 8 != 0)
        return a.windows + fill == 0 ? cudaSuccess
                                     : launch(k_sum_rows_any<S, D>, a.windows + fill, kThreads, 0, s, a);
    cudaError_t e = cudaSuccess;
    if ((int64_t)a.windows * a.slices + fill > 0)
        e = launch(k_sum_rows<S, D>, (int64_t)a.windows * a.slices + fill, kThreads, 0, s, a);
    if (e == cudaSuccess && a.windows > 1)
        e = launch(k_join_rows<D>, (int64_t)(a.windows - 1) * a.slices, kThreads, 0, s, a);
    return e;
}

}  // namespace

cudaError_t embed_fwd(sn_dtype tdt, const void *table, int64_t vocab, int d, const int32_t *ids, int64_t T,
                      float scale, sn_dtype xdt, void *X, unsigned int *err, cudaStream_t s)
{
    const LookupArgs a{table, vocab, d, ids, T, scale, X, err};
    if (tdt == SN_BF16)
        return xdt == SN_BF16 ? lookup<__nv_bfloat16, __nv_bfloat16>(a, s) : lookup<__nv_bfloat16, float>(a, s);
    return xdt == SN_BF16 ? lookup<float, __nv_bfloat16>(a, s) : lookup<float, float>(a, s);
}

size_t embed_bwd_workspace(int64_t T, int64_t vocab, int d) { return layout_of(T, vocab, d).total; }

cudaError_t embed_bwd(sn_dtype gdt, const void *G, int64_t ldg, int64_t T, int d, const int32_t *ids, float scale,
                      sn_dtype edt, void *dE, int64_t vocab, bool accumulate, void *ws, unsigned int *err,
                      cudaStream_t s)
{
    const Layout l = layout_of(T, vocab, d);
    char *m = (char *)ws;
    // a range of ids for every SM, whole words of `used`
    int64_t width = (vocab + device_sms() - 1) / device_sms();
    width = std::min<int64_t>((width + 31) / 32 * 32, kMaxWidth);
    SortArgs q{ids, T, vocab, (int)width, (int)((vocab + width - 1) / width), (int32_t *)(m + l.order),
               (int32_t *)(m + l.sorted), (int32_t *)(m + l.places), (uint32_t *)(m + l.used), err};
    const size_t smem = (size_t)width * 4 + 4 * kSortThreads * sizeof(int2);
    cudaError_t e = cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess)
        e = launch(k_sort_tokens, std::min(q.ranges, device_sms()), kSortThreads, smem, s, q);
    if (e != cudaSuccess)
        return e;
    const SumArgs a{G, ldg, T, vocab, d, scale, dE, accumulate, q.order, q.sorted, q.places, q.used,
                    l.window, l.windows, std::min(64, (d + 8 * kThreads - 1) / (8 * kThreads)), (float *)(m + l.part)};
    if (gdt == SN_BF16)
        return edt == SN_BF16 ? sum_rows<__nv_bfloat16, __nv_bfloat16>(a, s) : sum_rows<__nv_bfloat16, float>(a, s);
    return edt == SN_BF16 ? sum_rows<float, __nv_bfloat16>(a, s) : sum_rows<float, float>(a, s);
}

}  // namespace sn
