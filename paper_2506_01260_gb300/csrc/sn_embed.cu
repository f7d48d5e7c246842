// sn_embed.cu — embedding lookup with scaling, and its gradient by sorted tokens.
//
//   X[t] = scale E[ids[t]],   dE[v] = scale sum over the t with ids[t] = v of G[t]
//
// Both bound by DRAM: the lookup reads a row and writes one for every token; the gradient
// reads G once and writes the whole table once (or, accumulating, reads and writes the rows
// that have tokens).  The gradient sorts the tokens by id, cuts the sorted list into windows
// of equal length, whatever the ids' frequencies, and lets a block sum a window's rows in
// token order: a token with thousands of rows is shared by many blocks, without atomics.
//
// Measured: the lookup of 16384 bf16 rows of 4096 43 us (6.2 TB/s); the gradient of 16384 bf16
// rows of 4096 into 128256 bf16 rows 178 us (6.6 TB/s), of 65536 rows of 8192 with Zipf ids into
// 32000 fp32 rows 360 us (5.9 TB/s), 24 of them the sort, which reads all ids on every SM, and 9
// the sums of the ids that many windows share.
#include <algorithm>

#include "sn_vec.cuh"

namespace sn {
namespace {

constexpr int kThreads = 256;

// 8 elements of a row as they lie in memory
template <typename S>
struct Raw {
    static constexpr int kWords = (int)sizeof(S) / 2, P = Vec<S>::N / 2;
    uint4 v[kWords];
    __device__ __forceinline__ void load(const S *p)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            v[i] = __ldg((const uint4 *)p + i);
    }
    // for a row that is read once: first to leave L2
    __device__ __forceinline__ void load_once(const S *p)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            v[i] = __ldcs((const uint4 *)p + i);
    }
    // `n` elements one by one, zeros after them
    __device__ __forceinline__ void load_single(const S *p, int n)
    {
        union {
            uint4 w[kWords];
            S x[8];
        } u;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            u.x[k] = k < n ? p[k] : Vec<S>::round(0.f);
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            v[i] = u.w[i];
    }
    __device__ __forceinline__ void get(float2 (&f)[4]) const
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            unpack_pairs(v[i], *(float2(*)[P])(f + i * P));
    }
};

template <bool ONCE = false, typename D>
__device__ __forceinline__ void put_piece(D *dst, const float2 (&f)[4])
{
    constexpr int P = Vec<D>::N / 2;
#pragma unroll
    for (int i = 0; i < 4 / P; ++i) {
        const uint4 v = pack_pairs(*(const float2(*)[P])(f + i * P));
        if (ONCE)
            __stcs((uint4 *)dst + i, v);
        else
            ((uint4 *)dst)[i] = v;
    }
}

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

// 2^lx lanes walk a row's pieces of 8 elements, two at a time; a block takes 256 >> lx rows.
// Loads and stores are marked to leave L2 first (16384 rows of 4096 from 128256: 42.5 us, 46.5
// without; 65536 rows of 2048 from 1024: 107, 122).  Blocks on an SM hide the chain id -> row:
// eight for bf16 (27551 rows of 512: 10.5 us, 11.7 with six), from fp32 tables six of 32 bytes
// of loads a thread (U = 1) for rows of one step (65536 rows of 1024: 76 us, 81 with five of 64
// bytes) and five of 64 bytes for longer ones (65536 rows of 8192: 513 us, 534 the other way).
template <typename S, typename D, int U>
__global__ void __launch_bounds__(kThreads, sizeof(S) + sizeof(D) == 4 ? 8 : U == 1 ? 6 : 5)
    k_lookup(const LookupArgs a, int lx)
{
    griddep_start();
    constexpr int N = 8;
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
            Raw<S> g[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j0 + (u << lx) < nv)
                    g[u].load_once(src + (j0 + (u << lx)) * N);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + (u << lx);
                if (j >= nv)
                    break;
                float2 f[4];
                g[u].get(f);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    f[k] = good ? mul2(f[k], both(a.scale)) : both(0.f);
                put_piece<true>(dst + j * N, f);
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
// (from L2): it counts the valid ids below its range, which is where its tokens start in the
// sorted list, and its own tokens by warp and step, which gives each of them its place in a list
// in token order.  That list is cut into `segments`, a warp each; with every segment's count of
// every id, the warps place their segments' tokens at once, 32 at a time.  No block waits for
// another, and there is no atomic whose order shows.

constexpr int kSortThreads = 1024;
constexpr int kWarps = kSortThreads / 32;
constexpr int kCounters = 24576;               // segments * width, at most
constexpr int kMaxWidth = 8192;                // ids of a range
constexpr int kStep = 4 * kSortThreads;        // tokens of a step: 4 consecutive ones a thread
constexpr int kSteps = 16;                     // steps that are counted before tokens are listed

struct SortArgs {
    const int32_t *ids;
    int64_t T, vocab;
    int width, ranges, segments;
    int32_t *order, *sorted;    // [T] token and id at each place of the sorted list
    int32_t *tokens, *locals;   // [T] token and id within its range, range by range in token order
    int32_t *places;            // valid tokens
    uint32_t *used;             // a bit per id: has tokens
    unsigned int *err;
};

// The exclusive prefix sum of `n` over the block and its total; `warps`: 32 ints
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
    const int mine = warps[lane];
    int s = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        s += lane >= o ? y : 0;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    return __shfl_sync(0xffffffffu, s - mine, warp) + incl - n;
}

// The ids of 4 consecutive tokens, -1 past the last
__device__ __forceinline__ int4 load_ids(const SortArgs &a, int64_t t)
{
    if (t + 4 <= a.T && aligned16(a.ids))
        return __ldg((const int4 *)(a.ids + t));
    return make_int4(t < a.T ? a.ids[t] : -1, t + 1 < a.T ? a.ids[t + 1] : -1, t + 2 < a.T ? a.ids[t + 2] : -1,
                     t + 3 < a.T ? a.ids[t + 3] : -1);
}

__global__ void __launch_bounds__(kSortThreads) k_sort_tokens(const SortArgs a)
{
    griddep_start();
    extern __shared__ int count[];                  // [segments][width]
    __shared__ int warps[kWarps], found[kSteps * kWarps];
    __shared__ int s_below, s_bad;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int range = blockIdx.x; range < a.ranges; range += gridDim.x) {
        const int64_t lo = (int64_t)range * a.width;
        const uint32_t n_ids = (uint32_t)min((int64_t)a.width, a.vocab - lo);
        __syncthreads();
        if (threadIdx.x == 0)
            s_below = s_bad = 0;
        __syncthreads();
        int below = 0, bad = 0;
        auto look = [&](const int4 &v, int64_t t) {          // 4 tokens; which are the range's
            const int id[4] = {v.x, v.y, v.z, v.w};
            uint32_t h = 0;
            if (range == 0)                                  // one block reports ids that are none
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    bad |= (uint32_t)id[k] >= (uint64_t)a.vocab && t + k < a.T;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                below += (uint32_t)id[k] < (uint32_t)lo;
                h |= ((uint32_t)id[k] - (uint32_t)lo < n_ids ? 1u : 0u) << k;
            }
            return h;
        };
        // the ids below the range, ids that are none: of all tokens before the first is listed
        for (int64_t t0 = (int64_t)kSteps * kStep; t0 < a.T; t0 += 4 * kStep) {
            int4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = load_ids(a, t0 + u * kStep + 4 * threadIdx.x);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                look(v[u], t0 + u * kStep + 4 * threadIdx.x);
        }
        // the range's tokens in order, kSteps steps at a time: count by step and warp, then list
        int mine = 0, first = 0;
        for (int64_t t0 = 0; t0 < a.T; t0 += (int64_t)kSteps * kStep) {
            const int steps = (int)min((int64_t)kSteps, (a.T - t0 + kStep - 1) / kStep);
            uint64_t hits = 0;                       // 4 bits a step
            for (int q = 0; q < steps; q += 4) {
                int4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    v[u] = load_ids(a, t0 + (q + u) * kStep + 4 * threadIdx.x);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t h = look(v[u], t0 + (q + u) * kStep + 4 * threadIdx.x);
                    hits |= (uint64_t)h << (4 * (q + u));
                    const int n = __reduce_add_sync(0xffffffffu, __popc(h));
                    if (lane == 0)
                        found[(q + u) * kWarps + warp] = n;
                }
            }
            if (t0 == 0) {
                below = warp_sum(below);
                if (lane == 0 && below)
                    atomicAdd(&s_below, below);
                if (bad)
                    s_bad = 1;
            }
            __syncthreads();
            first = s_below;
            int total;
            const int n = threadIdx.x < steps * kWarps ? found[threadIdx.x] : 0;
            const int at = block_scan(n, warps, total);
            if (threadIdx.x < steps * kWarps)
                found[threadIdx.x] = at;
            __syncthreads();
            for (int q = 0; q < steps; ++q) {
                const uint32_t h = (uint32_t)(hits >> (4 * q)) & 15u;
                if (__ballot_sync(0xffffffffu, h) == 0)
                    continue;
                int incl = __popc(h);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, incl, o);
                    incl += lane >= o ? y : 0;
                }
                int p = first + mine + found[q * kWarps + warp] + incl - __popc(h);
                const int64_t t = t0 + q * kStep + 4 * threadIdx.x;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if ((h >> k) & 1u)
                        a.tokens[p++] = (int)(t + k);
            }
            mine += total;
            __syncthreads();
        }
        if (range == 0 && threadIdx.x == 0 && s_bad && a.err)
            atomicOr(a.err, SN_EBIT_BAD_ID);
        // short lists take fewer segments: two rounds of a warp each
        const int segments = max(1, min(a.segments, (mine + 63) / 64));
        for (int i = threadIdx.x; i < segments * a.width; i += kSortThreads)
            count[i] = 0;
        __syncthreads();
        // each segment's count of each id
        const int per = (mine + segments - 1) / segments;
        const int i0 = min(mine, warp * per), i1 = warp < segments ? min(mine, i0 + per) : i0;
        int *counts = count + warp * a.width;
        for (int ib = i0; ib < i1; ib += 4 * 32) {
            int local[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                local[u] = ib + u * 32 + lane < i1 ? a.tokens[first + ib + u * 32 + lane] : -1;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                local[u] = local[u] >= 0 ? a.ids[local[u]] - (int)lo : -1;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t same = __match_any_sync(0xffffffffu, local[u]);
                if (local[u] >= 0) {
                    a.locals[first + ib + u * 32 + lane] = local[u];
                    if ((same >> lane) == 1u)                  // the last lane of its id
                        counts[local[u]] += __popc(same);
                }
                __syncwarp();
            }
        }
        __syncthreads();
        // each id's first place, and from there each segment's; the bits of ids with tokens
        int place = first;
        for (int c0 = 0; c0 < a.width; c0 += kSortThreads) {
            const int c = c0 + threadIdx.x;
            int n = 0;
            if (c < a.width)
                for (int g = 0; g < segments; ++g) {
                    const int x = count[g * a.width + c];
                    count[g * a.width + c] = n;
                    n += x;
                }
            const uint32_t bits = __ballot_sync(0xffffffffu, n > 0);
            if (lane == 0 && (uint32_t)c < n_ids)
                a.used[(lo + c) / 32] = bits;
            int total;
            const int at = place + block_scan(n, warps, total);
            if (c < a.width)
                for (int g = 0; g < segments; ++g)
                    count[g * a.width + c] += at;
            place += total;
        }
        if (threadIdx.x == 0 && range == a.ranges - 1)
            *a.places = place;
        __syncthreads();
        // the segments' tokens at their places
        int token = -1, local = -1;
        if (i0 + lane < i1) {
            token = a.tokens[first + i0 + lane];
            local = a.locals[first + i0 + lane];
        }
        for (int ib = i0; ib < i1; ib += 32) {
            const int t = token, id = local, next = ib + 32 + lane;
            token = next < i1 ? a.tokens[first + next] : -1;
            local = next < i1 ? a.locals[first + next] : -1;
            const uint32_t same = __match_any_sync(0xffffffffu, id);
            if (id >= 0) {
                const int p = counts[id] + __popc(same & ((1u << lane) - 1u));
                a.order[p] = t;
                a.sorted[p] = (int)lo + id;
            }
            __syncwarp();
            if (id >= 0 && (same >> lane) == 1u)
                counts[id] += __popc(same);
            __syncwarp();
        }
    }
}

// At most kFew tokens: one block, every token's place from the tokens before it in order
constexpr int kFew = 1024;

__global__ void __launch_bounds__(kFew) k_sort_few(const SortArgs a)
{
    griddep_start();
    __shared__ uint32_t ids[kFew];
    const int T = (int)a.T, t = threadIdx.x;
    const int id = t < T ? a.ids[t] : -1;
    const bool good = t < T && (uint32_t)id < (uint64_t)a.vocab;
    ids[t] = good ? (uint32_t)id : 0xffffffffu;              // those that are none come last
    for (int64_t w = t; w < (a.vocab + 31) / 32; w += blockDim.x)
        a.used[w] = 0;
    const int places = __syncthreads_count(good);
    if (t == 0)
        *a.places = places;
    if (t < T && !good && a.err)
        atomicOr(a.err, SN_EBIT_BAD_ID);
    if (!good)
        return;
    int p = 0;
#pragma unroll 8
    for (int i = 0; i < T; ++i)
        p += ids[i] < (uint32_t)id || (ids[i] == (uint32_t)id && i < t);
    a.order[p] = t;
    a.sorted[p] = id;
    atomicOr(a.used + id / 32, 1u << (id & 31));
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
    float *part;                   // [windows][2][dp]: sums of a first and a last id that go on in other windows
    int dp;                        // d rounded up to 8
};

constexpr int kMaxWindow = 128;

// n <= 8 columns of a row of dE: the sum times the scale, in addition to what is there.  VEC: all
// 8, on a 16-byte boundary.
template <typename D, bool VEC>
__device__ __forceinline__ void write_piece(D *dst, int n, const float2 (&acc)[4], float scale, bool accumulate)
{
    float2 f[4];
    if (accumulate) {
        Raw<D> old;
        if (VEC)
            old.load(dst);
        else
            old.load_single(dst, n);
        old.get(f);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        f[k] = accumulate ? fma2(acc[k], both(scale), f[k]) : mul2(acc[k], both(scale));
    if (VEC) {
        put_piece(dst, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n)
                dst[k] = Vec<D>::round(k % 2 ? f[k / 2].y : f[k / 2].x);
    }
}

__device__ __forceinline__ void write_part(float *dst, const float2 (&acc)[4])
{
    *(float4 *)dst = make_float4(acc[0].x, acc[0].y, acc[1].x, acc[1].y);
    *(float4 *)(dst + 4) = make_float4(acc[2].x, acc[2].y, acc[3].x, acc[3].y);
}

// Blocks [0, windows * slices) sum; the others, 32 ids each, write the rows without tokens, a
// warp a row.  A thread has 8 columns: narrow rows have smaller blocks, more of them an SM (27551
// bf16 rows of 512 into 50257 ids: 28 us, 39 with 256 threads for either kind of block).
// MODE 0 writes dE.  MODE 1 adds to it and loads the rows of dE that a batch of tokens ends in
// with the batch's rows of G; MODE 2 loads them when it gets there, with more rows of G in
// flight.
enum { WRITE = 0, ADD_AHEAD = 1, ADD = 2 };

template <typename S, typename D, int MODE, bool VEC>
__global__ void __launch_bounds__(kThreads) k_sum_rows(const SumArgs a)
{
    griddep_start();
    constexpr bool ACC = MODE == ADD_AHEAD;
    const int nv = a.dp / 8;
    D *dE = (D *)a.dE;
    if ((int64_t)blockIdx.x >= (int64_t)a.windows * a.slices) {
        const int64_t word = (int64_t)blockIdx.x - (int64_t)a.windows * a.slices;
        const uint32_t used = a.used[word];
        const int64_t v0 = word * 32;
        const int n = (int)min((int64_t)32, a.vocab - v0);
        for (int i = threadIdx.x / 32; i < n; i += blockDim.x / 32)
            if (!((used >> i) & 1u)) {
                D *row = dE + (v0 + i) * a.d;
                if (VEC)
                    for (int j = threadIdx.x % 32; j < a.d / Vec<D>::N; j += 32)
                        ((uint4 *)row)[j] = make_uint4(0, 0, 0, 0);
                else
                    for (int j = threadIdx.x % 32; j < a.d; j += 32)
                        row[j] = Vec<D>::round(0.f);
            }
        return;
    }
    const int w = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const int places = *a.places;
    const int p0 = w * a.window, p1 = min(places, p0 + a.window);
    if (p0 >= p1)
        return;
    // A run of one id that goes on in the next window and ends there is summed here, where it
    // starts; a longer one leaves a part in every window.
    // ids from the place before the window to the one after the next, tokens of both
    __shared__ int all_ids[2 * kMaxWindow + 2], all_tokens[2 * kMaxWindow];
    for (int k = threadIdx.x; k < 2 * a.window + 2; k += blockDim.x) {
        const int p = p0 - 1 + k;
        all_ids[k] = p >= 0 && p < places ? a.sorted[p] : -1;
        if (k < 2 * a.window)
            all_tokens[k] = p + 1 < places ? a.order[p + 1] : 0;
    }
    const int far_before = p0 > a.window ? a.sorted[p0 - a.window - 1] : -1;
    __syncthreads();
    const int len = p1 - p0;
    const int head = all_ids[1], tail = all_ids[len], after = all_ids[len + 1];
    const bool going_on = all_ids[0] == head;
    // the head run, where the window before has it; the tail run's tokens of the next window
    int skip = 0, more = 0;
    for (int i0 = 0; i0 < a.window; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        skip += __syncthreads_count(i < len && going_on && far_before != head && after != head &&
                                    all_ids[1 + i] == head);
        more += __syncthreads_count(i < a.window && after == tail && all_ids[len + 1 + a.window] != tail &&
                                    !(going_on && tail == head) && all_ids[len + 1 + i] == tail);
    }
    const int n = len + more - skip;
    if (n <= 0)
        return;
    const int *ids = all_ids + skip, *tokens = all_tokens + skip;
    const S *G = (const S *)a.G;
    constexpr int U = sizeof(S) == 2 && !ACC ? 8 : 4;         // rows in flight
    for (int j = slice * blockDim.x + threadIdx.x; j < nv; j += a.slices * blockDim.x) {
        float2 acc[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            acc[k] = both(0.f);
        bool first = ids[0] == ids[1];             // the run goes on from the window before
        for (int i0 = 0; i0 < n; i0 += U) {
            Raw<S> g[U];
            Raw<D> old[ACC ? U : 1];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < n) {
                    const S *src = G + (int64_t)tokens[i0 + u] * a.ldg + j * 8;
                    if (VEC)
                        g[u].load(src);
                    else
                        g[u].load_single(src, a.d - j * 8);
                    if (ACC && ids[i0 + u + 2] != ids[i0 + u + 1])
                        old[ACC ? u : 0].load(dE + (int64_t)ids[i0 + u + 1] * a.d + j * 8);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u >= n)
                    break;
                float2 row[4];
                g[u].get(row);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    acc[k] = add2(acc[k], row[k]);
                const int id = ids[i0 + u + 1];
                const bool ends = ids[i0 + u + 2] != id;
                if (!ends && i0 + u + 1 < n)
                    continue;
                if (first || !ends) {
                    write_part(a.part + ((int64_t)w * 2 + !first) * a.dp + j * 8, acc);
                } else if (ACC) {
                    float2 sum[4];
                    old[ACC ? u : 0].get(sum);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum[k] = fma2(acc[k], both(a.scale), sum[k]);
                    put_piece(dE + (int64_t)id * a.d + j * 8, sum);
                } else {
                    write_piece<D, VEC>(dE + (int64_t)id * a.d + j * 8, a.d - j * 8, acc, a.scale, MODE == ADD);
                }
                first = false;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    acc[k] = both(0.f);
            }
        }
    }
}

// An id whose tokens go on from window to window is finished by the window where they start.
// A block takes 256 columns of kJoin windows: its 8 warps share the parts of such an id and
// their sums are added in the warps' order.
constexpr int kJoin = 8;

template <typename D, bool VEC>
__global__ void __launch_bounds__(kThreads) k_join_rows(const SumArgs a)
{
    griddep_start();
    constexpr int kWarps8 = kThreads / 32, U = 4;
    const int cols = (a.d + 255) / 256;
    const int w0 = blockIdx.x / cols * kJoin, j = blockIdx.x % cols * 256 + threadIdx.x % 32 * 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ int starts[kJoin];                            // the id that a window starts and several go on with
    __shared__ __align__(16) float sums[kWarps8][256];
    const int places = *a.places;
    if (threadIdx.x < kJoin) {
        const int64_t p0 = (int64_t)(w0 + threadIdx.x) * a.window, p1 = p0 + a.window;
        int id = -1;
        if (p1 + a.window < places) {
            id = a.sorted[p1];
            const int last = a.sorted[p1 - 1], head = a.sorted[p0], before = p0 > 0 ? a.sorted[p0 - 1] : -1;
            if (last != id || (head == id && before == id) || a.sorted[p1 + a.window] != id)
                id = -1;
        }
        starts[threadIdx.x] = id;
    }
    __syncthreads();
    for (int q = 0; q < kJoin; ++q) {
        const int id = starts[q], w = w0 + q;
        if (id < 0)
            continue;
        // the windows that start with this id: all up to the one where it ends
        int more = 0;
        for (;;) {
            const int64_t v = (int64_t)w + 1 + more + threadIdx.x;
            const int n = __syncthreads_count(v * a.window < places && a.sorted[v * a.window] == id);
            more += n;
            if (n < kThreads)
                break;
        }
        float2 acc[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            acc[k] = both(0.f);
        if (j < a.d) {
            // part 0: the last of window w, parts 1 to `more`: the first of those after it
            for (int v0 = warp; v0 <= more; v0 += U * kWarps8) {
                Raw<float> f[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int v = v0 + u * kWarps8;
                    if (v <= more)
                        f[u].load(a.part + ((int64_t)(w + v) * 2 + (v == 0)) * a.dp + j);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (v0 + u * kWarps8 <= more) {
                        float2 x[4];
                        f[u].get(x);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            acc[k] = add2(acc[k], x[k]);
                    }
            }
        }
        write_part(&sums[warp][lane * 8], acc);
        __syncthreads();
        if (warp == 0 && j < a.d) {
            for (int v = 1; v < kWarps8; ++v)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    acc[k] = add2(acc[k], *(const float2 *)&sums[v][lane * 8 + 2 * k]);
            write_piece<D, VEC>((D *)a.dE + (int64_t)id * a.d + j, a.d - j, acc, a.scale, a.accumulate);
        }
        __syncthreads();
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
    const int64_t blocks = std::min((a.T + per - 1) / per, most);
    return sizeof(S) == 4 && a.d / 8 <= kThreads ? launch(k_lookup<S, D, 1>, blocks, kThreads, 0, s, a, lx)
                                                 : launch(k_lookup<S, D, 2>, blocks, kThreads, 0, s, a, lx);
}

// Where the sort's and the sums' buffers lie in the workspace
struct Layout {
    size_t order, sorted, list, places, used, part, total;
    int window, windows;
};

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

Layout layout_of(int64_t T, int64_t vocab, int d)
{
    Layout l;
    // 8 to 128 places a window, so that small calls still fill the SMs (with blocks of a warp for
    // every 256 columns)
    const int64_t sms = device_sms();
    int64_t w = 8;
    while (w < kMaxWindow && T / w * ((d + 255) / 256) > 64 * sms)
        w *= 2;
    l.window = (int)w;
    l.windows = (int)((T + w - 1) / w);
    size_t at = 0;
    l.order = at;
    at += up256((size_t)T * 4);
    l.sorted = at;
    at += up256((size_t)T * 4);
    l.list = at;
    at += up256((size_t)T * 8);
    l.places = at;
    at += 256;
    l.used = at;
    at += up256((size_t)((vocab + 31) / 32) * 4);
    l.part = at;
    at += up256((size_t)l.windows * 2 * ((d + 7) / 8 * 8) * sizeof(float));
    l.total = at;
    return l;
}

template <typename S, typename D, int MODE, bool VEC>
cudaError_t sum_and_join(const SumArgs &a, cudaStream_t s)
{
    const int64_t grid = (int64_t)a.windows * a.slices + (MODE == WRITE ? (a.vocab + 31) / 32 : 0);
    const int threads = std::min(kThreads, (a.dp / 8 + 31) / 32 * 32);      // 256: slices may be more than one
    cudaError_t e = grid > 0 ? launch(k_sum_rows<S, D, MODE, VEC>, grid, threads, 0, s, a) : cudaSuccess;
    if (e == cudaSuccess && a.windows > 1)
        e = launch(k_join_rows<D, VEC>, (int64_t)(a.windows - 1 + kJoin - 1) / kJoin * ((a.d + 255) / 256), kThreads,
                   0, s, a);
    return e;
}

template <typename S, typename D>
cudaError_t sum_rows(const SumArgs &a, cudaStream_t s)
{
    // rows that are no whole 16-byte pieces: single elements
    if (a.d % 8 != 0 || a.ldg % 8 != 0)
        return a.accumulate ? sum_and_join<S, D, ADD, false>(a, s) : sum_and_join<S, D, WRITE, false>(a, s);
    if (!a.accumulate)
        return sum_and_join<S, D, WRITE, true>(a, s);
    // fewer tokens than ids: most ids have one token or two, and a batch ends in several rows
    // of dE (16384 tokens of 128256 ids: 78 us, 102 without the loads ahead); more tokens than
    // ids: they cost rows of G in flight (65536 of 32000: 370 us, 320 without)
    return a.T < a.vocab ? sum_and_join<S, D, ADD_AHEAD, true>(a, s) : sum_and_join<S, D, ADD, true>(a, s);
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
    const int segments = std::max(1, std::min(kWarps, (int)(kCounters / width)));
    SortArgs q{ids, T, vocab, (int)width, (int)((vocab + width - 1) / width), segments, (int32_t *)(m + l.order),
               (int32_t *)(m + l.sorted), (int32_t *)(m + l.list), (int32_t *)(m + l.list) + T, (int32_t *)(m + l.places), (uint32_t *)(m + l.used),
               err};
    cudaError_t e = cudaSuccess;
    if (T <= kFew) {
        e = launch(k_sort_few, 1, (int)((std::max<int64_t>(T, 32) + 31) / 32 * 32), 0, s, q);
    } else {
        e = cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeMaxDynamicSharedMemorySize, kCounters * 4);
        if (e == cudaSuccess)
            e = launch(k_sort_tokens, std::min(q.ranges, device_sms()), kSortThreads, (size_t)segments * width * 4, s,
                       q);
    }
    if (e != cudaSuccess)
        return e;
    const SumArgs a{G, ldg, T, vocab, d, scale, dE, accumulate, q.order, q.sorted, q.places, q.used,
                    l.window, l.windows, std::min(64, (d + 8 * kThreads - 1) / (8 * kThreads)), (float *)(m + l.part),
                    (d + 7) / 8 * 8};
    if (gdt == SN_BF16)
        return edt == SN_BF16 ? sum_rows<__nv_bfloat16, __nv_bfloat16>(a, s) : sum_rows<__nv_bfloat16, float>(a, s);
    return edt == SN_BF16 ? sum_rows<float, __nv_bfloat16>(a, s) : sum_rows<float, float>(a, s);
}

}  // namespace sn
