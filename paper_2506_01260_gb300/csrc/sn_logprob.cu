// sn_logprob.cu — log probabilities of given tokens from logits, with the entropy and the
// best alternatives, and the gradient of log probability and entropy.
//
//   m = max x,  z = scale (x - m),  S = sum e^z
//   logp = z[target] - ln S,   H = ln S - sum e^z z / S
//   dx[v] = scale (a ([v = target] - p[v]) - b p[v] (ln p[v] + H)),  ln p = z - ln S
//
// Bound by DRAM, at 2 or 4 bytes a logit (twice that for the gradient), as long as the
// arithmetic hides behind it: one pass over a row keeps a running maximum, S and the
// entropy's sum in each thread, in base 2 so that an exponential is one fma and one ex2.
// Sums are fp32.  A row is one block's, or, where rows are few, that of a cluster of blocks
// that join their sums in shared memory.
//
// The alternatives come out of the same pass: each thread keeps the largest logit it saw,
// and the n-th largest of those bounds the row's n-th largest from below, so only the few
// elements at or above the bound are looked at again (in L2) and ranked by value, the lower
// token first among equals.
#include <algorithm>

#include "sn_vec.cuh"

namespace sn {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxTop = 32;
constexpr int kCand = 1024;             // elements at or above the bound that a block ranks
constexpr int kMaxCluster = 8;
// 2^t below 2^-200 is 0 in fp32; clamped there, 0 * t is 0 where t is -infinity
constexpr float kFloor = -200.f;

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

struct LogpArgs {
    const void *x;
    int64_t T, ld;
    int V;
    const int32_t *target;     // may be null
    float scale;
    float *logp, *lse, *entropy;   // each may be null; lse: [T, 2]
    int top;
    int32_t *top_ids;
    float *top_logp;
    unsigned int *err;
};

// A row from its first 16-byte boundary on: `head` elements before it, `nv` whole pieces,
// then the rest.  The ends are read singly, so nothing outside the row is touched.
template <typename T>
struct RowView {
    const T *p;
    int head, nv, V;
    __device__ __forceinline__ RowView(const T *row, int V) : p(row), V(V)
    {
        const int off = (int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T));
        head = off < V ? off : V;
        nv = (V - head) / Vec<T>::N;
    }
    __device__ __forceinline__ uint4 piece(int i) const { return __ldg((const uint4 *)(p + head) + i); }
    // elements outside the pieces: 0 .. loose() - 1, and the column of each
    __device__ __forceinline__ int loose() const { return V - nv * Vec<T>::N; }
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + nv * Vec<T>::N; }
};

// Order of logits as whole numbers: larger logits first, -0 = +0, NaN above everything
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x)
        return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key == 0xffffffffu ? 0x7fffffffu : key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kLowestKey = 0x007fffffu;       // of -infinity
// The larger logit first, then the lower token
__device__ __forceinline__ uint64_t rank_key(uint32_t key, int v) { return (uint64_t)key << 32 | (0xffffffffu - (uint32_t)v); }

// A part of a row's softmax sums: the largest logit m, and the sums of e and e * t over
// e = 2^t, t = x c - base(m), c = scale log2(e).  One fma makes t; the base is m c rounded, which
// every part and the result agree on.  Where m c overflows (a row masked with the type's lowest
// value) t is (x - m) c instead.
struct Sums {
    float m, s, a;
};

// 0 for a part that has no logit above -infinity: its sums are 0
__device__ __forceinline__ float base_of(float m, float c) { return m == -INFINITY ? 0.f : __fmul_rn(m, c); }
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// What t loses when the maximum rises from m0 to m1
__device__ __forceinline__ float shift(float m0, float m1, float c)
{
    if (m0 == -INFINITY)
        return 0.f;
    const float b0 = base_of(m0, c), b1 = base_of(m1, c);
    return finite(b0) && finite(b1) ? b0 - b1 : (m0 - m1) * c;
}

__device__ __forceinline__ void join(Sums &x, const Sums &y, float c)
{
    const float m = fmaxf(x.m, y.m);
    const float dx = shift(x.m, m, c), dy = shift(y.m, m, c);
    const float fx = ex2(dx), fy = ex2(dy);
    x.a = fx * fmaf(x.s, fmaxf(dx, kFloor), x.a) + fy * fmaf(y.s, fmaxf(dy, kFloor), y.a);
    x.s = fx * x.s + fy * y.s;
    x.m = m;
}

template <int THREADS>
struct Shared {
    Sums sums[THREADS / 32];
    Sums block;                        // this block's sums, read by the cluster
    uint32_t lane_max[THREADS];
    uint32_t bound;
    int n_cand;
    uint64_t cand[kCand];
    uint64_t best[kMaxTop];            // this block's alternatives in order, read by the cluster
    uint64_t merged[kMaxCluster * kMaxTop];
    uint64_t found[THREADS / 32];
};

__device__ __forceinline__ uint64_t warp_max64(uint64_t v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t w = __shfl_xor_sync(0xffffffffu, v, o);
        v = w > v ? w : v;
    }
    return v;
}

// `fn(value, column)` for this thread's elements of the pieces [i0, i1) and, in the block
// that has them, the loose ends
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void each(const RowView<T> &row, int i0, int i1, bool ends, F fn)
{
    constexpr int N = Vec<T>::N;
    for (int i = i0 + threadIdx.x; i < i1; i += THREADS) {
        float f[N];
        Vec<T>::unpack(row.piece(i), f);
#pragma unroll
        for (int k = 0; k < N; ++k)
            fn(f[k], row.head + i * N + k);
    }
    if (ends)
        for (int i = threadIdx.x; i < row.loose(); i += THREADS) {
            const int v = row.loose_at(i);
            fn(Vec<T>::one(row.p[v]), v);
        }
}

// sh.cand = this block's elements whose key is at least `from`; how many there are (the list
// holds the first kCand of them)
template <typename T, int THREADS>
__device__ __forceinline__ int collect(Shared<THREADS> &sh, const RowView<T> &row, int i0, int i1, bool ends,
                                       uint32_t from, uint32_t mine)
{
    __syncthreads();
    if (threadIdx.x == 0)
        sh.n_cand = 0;
    __syncthreads();
    if (mine >= from)
        each<T, THREADS>(row, i0, i1, ends, [&](float x, int v) {
            const uint32_t k = key_of(x);
            if (k >= from) {
                const int at = atomicAdd(&sh.n_cand, 1);
                if (at < kCand)
                    sh.cand[at] = rank_key(k, v);
            }
        });
    __syncthreads();
    return sh.n_cand;
}

// sh.best[r0 .. r1) = the lowest tokens of this block whose key is `key`: steps of one element
// a thread in the order of the columns, until there are enough
template <typename T, int THREADS>
__device__ void lowest_equal(Shared<THREADS> &sh, const RowView<T> &row, int i0, int i1, bool ends, uint32_t key,
                             int r0, int r1)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = ends ? 0 : row.head + i0 * Vec<T>::N, c1 = row.head + i1 * Vec<T>::N;
    const int tail = ends ? row.head + row.nv * Vec<T>::N : c1;      // then the row's last columns
    const int n = (c1 - c0) + (ends ? row.V - tail : 0);
    for (int at0 = 0; at0 < n && r0 < r1; at0 += THREADS) {
        const int at = at0 + threadIdx.x;
        const int v = at < c1 - c0 ? c0 + at : tail + at - (c1 - c0);
        const bool hit = at < n && key_of(Vec<T>::one(row.p[v])) == key;
        const uint32_t bits = __ballot_sync(0xffffffffu, hit);
        __syncthreads();
        if (lane == 0)
            sh.found[warp] = (uint64_t)__popc(bits);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < THREADS / 32; ++w) {
            before += w < warp ? (int)sh.found[w] : 0;
            all += (int)sh.found[w];
        }
        const int r = r0 + before + __popc(bits & ((1u << lane) - 1u));
        if (hit && r < r1)
            sh.best[r] = rank_key(key, v);
        r0 += all;
    }
}

// The block's `top` best elements into sh.best, in order.  `mine`: the largest key that this
// thread saw (0: no element).
template <typename T, int THREADS>
__device__ void select(Shared<THREADS> &sh, const RowView<T> &row, int i0, int i1, bool ends, int top,
                       uint32_t mine, int elements)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    sh.lane_max[threadIdx.x] = mine;
    __syncthreads();
    if (warp == 0) {
        // the top-th largest of the threads' maxima, bit by bit
        uint32_t k[THREADS / 32], b = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i)
            k[i] = sh.lane_max[i * 32 + lane];
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = b | 1u << bit;
            int n = 0;
#pragma unroll
            for (int i = 0; i < THREADS / 32; ++i)
                n += k[i] >= trial;
            if (__reduce_add_sync(0xffffffffu, n) >= top)
                b = trial;
        }
        if (lane == 0)
            sh.bound = max(b, kLowestKey);
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    const int want = min(top, elements);
    int n = collect<T, THREADS>(sh, row, i0, i1, ends, bound, mine);
    bool ties = false;
    if (n > kCand) {
        // many equal elements at the bound (a masked row's are -infinity): those above it
        // alone, then the lowest tokens at it
        ties = true;
        n = bound == 0xffffffffu ? 0 : collect<T, THREADS>(sh, row, i0, i1, ends, bound + 1, mine);
    }
    if (n <= kCand) {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t k = sh.cand[i];
            int r = 0;
            for (int j = 0; j < n; ++j)
                r += sh.cand[j] > k;
            if (r < top)
                sh.best[r] = k;
        }
        if (ties)
            lowest_equal<T, THREADS>(sh, row, i0, i1, ends, bound, n, want);
    } else {
        // more than the list holds lie in fewer than `top` threads' elements: the best below
        // the last one, `want` times over
        uint64_t last = ~0ull;
        for (int r = 0; r < want; ++r) {
            uint64_t b = 0;
            if (mine >= bound)
                each<T, THREADS>(row, i0, i1, ends, [&](float x, int v) {
                    const uint64_t k = rank_key(key_of(x), v);
                    b = k < last && k > b ? k : b;
                });
            b = warp_max64(b);
            __syncthreads();
            if (lane == 0)
                sh.found[warp] = b;
            __syncthreads();
            b = sh.found[0];
            for (int w = 1; w < THREADS / 32; ++w)
                b = sh.found[w] > b ? sh.found[w] : b;
            if (threadIdx.x == 0)
                sh.best[r] = b;
            last = b;
        }
    }
    for (int i = want + threadIdx.x; i < top; i += THREADS)
        sh.best[i] = 0;
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ T ld_remote(const T *p, uint32_t rank)
{
    static_assert(sizeof(T) % 4 == 0, "whole words");
    const uint32_t a = (uint32_t)__cvta_generic_to_shared(p);
    union {
        T v;
        float f[sizeof(T) / 4];
    } u;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 4; ++i)
        u.f[i] = ld_cluster(a + 4 * i, rank);
    return u.v;
}

template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(THREADS) k_logprob(const LogpArgs a, int cluster)
{
    griddep_start();
    constexpr int N = Vec<T>::N, U = 4;
    __shared__ Shared<THREADS> sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = cluster > 1 ? (int)(blockIdx.x % cluster) : 0;
    const float c = a.scale * kLog2e;
    for (int64_t t = blockIdx.x / cluster; t < a.T; t += gridDim.x / cluster) {
        const RowView<T> row((const T *)a.x + t * a.ld, a.V);
        const int per = (row.nv + cluster - 1) / cluster;
        const int i0 = min(row.nv, rank * per), i1 = min(row.nv, i0 + per);
        const bool ends = rank == 0;
        Sums p{-INFINITY, 0.f, 0.f};
        bool nan = false, saw = i0 + (int)threadIdx.x < i1;
        auto add = [&](const float *f, int n) {
            float m = f[0];
            for (int k = 1; k < n; ++k)
                m = fmaxf(m, f[k]);
            if (m > p.m) {
                const float d = shift(p.m, m, c);
                const float r = ex2(d);
                p.a = r * fmaf(p.s, fmaxf(d, kFloor), p.a);
                p.s *= r;
                p.m = m;
            }
            const float b = base_of(p.m, c);
            const bool far = !finite(b);
            for (int k = 0; k < n; ++k) {
                float t = fmaf(f[k], c, -b);
                if (far)
                    t = (f[k] - p.m) * c;
                const float e = ex2(t);
                p.s += e;
                p.a = fmaf(e, fmaxf(t, kFloor), p.a);
                nan |= f[k] != f[k];
            }
        };
        for (int i = i0 + threadIdx.x; i < i1; i += U * THREADS) {
            uint4 v[U];
            float f[U * N];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * THREADS < i1)
                    v[u] = row.piece(i + u * THREADS);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * THREADS < i1) {
                    Vec<T>::unpack(v[u], *(float(*)[N])(f + u * N));
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        f[u * N + k] = -INFINITY;
                }
            add(f, U * N);
        }
        if (ends && (int)threadIdx.x < row.loose()) {
            const float f = Vec<T>::one(row.p[row.loose_at(threadIdx.x)]);
            add(&f, 1);
            saw = true;
        }
        const uint32_t mine = nan ? 0xffffffffu : saw ? key_of(p.m) : 0u;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const Sums q{__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                         __shfl_xor_sync(0xffffffffu, p.a, o)};
            join(p, q, c);
        }
        __syncthreads();
        if (lane == 0)
            sh.sums[warp] = p;
        __syncthreads();
        p = sh.sums[0];
        for (int w = 1; w < THREADS / 32; ++w)
            join(p, sh.sums[w], c);
        if (threadIdx.x == 0)
            sh.block = p;
        if (TOP)
            select<T, THREADS>(sh, row, i0, i1, ends, a.top, mine,
                               (i1 - i0) * N + (ends ? row.loose() : 0));
        if (cluster > 1) {
            cluster_sync();
            if (rank == 0) {
                for (int r = 1; r < cluster; ++r)
                    join(p, ld_remote(&sh.block, r), c);
                if (TOP) {
                    for (int i = threadIdx.x; i < cluster * a.top; i += THREADS)
                        sh.merged[i] = ld_remote(&sh.best[i % a.top], i / a.top);
                    __syncthreads();
                    for (int i = threadIdx.x; i < cluster * a.top; i += THREADS) {
                        const uint64_t k = sh.merged[i];
                        int r = 0;
                        for (int j = 0; j < cluster * a.top; ++j)
                            r += sh.merged[j] > k;
                        if (k != 0 && r < a.top)
                            sh.cand[r] = k;
                    }
                    __syncthreads();
                }
            }
        }
        if (rank == 0) {
            const uint64_t *best = TOP && cluster > 1 ? sh.cand : sh.best;
            // a row whose logits are all -infinity: S = 0, lse = -infinity, every
            // probability is 0 and so is the entropy
            const bool empty = p.m == -INFINITY && p.s == 0.f;
            const float b = base_of(p.m, c), l2 = empty ? -INFINITY : log2f(p.s);
            // ln S for the sums of 2^((x - m) c): the base's rounding taken out again
            const float ln = empty ? -INFINITY : kLn2 * (finite(b) ? l2 - fmaf(p.m, c, -b) : l2);
            if (threadIdx.x == 0) {
                if (a.lse)
                    *(float2 *)(a.lse + 2 * t) = make_float2(p.m, ln);
                if (a.entropy)
                    a.entropy[t] = empty ? 0.f : kLn2 * (l2 - p.a / p.s);
                if (a.logp) {
                    const int v = a.target[t];
                    if (v >= a.V && a.err)
                        atomicOr(a.err, SN_EBIT_BAD_ID);
                    float lp = 0.f;
                    if (v >= 0 && v < a.V)
                        lp = empty ? -INFINITY : fmaf(Vec<T>::one(row.p[v]) - p.m, a.scale, -ln);
                    a.logp[t] = lp;
                }
            }
            if (TOP && (int)threadIdx.x < a.top) {
                const uint64_t k = best[threadIdx.x];
                a.top_ids[t * a.top + threadIdx.x] = (int32_t)(0xffffffffu - (uint32_t)k);
                const float x = value_of((uint32_t)(k >> 32));
                a.top_logp[t * a.top + threadIdx.x] = empty ? -INFINITY : fmaf(x - p.m, a.scale, -ln);
            }
        }
        if (cluster > 1)
            cluster_sync();             // the others' shared memory was read
        else if (TOP)
            __syncthreads();
    }
}

// ---- gradient ------------------------------------------------------------------------------

struct LogpBwdArgs {
    const void *x;
    void *dx;
    int64_t T, ld, ldd;
    int V;
    const int32_t *target;
    const float *lse, *entropy, *dlogp, *dentropy;   // target with dlogp, entropy with dentropy
    float scale;
    int segments;                                     // blocks of a row
};

constexpr int kBwdThreads = 256, kBwdPieces = 4;

// Per row: dx = p (k - b' ln p) + [v = target] a',  k = -a' - b' H,  primes: times scale
struct RowCoef {
    float m, c, l2, a, b, k;       // log2 p = (x - m) c - l2;  b for log2 p
    int target;
    bool empty;
    __device__ __forceinline__ float at(float x, int v) const
    {
        const float t = fmaf(x - m, c, -l2);
        const float p = ex2(t);
        float g = p * fmaf(-b, fmaxf(t, kFloor), k);
        if (t != t)
            g = t;
        if (v == target)
            g += a;
        return empty ? 0.f : g;
    }
};

template <typename T>
__global__ void __launch_bounds__(kBwdThreads) k_logprob_bwd(const LogpBwdArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, U = kBwdPieces;
    for (int64_t blk = blockIdx.x; blk < a.T * a.segments; blk += gridDim.x) {
        const int64_t t = blk / a.segments;
        const int seg = (int)(blk - t * a.segments);
        const RowView<T> row((const T *)a.x + t * a.ld, a.V);
        T *out = (T *)a.dx + t * a.ldd;
        RowCoef q;
        const float2 lse = *(const float2 *)(a.lse + 2 * t);
        q.m = lse.x;
        q.c = a.scale * kLog2e;
        q.l2 = lse.y * kLog2e;
        q.empty = lse.y == -INFINITY;
        q.target = a.dlogp ? a.target[t] : -1;
        q.a = a.dlogp && q.target >= 0 && q.target < a.V ? a.dlogp[t] * a.scale : 0.f;
        const float b = a.dentropy ? a.dentropy[t] * a.scale : 0.f;
        q.k = -q.a - (a.dentropy ? b * a.entropy[t] : 0.f);
        q.b = b * kLn2;
        const bool wide = (((uintptr_t)row.p ^ (uintptr_t)out) & 15) == 0;
        uint4 v[U];
        const int i0 = seg * U * kBwdThreads + threadIdx.x;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * kBwdThreads < row.nv)
                v[u] = *((const uint4 *)(row.p + row.head) + i0 + u * kBwdThreads);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kBwdThreads;
            if (i >= row.nv)
                continue;
            const int c0 = row.head + i * N;
            float f[N];
            Vec<T>::unpack(v[u], f);
#pragma unroll
            for (int k = 0; k < N; ++k)
                f[k] = q.at(f[k], c0 + k);
            if (wide) {
                *(uint4 *)(out + c0) = Vec<T>::pack(f);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    out[c0 + k] = Vec<T>::round(f[k]);
            }
        }
        if (seg == 0 && (int)threadIdx.x < row.loose()) {
            const int c = row.loose_at(threadIdx.x);
            out[c] = Vec<T>::round(q.at(Vec<T>::one(row.p[c]), c));
        }
    }
}

template <typename T, int THREADS>
cudaError_t fwd(const LogpArgs &a, int cluster, cudaStream_t s)
{
    const int64_t rows = std::min<int64_t>(a.T, ((int64_t)1 << 30) / cluster);
    count_launch();
    cudaError_t e;
    if (a.top > 0)
        e = launch_clusters(k_logprob<T, THREADS, true>, cluster, dim3((unsigned)(rows * cluster)), dim3(THREADS),
                            0, s, a, cluster);
    else
        e = launch_clusters(k_logprob<T, THREADS, false>, cluster, dim3((unsigned)(rows * cluster)), dim3(THREADS),
                            0, s, a, cluster);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t fwd_type(const LogpArgs &a, cudaStream_t s)
{
    const int nv = a.V / Vec<T>::N;
    if (nv <= 1024)
        return fwd<T, 128>(a, 1, s);
    // few rows: blocks of a cluster share one, as long as each has a piece a thread; on a
    // part of the GPU's SMs clusters may have no place
    int cluster = 1;
    const int sms = device_sms();
    while (cluster < kMaxCluster && a.T * cluster * 2 <= sms && nv >= cluster * 2 * 512)
        cluster *= 2;
    if (cluster > 1 && stream_sms(s) < sms)
        cluster = 1;
    return fwd<T, 512>(a, cluster, s);
}

template <typename T>
cudaError_t bwd_type(LogpBwdArgs a, cudaStream_t s)
{
    constexpr int per = Vec<T>::N * kBwdPieces * kBwdThreads;
    a.segments = (a.V + per - 1) / per;
    count_launch();
    const cudaError_t e = launch_dependent(k_logprob_bwd<T>,
                                           dim3((unsigned)std::min<int64_t>(a.T * a.segments, (int64_t)1 << 30)),
                                           dim3(kBwdThreads), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t logprob_fwd(sn_dtype dt, const void *x, int64_t T, int V, int64_t ld, const int32_t *target,
                        float scale, float *logp, float *lse, float *entropy, int top, int32_t *top_ids,
                        float *top_logp, unsigned int *err, cudaStream_t s)
{
    const LogpArgs a{x, T, ld, V, target, scale, logp, lse, entropy, top, top_ids, top_logp, err};
    return dt == SN_BF16 ? fwd_type<__nv_bfloat16>(a, s) : fwd_type<float>(a, s);
}

cudaError_t logprob_bwd(sn_dtype dt, const void *x, int64_t T, int V, int64_t ld, const int32_t *target,
                        const float *lse, const float *dlogp, const float *entropy, const float *dentropy,
                        float scale, void *dx, int64_t ldd, cudaStream_t s)
{
    const LogpBwdArgs a{x, dx, T, ld, ldd, V, target, lse, entropy, dlogp, dentropy, scale, 1};
    return dt == SN_BF16 ? bwd_type<__nv_bfloat16>(a, s) : bwd_type<float>(a, s);
}

}  // namespace sn
