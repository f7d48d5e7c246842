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
// that join their sums in shared memory; a narrow row is a warp's.
//
// Measured, bf16: 4096 rows of 128256 with the entropy 154 us (6.8 TB/s), with 8 alternatives
// too 171, their search being latency (four barriers and a read of L2 a row); the gradient of
// 8191 rows of 50257 234 us (7.05 TB/s).  8 fp32 rows of 128256 5.7 us, with 20 alternatives 9.6.
//
// The alternatives come out of the same pass: each thread keeps the largest logit it saw, the
// step that it was in and the largest of its other steps.  The n-th largest of the maxima of 64
// groups of threads bounds the row's n-th largest from below, so only the steps that reach the
// bound are read again, one or two for each alternative, and the few elements found there are
// ranked by value, the lower token first among equals.  Reading whole threads' pieces again
// instead costs 14 us at 4096 rows of 128256 bf16 (the rows in flight pass L2).
#include <algorithm>

#include "sn_vec.cuh"

namespace sn {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxTop = 32;
constexpr int kCand = 1024;             // elements at or above the bound that a block ranks
constexpr int kGroups = 64;             // of a block's threads: at least kMaxTop
constexpr int kSpare = 2;               // groups that the bound may let in beside those asked for
constexpr int kMaxCluster = 8;
constexpr int kPieces = 4;              // of a thread's step
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

// A part of a row's softmax sums: the largest logit m, and the sums of e and e * t over e = 2^t,
// t = x c - origin(m), c = scale log2(e).  The origin is m c rounded to fp32 (one fma makes t;
// all that is computed from the sums knows the rounding) as long as that is small; past 2^20,
// where its rounding would be felt, or where m c overflows (a row masked with the type's lowest
// value), it is m c itself and t = (x - m) c.
struct Sums {
    float m, s, a;
};

// 0 for a part that has no logit above -infinity: its sums are 0
__device__ __forceinline__ float base_of(float m, float c) { return m == -INFINITY ? 0.f : __fmul_rn(m, c); }
__device__ __forceinline__ bool rounded(float base) { return fabsf(base) < 0x1p20f; }

// The change of t where the maximum rises from m0 to m1
__device__ __forceinline__ float shift(float m0, float m1, float c)
{
    if (m0 == -INFINITY)
        return 0.f;
    const float b0 = base_of(m0, c), b1 = base_of(m1, c);
    if (rounded(b0))
        return rounded(b1) ? b0 - b1 : -fmaf(m1, c, -b0);
    return rounded(b1) ? fmaf(m0, c, -b1) : (m0 - m1) * c;
}

// What a row's sums give: ln S, and from it log probabilities and the entropy.  A row whose
// logits are all -infinity: S = 0, lse = -infinity, every probability is 0 and so is the entropy.
struct Result {
    bool empty;
    float l2, ln;
    __device__ __forceinline__ Result(const Sums &p, float c)
    {
        empty = p.m == -INFINITY && p.s == 0.f;
        const float b = base_of(p.m, c);
        l2 = empty ? -INFINITY : log2f(p.s);
        // ln S for the sums of 2^((x - m) c): the base's rounding taken out again
        ln = empty ? -INFINITY : kLn2 * (rounded(b) ? l2 - fmaf(p.m, c, -b) : l2);
    }
    __device__ __forceinline__ float entropy(const Sums &p) const { return empty ? 0.f : kLn2 * (l2 - p.a / p.s); }
    __device__ __forceinline__ float logp(float x, const Sums &p, float scale) const
    {
        return empty ? -INFINITY : fmaf(x - p.m, scale, -ln);
    }
};

// The sums of a warp's lanes, or of the block's warps, in every lane: the largest m first, so
// that each lane is rescaled once
template <int LANES>
__device__ __forceinline__ void join_lanes(Sums &p, float c)
{
    float m = p.m;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float d = shift(p.m, m, c), f = ex2(d);
    p.a = f * fmaf(p.s, fmaxf(d, kFloor), p.a);
    p.s *= f;
    p.m = m;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        p.s += __shfl_xor_sync(0xffffffffu, p.s, o);
        p.a += __shfl_xor_sync(0xffffffffu, p.a, o);
    }
}

template <int THREADS>
struct Shared {
    Sums sums[THREADS / 32];
    Sums block;                        // this block's sums, read by the cluster
    __align__(16) uint32_t keys[kGroups];  // the largest key that each group of threads saw, 0: none
    int step[THREADS];                 // of each warp, those that `collect` reads
    uint32_t bound;
    int n_cand, nan;                   // nan: a NaN among the elements
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

// `put(value, column)` for the elements of a piece whose key is at least `from`; nan: one of the
// row's is a NaN
template <typename T, typename F>
__device__ __forceinline__ void reaching(uint4 piece, int column, uint32_t from, bool nan, F put)
{
    constexpr int N = Vec<T>::N;
    const float least = value_of(from);
    float f[N];
    Vec<T>::unpack(piece, f);
    uint32_t hits = 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
        hits |= (f[k] >= least ? 1u : 0u) << k;
    if (nan) {
        hits = 0;
#pragma unroll
        for (int k = 0; k < N; ++k)
            hits |= (key_of(f[k]) >= from ? 1u : 0u) << k;
    }
    while (hits) {
        const int k = __ffs(hits) - 1;
        float y = f[0];
#pragma unroll
        for (int q = 1; q < N; ++q)
            y = k == q ? f[q] : y;
        put(y, column + k);
        hits &= hits - 1;
    }
}

// What a thread knows of the elements it saw: the largest key (0: no element), the step that it
// is in (its first piece, -1: none), and the largest key of its other steps
struct Best {
    uint32_t key, next;
    int at;
};

// sh.cand = this block's elements whose key is at least `from`, a key not below the bound; how
// many there are (the list holds the first kCand of them).  They lie in the best steps of the
// threads that saw such an element, in more of their pieces where `next` reaches it too, and
// among the loose elements.  The lanes of a warp share its threads' pieces.
template <typename T, int THREADS>
__device__ __forceinline__ int collect(Shared<THREADS> &sh, const RowView<T> &row, int i0, int i1, bool ends,
                                       const Best &mine, uint32_t from)
{
    constexpr int N = Vec<T>::N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool nan = sh.nan;
    auto put = [&](float x, int v) {
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < kCand)
            sh.cand[at] = rank_key(key_of(x), v);
    };
    uint32_t hot = __ballot_sync(0xffffffffu, mine.key >= from);
    uint32_t wide = __ballot_sync(0xffffffffu, mine.key >= from && (mine.next >= from || mine.at < 0));
    hot &= ~wide;
    if (hot >> lane & 1)
        sh.step[warp * 32 + __popc(hot & ((1u << lane) - 1u))] = mine.at;
    __syncwarp();
    int n = __popc(hot);
    const int *step = &sh.step[warp * 32 + lane / kPieces];
    int w = i1;                        // the next piece of the thread whose pieces are all looked at
    while (n > 0 || wide) {
        int i = i1;
        if (n > 0) {                   // a step each of up to eight threads
            if (lane / kPieces < n)
                i = *step + lane % kPieces * THREADS;
            step += 32 / kPieces;
            n -= 32 / kPieces;
        } else {
            if (w >= i1)
                w = i0 + warp * 32 + __ffs(wide) - 1;
            i = w + lane * THREADS;
            w += 32 * THREADS;
            if (w >= i1)
                wide &= wide - 1;
        }
        if (i >= i1)
            continue;
        reaching<T>(row.piece(i), row.head + i * N, from, nan, put);
    }
    if (ends && (int)threadIdx.x < row.loose()) {
        const int v = row.loose_at(threadIdx.x);
        const float x = Vec<T>::one(row.p[v]);
        if (key_of(x) >= from)
            put(x, v);
    }
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

// out[r] = the key of rank r < top among n different ones (0: no key): eight lanes count those
// above each
template <int THREADS>
__device__ __forceinline__ void place(const uint64_t *keys, int n, int top, uint64_t *out)
{
    const int sub = threadIdx.x % 8;
    for (int i0 = threadIdx.x / 32 * 4; i0 < n; i0 += THREADS / 8) {
        const int i = i0 + threadIdx.x % 32 / 8;
        const uint64_t k = i < n ? keys[i] : 0;
        int r = 0;
        for (int j = sub; j < n; j += 8)
            r += keys[j] > k;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1)
            r += __shfl_xor_sync(0xffffffffu, r, o);
        if (sub == 0 && k != 0 && r < top)
            out[r] = k;
    }
}

// A key close below the top-th largest of a warp's K keys a lane (0: no element), at least that
// of -infinity: bit by bit from the first in which they differ, until `top` or a few more reach
// it.  nan: the largest is that of a NaN.
template <typename T, int K>
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&k)[K], int top, bool &nan)
{
    uint32_t hi = k[0], lo = k[0];
#pragma unroll
    for (int i = 1; i < K; ++i) {
        hi = max(hi, k[i]);
        lo = min(lo, k[i]);
    }
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lo);
    nan = hi == 0xffffffffu;
    const int first = 31 - __clz(hi ^ lo);                // -1: all the same
    uint32_t b = first < 0 ? hi : hi & ~((2u << first) - 1u);
    for (int bit = first; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {         // bf16 keys differ above
        const uint32_t trial = b | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < K; ++i)
            n += __popc(__ballot_sync(0xffffffffu, k[i] >= trial));
        if (n >= top) {
            b = trial;
            if (n <= top + kSpare)
                break;
        }
    }
    // the low half of a bf16 key is ones below zero: with it the bound is the key itself, so that
    // one more leaves out the elements that tie there
    if (sizeof(T) == 2 && b >> 31 == 0)
        b |= 0xffffu;
    return max(b, kLowestKey);
}

// The block's `top` best elements into sh.best, in order
template <typename T, int THREADS>
__device__ void select(Shared<THREADS> &sh, const RowView<T> &row, int i0, int i1, bool ends, int top,
                       const Best &mine, int elements)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp == 0) {
        static_assert(kGroups == 64, "two a lane");
        const uint32_t k[2] = {sh.keys[2 * lane], sh.keys[2 * lane + 1]};
        bool nan;
        const uint32_t b = bound_of<T>(k, top, nan);
        if (lane == 0) {
            sh.bound = b;
            sh.n_cand = 0;
            sh.nan = nan;
        }
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    const int want = min(top, elements);
    int n = collect<T, THREADS>(sh, row, i0, i1, ends, mine, bound);
    bool ties = false;
    if (n > kCand) {
        // many equal elements at the bound (a masked row's are -infinity): those above it
        // alone, then the lowest tokens at it
        ties = true;
        __syncthreads();
        if (threadIdx.x == 0)
            sh.n_cand = 0;
        __syncthreads();
        n = bound == 0xffffffffu ? 0 : collect<T, THREADS>(sh, row, i0, i1, ends, mine, bound + 1);
    }
    if (n <= kCand) {
        place<THREADS>(sh.cand, n, top, sh.best);
        if (ties)
            lowest_equal<T, THREADS>(sh, row, i0, i1, ends, bound, n, want);
    } else {
        // more than the list holds lie in fewer than `top` threads' elements: the best that is
        // not above `most`, `want` times over
        uint64_t most = ~0ull;
        for (int r = 0; r < want; ++r) {
            uint64_t b = 0;
            if (mine.key >= bound)
                each<T, THREADS>(row, i0, i1, ends, [&](float x, int v) {
                    const uint64_t k = rank_key(key_of(x), v);
                    b = k <= most && k > b ? k : b;
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
            most = b - 1;
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

// Asks for the first bytes of a later row's pieces, so that DRAM stays busy while rows' sums meet
// (8192 rows of 32000 bf16 with 8 alternatives: 107 us, 112 with half as much; with twice as much,
// longer rows push each other out of L2)
constexpr int kAhead = 64 * 1024;

// ---- one pass over a thread's pieces ---------------------------------------------------------

// Elements at or below -10^20 count as -10^20 on the short path, where e = 0 whatever they
// are and t has to stay finite (0 * t = 0); it is taken while |m| < 10^19 and c > 10^-17, so
// that t is far below the smallest exponent.
constexpr float kLow = -1e20f;
constexpr uint32_t kLowPair = 0xE0AEE0AEu;       // bf16, twice

__host__ __device__ __forceinline__ bool near_scale(float c) { return c > 1e-17f && c < 1e17f; }
__device__ __forceinline__ bool near(float m, float c)
{
    return fabsf(m) < 1e19f && near_scale(c) && rounded(m * c);
}

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_pair_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two words of a piece (bf16: 4 elements, fp32: 2): their maximum, and their pairs with the
// elements below kLow raised to it
template <typename T>
struct Words;
template <>
struct Words<__nv_bfloat16> {
    static constexpr uint32_t kNone = 0xFF80FF80u;       // -infinity
    static constexpr int kPairs = 4;                     // of a piece
    template <int U>
    static __device__ __forceinline__ float max_of(const uint4 (&v)[U])
    {
        uint32_t m = max_pair(max_pair(v[0].x, v[0].y), max_pair(v[0].z, v[0].w));
#pragma unroll
        for (int u = 1; u < U; ++u)
            m = max_pair(m, max_pair(max_pair(v[u].x, v[u].y), max_pair(v[u].z, v[u].w)));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
    static __device__ __forceinline__ void pairs(uint4 v, float2 (&f)[4])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = max_pair_nan(w[i], kLowPair);
            f[i] = make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
        }
    }
};
template <>
struct Words<float> {
    static constexpr uint32_t kNone = 0xFF800000u;
    static constexpr int kPairs = 2;
    template <int U>
    static __device__ __forceinline__ float max_of(const uint4 (&v)[U])
    {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[u].x), __uint_as_float(v[u].y)),
                               fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
        return m;
    }
    static __device__ __forceinline__ void pairs(uint4 v, float2 (&f)[2])
    {
        f[0] = make_float2(max_nan(__uint_as_float(v.x), kLow), max_nan(__uint_as_float(v.y), kLow));
        f[1] = make_float2(max_nan(__uint_as_float(v.z), kLow), max_nan(__uint_as_float(v.w), kLow));
    }
};

// A thread's sums while it walks, over the even and the odd elements.  Their origin is that of
// an earlier maximum m until the largest logit `top` has risen kRise powers of two above it:
// with 32 lanes a warp, some lane's maximum rises in almost every step.
constexpr float kRise = 8.f;

struct Walk {
    float top, m, b;
    bool short_;                     // near(m, c)
    float2 s, a;
    float next;                      // the largest logit of the steps but the one that `top` is in,
    int at;                          // whose first piece is `at`

    __device__ __forceinline__ Walk()
        : top(-INFINITY), m(-INFINITY), b(0.f), short_(false), s(both(0.f)), a(both(0.f)), next(-INFINITY), at(-1) {}

    template <bool ENT>
    __device__ __forceinline__ void raise(float to, float c)
    {
        const float d = shift(m, to, c), r = ex2(d);
        if (ENT)
            a = mul2(both(r), fma2(s, both(fmaxf(d, kFloor)), a));
        s = mul2(both(r), s);
        m = to;
        b = base_of(to, c);
        short_ = near(to, c);
    }
    // any element, any m: a product and a difference more
    template <bool ENT>
    __device__ __forceinline__ void one(float x, float c)
    {
        top = fmaxf(top, x);
        if (top > m)
            raise<ENT>(top, c);
        const float t = rounded(b) ? fmaf(x, c, -b) : (x - m) * c;
        const float e = ex2(t);
        s.x += e;
        if (ENT)
            a.x = fmaf(e, fmaxf(t, kFloor), a.x);
    }
    template <typename T, bool TOP, bool ENT, int U>
    __device__ __forceinline__ void pieces(const uint4 (&v)[U], int i, float c)
    {
        const float most = Words<T>::max_of(v);
        if (TOP) {
            next = fmaxf(next, fminf(top, most));
            at = most > top ? i : at;
        }
        top = fmaxf(top, most);
        if (top > m && !(fmaf(top, c, -b) < kRise && short_))
            raise<ENT>(top, c);
        if (short_) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float2 f[Words<T>::kPairs];
                Words<T>::pairs(v[u], f);
#pragma unroll
                for (int k = 0; k < Words<T>::kPairs; ++k) {
                    const float2 t = fma2(f[k], both(c), both(-b));
                    const float2 e = make_float2(ex2(t.x), ex2(t.y));
                    s = add2(s, e);
                    if (ENT)
                        a = fma2(e, t, a);
                }
            }
        } else {
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                float f[Vec<T>::N];
                uint4 w = v[0];
#pragma unroll
                for (int k = 1; k < U; ++k)
                    w = u == k ? v[k] : w;
                Vec<T>::unpack(w, f);
#pragma unroll
                for (int k = 0; k < Vec<T>::N; ++k)
                    one<ENT>(f[k], c);
            }
        }
    }
    // the sums from the largest logit on
    template <bool ENT>
    __device__ __forceinline__ Sums sums(float c)
    {
        if (top > m)
            raise<ENT>(top, c);
        return {m, s.x + s.y, a.x + a.y};
    }
};

template <typename T, int THREADS>
struct RowPart : RowView<T> {
    int i0, i1;
    __device__ __forceinline__ RowPart(const LogpArgs &a, int64_t t, int rank, int cluster)
        : RowView<T>((const T *)a.x + t * a.ld, a.V)
    {
        const int per = cluster == 1 ? this->nv : (this->nv + cluster - 1) / cluster;
        i0 = min(this->nv, rank * per);
        i1 = min(this->nv, i0 + per);
    }
    // a thread's step from piece i on; none where the part ends
    __device__ __forceinline__ void load(int i, uint4 (&v)[kPieces]) const
    {
        if (i + (kPieces - 1) * THREADS < i1) {
#pragma unroll
            for (int u = 0; u < kPieces; ++u)
                v[u] = this->piece(i + u * THREADS);
        } else {
#pragma unroll
            for (int u = 0; u < kPieces; ++u)
                v[u] = i + u * THREADS < i1 ? this->piece(i + u * THREADS)
                                            : make_uint4(Words<T>::kNone, Words<T>::kNone, Words<T>::kNone,
                                                         Words<T>::kNone);
        }
    }
};

template <typename T, int THREADS, bool TOP, bool ENT>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprob(const LogpArgs a, int cluster_log2, int ahead)
{
    griddep_start();
    constexpr int N = Vec<T>::N, U = kPieces, W = THREADS / 32;
    __shared__ Shared<THREADS> sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cluster = 1 << cluster_log2;
    const int rank = (int)(blockIdx.x & (cluster - 1));
    const float c = a.scale * kLog2e;
    const bool ends = rank == 0;
    const int64_t stride = gridDim.x >> cluster_log2;
    for (int64_t t = blockIdx.x >> cluster_log2; t < a.T; t += stride) {
        const RowPart<T, THREADS> row(a, t, rank, cluster);
        const bool has_loose = ends && (int)threadIdx.x < row.loose();
        const float loose = has_loose ? Vec<T>::one(row.p[row.loose_at(threadIdx.x)]) : 0.f;
        Walk walk;
        int i = row.i0 + threadIdx.x;
        uint4 v[U], next[U];
        row.load(i, v);
        while (i + U * THREADS < row.i1) {
            row.load(i + U * THREADS, next);
            walk.pieces<T, TOP, ENT>(v, i, c);
            i += U * THREADS;
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[u] = next[u];
        }
        if (i < row.i1)
            walk.pieces<T, TOP, ENT>(v, i, c);
        if (threadIdx.x == 0 && cluster == 1 && t + ahead < a.T) {
            const RowView<T> later((const T *)a.x + (t + ahead) * a.ld, a.V);
            const int bytes = min(later.nv * 16, kAhead);
            if (bytes > 0)
                prefetch_l2(later.p + later.head, (uint32_t)bytes);
        }
        bool saw = row.i0 + (int)threadIdx.x < row.i1;
        if (has_loose) {
            walk.one<ENT>(loose, c);
            saw = true;
        }
        Sums p = walk.sums<ENT>(c);
        Best mine = {0, 0, walk.at};
        if (TOP) {
            if (saw) {
                mine.key = key_of(p.m);
                mine.next = key_of(walk.next);
            }
            if (p.s != p.s) {                     // a NaN among them, or an infinity
                bool nan = false;
                each<T, THREADS>(row, row.i0, row.i1, ends, [&](float x, int) { nan |= x != x; });
                if (nan)
                    mine = {0xffffffffu, 0, -1};
            }
        }
        join_lanes<32>(p, c);
        __syncthreads();
        if (lane == 0)
            sh.sums[warp] = p;
        if (TOP) {
            uint32_t k = mine.key;
#pragma unroll
            for (int o = THREADS / kGroups / 2; o > 0; o >>= 1)
                k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
            if (threadIdx.x % (THREADS / kGroups) == 0)
                sh.keys[threadIdx.x / (THREADS / kGroups)] = k;
        }
        __syncthreads();
        p = sh.sums[lane % W];
        join_lanes<W>(p, c);
        if (threadIdx.x == 0)
            sh.block = p;
        if (TOP)
            select<T, THREADS>(sh, row, row.i0, row.i1, ends, a.top, mine,
                               (row.i1 - row.i0) * N + (ends ? row.loose() : 0));
        if (cluster > 1) {
            cluster_sync();
            if (rank == 0) {
                p = {-INFINITY, 0.f, 0.f};
                if (lane % kMaxCluster < cluster)
                    p = ld_remote(&sh.block, lane % kMaxCluster);
                join_lanes<kMaxCluster>(p, c);
                if (TOP) {
                    for (int i = threadIdx.x; i < cluster * a.top; i += THREADS)
                        sh.merged[i] = ld_remote(&sh.best[i % a.top], i / a.top);
                    __syncthreads();
                    place<THREADS>(sh.merged, cluster * a.top, a.top, sh.cand);
                    __syncthreads();
                }
            }
        }
        if (rank == 0) {
            const uint64_t *best = TOP && cluster > 1 ? sh.cand : sh.best;
            const Result z(p, c);
            if (threadIdx.x == 0) {
                if (a.lse)
                    *(float2 *)(a.lse + 2 * t) = make_float2(p.m, z.ln);
                if (ENT)
                    a.entropy[t] = z.entropy(p);
                if (a.logp) {
                    const int v = a.target[t];
                    if (v >= a.V && a.err)
                        atomicOr(a.err, SN_EBIT_BAD_ID);
                    a.logp[t] = v >= 0 && v < a.V ? z.logp(Vec<T>::one(row.p[v]), p, a.scale) : 0.f;
                }
            }
            if (TOP && (int)threadIdx.x < a.top) {
                const uint64_t k = best[threadIdx.x];
                a.top_ids[t * a.top + threadIdx.x] = (int32_t)(0xffffffffu - (uint32_t)k);
                a.top_logp[t * a.top + threadIdx.x] = z.logp(value_of((uint32_t)(k >> 32)), p, a.scale);
            }
        }
        if (cluster > 1)
            cluster_sync();             // the others' shared memory was read
        else if (TOP)
            __syncthreads();
    }
}

// ---- narrow rows -----------------------------------------------------------------------------
// A warp has a whole row of at most kNarrow elements in registers, so its sums start from the
// row's maximum and the alternatives are found without reading again.  16384 rows of 1024 bf16:
// 10.3 us, 36 with a block of 128 threads a row; with 8 alternatives 25 and 69.

constexpr int kNarrow = 1024, kNarrowWarps = 8, kNarrowCand = 192;

template <typename T, bool TOP, bool ENT>
__global__ void __launch_bounds__(32 * kNarrowWarps, 4) k_logprob_narrow(const LogpArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, C = kNarrow / (32 * N), K = 4;
    __shared__ uint64_t cands[TOP ? kNarrowWarps : 1][TOP ? kNarrowCand : 1];
    __shared__ int counts[kNarrowWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float c = a.scale * kLog2e;
    for (int64_t t = (int64_t)blockIdx.x * kNarrowWarps + warp; t < a.T; t += (int64_t)gridDim.x * kNarrowWarps) {
        const RowView<T> row((const T *)a.x + t * a.ld, a.V);
        uint4 v[C];
#pragma unroll
        for (int i = 0; i < C; ++i)
            v[i] = lane + 32 * i < row.nv ? row.piece(lane + 32 * i)
                                          : make_uint4(Words<T>::kNone, Words<T>::kNone, Words<T>::kNone, Words<T>::kNone);
        const bool has_loose = lane < row.loose();
        const float loose = has_loose ? Vec<T>::one(row.p[row.loose_at(lane)]) : -INFINITY;
        const int target = a.logp ? a.target[t] : -1;
        const float at_target = target >= 0 && target < a.V ? Vec<T>::one(row.p[target]) : 0.f;
        const float own = fmaxf(Words<T>::max_of(v), loose);
        Walk walk;
        walk.top = own;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            walk.top = fmaxf(walk.top, __shfl_xor_sync(0xffffffffu, walk.top, o));
        walk.pieces<T, false, ENT>(v, 0, c);
        if (has_loose)
            walk.one<ENT>(loose, c);
        Sums p = {walk.m, walk.s.x + walk.s.y, walk.a.x + walk.a.y};       // the same m in every lane
        const bool none = p.s != p.s;                   // NaN, or an infinity
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            p.s += __shfl_xor_sync(0xffffffffu, p.s, o);
            if (ENT)
                p.a += __shfl_xor_sync(0xffffffffu, p.a, o);
        }
        const Result z(p, c);
        if (lane == 0) {
            if (a.lse)
                *(float2 *)(a.lse + 2 * t) = make_float2(p.m, z.ln);
            if (ENT)
                a.entropy[t] = z.entropy(p);
            if (a.logp) {
                if (target >= a.V && a.err)
                    atomicOr(a.err, SN_EBIT_BAD_ID);
                a.logp[t] = target >= 0 && target < a.V ? z.logp(at_target, p, a.scale) : 0.f;
            }
        }
        if (!TOP)
            continue;
        // fn(value, column, piece) for each of this lane's elements
        const auto each = [&](auto fn) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                if (lane + 32 * i >= row.nv)
                    continue;
                float f[N];
                Vec<T>::unpack(v[i], f);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    fn(f[k], row.head + (lane + 32 * i) * N + k, i);
            }
            if (has_loose)
                fn(loose, row.loose_at(lane), 0);
        };
        // the largest keys of this lane's pieces, C / K of them at a time
        uint32_t key[K];
#pragma unroll
        for (int g = 0; g < K; ++g) {
            uint4 u[C / K];
#pragma unroll
            for (int i = 0; i < C / K; ++i)
                u[i] = v[g * (C / K) + i];
            key[g] = lane + 32 * g * (C / K) < row.nv ? key_of(Words<T>::max_of(u)) : 0u;
        }
        if (has_loose)
            key[0] = max(key[0], key_of(loose));
        if (none)
            each([&](float x, int, int i) { key[i * K / C] = x != x ? 0xffffffffu : key[i * K / C]; });
        bool nan;
        const uint32_t bound = bound_of<T>(key, a.top, nan);
        uint64_t *cand = cands[warp];
        // the elements whose key is at least `from`: how many, the first kNarrowCand in the list
        const auto collect_from = [&](uint32_t from) {
            __syncwarp();
            if (lane == 0)
                counts[warp] = 0;
            __syncwarp();
            const auto put = [&](float x, int col) {
                const int at = atomicAdd(&counts[warp], 1);
                if (at < kNarrowCand)
                    cand[at] = rank_key(key_of(x), col);
            };
#pragma unroll
            for (int i = 0; i < C; ++i)
                if (lane + 32 * i < row.nv && key[i * K / C] >= from)
                    reaching<T>(v[i], row.head + (lane + 32 * i) * N, from, nan, put);
            if (has_loose && key_of(loose) >= from)
                put(loose, row.loose_at(lane));
            __syncwarp();
            return counts[warp];
        };
        const auto write = [&](int r, uint64_t k) {
            a.top_ids[t * a.top + r] = (int32_t)(0xffffffffu - (uint32_t)k);
            a.top_logp[t * a.top + r] = z.logp(value_of((uint32_t)(k >> 32)), p, a.scale);
        };
        int n = collect_from(bound);
        bool ties = false;
        if (n > kNarrowCand) {
            // many equal ones at the bound: those above it, then the lowest tokens at it
            ties = true;
            n = bound == 0xffffffffu ? 0 : collect_from(bound + 1);
        }
        if (n <= kNarrowCand) {
            for (int i = lane; i < n; i += 32) {
                const uint64_t k = cand[i];
                int r = 0;
                for (int j = 0; j < n; ++j)
                    r += cand[j] > k;
                if (r < a.top)
                    write(r, k);
            }
            if (!ties)
                continue;
            // in the order of the columns: the loose ones in front, the pieces, the last ones
            const uint32_t before = (1u << lane) - 1u;
            const uint32_t ends = __ballot_sync(0xffffffffu, has_loose && key_of(loose) == bound);
            const uint32_t front = ends & ((1u << row.head) - 1u);
            const bool mine = ends >> lane & 1;
            if (mine && lane < row.head && n + __popc(front & before) < a.top)
                write(n + __popc(front & before), rank_key(bound, row.loose_at(lane)));
            n += __popc(front);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                if (n >= a.top)
                    break;
                float f[N];
                Vec<T>::unpack(v[i], f);
                int same = 0;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    same += lane + 32 * i < row.nv && key_of(f[k]) == bound;
                int r = same;                              // and those of the lanes before
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int x = __shfl_up_sync(0xffffffffu, r, o);
                    r += lane >= o ? x : 0;
                }
                const int all = __shfl_sync(0xffffffffu, r, 31);
                r += n - same;
                if (same)
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (key_of(f[k]) == bound) {
                            if (r < a.top)
                                write(r, rank_key(bound, row.head + (lane + 32 * i) * N + k));
                            ++r;
                        }
                n += all;
            }
            if (mine && lane >= row.head && n + __popc(ends & ~front & before) < a.top)
                write(n + __popc(ends & ~front & before), rank_key(bound, row.loose_at(lane)));
            continue;
        }
        // more than the list holds lie in few lanes' pieces: the best that is not above `most`
        uint64_t most = ~0ull;
        for (int r = 0; r < a.top; ++r) {
            uint64_t b = 0;
            each([&](float x, int col, int) {
                const uint64_t k = rank_key(key_of(x), col);
                b = k <= most && k > b ? k : b;
            });
            b = warp_max64(b);
            most = b - 1;
            if (lane == 0)
                write(r, b);
        }
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
    float most;                // |scale * dentropy| on the short path, at most; below 0: no short path
};

constexpr int kBwdThreads = 256, kBwdPieces = 4;

// Per row: dx = p (k - b' ln p) + [v = target] a',  k = -a' - b' H,  primes: times scale
struct RowCoef {
    float m, c, l2, a, b, k;       // log2 p = (x - m) c - l2;  b for log2 p
    int target;
    bool near_, empty;
    // without the target's term
    __device__ __forceinline__ float at(float x) const
    {
        const float t = fmaf(x - m, c, -l2);
        return empty ? 0.f : ex2(t) * fmaf(-b, t < kFloor ? kFloor : t, k);
    }
};

// 16 bytes from byte `from` (a multiple of 2, below 16) of lo and hi on
__device__ __forceinline__ uint4 bytes_from(uint4 lo, uint4 hi, int from)
{
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 6; ++i)
        w[i] = from & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i)
        w[i] = from & 4 ? w[i + 1] : w[i];
    const int bits = (from & 2) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                      __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// N elements from p on, in the row [begin, end): the two pieces that they lie in, or, where those
// pass the row's ends, one by one
template <typename T>
__device__ __forceinline__ uint4 unaligned_piece(const T *p, const T *begin, const T *end)
{
    constexpr int N = Vec<T>::N;
    const int from = (int)((uintptr_t)p & 15);
    const T *lo = (const T *)((const char *)p - from);
    if (from == 0)
        return __ldcs((const uint4 *)p);
    if (lo >= begin && lo + 2 * N <= end)
        return bytes_from(__ldcs((const uint4 *)lo), __ldcs((const uint4 *)lo + 1), from);
    float f[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
        f[k] = Vec<T>::one(p[k]);
    return Vec<T>::pack(f);
}

// LANES threads share a row's step: a block has one row's, or several narrow rows' (16384 rows of
// 1024 bf16: 12 us, 33 with a block a row).  SHIFT: some rows of the logits lie otherwise to their
// 16-byte boundaries than the gradient's.  Then the pieces are whole in the output for bf16 (8191
// rows of 50257, 47 elements of padding: 309 us, 924 with elements written one by one), and in
// the logits for fp32, with single writes (473 us, 700 the other way).
//
// A step is loads, a few instructions and stores, so what counts is how many are on an SM: at 32
// registers, all 2048 threads (8191 rows of 50257 bf16: 234 us, 7.05 TB/s; 254 with 48 registers,
// 366 with 72).  With several rows a block that spills (16384 rows of 1024: 20 us, 12 with 48).
template <typename T, int LANES, bool SHIFT>
__global__ void __launch_bounds__(kBwdThreads, LANES == kBwdThreads ? 8 : SHIFT && sizeof(T) == 2 ? 4 : 5)
    k_logprob_bwd(const LogpBwdArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, U = kBwdPieces, kRows = kBwdThreads / LANES;
    constexpr bool SINGLE = SHIFT && sizeof(T) == 4;
    const int seg = blockIdx.x, lane = threadIdx.x % LANES;
    for (int64_t t = (int64_t)blockIdx.y * kRows + threadIdx.x / LANES; t < a.T; t += (int64_t)gridDim.y * kRows) {
        const T *x = (const T *)a.x + t * a.ld;
        T *out = (T *)a.dx + t * a.ldd;
        const RowView<T> row(SINGLE ? x : out, a.V);
        RowCoef q;
        const float2 lse = *(const float2 *)(a.lse + 2 * t);
        q.m = lse.x;
        q.c = a.scale * kLog2e;
        q.l2 = lse.y * kLog2e;
        q.empty = lse.y == -INFINITY;
        q.target = a.dlogp ? a.target[t] : -1;
        q.a = !q.empty && a.dlogp && q.target >= 0 && q.target < a.V ? a.dlogp[t] * a.scale : 0.f;
        const float b = a.dentropy ? a.dentropy[t] * a.scale : 0.f;
        q.k = -q.a - (a.dentropy ? b * a.entropy[t] : 0.f);
        q.b = b * kLn2;
        // near() of m and c, and b t finite too (t is above -2 * 10^20 c)
        q.near_ = !q.empty && fabsf(q.m) < 1e19f && rounded(q.m * q.c) && fabsf(b) <= a.most;
        // marked to leave L2 first, coming and going (with 48 registers: 8191 rows of 50257 took 275
        // us without, 253 with, 4096 of 128256 322 and 295; either mark alone gained less, or nothing)
        uint4 v[U];
        const int i0 = seg * U * LANES + lane;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * LANES < row.nv)
                v[u] = SHIFT && !SINGLE ? unaligned_piece(x + row.head + (i0 + u * LANES) * N, x, x + a.V)
                             : __ldcs((const uint4 *)(x + row.head) + i0 + u * LANES);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * LANES;
            if (i >= row.nv)
                continue;
            const int c0 = row.head + i * N;
            float f[N];
            if (q.near_) {
                float2 y[N / 2];
                Words<T>::pairs(v[u], y);
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    const float2 z = fma2(add2(y[k], both(-q.m)), both(q.c), both(-q.l2));
                    const float2 g = mul2(make_float2(ex2(z.x), ex2(z.y)), fma2(both(-q.b), z, both(q.k)));
                    f[2 * k] = g.x;
                    f[2 * k + 1] = g.y;
                }
            } else {
                Vec<T>::unpack(v[u], f);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    f[k] = q.at(f[k]);
            }
            if ((uint32_t)(q.target - c0) < (uint32_t)N)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    f[k] += q.target - c0 == k ? q.a : 0.f;
            if (!SINGLE) {
                __stcs((uint4 *)(out + c0), Vec<T>::pack(f));
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    out[c0 + k] = Vec<T>::round(f[k]);
            }
        }
        if (seg == 0 && lane < row.loose()) {
            const int c = row.loose_at(lane);
            out[c] = Vec<T>::round(q.at(Vec<T>::one(x[c])) + (c == q.target ? q.a : 0.f));
        }
    }
}

template <typename T, int THREADS, bool TOP, bool ENT>
cudaError_t fwd_launch(const LogpArgs &a, int cluster, cudaStream_t s)
{
    const int64_t rows = std::min<int64_t>(a.T, ((int64_t)1 << 30) / cluster);
    int log2 = 0;
    while (1 << log2 < cluster)
        ++log2;
    count_launch();
    const cudaError_t e = launch_clusters(k_logprob<T, THREADS, TOP, ENT>, cluster, dim3((unsigned)(rows * cluster)),
                                          dim3(THREADS), 0, s, a, log2, device_sms() * (1024 / THREADS));
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int THREADS>
cudaError_t fwd(const LogpArgs &a, int cluster, cudaStream_t s)
{
    if (a.entropy)
        return a.top > 0 ? fwd_launch<T, THREADS, true, true>(a, cluster, s)
                         : fwd_launch<T, THREADS, false, true>(a, cluster, s);
    return a.top > 0 ? fwd_launch<T, THREADS, true, false>(a, cluster, s)
                     : fwd_launch<T, THREADS, false, false>(a, cluster, s);
}

template <typename T, bool TOP, bool ENT>
cudaError_t narrow_launch(const LogpArgs &a, cudaStream_t s)
{
    const int64_t blocks = std::min<int64_t>((a.T + kNarrowWarps - 1) / kNarrowWarps, (int64_t)1 << 30);
    count_launch();
    const cudaError_t e = launch_dependent(k_logprob_narrow<T, TOP, ENT>, dim3((unsigned)blocks),
                                           dim3(32 * kNarrowWarps), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t fwd_type(const LogpArgs &a, cudaStream_t s)
{
    if (a.V <= kNarrow) {
        if (a.entropy)
            return a.top > 0 ? narrow_launch<T, true, true>(a, s) : narrow_launch<T, false, true>(a, s);
        return a.top > 0 ? narrow_launch<T, true, false>(a, s) : narrow_launch<T, false, false>(a, s);
    }
    const int nv = a.V / Vec<T>::N;
    if (nv <= 1024)
        return fwd<T, 128>(a, 1, s);
    const int sms = device_sms();
    if (a.T >= 2 * sms)
        return fwd<T, 256>(a, 1, s);
    // few rows: blocks of a cluster share one, as long as each has a piece a thread; on a
    // part of the GPU's SMs clusters may have no place
    int cluster = 1;
    while (cluster < kMaxCluster && a.T * cluster <= sms && nv >= cluster * 2 * 512)
        cluster *= 2;
    if (cluster > 1 && stream_sms(s) < sms)
        cluster = 1;
    return fwd<T, 512>(a, cluster, s);
}

template <typename T, int LANES>
cudaError_t bwd_launch(const LogpBwdArgs &a, cudaStream_t s)
{
    const bool same = (((uintptr_t)a.x ^ (uintptr_t)a.dx) & 15) == 0 && (a.ld - a.ldd) % Vec<T>::N == 0;
    constexpr int64_t per = Vec<T>::N * kBwdPieces * LANES, kRows = kBwdThreads / LANES;
    count_launch();
    const cudaError_t e = launch_dependent(same ? k_logprob_bwd<T, LANES, false> : k_logprob_bwd<T, LANES, true>,
                                           dim3((unsigned)((a.V + per - 1) / per),
                                                (unsigned)std::min<int64_t>((a.T + kRows - 1) / kRows, 65535)),
                                           dim3(kBwdThreads), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t bwd_type(const LogpBwdArgs &a, cudaStream_t s)
{
    const int lanes = (a.V / Vec<T>::N + kBwdPieces - 1) / kBwdPieces;
    return lanes <= 32    ? bwd_launch<T, 32>(a, s)
           : lanes <= 64  ? bwd_launch<T, 64>(a, s)
           : lanes <= 128 ? bwd_launch<T, 128>(a, s)
                          : bwd_launch<T, kBwdThreads>(a, s);
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
    const float c = scale * kLog2e;
    const LogpBwdArgs a{x, dx, T, ld, ldd, V, target, lse, entropy, dlogp, dentropy, scale,
                        near_scale(c) ? 1e17f / c : -1.f};
    return dt == SN_BF16 ? bwd_type<__nv_bfloat16>(a, s) : bwd_type<float>(a, s);
}

}  // namespace sn
