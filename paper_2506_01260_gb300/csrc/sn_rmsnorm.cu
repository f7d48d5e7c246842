// sn_rmsnorm.cu — root-mean-square norm of a residual stream, with the residual's addition
// in front, an 8-bit output behind, and the gradient.
//
//   h = x + r,  rs = 1 / sqrt(mean(h^2) + eps),  y = h rs w
//   8-bit: a = max |y| over a row or a group of its columns, scale = a / qmax,
//          code = Q(y qmax / a)
//   gradient, from the stored h:  g = dy w,  c = mean(g h) rs^2,
//          dx = rs (g - h c) + dh,   dw = sum over the rows of dy h rs
//
// Bound by DRAM: every element of a row is read once and stays in registers as a 16-byte
// piece until it is written (`Shape` below gives the lanes of a width).  Sums are
// fp32 in every type; y is computed from the unrounded h and rounded once, the stored h once.
//
// Measured: 16384 bf16 rows of 4096 with a residual 79 us (6.8 TB/s), their gradient 82 us (6.6
// TB/s, the sum of dw's parts in it); e4m3 codes of 65536 bf16 rows of 8192 with a scale per 128
// columns 522 us (7.2 TB/s); the gradient of 4173 fp32 rows of 2056 26 us (5.3 TB/s), where the
// 14 rows a block walks and the sum of dw's parts cost latency.
#include <algorithm>
#include <type_traits>

#include <cuda_fp8.h>

#include "sn_norm.cuh"

namespace sn {
namespace {

struct NormArgs {
    const void *X, *R;      // R: null without a residual
    void *H;                // null: h is not stored
    const void *w;
    bool w_bf16;
    int64_t T, ldx;
    int d;
    float eps;
    void *Y;
    uint8_t *codes;
    float *scale;
    int group_log2;         // columns that share a scale: 2^group_log2; 0: the row
    float least, most;      // of a row's sum of squares that is taken as it is
    int ahead;              // rows that are in flight on the GPU at once; 0: no prefetch
};

// The smallest magnitude that a group's scale is made for: its reciprocal stays finite.
constexpr float kTiny = 0x1p-100f;

template <int FMT>
__device__ __forceinline__ float qmax_of() { return FMT == SN_Q_INT8 ? 127.f : 448.f; }

template <int FMT>
__device__ __forceinline__ float scale_of(float a)
{
    return (a > 0.f && a < kTiny ? kTiny : a) / qmax_of<FMT>();
}
template <int FMT>
__device__ __forceinline__ float reciprocal_of(float a)
{
    return a == 0.f ? 0.f : qmax_of<FMT>() / (a < kTiny ? kTiny : a);
}

// Four codes of y * rec, the first in the lowest byte: int8 rounds half to even (adding
// 1.5 * 2^23 leaves the rounded value in the low byte; |y * rec| <= 127 (1 + 2^-22)), e4m3
// rounds to nearest even and saturates.  What a NaN or an infinity gives does not matter: its
// scale is none.
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(float2 y0, float2 y1, float rec)
{
    const float2 x0 = mul2(y0, both(rec)), x1 = mul2(y1, both(rec));
    if (FMT == SN_Q_INT8) {
        const float2 q0 = add2(x0, both(12582912.f)), q1 = add2(x1, both(12582912.f));
        return __byte_perm(__byte_perm(__float_as_uint(q0.x), __float_as_uint(q0.y), 0x0040),
                           __byte_perm(__float_as_uint(q1.x), __float_as_uint(q1.y), 0x0040), 0x5410);
    }
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(x0, __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(x1, __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
template <int FMT>
__device__ __forceinline__ uint8_t code_of(float y, float rec)
{
    return (uint8_t)codes_of<FMT>(make_float2(y, 0.f), both(0.f), rec);
}

// A scaled row's dx, of y w, n, mean(g n), 1 / rms(h f) and f: the factor's root on either side of the
// reciprocal root, so that nothing on the way is smaller or larger than fp32 holds where dx is not
__device__ __forceinline__ float scaled_dx(float g, float n, float m, float rs, float f, float r)
{
    const float half = f > 1.f ? 0x1p50f : 0x1p-40f;
    return fmaf(fmaf(-n, m, g) * half * rs, half, r);
}

// ---- forward, rows in registers ------------------------------------------------------------

__device__ __forceinline__ float max_magnitude(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}

// The largest magnitude of a piece, a NaN if it holds one
template <int P>
__device__ __forceinline__ float magnitude(const float2 (&f)[P])
{
    float m = 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k)
        m = max_magnitude(m, f[k].x, f[k].y);
    return m;
}

// The maximum over 2^n neighbouring lanes (`lanes` of them, >= 4) of each of C values: lane i
// gets that of value i mod 4.  Two halvings, then one value a lane: 5 shuffles for 4 values of
// 16 lanes, not 16 (65536 rows of 8192 with 128 columns a scale: 576 us, 652).
template <int C>
__device__ __forceinline__ float max_of_lanes(const float (&v)[C], int lane, int lanes)
{
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = i < C ? v[i < C ? i : 0] : 0.f;
    const bool odd = lane & 1, high = lane & 2;
#pragma unroll
    for (int i = 0; i < 4; i += 2)
        if (i < C)
            x[i] = max_nan(odd ? x[i + 1] : x[i], __shfl_xor_sync(0xffffffffu, odd ? x[i] : x[i + 1], 1));
    float m = max_nan(high ? x[2] : x[0], __shfl_xor_sync(0xffffffffu, high ? x[0] : x[2], 2));
#pragma unroll
    for (int o = 4; o < 32; o *= 2)
        if (o < lanes)
            m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// A row by single elements, from memory.  SCALED: as h f; otherwise f is 1, and where the sum of
// squares is not in range nothing is written.  Returns that sum.
template <typename T, int S, bool EXACT, int FMT, bool SCALED>
__device__ float norm_singly(const NormArgs &a, int64_t t, float f, float *red, int &turn)
{
    const int d = a.d, G = Shape<S, EXACT>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const T *x = (const T *)a.X + t * a.ldx;
    const T *r = a.R ? (const T *)a.R + t * d : nullptr;
    T *H = a.H ? (T *)a.H + t * d : nullptr;
    auto h_at = [&](int j) { return Vec<T>::one(x[j]) + (r ? Vec<T>::one(r[j]) : 0.f); };
    float s[1] = {0.f};
#pragma unroll SCALED ? 1 : 4
    for (int j = lane; j < d; j += G) {
        const float h = SCALED ? h_at(j) * f : h_at(j);
        s[0] = fmaf(h, h, s[0]);
    }
    row_reduce<S, 1, false, EXACT>(s, red, turn);
    if (!SCALED && !in_range(a, s[0]))
        return s[0];
    const float mean = s[0] / (float)d + (SCALED ? a.eps * f * f : a.eps);
    const float rs = SCALED ? root_of(mean) : rsqrtf(mean);
    auto y_of = [&](float h, int j) { return (SCALED ? h * f : h) * rs * weight_at(a, j); };
    constexpr int F = FMT < 0 ? 0 : FMT;
    if (FMT < 0) {
#pragma unroll SCALED ? 1 : 4
        for (int j = lane; j < d; j += G) {
            const float h = h_at(j);
            if (H)
                H[j] = Vec<T>::round(h);
            ((T *)a.Y)[t * d + j] = Vec<T>::round(y_of(h, j));
        }
    } else if (a.group_log2 == 0) {
        float m[1] = {0.f};
#pragma unroll SCALED ? 1 : 4
        for (int j = lane; j < d; j += G)
            m[0] = max_nan(m[0], fabsf(y_of(h_at(j), j)));
        row_reduce<S, 1, true, EXACT>(m, red, turn);
        const float rec = reciprocal_of<F>(m[0]);
        if (lane == 0)
            a.scale[t] = scale_of<F>(m[0]);
#pragma unroll SCALED ? 1 : 4
        for (int j = lane; j < d; j += G) {
            const float h = h_at(j);
            a.codes[t * d + j] = code_of<F>(y_of(h, j), rec);
            if (H)
                H[j] = Vec<T>::round(h);
        }
    } else {
        // a warp takes whole groups
        const int group = 1 << a.group_log2, groups = (d + group - 1) / group;
#pragma unroll SCALED ? 1 : 4
        for (int g = lane / 32; g < groups; g += G / 32) {
            const int j0 = g * group, j1 = min(d, j0 + group);
            float m = 0.f;
#pragma unroll SCALED ? 1 : 4
            for (int j = j0 + lane % 32; j < j1; j += 32)
                m = max_nan(m, fabsf(y_of(h_at(j), j)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float rec = reciprocal_of<F>(m);
            if (lane % 32 == 0)
                a.scale[t * groups + g] = scale_of<F>(m);
#pragma unroll SCALED ? 1 : 4
            for (int j = j0 + lane % 32; j < j1; j += 32) {
                const float h = h_at(j);
                a.codes[t * d + j] = code_of<F>(y_of(h, j), rec);
                if (H)
                    H[j] = Vec<T>::round(h);
            }
        }
    }
    return s[0];
}

// Threads of an SM that registers are kept low enough for.  With a residual, codes from bf16 rows
// take up to 115 registers at 4 pieces a lane and are left them (at most 80, for 768 threads:
// 16384 rows of 4096 with bounds 95 us, 73 without that cap).  Blocks of 512 are two an SM (8192
// rows of 16384 bf16: 143 us, 230 with one block).  Without a residual (RES) a thread has half the
// loads in flight and fewer registers, so more threads pay: 16384 rows of 8192 bf16 take 85 us, 95
// with as many as with one.  Rows of one piece fit 32 registers, all of an SM's threads (65536 rows
// of 256 bf16 with a residual: 21.2 us, 22.5 with 1536).
template <typename T, int S, int C, int FMT, bool RES>
constexpr int kResident = S > 512    ? S
                          : S == 512 ? 1024
                          : C == 1   ? (FMT < 0 ? 2048 : 1536)
                          : C == 2   ? (RES || FMT >= 0 ? 1024 : 1536)
                          : RES      ? (FMT < 0 || sizeof(T) == 4 ? 768 : 512)
                                     : (sizeof(T) == 4 ? 1280 : FMT < 0 ? 1024 : 768);

template <typename T, int S, bool EXACT, int C, int FMT, bool RES>
__global__ void __launch_bounds__(Shape<S>::kThreads, kResident<T, S, C, FMT, RES> / Shape<S>::kThreads)
    k_rmsnorm(const NormArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, P = N / 2, kRows = Shape<S>::kRows;
    __shared__ __align__(16) float red[2 * 32];
    int turn = 0;
    const int G = Shape<S, EXACT>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const int nv = EXACT ? S * C : a.d / N;
    const T *X = (const T *)a.X, *R = RES ? (const T *)a.R : nullptr;
    T *H = (T *)a.H, *Y = (T *)a.Y;
    for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
        const int64_t t = t0 + (S == 32 ? threadIdx.x / 32 : 0);
        const bool live = S != 32 || t < a.T;
        uint4 xv[C], rv[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = live && j < nv;
            xv[i] = in ? *((const uint4 *)(X + t * a.ldx) + j) : make_uint4(0, 0, 0, 0);
            rv[i] = RES && in ? *((const uint4 *)(R + t * a.d) + j) : make_uint4(0, 0, 0, 0);
        }
        if (FMT >= 0 && a.ahead > 0 && threadIdx.x < 2 && t0 + a.ahead + kRows <= a.T) {
            const T *p = threadIdx.x == 0 ? X + (t0 + a.ahead) * a.ldx : RES ? R + (t0 + a.ahead) * a.d : nullptr;
            if (p)
                prefetch_l2(p, (uint32_t)(kRows * a.d * sizeof(T)));
        }
        float2 h[C][P], sq = both(0.f);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            unpack_pairs(xv[i], h[i]);
            if (RES) {
                float2 r[P];
                unpack_pairs(rv[i], r);
#pragma unroll
                for (int k = 0; k < P; ++k)
                    h[i][k] = add2(h[i][k], r[k]);
            }
#pragma unroll
            for (int k = 0; k < P; ++k)
                sq = fma2(h[i][k], h[i][k], sq);
            const int j = lane + G * i;
            if (H && live && j < nv)
                *((uint4 *)(H + t * a.d) + j) = pack_pairs(h[i]);
        }
        // The weights are asked for before the row's sums meet where they fit beside h: codes
        // without a residual (16384 rows of 4096, 128 columns a scale: 41.0 us, 44.4 behind the
        // sums) and norms with one (65536 rows of 512: 40.4, 41.1).  Elsewhere they cost more than
        // they hide: codes of 65536 rows of 8192 with a residual 545 us, 522 behind the sums,
        // norms of 16384 rows of 8192 without one 107 and 85.
        constexpr bool kWeights = EXACT && (FMT < 0 ? RES && C > 1 : !RES && S > 32);
        float wv[kWeights ? C : 1][N];
        if (kWeights)
#pragma unroll
            for (int i = 0; i < C; ++i)
                load_weight(a, (lane + G * i) * N, wv[kWeights ? i : 0]);
        float s[1] = {sq.x + sq.y}, eps = a.eps;
        const auto scale_row = [&] {
            const float f = factor_of(a, s[0]);
            sq = both(0.f);
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    h[i][k] = mul2(h[i][k], both(f));
                    sq = fma2(h[i][k], h[i][k], sq);
                }
            s[0] = sq.x + sq.y;
            eps = eps * f * f;
        };
        // A loop of two turns at most, the second for a row out of range; written out for one piece
        // a lane (65536 rows of 256 bf16: 21.2 us, 22.7 as a loop), more pieces spill so.
        if (FMT < 0 && C == 1) {
            row_reduce<S, 1, false, EXACT>(s, red, turn);
            if (!in_range(a, s[0])) {                // (every lane of the row)
                scale_row();
                row_reduce<S, 1, false, EXACT>(s, red, turn);
            }
        } else {
#pragma unroll 1
            for (bool scaled = false;; scaled = true) {
                row_reduce<S, 1, false, EXACT>(s, red, turn);
                if (scaled || in_range(a, s[0]))
                    break;
                scale_row();
            }
        }
        const float rs = root_of(s[0] / (float)a.d + eps);
        float m[1] = {0.f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j < nv) {
                float (&w)[N] = wv[kWeights ? i : 0];
                if (!kWeights)
                    load_weight(a, j * N, w);
#pragma unroll
                for (int k = 0; k < P; ++k)
                    h[i][k] = mul2(mul2(h[i][k], both(rs)), make_float2(w[2 * k], w[2 * k + 1]));
                if (FMT < 0) {
                    if (live)
                        *((uint4 *)(Y + t * a.d) + j) = pack_pairs(h[i]);
                } else if (a.group_log2 == 0) {
                    m[0] = max_nan(m[0], magnitude(h[i]));
                }
            }
        }
        if (FMT < 0)
            continue;
        constexpr int F = FMT < 0 ? 0 : FMT;
        float rec = 0.f;
        if (a.group_log2 == 0) {
            row_reduce<S, 1, true, EXACT>(m, red, turn);
            rec = reciprocal_of<F>(m[0]);
            if (live && lane == 0)
                a.scale[t] = scale_of<F>(m[0]);
        }
        // Groups: 2^log2 lanes share a scale, in each of their C pieces.  Lane i of them divides
        // for piece i and the others take it from there (every lane dividing for every piece:
        // 65536 rows of 8192 took 747 us).
        static_assert(C <= 4, "a group has 4 lanes at least");
        const int log2 = a.group_log2 - (N == 8 ? 3 : 2), lanes = a.group_log2 ? 1 << log2 : 0;
        float mine = 0.f;
        if (a.group_log2) {
            float each[C];
#pragma unroll
            for (int i = 0; i < C; ++i)
                each[i] = lane + G * i < nv ? magnitude(h[i]) : 0.f;
            const float big = max_of_lanes(each, lane, lanes);
            mine = reciprocal_of<F>(big);
            const int in_group = lane & (lanes - 1), j = lane - in_group + G * in_group;
            const int64_t groups = (a.d - 1 >> a.group_log2) + 1;
            if (live && in_group < C && j < nv)
                a.scale[t * groups + (j >> log2)] = scale_of<F>(big);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (a.group_log2)
                rec = __shfl_sync(0xffffffffu, mine, (threadIdx.x & 31 & ~(lanes - 1)) + i);
            if (live && j < nv) {
                uint32_t q[N / 4];
#pragma unroll
                for (int k = 0; k < P; k += 2)
                    q[k / 2] = codes_of<F>(h[i][k], h[i][k + 1], rec);
                uint32_t *dst = (uint32_t *)(a.codes + t * a.d + j * N);
                if (N == 8)
                    *(uint2 *)dst = make_uint2(q[0], q[N / 4 - 1]);
                else
                    *dst = q[0];
            }
        }
    }
}

// ---- forward, any width ------------------------------------------------------------------
// Widths that are no whole 16-byte pieces, rows off the alignment, and rows wider than
// registers hold: a block walks its row by single elements, the second time from L2.

template <typename T, int FMT>
__global__ void __launch_bounds__(kAnyThreads) k_rmsnorm_any(const NormArgs a)
{
    griddep_start();
    __shared__ __align__(16) float red[2 * 32];
    int turn = 0;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const float sum = norm_singly<T, kAnyThreads, true, FMT, false>(a, t, 1.f, red, turn);
        if (!in_range(a, sum))
            norm_singly<T, kAnyThreads, true, FMT, true>(a, t, factor_of(a, sum), red, turn);
    }
}

// ---- gradient --------------------------------------------------------------------------------

struct NormBwdArgs {
    const void *dY, *H, *dH;    // dH: null without a gradient along the residual stream
    const void *w;
    bool w_bf16;
    int64_t T, ldy;
    int d;
    float eps;
    void *dX;
    float least, most;          // of a row's sum of squares that is taken as it is
    float *part;                // [lanes of rows, d] partial sums of dw
    bool prefetch;
};

// A row of the gradient by single elements, from memory, M neighbouring ones a thread; its part of
// dw is added to what `part` has.  SCALED and the result as in norm_singly.
template <typename T, int S, int M, bool SCALED>
__device__ float norm_bwd_singly(const NormBwdArgs &a, int64_t t, float f, float *part, float *red, int &turn)
{
    const int d = a.d, G = Shape<S>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const T *H = (const T *)a.H + t * d, *dY = (const T *)a.dY + t * a.ldy;
    const T *dH = a.dH ? (const T *)a.dH + t * d : nullptr;
    T *dX = (T *)a.dX + t * d;
    auto h_at = [&](int j) { return SCALED ? Vec<T>::one(H[j]) * f : Vec<T>::one(H[j]); };
    float s[2] = {0.f, 0.f};
    for (int i = lane * M; i < d; i += G * M)
        for (int j = i; j < i + M; ++j) {
            const float h = h_at(j), y = Vec<T>::one(dY[j]);
            s[0] = fmaf(h, h, s[0]);
            s[1] = fmaf(y * weight_at(a, j), h, s[1]);
        }
    row_reduce<S, 2, false>(s, red, turn);
    if (!SCALED && !in_range(a, s[0]))
        return s[0];
    const float mean = s[0] / (float)d + (SCALED ? a.eps * f * f : a.eps);
    const float rs = SCALED ? root_of(mean) : rsqrtf(mean);
    const float m = s[1] / (float)d * rs, c = m * rs;
    for (int i = lane * M; i < d; i += G * M)
        for (int j = i; j < i + M; ++j) {
            const float h = h_at(j), y = Vec<T>::one(dY[j]);
            const float r = dH ? Vec<T>::one(dH[j]) : 0.f, g = y * weight_at(a, j);
            dX[j] = Vec<T>::round(SCALED ? scaled_dx(g, h * rs, m, rs, f, r) : fmaf(rs, fmaf(-h, c, g), r));
            part[j] = fmaf(y * h, rs, part[j]);
        }
    return s[0];
}

// Every group of G lanes walks the rows its place, its place + the number of groups, ...
// and keeps the part of dw of its columns in registers.  Threads of an SM:
template <typename T, int S, int C>
constexpr int kBwdResident = S > 512                        ? S
                             : S == 320                     ? 640
                             : C == 1                       ? (sizeof(T) == 4 ? 1024 : 768)
                             : sizeof(T) == 4 && S <= 256 ? 768
                                                            : 512;

template <typename T, int S, int C>
__global__ void __launch_bounds__(Shape<S>::kThreads, kBwdResident<T, S, C> / Shape<S>::kThreads)
    k_rmsnorm_bwd(const NormBwdArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, kRows = Shape<S>::kRows;
    __shared__ __align__(16) float red[2 * 2 * 32];
    int turn = 0;
    const int G = Shape<S>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const int nv = a.d / N;
    const T *dY = (const T *)a.dY, *H = (const T *)a.H, *dH = (const T *)a.dH;
    T *dX = (T *)a.dX;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    auto load = [&](int64_t t, uint4 (&hv)[C], uint4 (&yv)[C], uint4 (&rv)[C]) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = t < a.T && j < nv;
            hv[i] = in ? *((const uint4 *)(H + t * a.d) + j) : make_uint4(0, 0, 0, 0);
            yv[i] = in ? *((const uint4 *)(dY + t * a.ldy) + j) : make_uint4(0, 0, 0, 0);
            rv[i] = in && dH ? *((const uint4 *)(dH + t * a.d) + j) : make_uint4(0, 0, 0, 0);
        }
    };
    // The next row's loads run before this row's sums meet, where registers allow (65536 rows of
    // 8192: 604 us, 632 without; 4173 rows of 2056 in fp32: 29.6, 35.1; 65536 of 256 34.0, 36.2);
    // rows of 4 KB and more are asked for into L2 before that.
    constexpr bool kEarly = S <= 512;
    // A row out of range: from the registers that hold it (a warp's rows of two pieces a lane: 65536
    // rows of 256 fp32 49.3 us, 55.0 the other way), or behind the loop, which is then entered
    // again, by single elements (65536 rows of 8192 bf16: 605 us, 744 from the registers).
    constexpr bool kInside = S == 32 && C > 1;
    const int warp = S == 32 ? threadIdx.x / 32 : 0;
    float *part = a.part + ((int64_t)blockIdx.x * kRows + warp) * a.d;
    int64_t t0 = (int64_t)blockIdx.x * kRows;
    // (a warp's rows: each warp for itself)
    for (bool first = true;; first = false) {
        float dw[C][N], wv[C][N];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
#pragma unroll
            for (int k = 0; k < N; ++k)
                dw[i][k] = wv[i][k] = 0.f;
            if (j < nv)
                load_weight(a, j * N, wv[i]);
        }
        uint4 hv[C], yv[C], rv[C], hn[C], yn[C], rn[C];
        if (kEarly)
            load(t0 + warp, hn, yn, rn);
        float sum = 0.f;
        for (; t0 < a.T; t0 += stride) {
            const int64_t t = t0 + warp;
            const bool live = t < a.T;
            if (kEarly) {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    hv[i] = hn[i];
                    yv[i] = yn[i];
                    rv[i] = rn[i];
                }
                load(t + stride, hn, yn, rn);
            } else {
                load(t, hv, yv, rv);
            }
            const int64_t later = t0 + (kEarly ? 2 : 1) * stride;
            if (a.prefetch && threadIdx.x < 3 && later + kRows <= a.T) {
                const T *p = threadIdx.x == 0 ? H : threadIdx.x == 1 ? dY : dH;
                if (p)
                    prefetch_l2(p + later * a.d, (uint32_t)(kRows * a.d * sizeof(T)));
            }
            const auto forget = [&] {                // the compiler keeps nothing made from hv and yv
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    asm volatile("" : "+r"(yv[i].x), "+r"(yv[i].y), "+r"(yv[i].z), "+r"(yv[i].w));
                    asm volatile("" : "+r"(hv[i].x), "+r"(hv[i].y), "+r"(hv[i].z), "+r"(hv[i].w));
                }
            };
            float s[2];
            const auto sums = [&](auto scaled, float f) {
                s[0] = s[1] = 0.f;
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    float h[N], y[N];
                    Vec<T>::unpack(hv[i], h);
                    Vec<T>::unpack(yv[i], y);
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const float x = scaled ? h[k] * f : h[k];
                        s[0] = fmaf(x, x, s[0]);
                        s[1] = fmaf(y[k] * wv[i][k], x, s[1]);
                    }
                }
                row_reduce<S, 2, false>(s, red, turn);
            };
            const auto finish = [&](auto scaled, float rs, float f) {
                const float m = s[1] / (float)a.d * rs, c = m * rs;
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int j = lane + G * i;
                    if (!(live && j < nv))
                        continue;
                    float h[N], y[N], x[N];
                    Vec<T>::unpack(hv[i], h);
                    Vec<T>::unpack(yv[i], y);
                    Vec<T>::unpack(rv[i], x);
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const float hk = scaled ? h[k] * f : h[k], g = y[k] * wv[i][k];
                        x[k] = scaled ? scaled_dx(g, hk * rs, m, rs, f, x[k]) : fmaf(rs, fmaf(-hk, c, g), x[k]);
                        dw[i][k] = fmaf(y[k] * hk, rs, dw[i][k]);
                    }
                    *((uint4 *)(dX + t * a.d) + j) = Vec<T>::pack(x);
                }
            };
            sums(std::false_type(), 1.f);
            sum = s[0];
            if (kInside) {
                if (in_range(a, sum) || !live) {
                    finish(std::false_type(), rsqrtf(sum / (float)a.d + a.eps), 1.f);
                } else {
                    const float f = factor_of(a, sum);
                    forget();
                    sums(std::true_type(), f);
                    forget();
                    finish(std::true_type(), root_of(s[0] / (float)a.d + a.eps * f * f), f);
                }
            } else {
                if (live && !in_range(a, sum))       // (every lane of the row)
                    break;
                finish(std::false_type(), rsqrtf(sum / (float)a.d + a.eps), 1.f);
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j < nv)
#pragma unroll
                for (int k = 0; k < N; k += 4) {
                    float4 *to = (float4 *)(part + j * N + k);
                    const float4 was = kInside || first ? make_float4(0.f, 0.f, 0.f, 0.f) : *to;
                    *to = make_float4(was.x + dw[i][k], was.y + dw[i][k + 1], was.z + dw[i][k + 2],
                                      was.w + dw[i][k + 3]);
                }
        }
        if (kInside || t0 >= a.T)
            break;
        norm_bwd_singly<T, S, N, true>(a, t0 + warp, factor_of(a, sum), part, red, turn);
        t0 += stride;
    }
}

// Any width: the part of dw lies in memory and is added to row by row by the thread that
// owns the column.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) k_rmsnorm_bwd_any(const NormBwdArgs a)
{
    griddep_start();
    __shared__ __align__(16) float red[2 * 2 * 32];
    int turn = 0;
    float *part = a.part + (int64_t)blockIdx.x * a.d;
    for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
        part[j] = 0.f;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const float sum = norm_bwd_singly<T, kAnyThreads, 1, false>(a, t, 1.f, part, red, turn);
        if (!in_range(a, sum))
            norm_bwd_singly<T, kAnyThreads, 1, true>(a, t, factor_of(a, sum), part, red, turn);
    }
}

// dw[j] = the sum of the parts' column j, in their order: 32 columns and 32 runs of parts a
// block, so that the result is the same bits every time.
__global__ void __launch_bounds__(1024) k_rmsnorm_dw(const float *__restrict__ part, int parts, int d,
                                                      float *dw, int accumulate)
{
    griddep_start();
    __shared__ float red[32][33];
    const int j = blockIdx.x * 32 + threadIdx.x, per = (parts + 31) / 32;
    float s = 0.f;
    if (j < d)
#pragma unroll 8
        for (int p = threadIdx.y * per, end = min(parts, p + per); p < end; ++p)
            s += __ldg(part + (int64_t)p * d + j);
    red[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = warp_sum(red[threadIdx.x][threadIdx.y]);       // row y of the transpose: column y
    const int c = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && c < d)
        dw[c] = accumulate ? dw[c] + s : s;
}

// ---- launches ----------------------------------------------------------------------------------

// Pieces a lane holds, at most
constexpr int kPieces = 4;

// Whether a width takes the kernels that hold rows in registers
template <typename T>
bool in_registers(int d, int64_t ld)
{
    constexpr int N = Vec<T>::N;
    return d % N == 0 && ld % N == 0 && d / N <= 1024 * kPieces;
}

template <typename T, int S, bool EXACT, int C, int FMT, bool RES>
cudaError_t fwd_rows(NormArgs a, int lanes, cudaStream_t s)
{
    constexpr int kRows = Shape<S>::kRows;
    const int threads = S == 32 ? 256 : lanes;
    const int64_t blocks = (a.T + kRows - 1) / kRows;
    a.ahead = 0;
    if (FMT >= 0 && a.ldx == a.d && a.d * sizeof(T) >= 4096) {
        a.ahead = resident<k_rmsnorm<T, S, EXACT, C, FMT, RES>>(threads) * device_sms() * kRows;
    }
    return launch(k_rmsnorm<T, S, EXACT, C, FMT, RES>, std::min<int64_t>(blocks, (int64_t)1 << 30), threads, a, s);
}

template <typename T, int S, bool EXACT, int C, int FMT>
cudaError_t fwd_shape(const NormArgs &a, int lanes, cudaStream_t s)
{
    return a.R ? fwd_rows<T, S, EXACT, C, FMT, true>(a, lanes, s) : fwd_rows<T, S, EXACT, C, FMT, false>(a, lanes, s);
}

template <typename T, int FMT>
cudaError_t fwd(const NormArgs &a, cudaStream_t s)
{
    if (!in_registers<T>(a.d, a.ldx))
        return launch(k_rmsnorm_any<T, FMT>, std::min<int64_t>(a.T, (int64_t)1 << 30), kAnyThreads, a, s);
    const int nv = a.d / Vec<T>::N, g = lanes_of(nv, kPieces);
    if (g == 32)
        return nv == 32             ? fwd_shape<T, 32, true, 1, FMT>(a, g, s)
               : nv == 64           ? fwd_shape<T, 32, true, 2, FMT>(a, g, s)
               : nv == 32 * kPieces ? fwd_shape<T, 32, true, kPieces, FMT>(a, g, s)
               : nv < 64            ? fwd_shape<T, 32, false, 2, FMT>(a, g, s)
                                    : fwd_shape<T, 32, false, kPieces, FMT>(a, g, s);
    if (g == 64 && nv == 64 * kPieces)
        return fwd_shape<T, 64, true, kPieces, FMT>(a, g, s);
    if (g == 128 && nv == 128 * kPieces)
        return fwd_shape<T, 128, true, kPieces, FMT>(a, g, s);
    if (g == 256 && nv == 256 * kPieces)
        return fwd_shape<T, 256, true, kPieces, FMT>(a, g, s);
    return g <= 256   ? fwd_shape<T, 256, false, kPieces, FMT>(a, g, s)
           : g <= 512 ? fwd_shape<T, 512, false, kPieces, FMT>(a, g, s)
                      : fwd_shape<T, 1024, false, kPieces, FMT>(a, g, s);
}

template <typename T>
cudaError_t fwd_format(const NormArgs &a, int format, cudaStream_t s)
{
    return format < 0              ? fwd<T, -1>(a, s)
           : format == SN_Q_INT8 ? fwd<T, SN_Q_INT8>(a, s)
                                 : fwd<T, SN_Q_E4M3>(a, s);
}

// Pieces a lane of the gradient holds, fewer than in the forward: it also keeps w and dw
constexpr int kBwdPieces = 2;
constexpr int kBwdThreadsPerSm = 1024;

template <typename T>
bool bwd_in_registers(int d, int64_t ld)
{
    constexpr int N = Vec<T>::N;
    return d % N == 0 && ld % N == 0 && d / N <= 1024 * kBwdPieces;
}

// Threads and rows of a block
struct BwdShape {
    int threads, rows;
};
BwdShape bwd_shape(bool registers, int nv)
{
    const int g = registers ? lanes_of(nv, kBwdPieces) : kAnyThreads;
    return g == 32 ? BwdShape{256, 8} : BwdShape{g, 1};
}

// The gradient's grid: the blocks that are on the GPU at once, at most kBwdThreadsPerSm
// threads an SM
template <auto KERNEL>
cudaError_t bwd_launch(BwdShape p, NormBwdArgs a, int &parts, cudaStream_t s)
{
    const int n = std::max(1, std::min(resident<KERNEL>(p.threads), kBwdThreadsPerSm / p.threads));
    const int64_t grid = std::min<int64_t>((a.T + p.rows - 1) / p.rows, (int64_t)device_sms() * n);
    parts = (int)grid * p.rows;
    return launch(KERNEL, grid, p.threads, a, s);
}

template <typename T>
constexpr int kNext = sizeof(T) == 4 ? 320 : 512;

template <typename T>
cudaError_t bwd(const NormBwdArgs &a, float *dw, bool accumulate, cudaStream_t s)
{
    const bool registers = bwd_in_registers<T>(a.d, a.ldy);
    const int nv = a.d / Vec<T>::N;
    const BwdShape p = bwd_shape(registers, nv);
    int parts = 0;
    cudaError_t e;
    if (!registers)
        e = bwd_launch<k_rmsnorm_bwd_any<T>>(p, a, parts, s);
    else if (p.rows > 1)
        e = nv <= 32 ? bwd_launch<k_rmsnorm_bwd<T, 32, 1>>(p, a, parts, s)
                     : bwd_launch<k_rmsnorm_bwd<T, 32, kBwdPieces>>(p, a, parts, s);
    else
        // fp32 rows of a little more than 256 lanes: two blocks of up to 320 an SM (4173 rows of
        // 2056: 26 us, 29 with one; bf16, which has twice the sums, spills: 2000 of 5000 26, 22)
        e = p.threads <= 256   ? bwd_launch<k_rmsnorm_bwd<T, 256, kBwdPieces>>(p, a, parts, s)
            : p.threads <= kNext<T> ? bwd_launch<k_rmsnorm_bwd<T, kNext<T>, kBwdPieces>>(p, a, parts, s)
            : p.threads <= 512 ? bwd_launch<k_rmsnorm_bwd<T, 512, kBwdPieces>>(p, a, parts, s)
                               : bwd_launch<k_rmsnorm_bwd<T, 1024, kBwdPieces>>(p, a, parts, s);
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(k_rmsnorm_dw, dim3((unsigned)((a.d - 1) / 32 + 1)), dim3(32, 32), 0, s, a.part, parts,
                         a.d, dw, (int)accumulate);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t rmsnorm_fwd(sn_dtype dt, const void *X, int64_t ldx, const void *R, void *H, sn_dtype wdt,
                        const void *w, int64_t T, int d, float eps, void *Y, int format, int group,
                        uint8_t *codes, float *scale, cudaStream_t s)
{
    int log2 = 0;
    while (1 << log2 < group)
        ++log2;
    const NormArgs a{X, R, H, w, wdt == SN_BF16, T, ldx, d, eps, Y, codes, scale, log2,
                     least_sum(d, eps), most_sum(eps), 0};
    return dt == SN_BF16 ? fwd_format<__nv_bfloat16>(a, format, s) : fwd_format<float>(a, format, s);
}

size_t rmsnorm_bwd_workspace(int64_t T, int d)
{
    // the most parts that any type and alignment of this width take
    int64_t parts = 0;
    auto most = [&](BwdShape p) {
        const int64_t blocks = (T + p.rows - 1) / p.rows;
        const int64_t grid = (int64_t)device_sms() * std::max(1, kBwdThreadsPerSm / p.threads);
        parts = std::max(parts, std::min(blocks, grid) * p.rows);
    };
    most(bwd_shape(false, 0));
    for (int n = 4; n <= 8; n += 4)
        if (d % n == 0 && d / n <= 1024 * kBwdPieces)
            most(bwd_shape(true, d / n));
    return (size_t)parts * d * sizeof(float);
}

cudaError_t rmsnorm_bwd(sn_dtype dt, const void *dY, int64_t ldy, const void *H, const void *dH, sn_dtype wdt,
                        const void *w, int64_t T, int d, float eps, void *dX, float *dw, bool accumulate,
                        float *part, cudaStream_t s)
{
    const size_t esize = dt == SN_BF16 ? 2 : 4;
    const NormBwdArgs a{dY, H, dH, w, wdt == SN_BF16, T, ldy, d, eps, dX, least_sum(d, eps), most_sum(eps),
                        part, ldy == d && d * esize >= 4096};
    return dt == SN_BF16 ? bwd<__nv_bfloat16>(a, dw, accumulate, s) : bwd<float>(a, dw, accumulate, s);
}

}  // namespace sn
