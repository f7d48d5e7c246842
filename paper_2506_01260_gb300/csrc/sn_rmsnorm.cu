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
// piece until it is written (`Row` below gives the lanes and pieces of a width).  Sums are
// fp32 in every type; y is computed from the unrounded h and rounded once, the stored h once.
#include <algorithm>

#include <cuda_fp8.h>

#include "sn_vec.cuh"

namespace sn {
namespace {

// A row of d elements, in `nv` 16-byte pieces: lane l of the G that share the row has the
// pieces l, l + G, ... (C of them).  Up to 32 lanes lie in one warp and sum by shuffles (a
// block of 256 threads then takes several rows); more lanes are the whole block.
template <int G>
struct Lanes {
    static constexpr int kThreads = G < 256 && G <= 32 ? 256 : G;
    static constexpr int kRows = kThreads / G;
};

// The sums of K values over the lanes of a row, in every lane; `red`: 2 * K * 32 floats
// that calls alternate between (`turn`), so one barrier a call is enough.
template <int G, int K, bool MAX>
__device__ __forceinline__ void row_reduce(float (&v)[K], float *red, int &turn)
{
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float x = __shfl_xor_sync(0xffffffffu, v[k], o);
            v[k] = MAX ? max_nan(v[k], x) : v[k] + x;
        }
    if (G <= 32)
        return;
    constexpr int W = G / 32;
    float *at = red + turn * (K * 32);
    turn ^= 1;
    if (threadIdx.x % 32 == 0)
#pragma unroll
        for (int k = 0; k < K; ++k)
            at[k * 32 + threadIdx.x / 32] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = at[k * 32];
#pragma unroll
        for (int w = 1; w < W; ++w)
            s = MAX ? max_nan(s, at[k * 32 + w]) : s + at[k * 32 + w];
        v[k] = s;
    }
}

// The norm's weights, bf16 or fp32 (a branch that every thread takes alike)
template <typename A, int N>
__device__ __forceinline__ void load_weight(const A &a, int j, float (&f)[N])
{
    if (a.w_bf16)
        load_floats((const __nv_bfloat16 *)a.w + j, f);
    else
        load_floats((const float *)a.w + j, f);
}
template <typename A>
__device__ __forceinline__ float weight_at(const A &a, int j)
{
    return a.w_bf16 ? __bfloat162float(((const __nv_bfloat16 *)a.w)[j]) : ((const float *)a.w)[j];
}

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
    int group;              // columns that share a scale; 0: the row
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

// One code: int8 rounds half to even and clamps, e4m3 rounds to nearest even and saturates
template <int FMT>
__device__ __forceinline__ uint32_t code_of(float x)
{
    if (FMT == SN_Q_INT8)
        return (uint32_t)max(-127, min(127, __float2int_rn(x))) & 0xFFu;
    return (uint32_t)__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
}

// ---- forward, rows in registers ------------------------------------------------------------

template <typename T, int G, int C, int FMT>
__global__ void __launch_bounds__(Lanes<G>::kThreads) k_rmsnorm(const NormArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N;
    __shared__ float red[2 * 32];
    int turn = 0;
    const int lane = threadIdx.x % G;
    const int nv = a.d / N;
    const T *X = (const T *)a.X, *R = (const T *)a.R;
    T *H = (T *)a.H, *Y = (T *)a.Y;
    for (int64_t t0 = (int64_t)blockIdx.x * Lanes<G>::kRows; t0 < a.T; t0 += (int64_t)gridDim.x * Lanes<G>::kRows) {
        const int64_t t = t0 + threadIdx.x / G;
        const bool live = t < a.T;
        uint4 xv[C], rv[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = live && j < nv;
            xv[i] = in ? *((const uint4 *)(X + t * a.ldx) + j) : make_uint4(0, 0, 0, 0);
            rv[i] = in && R ? *((const uint4 *)(R + t * a.d) + j) : make_uint4(0, 0, 0, 0);
        }
        float h[C][N], s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            Vec<T>::unpack(xv[i], h[i]);
            if (R) {
                float r[N];
                Vec<T>::unpack(rv[i], r);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    h[i][k] += r[k];
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                s[0] = fmaf(h[i][k], h[i][k], s[0]);
            const int j = lane + G * i;
            if (H && live && j < nv)
                *((uint4 *)(H + t * a.d) + j) = Vec<T>::pack(h[i]);
        }
        row_reduce<G, 1, false>(s, red, turn);
        const float rs = rsqrtf(s[0] / (float)a.d + a.eps);
        float m[1] = {0.f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j < nv) {
                float wv[N];
                load_weight(a, j * N, wv);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    h[i][k] = h[i][k] * rs * wv[k];
                if (FMT < 0) {
                    if (live)
                        *((uint4 *)(Y + t * a.d) + j) = Vec<T>::pack(h[i]);
                } else if (a.group == 0) {
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        m[0] = max_nan(m[0], fabsf(h[i][k]));
                }
            }
        }
        if (FMT < 0)
            continue;
        constexpr int F = FMT < 0 ? 0 : FMT;
        float rec = 0.f;
        if (a.group == 0) {
            row_reduce<G, 1, true>(m, red, turn);
            rec = reciprocal_of<F>(m[0]);
            if (live && lane == 0)
                a.scale[t] = scale_of<F>(m[0]);
        }
        const int lanes = a.group / N, groups = a.group ? (a.d + a.group - 1) / a.group : 1;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (a.group) {
                float x = 0.f;
                if (j < nv)
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        x = max_nan(x, fabsf(h[i][k]));
                for (int o = lanes / 2; o > 0; o >>= 1)
                    x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
                rec = reciprocal_of<F>(x);
                if (live && j < nv && j % lanes == 0)
                    a.scale[t * groups + j / lanes] = scale_of<F>(x);
            }
            if (live && j < nv) {
                uint32_t q[N / 4];
#pragma unroll
                for (int k = 0; k < N; k += 4)
                    q[k / 4] = code_of<F>(h[i][k] * rec) | code_of<F>(h[i][k + 1] * rec) << 8 |
                               code_of<F>(h[i][k + 2] * rec) << 16 | code_of<F>(h[i][k + 3] * rec) << 24;
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

constexpr int kAnyThreads = 512;

template <typename T, int FMT>
__global__ void __launch_bounds__(kAnyThreads) k_rmsnorm_any(const NormArgs a)
{
    griddep_start();
    __shared__ float red[2 * 32];
    int turn = 0;
    const T *X = (const T *)a.X, *R = (const T *)a.R;
    T *H = (T *)a.H, *Y = (T *)a.Y;
    const int d = a.d;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T *x = X + t * a.ldx;
        const T *r = R ? R + t * d : nullptr;
        auto h_at = [&](int j) { return Vec<T>::one(x[j]) + (r ? Vec<T>::one(r[j]) : 0.f); };
        float s[1] = {0.f};
        for (int j = threadIdx.x; j < d; j += kAnyThreads) {
            const float h = h_at(j);
            s[0] = fmaf(h, h, s[0]);
        }
        row_reduce<kAnyThreads, 1, false>(s, red, turn);
        const float rs = rsqrtf(s[0] / (float)d + a.eps);
        auto y_at = [&](int j) { return h_at(j) * rs * weight_at(a, j); };
        constexpr int F = FMT < 0 ? 0 : FMT;
        if (FMT < 0) {
            for (int j = threadIdx.x; j < d; j += kAnyThreads) {
                const float h = h_at(j);
                if (H)
                    H[t * d + j] = Vec<T>::round(h);
                Y[t * d + j] = Vec<T>::round(h * rs * weight_at(a, j));
            }
        } else if (a.group == 0) {
            float m[1] = {0.f};
            for (int j = threadIdx.x; j < d; j += kAnyThreads)
                m[0] = max_nan(m[0], fabsf(y_at(j)));
            row_reduce<kAnyThreads, 1, true>(m, red, turn);
            const float rec = reciprocal_of<F>(m[0]);
            if (threadIdx.x == 0)
                a.scale[t] = scale_of<F>(m[0]);
            for (int j = threadIdx.x; j < d; j += kAnyThreads) {
                const float h = h_at(j);
                a.codes[t * d + j] = (uint8_t)code_of<F>(h * rs * weight_at(a, j) * rec);
                if (H)
                    H[t * d + j] = Vec<T>::round(h);
            }
        } else {
            // a warp takes whole groups
            const int groups = (d + a.group - 1) / a.group;
            for (int g = threadIdx.x / 32; g < groups; g += kAnyThreads / 32) {
                const int j0 = g * a.group, j1 = min(d, j0 + a.group);
                float m = 0.f;
                for (int j = j0 + threadIdx.x % 32; j < j1; j += 32)
                    m = max_nan(m, fabsf(y_at(j)));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float rec = reciprocal_of<F>(m);
                if (threadIdx.x % 32 == 0)
                    a.scale[t * groups + g] = scale_of<F>(m);
                for (int j = j0 + threadIdx.x % 32; j < j1; j += 32) {
                    const float h = h_at(j);
                    a.codes[t * d + j] = (uint8_t)code_of<F>(h * rs * weight_at(a, j) * rec);
                    if (H)
                        H[t * d + j] = Vec<T>::round(h);
                }
            }
        }
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
    float *part;                // [lanes of rows, d] partial sums of dw
};

// Every group of G lanes walks the rows its place, its place + the number of groups, ...
// and keeps the part of dw of its columns in registers.
template <typename T, int G, int C>
__global__ void __launch_bounds__(Lanes<G>::kThreads) k_rmsnorm_bwd(const NormBwdArgs a)
{
    griddep_start();
    constexpr int N = Vec<T>::N;
    __shared__ float red[2 * 2 * 32];
    int turn = 0;
    const int lane = threadIdx.x % G;
    const int nv = a.d / N;
    const T *dY = (const T *)a.dY, *H = (const T *)a.H, *dH = (const T *)a.dH;
    T *dX = (T *)a.dX;
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
    for (int64_t t0 = (int64_t)blockIdx.x * Lanes<G>::kRows; t0 < a.T; t0 += (int64_t)gridDim.x * Lanes<G>::kRows) {
        const int64_t t = t0 + threadIdx.x / G;
        const bool live = t < a.T;
        uint4 hv[C], yv[C], rv[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = live && j < nv;
            hv[i] = in ? *((const uint4 *)(H + t * a.d) + j) : make_uint4(0, 0, 0, 0);
            yv[i] = in ? *((const uint4 *)(dY + t * a.ldy) + j) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            rv[i] = live && dH && j < nv ? *((const uint4 *)(dH + t * a.d) + j) : make_uint4(0, 0, 0, 0);
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float h[N], y[N];
            Vec<T>::unpack(hv[i], h);
            Vec<T>::unpack(yv[i], y);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                s[0] = fmaf(h[k], h[k], s[0]);
                s[1] = fmaf(y[k] * wv[i][k], h[k], s[1]);
            }
        }
        row_reduce<G, 2, false>(s, red, turn);
        const float rs = rsqrtf(s[0] / (float)a.d + a.eps);
        const float c = s[1] / (float)a.d * rs * rs;
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
                x[k] = fmaf(rs, fmaf(-h[k], c, y[k] * wv[i][k]), x[k]);
                dw[i][k] = fmaf(y[k] * h[k], rs, dw[i][k]);
            }
            *((uint4 *)(dX + t * a.d) + j) = Vec<T>::pack(x);
        }
    }
    float *part = a.part + ((int64_t)blockIdx.x * Lanes<G>::kRows + threadIdx.x / G) * a.d;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int j = lane + G * i;
        if (j < nv)
#pragma unroll
            for (int k = 0; k < N; k += 4)
                *(float4 *)(part + j * N + k) = make_float4(dw[i][k], dw[i][k + 1], dw[i][k + 2], dw[i][k + 3]);
    }
}

// Any width: the part of dw lies in memory and is added to row by row by the thread that
// owns the column.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) k_rmsnorm_bwd_any(const NormBwdArgs a)
{
    griddep_start();
    __shared__ float red[2 * 2 * 32];
    int turn = 0;
    const T *dY = (const T *)a.dY, *H = (const T *)a.H, *dH = (const T *)a.dH;
    T *dX = (T *)a.dX;
    const int d = a.d;
    float *part = a.part + (int64_t)blockIdx.x * d;
    for (int j = threadIdx.x; j < d; j += kAnyThreads)
        part[j] = 0.f;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        float s[2] = {0.f, 0.f};
        for (int j = threadIdx.x; j < d; j += kAnyThreads) {
            const float h = Vec<T>::one(H[t * d + j]), y = Vec<T>::one(dY[t * a.ldy + j]);
            s[0] = fmaf(h, h, s[0]);
            s[1] = fmaf(y * weight_at(a, j), h, s[1]);
        }
        row_reduce<kAnyThreads, 2, false>(s, red, turn);
        const float rs = rsqrtf(s[0] / (float)d + a.eps);
        const float c = s[1] / (float)d * rs * rs;
        for (int j = threadIdx.x; j < d; j += kAnyThreads) {
            const float h = Vec<T>::one(H[t * d + j]), y = Vec<T>::one(dY[t * a.ldy + j]);
            const float r = dH ? Vec<T>::one(dH[t * d + j]) : 0.f;
            dX[t * d + j] = Vec<T>::round(fmaf(rs, fmaf(-h, c, y * weight_at(a, j)), r));
            part[j] = fmaf(y * h, rs, part[j]);
        }
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
        for (int p = threadIdx.y * per, end = min(parts, p + per); p < end; ++p)
            s += part[(int64_t)p * d + j];
    red[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = warp_sum(red[threadIdx.x][threadIdx.y]);       // row y of the transpose: column y
    const int c = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && c < d)
        dw[c] = accumulate ? dw[c] + s : s;
}

// ---- launches ----------------------------------------------------------------------------------

// The lanes of a row and their pieces: 1 piece each up to 32 lanes, then the fewest lanes
// with at most kPieces pieces
constexpr int kPieces = 4;

int lanes_of(int nv)
{
    int g = 32;
    while (g * kPieces < nv)
        g *= 2;
    return g;
}

// Whether a width takes the kernels that hold rows in registers
template <typename T>
bool in_registers(int d, int64_t ld)
{
    constexpr int N = Vec<T>::N;
    return d % N == 0 && ld % N == 0 && d / N <= 1024 * kPieces;
}

template <typename K, typename A>
cudaError_t launch(K kernel, int64_t grid, int threads, const A &a, cudaStream_t s)
{
    count_launch();
    const cudaError_t e = launch_dependent(kernel, dim3((unsigned)grid), dim3(threads), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int G, int FMT>
cudaError_t fwd_lanes(const NormArgs &a, cudaStream_t s)
{
    const int pieces = (a.d / Vec<T>::N + G - 1) / G;
    const int64_t blocks = (a.T + Lanes<G>::kRows - 1) / Lanes<G>::kRows;
    const int64_t grid = std::min<int64_t>(blocks, (int64_t)1 << 30);
    if (pieces == 1)
        return launch(k_rmsnorm<T, G, 1, FMT>, grid, Lanes<G>::kThreads, a, s);
    if (pieces == 2)
        return launch(k_rmsnorm<T, G, 2, FMT>, grid, Lanes<G>::kThreads, a, s);
    return launch(k_rmsnorm<T, G, kPieces, FMT>, grid, Lanes<G>::kThreads, a, s);
}

template <typename T, int FMT>
cudaError_t fwd(const NormArgs &a, cudaStream_t s)
{
    if (!in_registers<T>(a.d, a.ldx))
        return launch(k_rmsnorm_any<T, FMT>, std::min<int64_t>(a.T, (int64_t)1 << 30), kAnyThreads, a, s);
    switch (lanes_of(a.d / Vec<T>::N)) {
    case 32: return fwd_lanes<T, 32, FMT>(a, s);
    case 64: return fwd_lanes<T, 64, FMT>(a, s);
    case 128: return fwd_lanes<T, 128, FMT>(a, s);
    case 256: return fwd_lanes<T, 256, FMT>(a, s);
    case 512: return fwd_lanes<T, 512, FMT>(a, s);
    default: return fwd_lanes<T, 1024, FMT>(a, s);
    }
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

int bwd_lanes(int nv)
{
    int g = 32;
    while (g * kBwdPieces < nv)
        g *= 2;
    return g;
}

struct BwdPlan {
    int threads, rows;       // of a block
    int grid;
    int parts() const { return grid * rows; }
};

BwdPlan bwd_plan(bool registers, int nv, int64_t T)
{
    BwdPlan p;
    const int g = registers ? bwd_lanes(nv) : kAnyThreads;
    p.threads = g <= 32 ? 256 : g;
    p.rows = p.threads / g;
    const int64_t blocks = (T + p.rows - 1) / p.rows;
    p.grid = (int)std::min<int64_t>(blocks, (int64_t)device_sms() * (kBwdThreadsPerSm / p.threads));
    return p;
}

template <typename T, int G>
cudaError_t bwd_lanes_launch(const NormBwdArgs &a, int grid, cudaStream_t s)
{
    if ((a.d / Vec<T>::N + G - 1) / G == 1)
        return launch(k_rmsnorm_bwd<T, G, 1>, grid, Lanes<G>::kThreads, a, s);
    return launch(k_rmsnorm_bwd<T, G, kBwdPieces>, grid, Lanes<G>::kThreads, a, s);
}

template <typename T>
cudaError_t bwd(const NormBwdArgs &a, float *dw, bool accumulate, cudaStream_t s)
{
    const bool registers = bwd_in_registers<T>(a.d, a.ldy);
    const int nv = a.d / Vec<T>::N;
    const BwdPlan p = bwd_plan(registers, nv, a.T);
    cudaError_t e;
    if (!registers) {
        e = launch(k_rmsnorm_bwd_any<T>, p.grid, kAnyThreads, a, s);
    } else {
        switch (bwd_lanes(nv)) {
        case 32: e = bwd_lanes_launch<T, 32>(a, p.grid, s); break;
        case 64: e = bwd_lanes_launch<T, 64>(a, p.grid, s); break;
        case 128: e = bwd_lanes_launch<T, 128>(a, p.grid, s); break;
        case 256: e = bwd_lanes_launch<T, 256>(a, p.grid, s); break;
        case 512: e = bwd_lanes_launch<T, 512>(a, p.grid, s); break;
        default: e = bwd_lanes_launch<T, 1024>(a, p.grid, s); break;
        }
    }
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(k_rmsnorm_dw, dim3((unsigned)((a.d - 1) / 32 + 1)), dim3(32, 32), 0, s, a.part,
                         p.parts(), a.d, dw, (int)accumulate);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t rmsnorm_fwd(sn_dtype dt, const void *X, int64_t ldx, const void *R, void *H, sn_dtype wdt,
                        const void *w, int64_t T, int d, float eps, void *Y, int format, int group,
                        uint8_t *codes, float *scale, cudaStream_t s)
{
    const NormArgs a{X, R, H, w, wdt == SN_BF16, T, ldx, d, eps, Y, codes, scale, group};
    return dt == SN_BF16 ? fwd_format<__nv_bfloat16>(a, format, s) : fwd_format<float>(a, format, s);
}

size_t rmsnorm_bwd_workspace(int64_t T, int d)
{
    // the most parts that any type and alignment of this width take
    size_t parts = 0;
    for (int n = 4; n <= 8; n += 4) {
        parts = std::max<size_t>(parts, bwd_plan(false, 0, T).parts());
        if (d % n == 0 && d / n <= 1024 * kBwdPieces)
            parts = std::max<size_t>(parts, bwd_plan(true, d / n, T).parts());
    }
    return parts * (size_t)d * sizeof(float);
}

cudaError_t rmsnorm_bwd(sn_dtype dt, const void *dY, int64_t ldy, const void *H, const void *dH, sn_dtype wdt,
                        const void *w, int64_t T, int d, float eps, void *dX, float *dw, bool accumulate,
                        float *part, cudaStream_t s)
{
    const NormBwdArgs a{dY, H, dH, w, wdt == SN_BF16, T, ldy, d, eps, dX, part};
    return dt == SN_BF16 ? bwd<__nv_bfloat16>(a, dw, accumulate, s) : bwd<float>(a, dw, accumulate, s);
}

}  // namespace sn
