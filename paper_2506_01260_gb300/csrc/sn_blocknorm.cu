// sn_blocknorm.cu — the norms after and before a block of a residual stream, fused with the block's
// gate and residual scale, and their gradients.
//
//   n1 = y / rms(y),  h = r + m n1,  z = h / rms(h) w_pre,     m = s gate w_post,
//                                                              rms(x) = sqrt(mean(x^2) + eps)
//   gradients, from the stored h:
//   n2 = h / rms(h),  g = dz w_pre,  dh' = (g - n2 mean(g n2)) / rms(h) + dh  (r's gradient)
//   e = m dh',        dy = (e - n1 mean(e n1)) / rms(y)
//   dw_pre = sum dz n2,   S_i = sum over gate i's tokens of dh' n1,
//   dgate_i = s w_post S_i,   dw_post = s sum_i gate_i S_i
//
// Bound by DRAM: every element is read once and stays in registers as a 16-byte piece until it is
// written.  Sums are fp32 in every type; z comes from the unrounded h and every output is rounded
// once.  The gradient's second mean is taken with the first, before dh' is known:
//   sum e y = (sum m y g - mean(g n2) sum m y n2) / rms(h) + sum m y dh,
// so a row's six sums meet once.
//
// Measured: forward of 16384 bf16 rows of 4096 80 us (6.7 TB/s), of 65536 of 8192 with 16 gates 644 (6.7);
// gradient 126 us (6.4 TB/s, 5 us of it the sum of the parts) and 960 (6.7), of 4173 fp32 rows of 2056 37
// (5.6), where the 14 rows a block walks and the sum of the parts cost latency.  fp32 forward of 16384 rows
// of 4096 160 us (6.7).  A gate for every few tokens costs what happens between two of its rows: gradient of
// 16384 bf16 rows of 4096, each call behind a flush of L2, 133 us without a gate, 147 with one for 128
// tokens, 163 for 16, 200 for 3 and 307 for each.
#include <algorithm>
#include <atomic>

#include "sn_norm.cuh"

namespace sn {
namespace {

struct Weight {
    const void *w;
    bool w_bf16;
};

struct Args {
    const void *Y, *R;          // the gradient: Y, H
    const void *dZ, *dH;        // the gradient; dH may be null
    const void *gate;           // null: 1
    Weight post, pre;
    int64_t T, ldy, lddz;
    int64_t per_gate;           // tokens that share a row of the gate
    int d;
    float eps, scale, inverse_d;
    float least, most;          // of a row's sum of squares that is taken as it is
    void *H, *Z;                // the gradient: dR, dY
    int64_t workers;            // the gradient's, at most T
    float *dgate;               // written where a worker has all of a gate's tokens
    bool add;
    bool gated;                 // by more than one row: S is every gate's own
    // [parts, d], a part a block, of dw_pre and (gated: a part a worker) of dw_post, which is S
    // itself where it is one for all tokens
    float *part_pre, *part_post;
    // gated: S of a worker and a gate that it shares with others.  A worker shares two gates at most, its
    // first, at 2 w, and its last, at 2 w + 1; with fewer gates than workers (few_gates) worker w's of gate
    // i at w + i are fewer rows.
    float *part_gate;
    bool few_gates;
};

// half of a factor's exponent: taken on either side of a product, nothing in between leaves fp32
__device__ __forceinline__ float half_of(float f) { return f == 1.f ? 1.f : f > 1.f ? 0x1p50f : 0x1p-40f; }

template <typename T>
__device__ __forceinline__ float gate_at(const Args &a, int64_t i, int j)
{
    return a.gate ? Vec<T>::one(((const T *)a.gate)[i * a.d + j]) : 1.f;
}
__device__ __forceinline__ int64_t gate_of(const Args &a, int64_t t)
{
    return (uint32_t)t / (uint32_t)a.per_gate;      // both are below 2^31
}

// ---- forward -----------------------------------------------------------------------------------

// Threads of an SM that registers are kept low enough for
template <int S, int C>
constexpr int kResident = S > 512 ? S : S == 512 ? 1024 : C == 1 ? 1536 : C == 2 ? 1024 : 768;

template <typename T, int S, bool EXACT, int C, bool GATED>
__global__ void __launch_bounds__(Shape<S>::kThreads, kResident<S, C> / Shape<S>::kThreads)
    k_blocknorm(const Args a)
{
    griddep_start();
    constexpr int N = Vec<T>::N, P = N / 2, kRows = Shape<S>::kRows;
    __shared__ __align__(16) float red[2 * 32];
    int turn = 0;
    const int G = Shape<S, EXACT>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const int nv = EXACT ? S * C : a.d / N;
    const T *Y = (const T *)a.Y, *R = (const T *)a.R, *gate = (const T *)a.gate;
    T *H = (T *)a.H, *Z = (T *)a.Z;
    for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
        const int64_t t = t0 + (S == 32 ? threadIdx.x / 32 : 0);
        const bool live = S != 32 || t < a.T;
        uint4 yv[C], rv[C], gv[GATED ? C : 1];
        const T *g = GATED ? gate + gate_of(a, live ? t : 0) * a.d : nullptr;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = live && j < nv;
            yv[i] = in ? *((const uint4 *)(Y + t * a.ldy) + j) : make_uint4(0, 0, 0, 0);
            rv[i] = in ? *((const uint4 *)(R + t * a.d) + j) : make_uint4(0, 0, 0, 0);
            if (GATED)       // (asked for behind the sums, 32768 rows of 2048 with 128 gates took 96 us, 79 now)
                gv[GATED ? i : 0] = in ? __ldg((const uint4 *)g + j) : make_uint4(0, 0, 0, 0);
        }
        float2 h[C][P], sq;
        float s[1], eps = a.eps, f = 1.f;
        const auto sum_squares = [&] {
            sq = both(0.f);
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int k = 0; k < P; ++k)
                    sq = fma2(h[i][k], h[i][k], sq);
            s[0] = sq.x + sq.y;
        };
        // the reciprocal root of the row in h, which is scaled where its squares ask for it
        const auto root = [&] {
            eps = a.eps;
            f = 1.f;
            sum_squares();
#pragma unroll 1
            while (true) {
                row_reduce<S, 1, false, EXACT>(s, red, turn);
                if (f != 1.f || in_range(a, s[0]))
                    break;
                f = factor_of(a, s[0]);
                eps = a.eps * f * f;
#pragma unroll
                for (int i = 0; i < C; ++i)
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        h[i][k] = mul2(h[i][k], both(f));
                sum_squares();
            }
            return root_of(s[0] / (float)a.d + eps);
        };
#pragma unroll
        for (int i = 0; i < C; ++i)
            unpack_pairs(yv[i], h[i]);
        const float r1 = root() * a.scale;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            float2 r[P];
            unpack_pairs(rv[i], r);
            if (j < nv) {
                float w[N];
                load_weight(a.post, j * N, w);
#pragma unroll
                for (int k = 0; k < P; ++k)
                    h[i][k] = mul2(h[i][k], mul2(both(r1), make_float2(w[2 * k], w[2 * k + 1])));
                if (GATED) {
                    float2 m[P];
                    unpack_pairs(gv[GATED ? i : 0], m);
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        h[i][k] = mul2(h[i][k], m[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < P; ++k)
                h[i][k] = add2(h[i][k], r[k]);
            if (live && j < nv)
                *((uint4 *)(H + t * a.d) + j) = pack_pairs(h[i]);
        }
        const float r2 = root();
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (live && j < nv) {
                float w[N];
                load_weight(a.pre, j * N, w);
#pragma unroll
                for (int k = 0; k < P; ++k)
                    h[i][k] = mul2(mul2(h[i][k], both(r2)), make_float2(w[2 * k], w[2 * k + 1]));
                *((uint4 *)(Z + t * a.d) + j) = pack_pairs(h[i]);
            }
        }
    }
}

// Widths that are no whole 16-byte pieces, rows off the alignment, and rows wider than registers
// hold: a block walks its row by single elements, again from L2.  The sum of squares of at(j), the
// factor that it was taken with, and the reciprocal root.
template <typename F>
__device__ float root_singly(const Args &a, F at, float &f, float *red, int &turn)
{
    f = 1.f;
    while (true) {
        float s[1] = {0.f};
        for (int j = threadIdx.x; j < a.d; j += kAnyThreads) {
            const float x = at(j) * f;
            s[0] = fmaf(x, x, s[0]);
        }
        row_reduce<kAnyThreads, 1, false, true>(s, red, turn);
        if (f != 1.f || in_range(a, s[0]))
            return root_of(s[0] / (float)a.d + a.eps * f * f);
        f = factor_of(a, s[0]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kAnyThreads) k_blocknorm_any(const Args a)
{
    griddep_start();
    __shared__ __align__(16) float red[2 * 32];
    int turn = 0;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T *y = (const T *)a.Y + t * a.ldy, *r = (const T *)a.R + t * a.d;
        const int64_t i = gate_of(a, t);
        float f1, f2;
        const float r1 = root_singly(a, [&](int j) { return Vec<T>::one(y[j]); }, f1, red, turn) * a.scale;
        auto h_at = [&](int j) {
            return fmaf(Vec<T>::one(y[j]) * f1, r1 * weight_at(a.post, j) * gate_at<T>(a, i, j), Vec<T>::one(r[j]));
        };
        const float r2 = root_singly(a, h_at, f2, red, turn);
        for (int j = threadIdx.x; j < a.d; j += kAnyThreads) {
            const float h = h_at(j);
            ((T *)a.H)[t * a.d + j] = Vec<T>::round(h);
            ((T *)a.Z)[t * a.d + j] = Vec<T>::round(h * f2 * r2 * weight_at(a.pre, j));
        }
    }
}

// ---- gradient ----------------------------------------------------------------------------------

// Of T tokens, worker w of W takes those from w T / W on; token t is worker ((t + 1) W - 1) / T's.
__device__ __forceinline__ int64_t first_token(int64_t w, int64_t W, int64_t T) { return w * T / W; }
__device__ __forceinline__ int64_t worker_of(int64_t t, int64_t W, int64_t T) { return ((t + 1) * W - 1) / T; }

// The row of part_gate for worker w's tokens of gate i, its first gate or not
__device__ __forceinline__ int64_t shared_at(const Args &a, int64_t w, int64_t i, bool first)
{
    return a.few_gates ? w + i : 2 * w + !first;
}

// The six sums of a row, over its elements or pairs of them
template <typename F>
struct Sums {
    F s[6];         // h h, g h, y y, m y g, m y h, m y dh
};
__device__ __forceinline__ float fma_of(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float mul_of(float a, float b) { return a * b; }
__device__ __forceinline__ float2 fma_of(float2 a, float2 b, float2 c) { return fma2(a, b, c); }
__device__ __forceinline__ float2 mul_of(float2 a, float2 b) { return mul2(a, b); }
template <typename F>
__device__ __forceinline__ void add_element(Sums<F> &m, F h, F z, F y, F r, F pw, F mw)
{
    const F g = mul_of(z, pw), my = mul_of(y, mw);
    m.s[0] = fma_of(h, h, m.s[0]);
    m.s[1] = fma_of(g, h, m.s[1]);
    m.s[2] = fma_of(y, y, m.s[2]);
    m.s[3] = fma_of(my, g, m.s[3]);
    m.s[4] = fma_of(my, h, m.s[4]);
    m.s[5] = fma_of(my, r, m.s[5]);
}
template <typename F>
__device__ __forceinline__ F every(float x);
template <>
__device__ __forceinline__ float every<float>(float x) { return x; }
template <>
__device__ __forceinline__ float2 every<float2>(float x) { return both(x); }

// What the elements of a row share; h and y are scaled by factors where their squares ask for it
struct Row {
    float fh = 1.f, fy = 1.f;   // the factors, 1 for almost every row
    float r2, c2, a2, half2;    // 1 / rms(h f), -mean(g n2), and 1 / rms(h) in two factors
    float r1, c1, a1, half1;
    // whether h or y has to be taken again by a factor
    __device__ __forceinline__ bool again(const Args &a, const float (&s)[6])
    {
        const bool h = fh == 1.f && !in_range(a, s[0]), y = fy == 1.f && !in_range(a, s[2]);
        if (h)
            fh = factor_of(a, s[0]);
        if (y)
            fy = factor_of(a, s[2]);
        return h || y;
    }
    __device__ __forceinline__ void finish(const Args &a, const float (&s)[6])
    {
        r2 = root_of(fmaf(s[0], a.inverse_d, a.eps * fh * fh));
        r1 = root_of(fmaf(s[2], a.inverse_d, a.eps * fy * fy));
        half2 = half_of(fh);
        half1 = half_of(fy);
        a2 = r2 * half2;
        a1 = r1 * half1;
        c2 = -(s[1] * a.inverse_d) * r2;
        c1 = -(fmaf(fmaf(r2 * c2, s[4], s[3]) * a2, half2, s[5]) * a.inverse_d) * r1;
    }
    // dh' and dy of an element, and its parts of dw_pre and S
    template <typename F>
    __device__ __forceinline__ void element(F h, F z, F y, F r, F pw, F mw, F &dh, F &dy, F &pre, F &sum) const
    {
        const F n2 = mul_of(h, every<F>(r2)), n1 = mul_of(y, every<F>(r1));
        dh = fma_of(mul_of(fma_of(n2, every<F>(c2), mul_of(z, pw)), every<F>(a2)), every<F>(half2), r);
        dy = mul_of(mul_of(fma_of(n1, every<F>(c1), mul_of(mw, dh)), every<F>(a1)), every<F>(half1));
        pre = fma_of(z, n2, pre);
        sum = fma_of(dh, n1, sum);
    }
};

// The sums of six values over the lanes of a row, in every lane.  Three halvings leave a lane one
// value of its eighth of the warp (9 shuffles for the six, not 30), a lane then adds four warps'
// parts of one value.  `red`: 2 * 8 * 32 floats that calls alternate between (`turn`).
template <int S>
__device__ __forceinline__ void row_sums(float (&v)[6], float *red, int &turn)
{
    const int lane = threadIdx.x % 32;
    const bool b4 = lane & 16, b3 = lane & 8, b2 = lane & 4;
    // lanes with b4 keep values 4 and 5 (and two zeros), the others 0 to 3; then halves of those
    float x[4];
    x[0] = (b4 ? v[4] : v[0]) + __shfl_xor_sync(0xffffffffu, b4 ? v[0] : v[4], 16);
    x[1] = (b4 ? v[5] : v[1]) + __shfl_xor_sync(0xffffffffu, b4 ? v[1] : v[5], 16);
    x[2] = __shfl_xor_sync(0xffffffffu, v[2], 16) + v[2];
    x[3] = __shfl_xor_sync(0xffffffffu, v[3], 16) + v[3];
    if (b4)
        x[2] = x[3] = 0.f;
    float y[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        y[i] = (b3 ? x[2 + i] : x[i]) + __shfl_xor_sync(0xffffffffu, b3 ? x[i] : x[2 + i], 8);
    float z = (b2 ? y[1] : y[0]) + __shfl_xor_sync(0xffffffffu, b2 ? y[0] : y[1], 4);
    z += __shfl_xor_sync(0xffffffffu, z, 2);
    z += __shfl_xor_sync(0xffffffffu, z, 1);            // value lane / 4 of the warp
    if (S > 32) {
        const int warps = blockDim.x / 32, warp = threadIdx.x / 32;
        float *at = red + turn * (8 * 32);
        turn ^= 1;
        if (lane % 4 == 0)
            at[lane * 8 + warp] = z;                    // value lane / 4: 32 warps
        __syncthreads();
        z = 0.f;
#pragma unroll
        for (int w = 0; w < S / 32; w += 16) {
            const int first = w + lane % 4 * 4;
            if (first < warps) {
                const float4 p = *(const float4 *)(at + lane / 4 * 32 + first);
                z += (p.x + (first + 1 < warps ? p.y : 0.f)) +
                     ((first + 2 < warps ? p.z : 0.f) + (first + 3 < warps ? p.w : 0.f));
            }
        }
        z += __shfl_xor_sync(0xffffffffu, z, 2);
        z += __shfl_xor_sync(0xffffffffu, z, 1);
    }
#pragma unroll
    for (int k = 0; k < 6; ++k)
        v[k] = __shfl_sync(0xffffffffu, z, 4 * k);
}

// Piece j of an array of fours (see k_blocknorm_bwd), as pairs
template <int P>
__device__ __forceinline__ void from_fours(const float4 *w, int nv, int j, float2 (&f)[P])
{
#pragma unroll
    for (int k = 0; k < P; k += 2) {
        const float4 v = w[k / 2 * nv + j];
        f[k] = make_float2(v.x, v.y);
        f[k + 1] = make_float2(v.z, v.w);
    }
}

// 16 bytes to shared memory
__device__ __forceinline__ void copy16(uint4 *to, const uint4 *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from)
                 : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Whether a row is copied ahead (see k_blocknorm_bwd)
template <int S, int C>
constexpr bool is_ahead = S <= 512 && C <= 3;
// Threads of an SM that registers are kept low enough for
template <int S>
constexpr int kBwdResident = S > 512 ? S : 512;

// A worker (a warp or a block) walks its run of tokens, a row at a time, and keeps dw_pre and the
// present gate's S of its columns in registers; m and w_pre lie in shared memory, each thread's own
// columns.
template <typename T, int S, int C>
__global__ void __launch_bounds__(Shape<S>::kThreads, kBwdResident<S> / Shape<S>::kThreads)
    k_blocknorm_bwd(const Args a)
{
    griddep_start();
    extern __shared__ float4 weights[];
    constexpr int N = Vec<T>::N, P = N / 2, kRows = Shape<S>::kRows;
    __shared__ __align__(16) float red[2 * 8 * 32];
    int turn = 0;
    const int G = Shape<S>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const int warp = S == 32 ? threadIdx.x / 32 : 0, nv = a.d / N;
    const T *Y = (const T *)a.Y, *H = (const T *)a.R, *dZ = (const T *)a.dZ, *dH = (const T *)a.dH;
    T *dR = (T *)a.H, *dY = (T *)a.Z;
    // fours of a piece's elements, the pieces' first fours in front: lanes read neighbouring 16 bytes
    float4 *wp = weights + warp * (2 * (N / 4)) * nv, *wm = wp + (N / 4) * nv;
    const int64_t worker = (int64_t)blockIdx.x * kRows + warp, workers = a.workers;
    float2 pre[C][P];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int j = lane + G * i;
#pragma unroll
        for (int k = 0; k < P; ++k)
            pre[i][k] = both(0.f);
        if (j < nv) {
            float w[N];
            load_weight(a.pre, j * N, w);
#pragma unroll
            for (int k = 0; k < N; k += 4)
                wp[k / 4 * nv + j] = make_float4(w[k], w[k + 1], w[k + 2], w[k + 3]);
        }
    }
    // The next row is on its way to shared memory, each thread's own pieces, while this one is at work
    // (16384 rows of 4096 bf16 126 us, 134 when it was asked for into L2 instead, 137 with the row after
    // it asked for as well).  Rows of more than 512 lanes leave no room there, and with four pieces a lane
    // it costs (16384 of 8192 fp32 540 us, 480).
    constexpr bool kAhead = is_ahead<S, C>;
    uint4 *ahead = (uint4 *)(weights + kRows * (2 * (N / 4)) * nv) + threadIdx.x;
    uint4 hv[C], yv[C], zv[C], rv[C];
    // (of the last block's warps some may have none)
    const int64_t t1 = worker < workers ? first_token(worker + 1, workers, a.T) : 0;
    auto load = [&](int64_t t) {
        const T *h = H + t * a.d, *y = Y + t * a.ldy, *z = dZ + t * a.lddz, *r = dH + t * a.d;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = j < nv;
            if (kAhead) {
                if (in) {
                    copy16(ahead + (4 * i) * blockDim.x, (const uint4 *)h + j);
                    copy16(ahead + (4 * i + 1) * blockDim.x, (const uint4 *)y + j);
                    copy16(ahead + (4 * i + 2) * blockDim.x, (const uint4 *)z + j);
                    if (dH)
                        copy16(ahead + (4 * i + 3) * blockDim.x, (const uint4 *)r + j);
                }
            } else {
                hv[i] = in ? *((const uint4 *)h + j) : make_uint4(0, 0, 0, 0);
                yv[i] = in ? *((const uint4 *)y + j) : make_uint4(0, 0, 0, 0);
                zv[i] = in ? *((const uint4 *)z + j) : make_uint4(0, 0, 0, 0);
                rv[i] = in && dH ? *((const uint4 *)r + j) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    int64_t t = first_token(worker, workers, a.T);
    if (kAhead) {
        if (!dH)                               // nothing is ever copied there
#pragma unroll
            for (int i = 0; i < C; ++i)
                ahead[(4 * i + 3) * blockDim.x] = make_uint4(0, 0, 0, 0);
        if (t < t1)
            load(t);
    }
    float2 sum[C][P];
    const auto clear = [&] {
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int k = 0; k < P; ++k)
                sum[i][k] = both(0.f);
    };
    clear();
    for (bool first = true; t < t1; first = false) {
        const int64_t i_gate = a.gated ? gate_of(a, t) : 0, t0 = t;
        const int64_t end = a.gated ? min(t1, (i_gate + 1) * a.per_gate) : t1;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j < nv) {
                float w[N], g[N];
                load_weight(a.post, j * N, w);
                if (a.gate)
                    Vec<T>::unpack(__ldg((const uint4 *)((const T *)a.gate + i_gate * a.d) + j), g);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    w[k] = a.scale * (a.gate ? g[k] * w[k] : w[k]);
#pragma unroll
                for (int k = 0; k < N; k += 4)
                    wm[k / 4 * nv + j] = make_float4(w[k], w[k + 1], w[k + 2], w[k + 3]);
            }
        }
        for (; t < end; ++t) {
            if (kAhead) {
                copies_done();
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    hv[i] = ahead[(4 * i) * blockDim.x];
                    yv[i] = ahead[(4 * i + 1) * blockDim.x];
                    zv[i] = ahead[(4 * i + 2) * blockDim.x];
                    rv[i] = ahead[(4 * i + 3) * blockDim.x];
                }
                if (t + 1 < t1)
                    load(t + 1);
            } else {
                load(t);
            }
            Row row;
            float m[6];
#pragma unroll 1
            while (true) {
                Sums<float2> sums;
#pragma unroll
                for (int k = 0; k < 6; ++k)
                    sums.s[k] = both(0.f);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int j = lane + G * i;
                    if (j < nv) {
                        float2 h[P], y[P], z[P], r[P], pw[P], mw[P];
                        from_fours(wp, nv, j, pw);
                        from_fours(wm, nv, j, mw);
                        unpack_pairs(hv[i], h);
                        unpack_pairs(yv[i], y);
                        unpack_pairs(zv[i], z);
                        unpack_pairs(rv[i], r);
#pragma unroll
                        for (int k = 0; k < P; ++k)
                            add_element(sums, h[k], z[k], y[k], r[k], pw[k], mw[k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < 6; ++k)
                    m[k] = sums.s[k].x + sums.s[k].y;
                row_sums<S>(m, red, turn);
                const float fh = row.fh, fy = row.fy;
                if (!row.again(a, m))          // (every lane of the row)
                    break;
                // a row out of range is scaled where it lies: exact but for elements that vanish
                // beside the row's largest
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    float2 x[P];
                    unpack_pairs(hv[i], x);
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        x[k] = mul2(x[k], both(fh == row.fh ? 1.f : row.fh));
                    hv[i] = pack_pairs(x);
                    unpack_pairs(yv[i], x);
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        x[k] = mul2(x[k], both(fy == row.fy ? 1.f : row.fy));
                    yv[i] = pack_pairs(x);
                }
            }
            row.finish(a, m);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int j = lane + G * i;
                if (j < nv) {
                    float2 h[P], y[P], z[P], r[P], pw[P], mw[P];
                    from_fours(wp, nv, j, pw);
                    from_fours(wm, nv, j, mw);
                    unpack_pairs(hv[i], h);
                    unpack_pairs(yv[i], y);
                    unpack_pairs(zv[i], z);
                    unpack_pairs(rv[i], r);
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        row.element(h[k], z[k], y[k], r[k], pw[k], mw[k], h[k], y[k], pre[i][k], sum[i][k]);
                    *((uint4 *)(dR + t * a.d) + j) = pack_pairs(h);
                    *((uint4 *)(dY + t * a.d) + j) = pack_pairs(y);
                }
            }
        }
        if (!a.gated)
            break;
        // S goes to w_post's gradient and to its gate's
        const bool whole = end - t0 == a.per_gate;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j >= nv)
                continue;
            float w[N], g[N];
            load_weight(a.post, j * N, w);
            Vec<T>::unpack(__ldg((const uint4 *)((const T *)a.gate + i_gate * a.d) + j), g);
            float *post = a.part_post + worker * a.d + j * N;
            float *to = (whole ? a.dgate + i_gate * a.d : a.part_gate + shared_at(a, worker, i_gate, first) * a.d) + j * N;
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                float4 q = make_float4(sum[i][k / 2].x, sum[i][k / 2].y, sum[i][k / 2 + 1].x, sum[i][k / 2 + 1].y);
                float4 p = first ? make_float4(0.f, 0.f, 0.f, 0.f) : *(float4 *)(post + k);
                *(float4 *)(post + k) = make_float4(fmaf(a.scale * g[k], q.x, p.x), fmaf(a.scale * g[k + 1], q.y, p.y),
                                                    fmaf(a.scale * g[k + 2], q.z, p.z),
                                                    fmaf(a.scale * g[k + 3], q.w, p.w));
                if (whole) {
                    p = a.add ? *(float4 *)(to + k) : make_float4(0.f, 0.f, 0.f, 0.f);
                    q = make_float4(fmaf(a.scale * w[k], q.x, p.x), fmaf(a.scale * w[k + 1], q.y, p.y),
                                    fmaf(a.scale * w[k + 2], q.z, p.z), fmaf(a.scale * w[k + 3], q.w, p.w));
                }
                *(float4 *)(to + k) = q;
            }
        }
        clear();
    }
    // What a block has summed: a row's lanes each their columns, or with a row a warp the sum of its
    // warps', through their shared memory
    if (S == 32)
        __syncwarp();
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int j = lane + G * i;
        if (j < nv)
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 p = make_float4(pre[i][k / 2].x, pre[i][k / 2].y, pre[i][k / 2 + 1].x, pre[i][k / 2 + 1].y);
                const float4 q = make_float4(sum[i][k / 2].x, sum[i][k / 2].y, sum[i][k / 2 + 1].x, sum[i][k / 2 + 1].y);
                if (S == 32) {
                    wp[k / 4 * nv + j] = p;
                    wm[k / 4 * nv + j] = q;
                } else {
                    *(float4 *)(a.part_pre + worker * a.d + j * N + k) = p;
                    if (!a.gated)
                        *(float4 *)(a.part_post + worker * a.d + j * N + k) = q;
                }
            }
    }
    if (S == 32) {
        __syncthreads();
        const int fours = N / 4 * nv;
        for (int e = threadIdx.x; e < (a.gated ? fours : 2 * fours); e += blockDim.x) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int w = 0; w < kRows; ++w) {
                const float4 v = weights[w * 2 * fours + e];
                s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
            }
            const int at = e % fours;
            float *to = (e < fours ? a.part_pre : a.part_post) + (int64_t)blockIdx.x * a.d;
            *(float4 *)(to + at % nv * N + at / nv * 4) = s;
        }
    }
}

// Any width: the parts lie in memory and are added to by the thread that owns the column.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) k_blocknorm_bwd_any(const Args a)
{
    griddep_start();
    __shared__ __align__(16) float red[2 * 8 * 32];
    int turn = 0;
    float *pre = a.part_pre + (int64_t)blockIdx.x * a.d, *post = a.part_post + (int64_t)blockIdx.x * a.d;
    for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
        pre[j] = post[j] = 0.f;
    const int64_t t1 = first_token(blockIdx.x + 1, gridDim.x, a.T);
    int64_t t = first_token(blockIdx.x, gridDim.x, a.T);
    for (bool first = true; t < t1; first = false) {
        const int64_t i = a.gated ? gate_of(a, t) : 0, end = a.gated ? min(t1, (i + 1) * a.per_gate) : t1;
        const bool whole = end - t == a.per_gate;
        float *to = !a.gated ? nullptr : whole ? a.dgate + i * a.d : a.part_gate + shared_at(a, blockIdx.x, i, first) * a.d;
        if (to && !(whole && a.add))
            for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
                to[j] = 0.f;
        for (; t < end; ++t) {
            const T *H = (const T *)a.R + t * a.d, *Y = (const T *)a.Y + t * a.ldy, *dZ = (const T *)a.dZ + t * a.lddz;
            const T *dH = a.dH ? (const T *)a.dH + t * a.d : nullptr;
            float m[6];
            Row row;
            auto m_at = [&](int j) { return a.scale * (gate_at<T>(a, i, j) * weight_at(a.post, j)); };
            do {
                Sums<float> sums = {};
                for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
                    add_element(sums, Vec<T>::one(H[j]) * row.fh, Vec<T>::one(dZ[j]), Vec<T>::one(Y[j]) * row.fy,
                                dH ? Vec<T>::one(dH[j]) : 0.f, weight_at(a.pre, j), m_at(j));
                for (int k = 0; k < 6; ++k)
                    m[k] = sums.s[k];
                row_sums<kAnyThreads>(m, red, turn);
            } while (row.again(a, m));
            row.finish(a, m);
            for (int j = threadIdx.x; j < a.d; j += kAnyThreads) {
                float dh, dy, s = 0.f, p = pre[j];
                row.element(Vec<T>::one(H[j]) * row.fh, Vec<T>::one(dZ[j]), Vec<T>::one(Y[j]) * row.fy,
                            dH ? Vec<T>::one(dH[j]) : 0.f, weight_at(a.pre, j), m_at(j), dh, dy, p, s);
                ((T *)a.H)[t * a.d + j] = Vec<T>::round(dh);
                ((T *)a.Z)[t * a.d + j] = Vec<T>::round(dy);
                pre[j] = p;
                post[j] = fmaf(a.gated ? a.scale * gate_at<T>(a, i, j) : 1.f, s, post[j]);
                if (to)
                    to[j] = fmaf(whole ? a.scale * weight_at(a.post, j) : 1.f, s, to[j]);
            }
        }
    }
}

// The sums of the workers' parts, in their order, so that the result is the same bits every time.
struct JoinArgs {
    const float *pre, *post, *gate;
    int pre_parts, post_parts;
    float *dw_pre, *dw_post, *dgate;
    Weight w_post;
    const void *one_gate;       // the gate where it is one row for all tokens, in T
    bool one_bf16;
    float scale;
    int d;
    int64_t T, workers, gates, per_gate, looked;
    int runs;
    bool few_gates, add;
};
// dw_pre and dw_post (blockIdx.y): 32 columns and 32 runs of parts a block.  Where S is one for all
// tokens, it makes dw_post and dgate.
__global__ void __launch_bounds__(1024) k_blocknorm_dw(const JoinArgs a)
{
    griddep_start();
    __shared__ float red[32][33];
    const float *part = blockIdx.y == 0 ? a.pre : a.post;
    const int parts = blockIdx.y == 0 ? a.pre_parts : a.post_parts, per = (parts + 31) / 32;
    const int j = blockIdx.x * 32 + threadIdx.x;
    float s = 0.f;
    if (j < a.d)
#pragma unroll 8
        for (int p = threadIdx.y * per, end = min(parts, p + per); p < end; ++p)
            s += __ldg(part + (int64_t)p * a.d + j);
    red[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = warp_sum(red[threadIdx.x][threadIdx.y]);       // row y of the transpose: column y
    const int c = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x > 0 || c >= a.d)
        return;
    if (blockIdx.y == 1 && a.gates <= 1) {
        s *= a.scale;
        if (a.one_gate) {
            const float g = s * weight_at(a.w_post, c);
            a.dgate[c] = a.add ? a.dgate[c] + g : g;
            s *= weight_at(Weight{a.one_gate, a.one_bf16}, c);
        }
    }
    float *to = (blockIdx.y == 0 ? a.dw_pre : a.dw_post) + c;
    *to = a.add ? *to + s : s;
}
// The gates whose tokens several workers had, looked for among all gates, or with more gates than
// workers among those in which a worker's tokens start.  A warp sums 32 columns of a gate's parts, or
// 8 warps do where a gate has many.
__global__ void __launch_bounds__(256) k_blocknorm_dgate(const JoinArgs a)
{
    griddep_start();
    __shared__ float red[8][32];
    const int at_once = 8 / a.runs, run = threadIdx.y % a.runs, j = blockIdx.x * 32 + threadIdx.x;
    for (int64_t y0 = (int64_t)blockIdx.y * at_once; y0 < a.looked; y0 += (int64_t)gridDim.y * at_once) {
        const int64_t y = y0 + threadIdx.y / a.runs;
        float s = 0.f, *to = nullptr;
        if (y < a.looked && j < a.d) {
            int64_t i = y, at;                  // the gate's first part (see shared_at)
            int parts;
            if (a.few_gates) {
                const int64_t w0 = worker_of(i * a.per_gate, a.workers, a.T);
                parts = (int)(worker_of((i + 1) * a.per_gate - 1, a.workers, a.T) - w0) + 1;
                at = w0 + i;
            } else {
                // a worker has a gate's tokens at least, so that two share one at most: the last of
                // worker y's and the first of the next one's, unless that one's tokens start with it
                const int64_t t = first_token(y + 1, a.workers, a.T);
                i = (uint32_t)t / (uint32_t)a.per_gate;
                parts = t > i * a.per_gate ? 2 : 1;
                at = 2 * y + 1;
            }
            if (parts > 1) {                    // (else one worker has written it)
                to = a.dgate + i * a.d + j;
                const float *part = a.gate + at * a.d + j;
                const int per = (parts + a.runs - 1) / a.runs;
#pragma unroll 8
                for (int p = run * per, end = min(parts, p + per); p < end; ++p)
                    s += __ldg(part + (int64_t)p * a.d);
            }
        }
        if (a.runs > 1) {
            red[threadIdx.y][threadIdx.x] = s;
            __syncthreads();
            s = 0.f;
            if (run == 0)
                for (int r = 0; r < a.runs; ++r)
                    s += red[threadIdx.y + r][threadIdx.x];
            __syncthreads();
        }
        if (to && run == 0) {
            s *= a.scale * weight_at(a.w_post, j);
            *to = a.add ? *to + s : s;
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------

constexpr int kPieces = 4;

template <typename T>
bool pieces(int d, int64_t ld, int most)
{
    constexpr int N = Vec<T>::N;
    return d % N == 0 && ld % N == 0 && d / N <= 1024 * most;
}

template <typename T, int S, bool EXACT, int C>
cudaError_t fwd_rows(const Args &a, int lanes, cudaStream_t s)
{
    constexpr int kRows = Shape<S>::kRows;
    const int64_t blocks = (a.T + kRows - 1) / kRows;
    const int64_t grid = std::min<int64_t>(blocks, (int64_t)1 << 30);
    const int threads = S == 32 ? 256 : lanes;
    return a.gate ? launch(k_blocknorm<T, S, EXACT, C, true>, grid, threads, a, s)
                  : launch(k_blocknorm<T, S, EXACT, C, false>, grid, threads, a, s);
}

template <typename T>
cudaError_t fwd(const Args &a, cudaStream_t s)
{
    if (!pieces<T>(a.d, a.ldy, kPieces))
        return launch(k_blocknorm_any<T>, std::min<int64_t>(a.T, (int64_t)1 << 30), kAnyThreads, a, s);
    const int nv = a.d / Vec<T>::N, g = lanes_of(nv, kPieces);
    if (g == 32)
        return nv <= 32 ? fwd_rows<T, 32, false, 1>(a, g, s)
             : nv <= 64 ? fwd_rows<T, 32, false, 2>(a, g, s)
                        : fwd_rows<T, 32, false, kPieces>(a, g, s);
    if (g == 64 && nv == 64 * kPieces)
        return fwd_rows<T, 64, true, kPieces>(a, g, s);
    if (g == 128 && nv == 128 * kPieces)
        return fwd_rows<T, 128, true, kPieces>(a, g, s);
    if (g == 256 && nv == 256 * kPieces)
        return fwd_rows<T, 256, true, kPieces>(a, g, s);
    return g <= 256 ? fwd_rows<T, 256, false, kPieces>(a, g, s)
         : g <= 512 ? fwd_rows<T, 512, false, kPieces>(a, g, s)
                    : fwd_rows<T, 1024, false, kPieces>(a, g, s);
}

// Pieces a lane of the gradient holds of rows of nv.  With two of bf16, two blocks of up to 256 threads
// are on an SM (one of 512 with one piece: 16384 rows of 4096 173 us when two took 137); three of fp32
// keep more on the way (16384 of 4096 238 us, 275 with four; 4173 of 2056 37.3, 41.6).
template <typename T>
int pieces_of(int nv) { return nv <= 32 ? 1 : sizeof(T) == 2 || nv <= 512 ? 2 : nv <= 512 * 3 ? 3 : 4; }

// The gradient's grid
struct Plan {
    int threads, rows_at_once;
    int64_t workers;
    size_t part, gate_parts;          // floats
};

template <typename T>
Plan plan_of(int64_t T_, int d, bool registers, int64_t gates)
{
    Plan p;
    const int nv = d / Vec<T>::N;
    int per_sm;
    if (!registers) {
        p.threads = kAnyThreads;
        p.rows_at_once = 1;
        per_sm = 2;
    } else {
        const int g = lanes_of(nv, pieces_of<T>(nv));
        p.threads = g == 32 ? 256 : g;
        p.rows_at_once = g == 32 ? 8 : 1;
        per_sm = std::max(1, std::min(8, 512 / p.threads));
    }
    p.workers = std::min<int64_t>(T_, (int64_t)device_sms() * per_sm * p.rows_at_once);
    p.part = (size_t)p.workers * d;
    // (none where every gate is one worker's)
    const int64_t per = p.workers > 0 && T_ % p.workers == 0 ? T_ / p.workers : 1;
    const bool shared = gates > 1 && gates < T_ && per % (T_ / gates) != 0;
    p.gate_parts = shared ? (size_t)(p.workers + std::min(p.workers, gates)) * d : 0;
    return p;
}

template <typename T>
bool bwd_registers(const Args &a) { return pieces<T>(a.d, a.ldy, 2) && a.lddz % Vec<T>::N == 0; }

template <typename T, int S, int C>
cudaError_t bwd_rows(const Plan &p, const Args &a, cudaStream_t s)
{
    // m and w_pre, and the next row's pieces
    const size_t smem = (size_t)p.rows_at_once * 2 * a.d * sizeof(float) + (is_ahead<S, C> ? (size_t)p.threads * C * 64 : 0);
    cudaError_t e = cudaFuncSetAttribute(k_blocknorm_bwd<T, S, C>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         147456);   // rows of 6144 fp32: 48 KB, and 96 on the way
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(k_blocknorm_bwd<T, S, C>,
                         dim3((unsigned)((p.workers + p.rows_at_once - 1) / p.rows_at_once)), dim3(p.threads), smem, s,
                         a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t bwd(Args a, int64_t gates, float *dw_post, float *dw_pre, float *ws, cudaStream_t s)
{
    const bool registers = bwd_registers<T>(a);
    const Plan p = plan_of<T>(a.T, a.d, registers, gates);
    a.workers = p.workers;
    a.gated = gates > 1;
    a.part_pre = ws;
    a.part_post = ws + p.part;
    a.part_gate = ws + 2 * p.part;
    a.few_gates = gates < p.workers;
    const int nv = a.d / Vec<T>::N;
    cudaError_t e;
    if (!registers)
        e = launch(k_blocknorm_bwd_any<T>, p.workers, kAnyThreads, a, s);
    else if (p.rows_at_once > 1)
        e = nv <= 32 ? bwd_rows<T, 32, 1>(p, a, s) : bwd_rows<T, 32, 2>(p, a, s);
    else if (nv <= 512)
        e = bwd_rows<T, 256, 2>(p, a, s);
    else if constexpr (sizeof(T) == 4)
        e = pieces_of<T>(nv) == 3 ? bwd_rows<T, 512, 3>(p, a, s) : bwd_rows<T, 512, 4>(p, a, s);
    else
        e = p.threads <= 512 ? bwd_rows<T, 512, 2>(p, a, s) : bwd_rows<T, 1024, 2>(p, a, s);
    if (e != cudaSuccess)
        return e;
    const int64_t looked = gates > 1 ? std::min(gates, p.workers - 1) : 0;
    const int blocks = (int)((p.workers + p.rows_at_once - 1) / p.rows_at_once);
    const JoinArgs j{a.part_pre, a.part_post, a.part_gate, blocks, gates > 1 ? (int)p.workers : blocks, dw_pre, dw_post,
                     a.dgate, a.post, gates == 1 ? a.gate : nullptr, sizeof(T) == 2, a.scale, a.d, a.T, p.workers,
                     gates, a.per_gate, looked, p.workers >= 8 * gates ? 8 : 1, a.few_gates, a.add};
    const unsigned across = (unsigned)((a.d - 1) / 32 + 1);
    count_launch();
    e = launch_dependent(k_blocknorm_dw, dim3(across, 2), dim3(32, 32), 0, s, j);
    if (e == cudaSuccess && looked > 0) {
        count_launch();
        e = launch_dependent(k_blocknorm_dgate,
                             dim3(across, (unsigned)std::min<int64_t>((looked * j.runs + 7) / 8, 65535)), dim3(32, 8),
                             0, s, j);
    }
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t blocknorm_fwd(sn_dtype dt, const void *Y, int64_t ldy, const void *R, const void *gate, int64_t gates,
                          sn_dtype wdt, const void *w_post, const void *w_pre, int64_t T, int d, float eps,
                          float scale, void *H, void *Z, cudaStream_t s)
{
    Args a = {};
    a.Y = Y;
    a.R = R;
    a.gate = gate;
    a.post = Weight{w_post, wdt == SN_BF16};
    a.pre = Weight{w_pre, wdt == SN_BF16};
    a.T = T;
    a.ldy = ldy;
    a.per_gate = T / std::max<int64_t>(1, gates);
    a.d = d;
    a.inverse_d = 1.f / (float)d;
    a.eps = eps;
    a.scale = scale;
    a.least = least_sum(d, eps);
    a.most = most_sum(eps);
    a.H = H;
    a.Z = Z;
    return dt == SN_BF16 ? fwd<__nv_bfloat16>(a, s) : fwd<float>(a, s);
}

size_t blocknorm_bwd_workspace(int64_t T, int d, int64_t gates)
{
    // the most that any type and alignment of this width takes
    size_t most = 0;
    auto take = [&](const Plan &p) { most = std::max(most, 2 * p.part + p.gate_parts); };
    take(plan_of<float>(T, d, false, gates));
    if (pieces<float>(d, d, 2))
        take(plan_of<float>(T, d, true, gates));
    if (pieces<__nv_bfloat16>(d, d, 2))
        take(plan_of<__nv_bfloat16>(T, d, true, gates));
    return most * sizeof(float);
}

cudaError_t blocknorm_bwd(sn_dtype dt, const void *dZ, int64_t lddz, const void *H, const void *Y, int64_t ldy,
                          const void *dH, const void *gate, int64_t gates, sn_dtype wdt, const void *w_post,
                          const void *w_pre, int64_t T, int d, float eps, float scale, void *dY, void *dR,
                          float *dw_post, float *dw_pre, float *dgate, bool accumulate, float *ws, cudaStream_t s)
{
    Args a = {};
    a.Y = Y;
    a.R = H;
    a.dZ = dZ;
    a.dH = dH;
    a.gate = gate;
    a.post = Weight{w_post, wdt == SN_BF16};
    a.pre = Weight{w_pre, wdt == SN_BF16};
    a.T = T;
    a.ldy = ldy;
    a.lddz = lddz;
    a.per_gate = T / std::max<int64_t>(1, gates);
    a.d = d;
    a.inverse_d = 1.f / (float)d;
    a.eps = eps;
    a.scale = scale;
    a.least = least_sum(d, eps);
    a.most = most_sum(eps);
    a.H = dR;
    a.Z = dY;
    a.dgate = dgate;
    a.add = accumulate;
    return dt == SN_BF16 ? bwd<__nv_bfloat16>(a, gates, dw_post, dw_pre, ws, s)
                         : bwd<float>(a, gates, dw_post, dw_pre, ws, s);
}

}  // namespace sn
