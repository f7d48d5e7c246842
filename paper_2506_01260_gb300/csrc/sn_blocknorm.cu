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
    float eps, scale;
    float least, most;          // of a row's sum of squares that is taken as it is
    void *H, *Z;                // the gradient: dR, dY
    // the gradient's work: chunks of `rows` tokens, `split` of them to a gate's tokens
    int64_t chunks, rows, split;
    float *dgate;               // written where a chunk has all of a gate's tokens
    bool add;
    float *part_pre, *part_post;    // [workers, d]
    float *part_gate;               // [chunks, d], where split > 1
    bool prefetch;
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

template <typename T, int S, bool EXACT, int C>
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
        uint4 yv[C], rv[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            const bool in = live && j < nv;
            yv[i] = in ? *((const uint4 *)(Y + t * a.ldy) + j) : make_uint4(0, 0, 0, 0);
            rv[i] = in ? *((const uint4 *)(R + t * a.d) + j) : make_uint4(0, 0, 0, 0);
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
        const T *g = gate && live ? gate + gate_of(a, t) * a.d : nullptr;
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
                if (g) {
                    float2 m[P];
                    unpack_pairs(__ldg((const uint4 *)g + j), m);
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

// A row's sums, of h and y scaled by their factors where their squares ask for it
struct Sums {
    float s[6];     // h h, g h, y y, m y g, m y h, m y dh
    __device__ __forceinline__ void add(float h, float g, float y, float m, float r)
    {
        const float my = m * y;
        s[0] = fmaf(h, h, s[0]);
        s[1] = fmaf(g, h, s[1]);
        s[2] = fmaf(y, y, s[2]);
        s[3] = fmaf(my, g, s[3]);
        s[4] = fmaf(my, h, s[4]);
        s[5] = fmaf(my, r, s[5]);
    }
};
// What the elements of a row share
struct Row {
    float fh, fy;               // the factors, 1 for almost every row
    float r2, c2, a2, half2;    // 1 / rms(h f), mean(g n2), and 1 / rms(h) in two factors
    float r1, c1, a1, half1;
    __device__ __forceinline__ void finish(const Args &a, const float (&s)[6])
    {
        const float n = (float)a.d;
        r2 = root_of(s[0] / n + a.eps * fh * fh);
        r1 = root_of(s[2] / n + a.eps * fy * fy);
        half2 = half_of(fh);
        half1 = half_of(fy);
        a2 = r2 * half2;
        a1 = r1 * half1;
        c2 = s[1] / n * r2;
        const float ey = fmaf(fmaf(-r2 * c2, s[4], s[3]) * a2, half2, s[5]);
        c1 = ey / n * r1;
    }
    // dh' and dy of an element, and n1 and n2
    __device__ __forceinline__ void element(float h, float g, float y, float m, float r, float &dh, float &dy,
                                            float &n1, float &n2) const
    {
        n2 = h * r2;
        n1 = y * r1;
        dh = fmaf(fmaf(-n2, c2, g) * a2, half2, r);
        dy = fmaf(-n1, c1, m * dh) * a1 * half1;
    }
};

// Threads of an SM that registers are kept low enough for
template <typename T, int S, int C>
constexpr int kBwdResident = S > 512 ? S : S == 320 ? 640 : S == 32 && C == 1 ? 768 : 512;

// A worker (a warp or a block) walks its chunks of tokens, a row at a time, and keeps dw_pre and
// S of its columns in registers; m and w_pre lie in shared memory, each thread's own columns.
template <typename T, int S, int C>
__global__ void __launch_bounds__(Shape<S>::kThreads, kBwdResident<T, S, C> / Shape<S>::kThreads)
    k_blocknorm_bwd(const Args a)
{
    griddep_start();
    extern __shared__ __align__(16) float weights[];
    constexpr int N = Vec<T>::N, kRows = Shape<S>::kRows;
    __shared__ __align__(16) float red[2 * 6 * 32];
    int turn = 0;
    const int G = Shape<S>::lanes(), lane = S == 32 ? threadIdx.x % 32 : threadIdx.x;
    const int warp = S == 32 ? threadIdx.x / 32 : 0, nv = a.d / N;
    const T *Y = (const T *)a.Y, *H = (const T *)a.R, *dZ = (const T *)a.dZ, *dH = (const T *)a.dH;
    T *dR = (T *)a.H, *dY = (T *)a.Z;
    float *wp = weights + (int64_t)warp * 2 * a.d, *wm = wp + a.d;
    const int64_t worker = (int64_t)blockIdx.x * kRows + warp, workers = (int64_t)gridDim.x * kRows;
    float pre[C][N];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int j = lane + G * i;
#pragma unroll
        for (int k = 0; k < N; ++k)
            pre[i][k] = 0.f;
        if (j < nv) {
            float w[N];
            load_weight(a.pre, j * N, w);
#pragma unroll
            for (int k = 0; k < N; k += 4)
                *(float4 *)(wp + j * N + k) = make_float4(w[k], w[k + 1], w[k + 2], w[k + 3]);
        }
    }
    // The next row's loads run before this row's sums meet, where registers allow
    constexpr bool kEarly = C == 1 || sizeof(T) == 4;
    bool first = true;
    for (int64_t c = worker; c < a.chunks; c += workers, first = false) {
        const int64_t i_gate = c / a.split, in = c - i_gate * a.split;
        const int64_t t0 = i_gate * a.per_gate + in * a.rows, t1 = min(t0 + a.rows, (i_gate + 1) * a.per_gate);
        float sum[C][N];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
#pragma unroll
            for (int k = 0; k < N; ++k)
                sum[i][k] = 0.f;
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
                    *(float4 *)(wm + j * N + k) = make_float4(w[k], w[k + 1], w[k + 2], w[k + 3]);
            }
        }
        uint4 hv[C], yv[C], zv[C], rv[C], hn[C], yn[C], zn[C], rn[C];
        auto load = [&](int64_t t, uint4 (&h)[C], uint4 (&y)[C], uint4 (&z)[C], uint4 (&r)[C]) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int j = lane + G * i;
                const bool live = t < t1 && j < nv;
                h[i] = live ? *((const uint4 *)(H + t * a.d) + j) : make_uint4(0, 0, 0, 0);
                y[i] = live ? *((const uint4 *)(Y + t * a.ldy) + j) : make_uint4(0, 0, 0, 0);
                z[i] = live ? *((const uint4 *)(dZ + t * a.lddz) + j) : make_uint4(0, 0, 0, 0);
                r[i] = live && dH ? *((const uint4 *)(dH + t * a.d) + j) : make_uint4(0, 0, 0, 0);
            }
        };
        if (kEarly)
            load(t0, hn, yn, zn, rn);
        for (int64_t t = t0; t < t1; ++t) {
            if (kEarly) {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    hv[i] = hn[i];
                    yv[i] = yn[i];
                    zv[i] = zn[i];
                    rv[i] = rn[i];
                }
                load(t + 1, hn, yn, zn, rn);
            } else {
                load(t, hv, yv, zv, rv);
            }
            const int64_t later = t + (kEarly ? 2 : 1);
            if (a.prefetch && lane < 4 && later < t1) {
                const T *p = lane == 0 ? H + later * a.d : lane == 1 ? Y + later * a.ldy
                           : lane == 2 ? dZ + later * a.lddz : dH ? dH + later * a.d : nullptr;
                if (p)
                    prefetch_l2(p, (uint32_t)(a.d * sizeof(T)));
            }
            Sums m;
            Row row;
            row.fh = row.fy = 1.f;
#pragma unroll 1
            while (true) {                     // again for a row out of range
#pragma unroll
                for (int k = 0; k < 6; ++k)
                    m.s[k] = 0.f;
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int j = lane + G * i;
                    if (j < nv) {
                        float h[N], y[N], z[N], r[N];
                        Vec<T>::unpack(hv[i], h);
                        Vec<T>::unpack(yv[i], y);
                        Vec<T>::unpack(zv[i], z);
                        Vec<T>::unpack(rv[i], r);
#pragma unroll
                        for (int k = 0; k < N; ++k)
                            m.add(h[k] * row.fh, z[k] * wp[j * N + k], y[k] * row.fy, wm[j * N + k], r[k]);
                    }
                }
                row_reduce<S, 6, false>(m.s, red, turn);
                const bool h_again = row.fh == 1.f && !in_range(a, m.s[0]);
                const bool y_again = row.fy == 1.f && !in_range(a, m.s[2]);
                if (!(h_again || y_again))     // (every lane of the row)
                    break;
                if (h_again)
                    row.fh = factor_of(a, m.s[0]);
                if (y_again)
                    row.fy = factor_of(a, m.s[2]);
            }
            row.finish(a, m.s);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int j = lane + G * i;
                if (j < nv) {
                    float h[N], y[N], z[N], r[N];
                    Vec<T>::unpack(hv[i], h);
                    Vec<T>::unpack(yv[i], y);
                    Vec<T>::unpack(zv[i], z);
                    Vec<T>::unpack(rv[i], r);
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        float dh, dy, n1, n2;
                        row.element(h[k] * row.fh, z[k] * wp[j * N + k], y[k] * row.fy, wm[j * N + k], r[k], dh, dy,
                                    n1, n2);
                        pre[i][k] = fmaf(z[k], n2, pre[i][k]);
                        sum[i][k] = fmaf(dh, n1, sum[i][k]);
                        h[k] = dh;
                        y[k] = dy;
                    }
                    *((uint4 *)(dR + t * a.d) + j) = Vec<T>::pack(h);
                    *((uint4 *)(dY + t * a.d) + j) = Vec<T>::pack(y);
                }
            }
        }
        // the chunk's S goes to w_post's gradient and to its gate's
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = lane + G * i;
            if (j >= nv)
                continue;
            float w[N], g[N];
            load_weight(a.post, j * N, w);
            if (a.gate)
                Vec<T>::unpack(__ldg((const uint4 *)((const T *)a.gate + i_gate * a.d) + j), g);
            float *post = a.part_post + worker * a.d + j * N;
            float *to = a.split > 1 ? a.part_gate + c * a.d + j * N : a.dgate + i_gate * a.d + j * N;
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                float4 p = first ? make_float4(0.f, 0.f, 0.f, 0.f) : *(float4 *)(post + k);
                p.x = fmaf(a.scale * (a.gate ? g[k] : 1.f), sum[i][k], p.x);
                p.y = fmaf(a.scale * (a.gate ? g[k + 1] : 1.f), sum[i][k + 1], p.y);
                p.z = fmaf(a.scale * (a.gate ? g[k + 2] : 1.f), sum[i][k + 2], p.z);
                p.w = fmaf(a.scale * (a.gate ? g[k + 3] : 1.f), sum[i][k + 3], p.w);
                *(float4 *)(post + k) = p;
                if (a.gate) {
                    float4 q = make_float4(sum[i][k], sum[i][k + 1], sum[i][k + 2], sum[i][k + 3]);
                    if (a.split == 1) {
                        const float4 was = a.add ? *(float4 *)(to + k) : make_float4(0.f, 0.f, 0.f, 0.f);
                        q = make_float4(fmaf(a.scale * w[k], q.x, was.x), fmaf(a.scale * w[k + 1], q.y, was.y),
                                        fmaf(a.scale * w[k + 2], q.z, was.z), fmaf(a.scale * w[k + 3], q.w, was.w));
                    }
                    *(float4 *)(to + k) = q;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int j = lane + G * i;
        if (j < nv)
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
                *(float4 *)(a.part_pre + worker * a.d + j * N + k) =
                    make_float4(pre[i][k], pre[i][k + 1], pre[i][k + 2], pre[i][k + 3]);
                if (first)                     // no chunk was this worker's
                    *(float4 *)(a.part_post + worker * a.d + j * N + k) = zero;
            }
    }
}

// Any width: the parts lie in memory and are added to by the thread that owns the column.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) k_blocknorm_bwd_any(const Args a)
{
    griddep_start();
    __shared__ __align__(16) float red[2 * 6 * 32];
    int turn = 0;
    float *pre = a.part_pre + (int64_t)blockIdx.x * a.d, *post = a.part_post + (int64_t)blockIdx.x * a.d;
    for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
        pre[j] = post[j] = 0.f;
    for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int64_t i = c / a.split, in = c - i * a.split;
        const int64_t t0 = i * a.per_gate + in * a.rows, t1 = min(t0 + a.rows, (i + 1) * a.per_gate);
        float *to = !a.gate ? nullptr : a.split > 1 ? a.part_gate + c * a.d : a.dgate + i * a.d;
        if (to && (a.split > 1 || !a.add))
            for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
                to[j] = 0.f;
        for (int64_t t = t0; t < t1; ++t) {
            const T *H = (const T *)a.R + t * a.d, *Y = (const T *)a.Y + t * a.ldy, *dZ = (const T *)a.dZ + t * a.lddz;
            const T *dH = a.dH ? (const T *)a.dH + t * a.d : nullptr;
            Sums m;
            Row row;
            row.fh = row.fy = 1.f;
            auto m_at = [&](int j) { return a.scale * (gate_at<T>(a, i, j) * weight_at(a.post, j)); };
            while (true) {
                for (int k = 0; k < 6; ++k)
                    m.s[k] = 0.f;
                for (int j = threadIdx.x; j < a.d; j += kAnyThreads)
                    m.add(Vec<T>::one(H[j]) * row.fh, Vec<T>::one(dZ[j]) * weight_at(a.pre, j),
                          Vec<T>::one(Y[j]) * row.fy, m_at(j), dH ? Vec<T>::one(dH[j]) : 0.f);
                row_reduce<kAnyThreads, 6, false, true>(m.s, red, turn);
                const bool h_again = row.fh == 1.f && !in_range(a, m.s[0]);
                const bool y_again = row.fy == 1.f && !in_range(a, m.s[2]);
                if (!(h_again || y_again))
                    break;
                if (h_again)
                    row.fh = factor_of(a, m.s[0]);
                if (y_again)
                    row.fy = factor_of(a, m.s[2]);
            }
            row.finish(a, m.s);
            for (int j = threadIdx.x; j < a.d; j += kAnyThreads) {
                const float z = Vec<T>::one(dZ[j]), w = weight_at(a.post, j);
                float dh, dy, n1, n2;
                row.element(Vec<T>::one(H[j]) * row.fh, z * weight_at(a.pre, j), Vec<T>::one(Y[j]) * row.fy, m_at(j),
                            dH ? Vec<T>::one(dH[j]) : 0.f, dh, dy, n1, n2);
                ((T *)a.H)[t * a.d + j] = Vec<T>::round(dh);
                ((T *)a.Z)[t * a.d + j] = Vec<T>::round(dy);
                pre[j] = fmaf(z, n2, pre[j]);
                post[j] = fmaf(a.scale * gate_at<T>(a, i, j), dh * n1, post[j]);
                if (to)
                    to[j] = fmaf(a.split > 1 ? 1.f : a.scale * w, dh * n1, to[j]);
            }
        }
    }
}

// The sums of parts, in their order: 32 columns and 32 runs of parts a block, so that the result
// is the same bits every time.  blockIdx.y: dw_pre, dw_post, then the gates whose tokens were split.
struct JoinArgs {
    const float *pre, *post, *gate;
    float *dw_pre, *dw_post, *dgate;
    Weight w_post;
    float scale;
    int parts, split, d;
    int64_t gates;          // rows of dgate that are joined
    bool add;
};
__global__ void __launch_bounds__(1024) k_blocknorm_join(const JoinArgs a)
{
    griddep_start();
    __shared__ float red[32][33];
    for (int64_t y = blockIdx.y; y < 2 + a.gates; y += gridDim.y) {
        const float *part = y == 0 ? a.pre : y == 1 ? a.post : a.gate + (y - 2) * a.split * a.d;
        const int parts = y < 2 ? a.parts : a.split, per = (parts + 31) / 32;
        const int j = blockIdx.x * 32 + threadIdx.x;
        float s = 0.f;
        if (j < a.d)
#pragma unroll 8
            for (int p = threadIdx.y * per, end = min(parts, p + per); p < end; ++p)
                s += __ldg(part + (int64_t)p * a.d + j);
        red[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        s = warp_sum(red[threadIdx.x][threadIdx.y]);
        const int c = blockIdx.x * 32 + threadIdx.y;
        if (threadIdx.x == 0 && c < a.d) {
            float *to = y == 0 ? a.dw_pre : y == 1 ? a.dw_post : a.dgate + (y - 2) * a.d;
            if (y >= 2)
                s *= a.scale * weight_at(a.w_post, c);
            to[c] = a.add ? to[c] + s : s;
        }
        __syncthreads();
    }
}

// ---- launches ------------------------------------------------------------------------------------

constexpr int kPieces = 4, kBwdPieces = 2;

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
    return launch(k_blocknorm<T, S, EXACT, C>, std::min<int64_t>(blocks, (int64_t)1 << 30), S == 32 ? 256 : lanes, a,
                  s);
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
    if (g == 128 && nv == 128 * kPieces)
        return fwd_rows<T, 128, true, kPieces>(a, g, s);
    if (g == 256 && nv == 256 * kPieces)
        return fwd_rows<T, 256, true, kPieces>(a, g, s);
    return g <= 256 ? fwd_rows<T, 256, false, kPieces>(a, g, s)
         : g <= 512 ? fwd_rows<T, 512, false, kPieces>(a, g, s)
                    : fwd_rows<T, 1024, false, kPieces>(a, g, s);
}

// The gradient's grid and its division of the tokens.  Without a gate, and with one row of it, every
// worker has one chunk; with more, a gate's tokens are divided into about four chunks a worker, of
// at least eight tokens (a chunk writes its S).
struct Plan {
    int threads, rows_at_once;
    int64_t workers, chunks, rows, split;
    size_t part, gate_parts;          // floats
};

template <typename T>
Plan plan_of(int64_t T_, int d, bool registers, int64_t gates)
{
    Plan p;
    const int nv = d / Vec<T>::N, sms = device_sms();
    int per_sm;
    if (!registers) {
        p.threads = kAnyThreads;
        p.rows_at_once = 1;
        per_sm = 2;
    } else {
        const int g = nv <= 64 ? 32 : lanes_of(nv, nv <= 512 ? 1 : kBwdPieces);
        p.threads = g == 32 ? 256 : g;
        p.rows_at_once = g == 32 ? 8 : 1;
        per_sm = std::max(1, std::min(4, (g <= 320 && sizeof(T) == 4 ? 640 : 512) / p.threads));
    }
    p.workers = std::min<int64_t>((T_ + p.rows_at_once - 1) / p.rows_at_once, (int64_t)sms * per_sm) * p.rows_at_once;
    const int64_t n = std::max<int64_t>(1, gates), per_gate = T_ / n;
    const int64_t want = n == 1 ? (T_ + p.workers - 1) / p.workers
                                : std::max<int64_t>(8, (T_ + 4 * p.workers - 1) / (4 * p.workers));
    p.rows = std::min(want, per_gate);
    p.split = (per_gate + p.rows - 1) / p.rows;
    p.chunks = n * p.split;
    p.part = (size_t)p.workers * d;
    p.gate_parts = gates > 0 && p.split > 1 ? (size_t)p.chunks * d : 0;
    return p;
}

template <typename T>
bool bwd_registers(const Args &a) { return pieces<T>(a.d, a.ldy, kBwdPieces) && a.lddz % Vec<T>::N == 0; }

template <typename T, int S, int C>
cudaError_t bwd_rows(const Plan &p, const Args &a, cudaStream_t s)
{
    const size_t smem = (size_t)p.rows_at_once * 2 * a.d * sizeof(float);
    cudaError_t e = cudaFuncSetAttribute(k_blocknorm_bwd<T, S, C>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         131072);   // of rows of 16384 bf16
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(k_blocknorm_bwd<T, S, C>, dim3((unsigned)(p.workers / p.rows_at_once)), dim3(p.threads), smem,
                         s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t bwd(Args a, int64_t gates, float *dw_post, float *dw_pre, float *ws, cudaStream_t s)
{
    const bool registers = bwd_registers<T>(a);
    const Plan p = plan_of<T>(a.T, a.d, registers, gates);
    a.chunks = p.chunks;
    a.rows = p.rows;
    a.split = p.split;
    a.part_pre = ws;
    a.part_post = ws + p.part;
    a.part_gate = ws + 2 * p.part;
    const int nv = a.d / Vec<T>::N;
    cudaError_t e;
    if (!registers)
        e = launch(k_blocknorm_bwd_any<T>, p.workers, kAnyThreads, a, s);
    else if (p.rows_at_once > 1)
        e = nv <= 32 ? bwd_rows<T, 32, 1>(p, a, s) : bwd_rows<T, 32, 2>(p, a, s);
    else if (nv <= 512)
        e = p.threads <= 256 ? bwd_rows<T, 256, 1>(p, a, s) : bwd_rows<T, 512, 1>(p, a, s);
    else if (sizeof(T) == 4 && p.threads <= 320)
        e = bwd_rows<T, 320, kBwdPieces>(p, a, s);
    else
        e = p.threads <= 512 ? bwd_rows<T, 512, kBwdPieces>(p, a, s) : bwd_rows<T, 1024, kBwdPieces>(p, a, s);
    if (e != cudaSuccess)
        return e;
    const int64_t joined = p.gate_parts ? gates : 0;
    const JoinArgs j{a.part_pre, a.part_post, a.part_gate, dw_pre, dw_post, a.dgate, a.post, a.scale,
                     (int)p.workers, (int)p.split, a.d, joined, a.add};
    count_launch();
    e = launch_dependent(k_blocknorm_join, dim3((unsigned)((a.d - 1) / 32 + 1),
                                                (unsigned)std::min<int64_t>(2 + joined, 65535)),
                         dim3(32, 32), 0, s, j);
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
    if (pieces<float>(d, d, kBwdPieces))
        take(plan_of<float>(T, d, true, gates));
    if (pieces<__nv_bfloat16>(d, d, kBwdPieces))
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
    a.eps = eps;
    a.scale = scale;
    a.least = least_sum(d, eps);
    a.most = most_sum(eps);
    a.H = dR;
    a.Z = dY;
    a.dgate = dgate;
    a.add = accumulate;
    a.prefetch = (size_t)d * (dt == SN_BF16 ? 2 : 4) >= 4096;
    return dt == SN_BF16 ? bwd<__nv_bfloat16>(a, gates, dw_post, dw_pre, ws, s)
                         : bwd<float>(a, gates, dw_post, dw_pre, ws, s);
}

}  // namespace sn
