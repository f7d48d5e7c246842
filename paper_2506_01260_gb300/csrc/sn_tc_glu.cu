// sn_tc_glu.cu — the gated pair of projections of a feed-forward block, and its gradients, on the
// tcgen05 tensor cores.
//
//   G = X Wg^T,  U = X Wu^T,  H = act(G) . U                     X [T, d], Wg and Wu [f, d]
//   dG = dH . U . act'(G),  dU = dH . act(G)                     from the stored G and U
//   dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X
//
// Products read bf16 and accumulate in fp32 (TMEM); every output is rounded once.  dG and dU are
// outputs and the operands of the products behind them, so they are rounded to bf16 in between, as
// the stored G and U are: the tensor cores read 16 bits.
#include <algorithm>
#include <atomic>

#include "sn_tc.cuh"
#include "sn_tc_kernels.cuh"
#include "sn_vec.cuh"

namespace sn {
namespace tc {
namespace {

enum { GLU_FWD = 0, GLU_DX = 1, GLU_DW = 2 };

// ---- the activations ---------------------------------------------------------------------

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// gelu's tanh form is g sigmoid(2 x), x = sqrt(2 / pi) (g + 0.044715 g^3)
constexpr float kTanhA = 1.5957691216057308f, kTanhB = 0.044715f;

// act(g); with `slope` also act'(g).  The shares p of g are taken as sigmoids and as erfc, whose
// relative error does not grow where they vanish.
template <bool SLOPE>
__device__ __forceinline__ float activate(float g, int act, float *slope)
{
    float p;
    switch (act) {
    case SN_ACT_SILU:
        p = sigmoid(g);
        if (SLOPE)
            *slope = fmaf(g * p, 1.f - p, p);
        return g * p;
    case SN_ACT_GELU:
        p = 0.5f * erfcf(-0.7071067811865476f * g);
        if (SLOPE)
            *slope = fmaf(g, 0.3989422804014327f * __expf(-0.5f * g * g), p);
        return g * p;
    case SN_ACT_GELU_TANH:
        p = sigmoid(kTanhA * g * fmaf(kTanhB * g, g, 1.f));
        if (SLOPE) {
            const float q = p * (1.f - p);                  // 0 where g^2 may pass fp32's range
            *slope = q > 0.f ? fmaf(g * q, kTanhA * fmaf(3.f * kTanhB * g, g, 1.f), p) : p;
        }
        return g * p;
    default:
        if (SLOPE)
            *slope = g > 0.f ? 1.f : 0.f;
        return fmaxf(g, 0.f);
    }
}

// ---- pairs of CTAs -----------------------------------------------------------------------
// With CG = 2 the two CTAs of a cluster share one 256 x 256 tile: each holds 128 rows of A and 128
// of B's 256 rows in its shared memory and 128 rows of the accumulator in its TMEM; the first CTA
// (the leader) issues the products for both.

// the address of the leader's `a`
__device__ __forceinline__ uint32_t leaders(uint32_t a)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
template <int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *m, int x, int y, uint32_t bar)
{
    if (CG == 1)
        tma_load_2d(dst, m, x, y, bar);
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
            "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(m), "r"(x), "r"(y), "r"(bar)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void alloc_columns(uint32_t dst_smem, uint32_t ncols)
{
    if (CG == 1) {
        tmem_alloc(dst_smem, ncols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem),
                     "r"(ncols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void free_columns(uint32_t taddr, uint32_t ncols)
{
    if (CG == 1)
        tmem_dealloc(taddr, ncols);
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void multiply(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                         uint32_t accumulate)
{
    if (CG == 1)
        mma_bf16(d_tmem, adesc, bdesc, idesc, accumulate);
    else
        asm volatile(
            "{ .reg .pred p; setp.ne.u32 p, %4, 0; "
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d_tmem),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
            : "memory");
}
// Arrive on `bar` (of both CTAs) once every product issued so far has completed
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if (CG == 1)
        mma_commit(bar);
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
            "[%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
}
// Arrive on the leader's `bar`
template <int CG>
__device__ __forceinline__ void arrive_leader(uint32_t bar)
{
    if (CG == 1)
        mbar_arrive(bar);
    else
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leaders(bar))
                     : "memory");
}
template <int CG>
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity)
{
    if (CG == 1)
        return mbar_test(bar, parity);
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; "
        "selp.u32 %0, 1, 0, p; }"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// A bounded wait as mbar_wait's; `err` may be null
template <int CG>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *abort, unsigned int *err)
{
    if (test<CG>(bar, parity))
        return true;
    const uint64_t t0 = global_ns();
    while (true) {
        if (test<CG>(bar, parity))
            return true;
        if (*abort)
            return false;
        if (global_ns() - t0 > kWaitLimitNs) {
            *abort = 1;
            if (err)
                atomicOr(err, SN_EBIT_TIMEOUT);
            return false;
        }
    }
}
template <int CG>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int *abort, unsigned int *err)
{
    int ok = 1;
    if ((threadIdx.x & 31) == 0)
        ok = wait<CG>(bar, parity, abort, err);
    ok = __shfl_sync(0xffffffffu, ok, 0);
    if (ok && (threadIdx.x & 31))
        test<CG>(bar, parity);
    return ok != 0;
}
// Instruction descriptor as idesc_bf16's, with either operand MN-major
constexpr uint32_t idesc_of(int M, int N, bool a_mn, bool b_mn)
{
    return idesc_bf16(M, N, false, a_mn) | (b_mn ? 1u << 16 : 0u);
}

// ---- the products, tiles of 128 CG x 256 -----------------------------------------------------

constexpr int kRows = 128, kCols = 256, kK = 64;
constexpr uint32_t kABytes = kRows * kK * 2;
constexpr int kEpilogueWarps = 4;
constexpr int kGluThreads = 64 + 32 * kEpilogueWarps;

template <int CG>
struct Stage {
    static constexpr uint32_t kBBytes = kCols / CG * kK * 2;
    static constexpr uint32_t kBytes = kABytes + kBBytes;      // of one CTA
    static constexpr int kStages = CG == 1 ? 4 : 6;
    static constexpr uint32_t kSmem = kStages * kBytes + 1024 /* alignment */ + 256 /* barriers */;
};
static_assert(Stage<1>::kSmem <= 232448 && Stage<2>::kSmem <= 232448, "shared memory of a CTA");

struct GluParams {
    CUtensorMap A[2], B[2];
    int64_t rows;           // of an output
    int cols;               // of an output (the forward: f)
    int64_t mt;             // tiles along the rows and the columns
    int nt;
    int64_t items;
    int64_t chunks;         // of 64 along a product's inner dimension
    int act;
    bool add;               // to what the output holds
    bool out_f32;
    void *out[3];           // forward: H, G, U (G and U may be null); else the outputs
    unsigned int *err;
};

struct Item {
    int which;              // dW: gate or up
    int64_t m0;
    int n0;
};
// Tiles run down the rows in bands, so that the tiles at work share rows and columns in L2.
constexpr int kBand = 8;
template <int MODE, int CG>
__device__ __forceinline__ Item item_at(const GluParams &p, int64_t i)
{
    Item t;
    const int64_t all = p.mt * p.nt;
    t.which = 0;
    if (MODE == GLU_DW && i >= all) {
        t.which = 1;
        i -= all;
    }
    const int64_t band = i / ((int64_t)kBand * p.nt);
    const int in = (int)(i - band * kBand * p.nt);
    const int h = (int)min((int64_t)kBand, p.mt - band * kBand);
    t.m0 = (band * kBand + in % h) * (kRows * CG);
    t.n0 = in / h * (MODE == GLU_FWD ? kCols / 2 : kCols);
    return t;
}

// 16 columns of a row, from `col` on, as bf16 or fp32
__device__ __forceinline__ void store_bf16(__nv_bfloat16 *row, int col, int cols, const float (&v)[16])
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (col + 8 * h < cols) {
            uint4 w;
            w.x = pack_bf16(v[8 * h], v[8 * h + 1]);
            w.y = pack_bf16(v[8 * h + 2], v[8 * h + 3]);
            w.z = pack_bf16(v[8 * h + 4], v[8 * h + 5]);
            w.w = pack_bf16(v[8 * h + 6], v[8 * h + 7]);
            *(uint4 *)(row + col + 8 * h) = w;
        }
}

template <int MODE>
__device__ __forceinline__ void put(const GluParams &p, int which, int64_t row, int col, float (&v)[16])
{
    if (MODE == GLU_DW && p.out_f32) {
        float *at = (float *)p.out[which] + row * p.cols + col;
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            if (col + j < p.cols) {
                float4 x = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                if (p.add) {
                    const float4 y = *(const float4 *)(at + j);
                    x = make_float4(y.x + x.x, y.y + x.y, y.z + x.z, y.w + x.w);
                }
                *(float4 *)(at + j) = x;
            }
        return;
    }
    __nv_bfloat16 *at = (__nv_bfloat16 *)p.out[which] + row * p.cols;
    if (MODE == GLU_DW && p.add)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (col + 8 * h < p.cols) {
                float y[8];
                Vec<__nv_bfloat16>::unpack(*(const uint4 *)(at + col + 8 * h), y);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[8 * h + j] += y[j];
            }
    store_bf16(at, col, p.cols, v);
}

template <int MODE, int CG>
__global__ void __launch_bounds__(kGluThreads, 1) k_glu(const __grid_constant__ GluParams p)
{
    extern __shared__ uint8_t smem_raw[];
    typedef Stage<CG> St;
    constexpr int S = St::kStages;
    uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    base += pad;
    const uint32_t bar = base + S * St::kBytes;
    const uint32_t full_b = bar, empty_b = bar + 8 * S, accf_b = bar + 16 * S, acce_b = accf_b + 16,
                   drain_b = acce_b + 16;
    uint32_t *tmem_slot = (uint32_t *)(smem_raw + pad + S * St::kBytes + 8 * (2 * S + 5));
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_b + 8 * s, 1);
            mbar_init(empty_b + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(accf_b + 8 * b, 1);
            mbar_init(acce_b + 8 * b, kEpilogueWarps * CG);
        }
        mbar_init(drain_b, 1);
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch(&p.A[0]);
        tma_prefetch(&p.B[0]);
    }
    if (warp == 1)
        alloc_columns<CG>(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_start();

    const int64_t first = blockIdx.x / CG, step = gridDim.x / CG;
    constexpr int kSegments = MODE == GLU_DX ? 2 : 1;

    if (warp == 0) {
        // ---------------------------------------------------------------- TMA producer
        if (lane == 0) {
            Ring ring;
            int64_t g = 0;
            bool ok = true;
            for (int64_t i = first; i < p.items && ok; i += step) {
                const Item t = item_at<MODE, CG>(p, i);
                const int m = (int)t.m0 + kRows * (int)rank;
                const int n = MODE == GLU_FWD ? t.n0 : t.n0 + (kCols / CG) * (int)rank;
                for (int seg = 0; seg < kSegments && ok; ++seg)
                    for (int64_t c = 0; c < p.chunks; ++c, ++g, ring.next(S)) {
                        if (!wait<CG>(empty_b + 8 * ring.s, ring.ph ^ 1, abort_flag, p.err)) {
                            ok = false;
                            break;
                        }
                        const uint32_t a = base + ring.s * St::kBytes, b = a + kABytes;
                        uint32_t fb = full_b + 8 * ring.s;
                        if (rank == 0)
                            mbar_arrive_tx(fb, CG * St::kBytes);
                        if (CG == 2)
                            fb = leaders(fb);
                        const int k = (int)c * kK;
                        if (MODE == GLU_DW) {
                            for (int j = 0; j < 2; ++j)
                                load_tile<CG>(a + 8192 * j, &p.A[t.which], m + 64 * j, k, fb);
                        } else {
                            load_tile<CG>(a, &p.A[seg], k, m, fb);
                        }
                        if (MODE == GLU_FWD) {
                            if (CG == 2) {
                                load_tile<CG>(b, &p.B[rank], k, n, fb);
                            } else {
                                load_tile<CG>(b, &p.B[0], k, n, fb);
                                load_tile<CG>(b + 16384, &p.B[1], k, n, fb);
                            }
                        } else {
                            for (int j = 0; j < 4 / CG; ++j)
                                load_tile<CG>(b + 8192 * j, &p.B[seg], n + 64 * j, k, fb);
                        }
                    }
            }
            if (!ok && rank == 0)      // copies already issued land before the CTAs exit
                for (int64_t j = g > S ? g - S : 0; j < g; ++j)
                    drain_wait(full_b + 8 * (uint32_t)(j % S), (uint32_t)(j / S) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products
        if (lane == 0 && rank == 0) {
            constexpr bool kAmn = MODE == GLU_DW, kBmn = MODE != GLU_FWD;
            constexpr uint32_t idesc = idesc_of(kRows * CG, kCols, kAmn, kBmn);
            Ring ring;
            uint32_t it = 0;
            bool ok = true;
            for (int64_t i = first; i < p.items && ok; i += step, ++it) {
                const uint32_t b = it & 1, nb = it >> 1;
                if (!wait<CG>(acce_b + 8 * b, (nb & 1) ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t d_tmem = tmem + b * kCols;
                for (int64_t c = 0; c < p.chunks * kSegments; ++c, ring.next(S)) {
                    if (!wait<CG>(full_b + 8 * ring.s, ring.ph, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = base + ring.s * St::kBytes, w = a + kABytes;
#pragma unroll
                    for (int kk = 0; kk < kK / 16; ++kk) {
                        const uint64_t ad = kAmn ? sdesc_mn_sw128(a + kk * 2048, 8192, 1024) : sdesc_sw128(a + kk * 32);
                        const uint64_t bd = kBmn ? sdesc_mn_sw128(w + kk * 2048, 8192, 1024) : sdesc_sw128(w + kk * 32);
                        multiply<CG>(d_tmem, ad, bd, idesc, c > 0 || kk > 0 ? 1u : 0u);
                    }
                    commit<CG>(empty_b + 8 * ring.s);
                }
                if (ok)
                    commit<CG>(accf_b + 8 * b);
            }
            if (!ok) {                 // products already issued end before TMEM is freed
                commit<CG>(drain_b);
                drain_wait(drain_b, 0);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- epilogue
        const int q = warp & 3;        // TMEM lane quarter of this warp
        uint32_t it = 0;
        for (int64_t i = first; i < p.items; i += step, ++it) {
            const Item t = item_at<MODE, CG>(p, i);
            const uint32_t b = it & 1, nb = it >> 1;
            if (!wait_warp<CG>(accf_b + 8 * b, nb & 1, abort_flag, p.err))
                break;
            tc_fence_after();
            const uint32_t taddr = tmem + b * kCols + ((uint32_t)(32 * q) << 16);
            const int64_t row = t.m0 + kRows * rank + 32 * q + lane;
            const bool in = row < p.rows;
            if (MODE == GLU_FWD) {
                for (int c = 0; c < kCols / 2; c += 16) {
                    float g[16], u[16];
                    __syncwarp();
                    tmem_ld16(taddr + c, g);
                    tmem_ld16(taddr + kCols / 2 + c, u);
                    tmem_ld_wait();
                    const int col = t.n0 + c;
                    if (!in || col >= p.cols)
                        continue;
                    if (p.out[1]) {
                        store_bf16((__nv_bfloat16 *)p.out[1] + row * p.cols, col, p.cols, g);
                        store_bf16((__nv_bfloat16 *)p.out[2] + row * p.cols, col, p.cols, u);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        g[j] = activate<false>(g[j], p.act, nullptr) * u[j];
                    store_bf16((__nv_bfloat16 *)p.out[0] + row * p.cols, col, p.cols, g);
                }
            } else {
                for (int c = 0; c < kCols; c += 16) {
                    float v[16];
                    __syncwarp();
                    tmem_ld16(taddr + c, v);
                    tmem_ld_wait();
                    if (in && t.n0 + c < p.cols)
                        put<MODE>(p, t.which, row, t.n0 + c, v);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                arrive_leader<CG>(acce_b + 8 * b);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();                // neither CTA leaves while the other may reach it
    if (warp == 1) {
        tc_fence_after();
        free_columns<CG>(tmem, 512);
    }
}

// ---- few tokens ------------------------------------------------------------------------------
// A server's step: the weights are read once and bound the call.  Here the weights are the products'
// M side: a CTA takes `take` rows of Wg and as many of Wu (so that the rows of a round divide over
// the SMs), the tokens are the N side, and a lane of the accumulators is a feature.

constexpr int kFewThreads = 192;
constexpr int kFewTokens = 256;

struct FewParams {
    CUtensorMap X, Wg, Wu;
    int T, f, n;            // n: T rounded up to 16
    int take;               // rows of each weight that a CTA takes at a time
    int tiles, chunks, stages;
    uint32_t stage_bytes, columns;
    int act;
    __nv_bfloat16 *H, *G, *U;
    unsigned int *err;
};

__global__ void __launch_bounds__(kFewThreads, 1) k_glu_few(const __grid_constant__ FewParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    base += pad;
    const int S = p.stages;
    const uint32_t w_bytes = (uint32_t)p.take * 128;
    // (a product reads 128 rows of each weight; those past `take` lie in what follows, up to 16 KB
    // past the last stage, and give lanes that nobody reads)
    const uint32_t bar_off = (uint32_t)S * p.stage_bytes + 16384;
    const uint32_t bar = base + bar_off;
    const uint32_t full_b = bar, empty_b = bar + 8 * S, accf_b = bar + 16 * S, acce_b = accf_b + 8,
                   drain_b = acce_b + 8;
    uint32_t *tmem_slot = (uint32_t *)(smem_raw + pad + bar_off + 8 * (2 * S + 3));
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_b + 8 * s, 1);
            mbar_init(empty_b + 8 * s, 1);
        }
        mbar_init(accf_b, 1);
        mbar_init(acce_b, 4);
        mbar_init(drain_b, 1);
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch(&p.X);
        tma_prefetch(&p.Wg);
        tma_prefetch(&p.Wu);
    }
    if (warp == 1)
        tmem_alloc(smem_u32(tmem_slot), p.columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_start();

    if (warp == 0) {
        if (lane == 0) {
            Ring ring;
            int g = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x)
                for (int c = 0; c < p.chunks; ++c, ++g, ring.next(S)) {
                    if (!wait<1>(empty_b + 8 * ring.s, ring.ph ^ 1, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    const uint32_t at = base + ring.s * p.stage_bytes, fb = full_b + 8 * ring.s;
                    mbar_arrive_tx(fb, p.stage_bytes);
                    tma_load_2d(at, &p.Wg, c * kK, tile * p.take, fb);
                    tma_load_2d(at + w_bytes, &p.Wu, c * kK, tile * p.take, fb);
                    tma_load_2d(at + 2 * w_bytes, &p.X, c * kK, 0, fb);
                }
            if (!ok)
                for (int j = g > S ? g - S : 0; j < g; ++j)
                    drain_wait(full_b + 8 * (uint32_t)(j % S), (uint32_t)(j / S) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16(128, p.n);
            Ring ring;
            uint32_t it = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x, ++it) {
                if (!wait<1>(acce_b, (it & 1) ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                for (int c = 0; c < p.chunks; ++c, ring.next(S)) {
                    if (!wait<1>(full_b + 8 * ring.s, ring.ph, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t at = base + ring.s * p.stage_bytes;
#pragma unroll
                    for (int kk = 0; kk < kK / 16; ++kk) {
                        const uint64_t bd = sdesc_sw128(at + 2 * w_bytes + kk * 32);
                        const uint32_t more = c > 0 || kk > 0 ? 1u : 0u;
                        mma_bf16(tmem, sdesc_sw128(at + kk * 32), bd, idesc, more);
                        mma_bf16(tmem + p.n, sdesc_sw128(at + w_bytes + kk * 32), bd, idesc, more);
                    }
                    mma_commit(empty_b + 8 * ring.s);
                }
                if (ok)
                    mma_commit(accf_b);
            }
            if (!ok) {
                mma_commit(drain_b);
                drain_wait(drain_b, 0);
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3;
        uint32_t it = 0;
        for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++it) {
            if (!wait_warp<1>(accf_b, it & 1, abort_flag, p.err))
                break;
            tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16);
            const int feature = tile * p.take + 32 * q + lane;
            const bool in = 32 * q + lane < p.take && feature < p.f;
            for (int c = 0; c < p.n; c += 16) {
                float g[16], u[16];
                __syncwarp();
                tmem_ld16(taddr + c, g);
                tmem_ld16(taddr + p.n + c, u);
                tmem_ld_wait();
                if (!in)
                    continue;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c + j < p.T) {
                        const int64_t at = (int64_t)(c + j) * p.f + feature;
                        if (p.G) {
                            p.G[at] = __float2bfloat16_rn(g[j]);
                            p.U[at] = __float2bfloat16_rn(u[j]);
                        }
                        p.H[at] = __float2bfloat16_rn(activate<false>(g[j], p.act, nullptr) * u[j]);
                    }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(acce_b);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, p.columns);
    }
}

// ---- dG and dU ---------------------------------------------------------------------------------
// Bound by DRAM: three bf16 arrays read, two written.
struct GradArgs {
    const __nv_bfloat16 *dH, *G, *U;
    __nv_bfloat16 *dG, *dU;
    int64_t T, lddh;
    int f8;                 // pieces of 8 in a row
    int act;
};
__global__ void __launch_bounds__(256) k_glu_grad(const GradArgs a)
{
    griddep_start();
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y)
        for (int j = blockIdx.x * 256 + threadIdx.x; j < a.f8; j += gridDim.x * 256) {
            const int64_t at = t * a.f8 + j;
            float h[8], g[8], u[8];
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)(a.dH + t * a.lddh) + j), h);
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)a.G + at), g);
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)a.U + at), u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float slope;
                const float x = activate<true>(g[i], a.act, &slope);
                g[i] = h[i] * u[i] * slope;
                u[i] = h[i] * x;
            }
            *((uint4 *)a.dG + at) = Vec<__nv_bfloat16>::pack(g);
            *((uint4 *)a.dU + at) = Vec<__nv_bfloat16>::pack(u);
        }
}

// ---- launches ------------------------------------------------------------------------------------

template <int MODE, int CG>
cudaError_t launch_tiles(GluParams p, int sms, cudaStream_t s)
{
    p.mt = (p.rows + kRows * CG - 1) / (kRows * CG);
    const int width = MODE == GLU_FWD ? kCols / 2 : kCols;
    p.nt = (p.cols + width - 1) / width;
    p.items = p.mt * p.nt * (MODE == GLU_DW ? 2 : 1);
    const int grid = (int)std::min<int64_t>(p.items, std::max(1, sms / CG)) * CG;
    cudaError_t e = cudaFuncSetAttribute(k_glu<MODE, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         Stage<CG>::kSmem);
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_clusters(k_glu<MODE, CG>, CG, dim3(grid), dim3(kGluThreads), Stage<CG>::kSmem, s, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// Pairs of CTAs where the stream's context has the whole GPU; with a part of it a pair might find
// no place.
template <int MODE>
cudaError_t launch_products(const GluParams &p, cudaStream_t s)
{
    const int all = device_sms(), sms = stream_sms(s);
    return sms < all ? launch_tiles<MODE, 1>(p, sms, s) : launch_tiles<MODE, 2>(p, sms, s);
}

cudaError_t launch_few(FewParams p, const __nv_bfloat16 *X, int64_t ldx, const __nv_bfloat16 *Wg,
                       const __nv_bfloat16 *Wu, int d, cudaStream_t s)
{
    const int sms = stream_sms(s);
    p.n = (p.T + 15) / 16 * 16;
    const int rounds = (int)(((int64_t)p.f + sms * 128 - 1) / (sms * 128));
    p.take = std::min(128, ((p.f + sms * rounds - 1) / (sms * rounds) + 7) / 8 * 8);
    p.tiles = (p.f + p.take - 1) / p.take;
    p.chunks = (d + kK - 1) / kK;
    p.stage_bytes = (uint32_t)(2 * p.take + p.n) * 128;
    const uint32_t rest = 16384 + 1024 + 512;
    p.stages = std::max(2, std::min(16, (int)((232448 - rest) / p.stage_bytes)));
    p.columns = 32;
    while (p.columns < 2u * p.n)
        p.columns *= 2;
    if (!tensor_map_2d(&p.X, X, d, p.T, (uint64_t)ldx * 2, kK, p.n, true) ||
        !tensor_map_2d(&p.Wg, Wg, d, p.f, (uint64_t)d * 2, kK, p.take, true) ||
        !tensor_map_2d(&p.Wu, Wu, d, p.f, (uint64_t)d * 2, kK, p.take, true))
        return cudaErrorInvalidValue;
    const uint32_t smem = (uint32_t)p.stages * p.stage_bytes + rest;
    cudaError_t e = cudaFuncSetAttribute(k_glu_few, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(k_glu_few, dim3(std::min(p.tiles, sms)), dim3(kFewThreads), smem, s, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace
}  // namespace tc

cudaError_t glu_fwd(const void *X, int64_t ldx, const void *Wg, const void *Wu, int64_t T, int d, int f, int act,
                    void *G, void *U, void *H, unsigned int *err, cudaStream_t s)
{
    using namespace tc;
    typedef __nv_bfloat16 b16;
    if (T <= 128) {
        FewParams p = {};
        p.T = (int)T;
        p.f = f;
        p.act = act;
        p.H = (b16 *)H;
        p.G = (b16 *)G;
        p.U = (b16 *)U;
        p.err = err;
        return launch_few(p, (const b16 *)X, ldx, (const b16 *)Wg, (const b16 *)Wu, d, s);
    }
    GluParams p = {};
    p.rows = T;
    p.cols = f;
    p.chunks = (d + kK - 1) / kK;
    p.act = act;
    p.out[0] = H;
    p.out[1] = G;
    p.out[2] = U;
    p.err = err;
    if (!tensor_map_2d(&p.A[0], X, d, T, (uint64_t)ldx * 2, kK, kRows, true) ||
        !tensor_map_2d(&p.B[0], Wg, d, f, (uint64_t)d * 2, kK, 128, true) ||
        !tensor_map_2d(&p.B[1], Wu, d, f, (uint64_t)d * 2, kK, 128, true))
        return cudaErrorInvalidValue;
    return launch_products<GLU_FWD>(p, s);
}

size_t glu_bwd_workspace(int64_t T, int d, int f) { return 0; }

cudaError_t glu_bwd(const void *dH, int64_t lddh, const void *X, int64_t ldx, const void *Wg, const void *Wu,
                    const void *G, const void *U, int64_t T, int d, int f, int act, void *dG, void *dU, void *dX,
                    sn_dtype grad_dt, void *dWg, void *dWu, bool accumulate, void *ws, unsigned int *err,
                    cudaStream_t s)
{
    using namespace tc;
    typedef __nv_bfloat16 b16;
    const GradArgs a{(const b16 *)dH, (const b16 *)G, (const b16 *)U, (b16 *)dG, (b16 *)dU, T, lddh, f / 8, act};
    const int across = (a.f8 + 255) / 256;
    count_launch();
    cudaError_t e = launch_dependent(
        k_glu_grad, dim3((unsigned)across, (unsigned)std::min<int64_t>(T, std::max(1, 65535 / across))), dim3(256), 0,
        s, a);
    if (e == cudaSuccess)
        e = cudaGetLastError();
    if (e == cudaSuccess && dX) {
        GluParams p = {};
        p.rows = T;
        p.cols = d;
        p.chunks = (f + kK - 1) / kK;
        p.out[0] = dX;
        p.err = err;
        if (!tensor_map_2d(&p.A[0], dG, f, T, (uint64_t)f * 2, kK, kRows, true) ||
            !tensor_map_2d(&p.A[1], dU, f, T, (uint64_t)f * 2, kK, kRows, true) ||
            !tensor_map_2d(&p.B[0], Wg, d, f, (uint64_t)d * 2, 64, kK, true) ||
            !tensor_map_2d(&p.B[1], Wu, d, f, (uint64_t)d * 2, 64, kK, true))
            return cudaErrorInvalidValue;
        e = launch_products<GLU_DX>(p, s);
    }
    if (e == cudaSuccess && dWg) {
        GluParams p = {};
        p.rows = f;
        p.cols = d;
        p.chunks = (T + kK - 1) / kK;
        p.out[0] = dWg;
        p.out[1] = dWu;
        p.out_f32 = grad_dt == SN_F32;
        p.add = accumulate;
        p.err = err;
        if (!tensor_map_2d(&p.A[0], dG, f, T, (uint64_t)f * 2, 64, kK, true) ||
            !tensor_map_2d(&p.A[1], dU, f, T, (uint64_t)f * 2, 64, kK, true) ||
            !tensor_map_2d(&p.B[0], X, d, T, (uint64_t)ldx * 2, 64, kK, true))
            return cudaErrorInvalidValue;
        e = launch_products<GLU_DW>(p, s);
    }
    return e;
}

}  // namespace sn
