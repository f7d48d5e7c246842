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
//
// The products of many tokens are bound by the tensor cores: a pair of CTAs multiplies 256 x 256 tiles
// of 64 deep chunks, which a ring of TMA loads feeds, a chunk in 555 cycles where its four products
// take 547, and eight warps drain one accumulator while the other fills.  (Two CTAs each for itself would
// read B twice: 1.5 times the shared memory's traffic.)  Those of a few tokens are bound by the weights'
// bytes, dG and dU by theirs.
//
// Measured, 8192 x 4096 x 14336 (T, d, f), in bursts of 20 calls: forward 949 us (2.03 PFLOP/s), with G and U
// 981, dG and dU 171 (6.9 TB/s), beyond those dX 1041 and the weights' gradients 973; a product of the same
// size of the vendor's library, in turn with them, 937, 1013 and 956.  The chip's power sets the clock where
// the tensor cores are at work 93 to 95% of the cycles, in a step lower (1.46 GHz at 1.4 kW): the forward for
// seconds 1117 us, the library's product 1107, and forward and gradients in turn 3650 us (1.58 PFLOP/s), 15%
// more than the bursts' sum.  1 token of 4096 x 14336 37.5 us (6.3 TB/s), 75 tokens 40.5, 1 of 8192 x 28672
// 139 (6.8 TB/s).
#include <algorithm>
#include <type_traits>

#include "sn_tc.cuh"
#include "sn_tc_kernels.cuh"
#include "sn_vec.cuh"

namespace sn {
namespace tc {
namespace {

enum { GLU_FWD = 0, GLU_DX = 1, GLU_DW = 2 };

// ---- the activations ---------------------------------------------------------------------

// From the exponential that is at most 1, so that the quotient's denominator is from 1 to 2 (from e^-x,
// a share below 2^-126 came out 0: __fdividef's, beyond 2^126)
__device__ __forceinline__ float sigmoid(float x)
{
    const float t = __expf(-fabsf(x));
    return __fdividef(x < 0.f ? t : 1.f, 1.f + t);
}

// gelu's tanh form is g sigmoid(2 x), x = sqrt(2 / pi) (g + 0.044715 g^3)
constexpr float kTanhA = 1.5957691216057308f, kTanhB = 0.044715f;

// act(g); with SLOPE also act'(g).  The shares p of g are taken as sigmoids and as erfc, so that nothing
// cancels where they vanish.  Their relative error grows there with the exponential's argument x, by
// 2^-23 |x| for its own and as much for each two roundings of x: below 2^-14 wherever bf16 still shows the
// result, where an output's is 2^-8.
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate(float g, float &slope)
{
    if (ACT == SN_ACT_RELU) {
        if (SLOPE)
            slope = g > 0.f ? 1.f : 0.f;
        return max_nan(g, 0.f);
    }
    if (ACT == SN_ACT_SILU) {
        const float p = sigmoid(g);
        if (SLOPE)
            slope = fmaf(g * p, 1.f - p, p);
        return g * p;
    }
    if (ACT == SN_ACT_GELU) {
        const float p = 0.5f * erfcf(-0.7071067811865476f * g);
        if (SLOPE)
            slope = fmaf(g, 0.3989422804014327f * __expf(-0.5f * g * g), p);
        return g * p;
    }
    const float p = sigmoid(kTanhA * g * fmaf(kTanhB * g, g, 1.f));
    if (SLOPE) {
        const float q = p * (1.f - p);                  // 0 where g^2 may pass fp32's range
        slope = q > 0.f ? fmaf(g * q, kTanhA * fmaf(3.f * kTanhB * g, g, 1.f), p) : p;
    }
    return g * p;
}
// F with the activation as a constant: a branch for many elements, whose chains of exponentials and
// divisions then run beside one another (decided at each element, the epilogue of 75 tokens took 8 us)
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f)
{
    switch (act) {
    case SN_ACT_SILU: f(std::integral_constant<int, SN_ACT_SILU>()); break;
    case SN_ACT_GELU: f(std::integral_constant<int, SN_ACT_GELU>()); break;
    case SN_ACT_GELU_TANH: f(std::integral_constant<int, SN_ACT_GELU_TANH>()); break;
    default: f(std::integral_constant<int, SN_ACT_RELU>()); break;
    }
}
// g = act(g) u
__device__ __forceinline__ void gate_all(float (&g)[16], const float (&u)[16], int act)
{
    with_activation(act, [&](auto a) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float none;
            g[j] = activate<decltype(a)::value, false>(g[j], none) * u[j];
        }
    });
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
// Whether a phase has completed, with acquire semantics toward the other CTA's threads too
__device__ __forceinline__ bool mbar_test_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; "
        "selp.u32 %0, 1, 0, p; }"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Whether a phase has completed, without waiting at all
__device__ __forceinline__ uint32_t peek(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.test_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2; "
        "selp.u32 %0, 1, 0, p; }"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
// Where a wait that expires is recorded in calls without an error word of their own, one a device
__device__ unsigned int g_unclaimed;

// A bounded wait of a whole warp, as warp_wait's; `err` may be null (g_unclaimed).  The votes tell the
// compiler that the warp stays together.  CLUSTER: for what the other CTA's threads have done.
// `moving`: a barrier whose phases go on while what the wait is for is at work, and the limit starts
// again at each: a tile of dW may take longer than it (one CTA's of 640 million tokens 3.3 s).
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *abort, unsigned int *err,
                                     uint32_t moving = 0)
{
    const auto test = [&] {
        return __all_sync(0xffffffffu, CLUSTER ? mbar_test_cluster(bar, parity) : mbar_test(bar, parity));
    };
    if (test())
        return true;
    uint64_t t0 = global_ns();
    bool phase = false;
    while (true) {
        if (test())
            return true;
        if (__any_sync(0xffffffffu, *abort))
            return false;
        if (moving && __any_sync(0xffffffffu, peek(moving, 0)) != phase) {
            phase = !phase;
            t0 = global_ns();
        }
        if (__any_sync(0xffffffffu, global_ns() - t0 > kWaitLimitNs)) {
            *abort = 1;
            if (threadIdx.x % 32 == 0)
                atomicOr(err ? err : &g_unclaimed, SN_EBIT_TIMEOUT);
            return false;
        }
    }
}
// Whether `is` holds in all 256 threads of the eight epilogue warps; a barrier for them
__device__ __forceinline__ bool all_of_eight(bool is)
{
    uint32_t all;
    asm volatile(
        "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; bar.red.and.pred q, 1, 256, p; selp.u32 %0, 1, 0, q; }"
        : "=r"(all)
        : "r"((uint32_t)is)
        : "memory");
    return all != 0;
}
// One lane of the warp
__device__ __forceinline__ bool elected()
{
    uint32_t is;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(is));
    return is != 0;
}

// A stage operand's descriptor at 16-element step kk (see sdesc_sw128, sdesc_mn_sw128): 32 bytes on in
// a K-major row, two groups of 8 rows on in MN-major tiles
template <bool MN>
__device__ __forceinline__ uint64_t step_desc(uint32_t at, int kk)
{
    return MN ? sdesc_mn_sw128(at + kk * 2048, 8192, 1024) : sdesc_sw128(at + kk * 32);
}

// Instruction descriptor as idesc_bf16's, with either operand MN-major
constexpr uint32_t idesc_of(int M, int N, bool a_mn, bool b_mn)
{
    return idesc_bf16(M, N, false, a_mn) | (b_mn ? 1u << 16 : 0u);
}

// ---- the products, tiles of 128 CG x 256 -----------------------------------------------------

constexpr int kRows = 128, kCols = 256, kK = 64;
constexpr uint32_t kABytes = kRows * kK * 2;
constexpr int kEpilogueWarps = 8;
constexpr uint32_t kOutBytes = 32 * 128;       // an epilogue warp's rows of 128 bytes of an output
constexpr int kGluThreads = 64 + 32 * kEpilogueWarps;

template <int CG>
struct Stage {
    static constexpr uint32_t kBBytes = kCols / CG * kK * 2;
    static constexpr uint32_t kBytes = kABytes + kBBytes;      // of one CTA
    static constexpr int kStages = CG == 1 ? 4 : 6;
    static constexpr uint32_t kOut = kStages * kBytes, kBar = kOut + kEpilogueWarps * kOutBytes;
    static constexpr uint32_t kSmem = kBar + 1024 /* alignment */ + 256 /* barriers */;
};
static_assert(Stage<1>::kSmem <= 232448 && Stage<2>::kSmem <= 232448, "shared memory of a CTA");

struct GluParams {
    CUtensorMap A[2], B[2], out[3];
    int64_t rows;           // of an output
    int cols;               // of an output (the forward: f)
    int64_t mt;             // tiles along the rows and the columns
    int nt;
    int64_t chunks;         // of 64 along a product's inner dimension (dX: of each of its two)
    // Work: whole tiles, then the tiles that would leave most pairs idle, cut into runs of `run`
    // chunks, a pair each (0: none is cut)
    int64_t whole, cut, run;
    int64_t span;           // chunks of a cut tile as the runs count them: at least its own
    float *parts;           // of cut tiles, fp32: pair u's of tile j at u + j
    int act;
    bool add;               // to what the output holds
    bool out_f32, keep;     // dW's type; whether the forward stores G and U
    void *at[2];            // dX or dW, where threads write it
    unsigned int *err;
};

// Tiles run down the rows in bands, so that the tiles at work share rows and columns in L2.
constexpr int kBand = 8;
struct Tile {
    int which;              // dW: gate or up
    int64_t m0;
    int n0;
};
template <int MODE, int CG>
__device__ __forceinline__ Tile tile_at(const GluParams &p, int64_t i)
{
    Tile t;
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
// A pair's n-th piece of work: a tile, and its chunks k0 to k1
struct Work {
    Tile t;
    int64_t k0, k1, part;   // part: where its sums go, -1 where they are the output
};
template <int MODE, int CG>
__device__ __forceinline__ bool work_at(const GluParams &p, int64_t n, Work &w)
{
    const int64_t u = blockIdx.x / CG, units = gridDim.x / CG, all = p.chunks * (MODE == GLU_DX ? 2 : 1);
    const int64_t i = u + n * units;
    w.k0 = 0;
    w.k1 = all;
    w.part = -1;
    if (i < p.whole) {
        w.t = tile_at<MODE, CG>(p, i);
        return true;
    }
    if (MODE == GLU_FWD || p.run == 0)
        return false;
    // (p.whole is a multiple of units where tiles are cut)
    const int64_t lo = u * p.run, hi = min(lo + p.run, p.cut * p.span);
    const int64_t j = lo / p.span + (n - p.whole / units);
    w.k0 = max(lo, j * p.span) - j * p.span;
    w.k1 = min(hi - j * p.span, all);
    if (w.k0 >= w.k1)
        return false;
    if (w.k1 - w.k0 < all)
        w.part = u + j;
    w.t = tile_at<MODE, CG>(p, p.whole + j);
    return true;
}

// Two fours of packed bf16 pairs, or eight fp32, of a warp's row `lane` at 16-byte pieces `c` and on
// of its 128 bytes
__device__ __forceinline__ void stage(uint32_t out, int lane, int c, const uint32_t *w)
{
    sts128(out + sw128(lane, c), make_uint4(w[0], w[1], w[2], w[3]));
    sts128(out + sw128(lane, c + 1), make_uint4(w[4], w[5], w[6], w[7]));
}
__device__ __forceinline__ void pack16(const float (&v)[16], uint32_t *w)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
}
// The warp's 32 rows of 128 bytes go to the output's box at (x, y); what lies past its edges stays
__device__ __forceinline__ void send(const CUtensorMap *m, uint32_t out, int lane, int x, int64_t y, bool in)
{
    fence_async_smem();
    __syncwarp();
    if (lane == 0 && in) {
        tma_store_2d(m, out, x, (int)y);
        bulk_commit();
    }
}
// The staging rows have been read and may be written again
__device__ __forceinline__ void sent(int lane)
{
    if (lane == 0)
        bulk_wait_read0();
    __syncwarp();
}

// 16 columns of dW added to what it holds
__device__ __forceinline__ void add_to(const GluParams &p, int which, int64_t row, int col, const float (&v)[16])
{
    if (p.out_f32) {
        float *at = (float *)p.at[which] + row * p.cols + col;
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            if (col + j < p.cols) {
                const float4 y = *(const float4 *)(at + j);
                *(float4 *)(at + j) = make_float4(y.x + v[j], y.y + v[j + 1], y.z + v[j + 2], y.w + v[j + 3]);
            }
        return;
    }
    __nv_bfloat16 *at = (__nv_bfloat16 *)p.at[which] + row * p.cols + col;
#pragma unroll
    for (int j = 0; j < 16; j += 8)
        if (col + j < p.cols) {
            float y[8];
            Vec<__nv_bfloat16>::unpack(*(const uint4 *)(at + j), y);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                y[k] += v[j + k];
            *(uint4 *)(at + j) = Vec<__nv_bfloat16>::pack(y);
        }
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
    const uint32_t bar = base + St::kBar;
    const uint32_t full_b = bar, empty_b = bar + 8 * S, accf_b = bar + 16 * S, acce_b = accf_b + 16,
                   drain_b = acce_b + 16;
    uint32_t *tmem_slot = (uint32_t *)(smem_raw + pad + St::kBar + 8 * (2 * S + 5));
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

    // A warp issues copies and one issues products: all its lanes walk the loop and one is elected
    // at each issue, so that what the instructions read is the warp's alike and lies in uniform
    // registers.  (With one lane in the loop, a chunk's four products took that lane 630 cycles to
    // issue, and the tensor cores 547 to do.)
    if (warp == 0) {
        // ---------------------------------------------------------------- TMA producer
        Ring ring;
        int64_t g = 0;
        bool ok = true;
        Work w;
        for (int64_t i = 0; ok && work_at<MODE, CG>(p, i, w); ++i) {
            const int m = (int)w.t.m0 + kRows * (int)rank;
            const int n = MODE == GLU_FWD ? w.t.n0 : w.t.n0 + (kCols / CG) * (int)rank;
            for (int64_t c = w.k0; c < w.k1; ++c, ++g, ring.next(S)) {
                if (!wait(empty_b + 8 * ring.s, ring.ph ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                const uint32_t a = base + ring.s * St::kBytes, b = a + kABytes;
                const uint32_t own = full_b + 8 * ring.s, fb = CG == 2 ? leaders(own) : own;
                const int seg = MODE == GLU_DX && c >= p.chunks;
                const int k = (int)(seg ? c - p.chunks : c) * kK;
                if (elected()) {
                    if (rank == 0)
                        mbar_arrive_tx(own, CG * St::kBytes);
                    if (MODE == GLU_DW) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            load_tile<CG>(a + 8192 * j, &p.A[w.t.which], m + 64 * j, k, fb);
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
#pragma unroll
                        for (int j = 0; j < 4 / CG; ++j)
                            load_tile<CG>(b + 8192 * j, &p.B[seg], n + 64 * j, k, fb);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok && rank == 0 && lane == 0)     // copies already issued land before the CTAs exit
            for (int64_t j = g > S ? g - S : 0; j < g; ++j)
                drain_wait(full_b + 8 * (uint32_t)(j % S), (uint32_t)(j / S) & 1);
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products
        if (rank == 0) {
            constexpr bool kAmn = MODE == GLU_DW, kBmn = MODE != GLU_FWD;
            constexpr uint32_t idesc = idesc_of(kRows * CG, kCols, kAmn, kBmn);
            Ring ring;
            uint32_t it = 0, ready = 0;
            bool ok = true;
            Work v;
            for (; ok && work_at<MODE, CG>(p, it, v); ++it) {
                const uint32_t b = it & 1, nb = it >> 1;
                if (!wait<CG == 2>(acce_b + 8 * b, (nb & 1) ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t d_tmem = tmem + b * kCols;
                for (int64_t c = v.k0; c < v.k1; ++c) {
                    if (!__all_sync(0xffffffffu, ready) && !wait(full_b + 8 * ring.s, ring.ph, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = base + ring.s * St::kBytes, w = a + kABytes, done = empty_b + 8 * ring.s;
                    // the next stage is looked at ahead of this one's products, which hide the look
                    ring.next(S);
                    ready = peek(full_b + 8 * ring.s, ring.ph);
                    uint64_t ad[kK / 16], bd[kK / 16];
#pragma unroll
                    for (int kk = 0; kk < kK / 16; ++kk) {
                        ad[kk] = step_desc<kAmn>(a, kk);
                        bd[kk] = step_desc<kBmn>(w, kk);
                    }
                    if (elected()) {
#pragma unroll
                        for (int kk = 0; kk < kK / 16; ++kk)
                            multiply<CG>(d_tmem, ad[kk], bd[kk], idesc, c > v.k0 || kk > 0 ? 1u : 0u);
                        commit<CG>(done);
                    }
                    __syncwarp();
                }
                if (ok && elected())
                    commit<CG>(accf_b + 8 * b);
                __syncwarp();
            }
            if (!ok && elected()) {    // products already issued end before TMEM is freed
                commit<CG>(drain_b);
                drain_wait(drain_b, 0);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- epilogue
        // A warp has 32 rows (its TMEM lane quarter) and half of the columns, and sends 128 bytes
        // of its rows at a time through its staging rows, whole lines of the output.
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t out = base + St::kOut + (warp - 2) * kOutBytes;
        Work w;
        for (uint32_t it = 0; work_at<MODE, CG>(p, it, w); ++it) {
            const Tile &t = w.t;
            const uint32_t b = it & 1, nb = it >> 1;
            if (!wait(accf_b + 8 * b, nb & 1, abort_flag, p.err, empty_b))
                break;
            tc_fence_after();
            const uint32_t taddr = tmem + b * kCols + ((uint32_t)(32 * q) << 16);
            const int64_t row0 = t.m0 + kRows * rank + 32 * q;
            const auto release = [&] {          // the accumulator has been read
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    arrive_leader<CG>(acce_b + 8 * b);
            };
            if (MODE == GLU_FWD) {
                const int col = t.n0 + 64 * half;
                const bool in = row0 < p.rows && col < p.cols;
                uint32_t gw[32], uw[32];
                sent(lane);
#pragma unroll
                for (int c = 0; c < 64; c += 16) {
                    float g[16], u[16];
                    tmem_ld16(taddr + 64 * half + c, g);
                    tmem_ld16(taddr + kCols / 2 + 64 * half + c, u);
                    tmem_ld_wait();
                    if (p.keep) {
                        pack16(g, gw + c / 2);
                        pack16(u, uw + c / 2);
                    }
                    gate_all(g, u, p.act);
                    uint32_t hw[8];
                    pack16(g, hw);
                    stage(out, lane, c / 8, hw);
                }
                release();
                send(&p.out[0], out, lane, col, row0, in);
                if (p.keep) {
                    sent(lane);
#pragma unroll
                    for (int c = 0; c < 64; c += 16)
                        stage(out, lane, c / 8, gw + c / 2);
                    send(&p.out[1], out, lane, col, row0, in);
                    sent(lane);
#pragma unroll
                    for (int c = 0; c < 64; c += 16)
                        stage(out, lane, c / 8, uw + c / 2);
                    send(&p.out[2], out, lane, col, row0, in);
                }
            } else if (w.part >= 0) {
                // lanes next to one another, four columns each
                float *to = p.parts + w.part * (kRows * CG * kCols) + (kRows * rank + 32 * q) * kCols + 4 * lane;
                const bool in = row0 + lane < p.rows;
                for (int c = 128 * half; c < 128 * half + 128; c += 16) {
                    float v[16];
                    __syncwarp();
                    tmem_ld16(taddr + c, v);
                    tmem_ld_wait();
                    if (in && t.n0 + c < p.cols)
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            *(float4 *)(to + (c + j) * 32) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                }
                release();
            } else if (MODE == GLU_DW && p.add) {
                for (int c = 128 * half; c < 128 * half + 128; c += 16) {
                    float v[16];
                    __syncwarp();
                    tmem_ld16(taddr + c, v);
                    tmem_ld_wait();
                    if (row0 + lane < p.rows && t.n0 + c < p.cols)
                        add_to(p, t.which, row0 + lane, t.n0 + c, v);
                }
                release();
            } else {
                // 128 bytes: 64 columns in bf16, 32 in fp32
                const bool wide = MODE == GLU_DW && p.out_f32;
                const int each = wide ? 32 : 64;
                for (int c0 = 128 * half; c0 < 128 * half + 128; c0 += each) {
                    const int col = t.n0 + c0;
                    sent(lane);
#pragma unroll
                    for (int c = 0; c < 64; c += 16) {
                        if (c >= each)
                            break;
                        float v[16];
                        tmem_ld16(taddr + c0 + c, v);
                        tmem_ld_wait();
                        if (wide) {
                            uint32_t w[16];
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                w[j] = __float_as_uint(v[j]);
                            stage(out, lane, c / 4, w);
                            stage(out, lane, c / 4 + 2, w + 8);
                        } else {
                            uint32_t w[8];
                            pack16(v, w);
                            stage(out, lane, c / 8, w);
                        }
                    }
                    if (c0 + each == 128 * half + 128)
                        release();
                    send(&p.out[t.which], out, lane, wide ? 2 * col : col, row0, row0 < p.rows && col < p.cols);
                }
            }
        }
        if (lane == 0)
            bulk_wait_all0();
        __syncwarp();
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

// The sums of cut tiles' parts, in the order of their chunks.  A thread takes eight columns of a row.
template <int MODE>
__global__ void __launch_bounds__(256) k_glu_join(const __grid_constant__ GluParams p)
{
    griddep_start();
    const int64_t all = p.chunks * (MODE == GLU_DX ? 2 : 1), j = blockIdx.y;
    const int64_t u0 = j * p.span / p.run, u1 = (j * p.span + all - 1) / p.run;
    if (u0 == u1)                      // one pair had it whole
        return;
    const Tile t = tile_at<MODE, 2>(p, p.whole + j);
    const int at = blockIdx.x * 8 + threadIdx.x / 32;             // 32 rows x 8 columns of the tile
    const int64_t row = t.m0 + at / 32 * 32 + threadIdx.x % 32;
    const int col = t.n0 + at % 32 * 8;
    if (row >= p.rows || col >= p.cols)
        return;
    const float *from = p.parts + (u0 + j) * (2 * kRows * kCols) + at / 32 * 32 * kCols + at % 32 * 256 +
                        4 * (threadIdx.x % 32);
    float v[8] = {};
    for (int64_t u = u0; u <= u1; ++u, from += 2 * kRows * kCols) {
        const float4 a = __ldcs((const float4 *)from), b = __ldcs((const float4 *)(from + 128));
        v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
        v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
    }
    if (MODE == GLU_DW && p.out_f32) {
        float *to = (float *)p.at[t.which] + row * p.cols + col;
#pragma unroll
        for (int k = 0; k < 8; k += 4) {
            const float4 y = p.add ? *(const float4 *)(to + k) : make_float4(0.f, 0.f, 0.f, 0.f);
            *(float4 *)(to + k) = make_float4(y.x + v[k], y.y + v[k + 1], y.z + v[k + 2], y.w + v[k + 3]);
        }
        return;
    }
    uint4 *to = (uint4 *)((__nv_bfloat16 *)p.at[t.which] + row * p.cols + col);
    float y[8] = {};
    if (p.add)
        Vec<__nv_bfloat16>::unpack(*to, y);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        y[k] += v[k];
    *to = Vec<__nv_bfloat16>::pack(y);
}

// ---- few tokens ------------------------------------------------------------------------------
// A server's step: the weights are read once and bound the call.  Here the weights are the products'
// M side: a CTA takes `take` rows of Wg and as many of Wu (so that the rows of a round divide over
// the SMs), the tokens are the N side, and a lane of the accumulators is a feature.  Up to 64 rows of
// each share one product's 128 (JOINED: Wu's are the upper lanes, and reach the lower lanes' threads
// through shared memory); more take a product each.

constexpr int kFewThreads = 320;

// Up to how many tokens: 128, and 224 where a CTA has one round of more than 64 rows of each weight
// (us, this kernel and the tiles': 160 tokens of 4096 x 14336 44.1 and 51.1, 224 47.1 and 51.4; 160 of
// 8192 x 28672, two rounds, 162.8 and 162.7, of 1024 x 4096, 32 rows, 11.1 and 10.1; 128 of
// 2048 x 8192 16.4 and 18.4)
constexpr int kFewTokens = 128, kMoreTokens = 224;

struct FewParams {
    CUtensorMap X, Wg, Wu;
    int T, f, n;            // n: T rounded up to 16
    int take;               // rows of each weight that a CTA takes at a time
    int tiles, steps, stages;
    int per;                // chunks of 64 along d in a stage: `steps` stages have them all
    uint32_t chunk_bytes, load_bytes, columns;
    int act;
    __nv_bfloat16 *H, *G, *U;
    unsigned int *err;
};

template <bool JOINED>
__global__ void __launch_bounds__(kFewThreads, 1) k_glu_few(const __grid_constant__ FewParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    base += pad;
    const int S = p.stages;
    const uint32_t stage_bytes = p.per * p.chunk_bytes;
    // Wu's rows lie behind Wg's `take`, or where they share a product behind 64.  (A product reads
    // 128 rows; those that hold no row of its weight give lanes that nobody reads: they lie in what
    // follows, up to 16 KB past the last stage.)
    const uint32_t up = JOINED ? 64 * 128 : (uint32_t)p.take * 128, x_off = JOINED ? 2 * up : 2 * (uint32_t)p.take * 128;
    const uint32_t bar_off = (uint32_t)S * stage_bytes + 16384;
    const uint32_t bar = base + bar_off;
    const uint32_t full_b = bar, empty_b = bar + 8 * S, accf_b = bar + 16 * S, acce_b = accf_b + 8,
                   drain_b = acce_b + 8;
    uint32_t *tmem_slot = (uint32_t *)(smem_raw + pad + bar_off + 8 * (2 * S + 3));
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    float *staged = (float *)(smem_raw + pad + (uint32_t)S * stage_bytes);      // (of the 16 KB)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_b + 8 * s, 1);
            mbar_init(empty_b + 8 * s, 1);
        }
        mbar_init(accf_b, 1);
        mbar_init(acce_b, 8);
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
        Ring ring;
        int g = 0;
        bool ok = true;
        for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x)
            for (int c = 0; c < p.steps; ++c, ++g, ring.next(S)) {
                if (!wait(empty_b + 8 * ring.s, ring.ph ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                const uint32_t at = base + ring.s * stage_bytes, fb = full_b + 8 * ring.s;
                if (elected()) {
                    mbar_arrive_tx(fb, p.load_bytes);
                    for (int h = 0; h < p.per; ++h) {
                        const int k = (c * p.per + h) * kK;
                        const uint32_t to = at + h * p.chunk_bytes;
                        tma_load_2d(to, &p.Wg, k, tile * p.take, fb);
                        tma_load_2d(to + up, &p.Wu, k, tile * p.take, fb);
                        tma_load_2d(to + x_off, &p.X, k, 0, fb);
                    }
                }
                __syncwarp();
            }
        if (!ok && lane == 0)
            for (int j = g > S ? g - S : 0; j < g; ++j)
                drain_wait(full_b + 8 * (uint32_t)(j % S), (uint32_t)(j / S) & 1);
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t idesc = idesc_bf16(128, p.n);
        Ring ring;
        uint32_t it = 0, ready = 0;
        bool ok = true;
        for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x, ++it) {
            if (!wait(acce_b, (it & 1) ^ 1, abort_flag, p.err)) {
                ok = false;
                break;
            }
            tc_fence_after();
            for (int c = 0; c < p.steps; ++c) {
                if (!__all_sync(0xffffffffu, ready) && !wait(full_b + 8 * ring.s, ring.ph, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t at = base + ring.s * stage_bytes, done = empty_b + 8 * ring.s;
                ring.next(S);
                ready = peek(full_b + 8 * ring.s, ring.ph);
                if (elected()) {
                    for (int h = 0; h < p.per; ++h) {
                        const uint32_t a = at + h * p.chunk_bytes;
#pragma unroll
                        for (int kk = 0; kk < kK / 16; ++kk) {
                            const uint64_t bd = sdesc_sw128(a + x_off + kk * 32);
                            const uint32_t more = c > 0 || h > 0 || kk > 0 ? 1u : 0u;
                            mma_bf16(tmem, sdesc_sw128(a + kk * 32), bd, idesc, more);
                            if (!JOINED)
                                mma_bf16(tmem + p.n, sdesc_sw128(a + up + kk * 32), bd, idesc, more);
                        }
                    }
                    mma_commit(done);
                }
                __syncwarp();
            }
            if (ok && elected())
                mma_commit(accf_b);
            __syncwarp();
        }
        if (!ok && elected()) {        // (by the lane that issued them)
            mma_commit(drain_b);
            drain_wait(drain_b, 0);
        }
        __syncwarp();
    } else {
        const int q = warp & 3, second = (warp - 2) >> 2;
        uint32_t it = 0;
        for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++it) {
            const bool ok = wait(accf_b, it & 1, abort_flag, p.err);
            if (!(JOINED ? all_of_eight(ok) : ok))       // (the warps meet below: all leave or none)
                break;
            tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16);
            const int row = JOINED ? 32 * (q & 1) + lane : 32 * q + lane;
            const int feature = tile * p.take + row;
            const bool in = row < p.take && feature < p.f;
            const auto store = [&](__nv_bfloat16 *to, int c, const float (&v)[16]) {
                to += (int64_t)c * p.f + feature;
#pragma unroll
                for (int j = 0; j < 16; ++j, to += p.f)
                    if (in && c + j < p.T)
                        *to = __float2bfloat16_rn(v[j]);
            };
            const auto finish = [&](int c, float (&g)[16], const float (&u)[16]) {
                if (p.G) {
                    store(p.G, c, g);
                    store(p.U, c, u);
                }
                gate_all(g, u, p.act);
                store(p.H, c, g);
            };
            if (JOINED) {
                // 32 tokens at a time, 16 for each of a lane quarter's two warps; U's lanes leave
                // them in shared memory for G's
                for (int c0 = 0; c0 < p.n; c0 += 32) {
                    const int c = c0 + 16 * second;
                    float v[16];
                    __syncwarp();
                    if (c < p.n) {
                        tmem_ld16(taddr + c, v);
                        tmem_ld_wait();
                    }
                    if (q >= 2 && c < p.n)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            staged[(16 * second + j) * 64 + row] = v[j];
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (q < 2 && c < p.n) {
                        float u[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            u[j] = staged[(16 * second + j) * 64 + row];
                        finish(c, v, u);
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                }
            } else {
                // (a lane quarter's two warps take the tokens in turn)
                for (int c = 16 * second; c < p.n; c += 32) {
                    float g[16], u[16];
                    __syncwarp();
                    tmem_ld16(taddr + c, g);
                    tmem_ld16(taddr + p.n + c, u);
                    tmem_ld_wait();
                    finish(c, g, u);
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
// Bound by DRAM: three bf16 arrays read, two written.  8 blocks an SM walk them (8192 x 14336, silu
// 171 us, 6.9 TB/s, relu 177, gelu_tanh 182; a block for every 256 pieces 185).  gelu's erfc takes longer
// than the memory: 251.
struct GradArgs {
    const __nv_bfloat16 *dH, *G, *U;
    __nv_bfloat16 *dG, *dU;
    int64_t T, lddh;
    int64_t f8;             // pieces of 8 in a row
    int act;
};
__global__ void __launch_bounds__(256) k_glu_grad(const GradArgs a)
{
    griddep_start();
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y)
        for (int64_t j = blockIdx.x * 256 + threadIdx.x; j < a.f8; j += gridDim.x * 256) {
            const int64_t at = t * a.f8 + j;
            float h[8], g[8], u[8];
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)(a.dH + t * a.lddh) + j), h);
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)a.G + at), g);
            Vec<__nv_bfloat16>::unpack(*((const uint4 *)a.U + at), u);
            with_activation(a.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float slope;
                    const float x = activate<decltype(act)::value, true>(g[i], slope);
                    g[i] = h[i] * u[i] * slope;
                    u[i] = h[i] * x;
                }
            });
            *((uint4 *)a.dG + at) = Vec<__nv_bfloat16>::pack(g);
            *((uint4 *)a.dU + at) = Vec<__nv_bfloat16>::pack(u);
        }
}

// ---- rows on 128-byte boundaries -----------------------------------------------------------------
// A box row of 128 bytes that starts off a 128-byte boundary is two requests of a copy, and where both
// of a product's operands have such rows, requests bound it (copies alone, 4096 tokens: forward of
// 2056 x 5504 120 us, of 2048 x 5504 72).  So the gradients' X and weights are laid out anew, rows
// `ld` apart, where that is a small part of the products.
struct LayArgs {
    const uint4 *from[2];
    uint4 *to[2];
    int64_t rows, ld_from, ld_to;   // in 16-byte pieces
    int across;
};
__global__ void __launch_bounds__(256) k_glu_lay(const LayArgs a)
{
    griddep_start();
    const uint4 *from = a.from[blockIdx.y];
    uint4 *to = a.to[blockIdx.y];
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < a.rows * a.across; i += gridDim.x * 256) {
        const int64_t r = i / a.across, c = i - r * a.across;
        to[r * a.ld_to + c] = from[r * a.ld_from + c];
    }
}

// A wait for a phase that nothing completes, without an error word
__global__ void __launch_bounds__(32) k_unclaimed_timeout()
{
    __shared__ __align__(8) uint64_t bar;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bar), 1);
        abort_flag = 0;
        mbar_fence_init();
    }
    __syncthreads();
    wait(smem_u32(&bar), 0, &abort_flag, nullptr);
}

// ---- launches ------------------------------------------------------------------------------------

// Whether X (for the weights' gradients) and the weights (for dX) are laid out anew: where neither d nor
// f is a multiple of 64, and a copy of T d elements stands against f of their products, or one of f d
// against T.  us, as they lie and anew.
//   dW by f: 2088 (8192 x 520) 49.9 and 52.9, (16384 x 1032) 122 and 123; 3000 (2000 x 2056) 43.7 and 43.8,
//   (8192) 147 and 138; 4088 (4173 x 2056) 108 and 97, 4104 111 and 102, 5512 142 and 128; 8200 (8192 x 4104)
//   743 and 661.  (From about 3000 on it pays already, by 5 to 10%.)
//   dX by T: 2000 (2056 x 5512) 67.9 and 80.7; 4173 144 and 148; 6000 196 and 191; 8192 259 and 253; 16384
//   509 and 463; 8192 of 520 x 2088 44.0 and 44.6, of 4104 x 8200 702 and 662.
// Below 2^33 products neither makes much (8192 x 520 x 1032, 0.5 of that: dX 30.9 and 29.6, dW 31.4 and 35.4).
struct Laid {
    bool X, W;
    int64_t ld;             // elements
    size_t x_bytes, w_bytes;
};
Laid laid_of(int64_t T, int d, int f, int64_t ldx)
{
    Laid l;
    const bool odd = d % 64 && f % 64 && T * d >= ((int64_t)1 << 33) / f;
    l.X = odd && ldx % 64 && f >= 4096;
    l.W = odd && T >= 8192;
    l.ld = (d + 63) / 64 * 64;
    l.x_bytes = (size_t)T * l.ld * 2;
    l.w_bytes = (size_t)f * l.ld * 2;
    return l;
}
cudaError_t lay(const void *a, const void *b, void *a_to, void *b_to, int64_t rows, int d, int64_t ld_from,
                int64_t ld_to, cudaStream_t s)
{
    const LayArgs l{{(const uint4 *)a, (const uint4 *)b}, {(uint4 *)a_to, (uint4 *)b_to}, rows, ld_from / 8, ld_to / 8,
                    d / 8};
    count_launch();
    const cudaError_t e = launch_dependent(
        k_glu_lay, dim3((unsigned)std::min<int64_t>((rows * l.across + 255) / 256, 8 * device_sms()), b ? 2 : 1),
        dim3(256), 0, s, l);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// The work of `tiles` tiles (`down` of them down the rows) of `all` chunks on `units` pairs: rounds of
// whole tiles, and the last round's cut where that ends it at least kSaved chunks earlier (a chunk is
// 0.3 us; the parts and their sum take about 10).  A run is at least kRun chunks.  Runs of one length,
// end to end, keep every pair at work; where tiles lie below one another, runs that divide each tile
// alike, if they are hardly longer, let them read their common columns at the same time: dX of 512 x
// 4096 x 14336 105 us with runs of 189, the weights read twice from DRAM, and 82 with runs of 224.
constexpr int64_t kSaved = 32, kRun = 8;
struct Cut {
    int64_t whole, cut, run, span, parts;       // parts: places of 256 x 256
};
Cut cut_of(int64_t tiles, int64_t down, int64_t all, int64_t units)
{
    const int64_t left = tiles % units;
    int64_t run = left ? std::max(kRun, (left * all + units - 1) / units) : 0, span = all;
    if (left == 0 || all - run < kSaved)
        return Cut{tiles, 0, 0, all, 0};
    const int64_t each = units / left, alike = (all + each - 1) / each;
    if (down > 1 && each > 1 && alike >= kRun && 4 * alike <= 5 * run) {
        run = alike;
        span = each * run;
    }
    return Cut{tiles - left, left, run, span, (left * span + run - 1) / run + left};
}

template <int MODE, int CG>
cudaError_t launch_tiles(GluParams p, int sms, cudaStream_t s)
{
    const int units = std::max(1, sms / CG);
    p.mt = (p.rows + kRows * CG - 1) / (kRows * CG);
    constexpr int width = MODE == GLU_FWD ? kCols / 2 : kCols;
    p.nt = (p.cols + width - 1) / width;
    const int64_t tiles = p.mt * p.nt * (MODE == GLU_DW ? 2 : 1);
    const Cut c = MODE != GLU_FWD && CG == 2 ? cut_of(tiles, p.mt, p.chunks * (MODE == GLU_DX ? 2 : 1), units)
                                             : Cut{tiles, 0, 0, 1, 0};
    p.whole = c.whole;
    p.cut = c.cut;
    p.run = c.run;
    p.span = c.span;
    const int grid = (int)(c.cut ? units : std::min<int64_t>(tiles, units)) * CG;
    cudaError_t e = cudaFuncSetAttribute(k_glu<MODE, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, Stage<CG>::kSmem);
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_clusters(k_glu<MODE, CG>, CG, dim3(grid), dim3(kGluThreads), Stage<CG>::kSmem, s, p);
    if constexpr (MODE != GLU_FWD)
        if (e == cudaSuccess && c.cut) {
            count_launch();
            e = launch_dependent(k_glu_join<MODE>, dim3(32, (unsigned)c.cut), dim3(256), 0, s, p);
        }
    return e != cudaSuccess ? e : cudaGetLastError();
}

// An output of `rows` rows of `cols` elements, written in boxes of 32 rows of 128 bytes; fp32 ones as
// twice as many of 16 bits, which a copy does not tell apart
bool out_map(CUtensorMap *m, const void *out, int cols, int64_t rows, bool f32)
{
    return tensor_map_2d(m, out, (uint64_t)cols * (f32 ? 2 : 1), rows, (uint64_t)cols * (f32 ? 4 : 2), 64, 32);
}

// Whether the forward is expected earlier from CTAs each for itself, in cycles: a chunk takes them 650 and
// a pair 547, a pair's start and end 3300 more, and tiles of half the rows may fill the rounds better (us,
// pairs and single CTAs: 1024 tokens of 512 x 2048 9.2 and 7.9, 300 of 1024 x 4096 11.8 and 10.8, 640 of
// 4096 x 14336 109 and 102; 300 of 2048 x 8192 26.0 and 30.6, 2048 of 4096 x 14336 267 and 310).
bool alone(const GluParams &p, int sms)
{
    const int64_t nt = (p.cols + kCols / 2 - 1) / (kCols / 2);
    const auto rounds = [&](int rows, int units) {
        return ((p.rows + rows - 1) / rows * nt + units - 1) / units;
    };
    return rounds(kRows, sms) * p.chunks * 650 < rounds(2 * kRows, std::max(1, sms / 2)) * p.chunks * 547 + 3300;
}

// Pairs of CTAs where the stream's context has the whole GPU; with a part of it a pair might find
// no place.
template <int MODE>
cudaError_t launch_products(const GluParams &p, int all, int sms, cudaStream_t s)
{
    return sms < all || (MODE == GLU_FWD && alone(p, sms)) ? launch_tiles<MODE, 1>(p, sms, s)
                                                           : launch_tiles<MODE, 2>(p, sms, s);
}

// Rows of each weight that a CTA takes at a time, in as few rounds as 128 rows allow
int few_rounds(int f, int sms) { return (int)(((int64_t)f + sms * 128 - 1) / (sms * 128)); }
int few_rows(int f, int sms)
{
    const int rounds = few_rounds(f, sms);
    return std::min(128, ((f + sms * rounds - 1) / (sms * rounds) + 7) / 8 * 8);
}
bool is_few(int64_t T, int f, int sms)
{
    return T <= (few_rounds(f, sms) == 1 && few_rows(f, sms) > 64 ? kMoreTokens : kFewTokens);
}

cudaError_t launch_few(FewParams p, const __nv_bfloat16 *X, int64_t ldx, const __nv_bfloat16 *Wg,
                       const __nv_bfloat16 *Wu, int d, int sms, cudaStream_t s)
{
    p.n = (p.T + 15) / 16 * 16;
    p.take = few_rows(p.f, sms);
    p.tiles = (p.f + p.take - 1) / p.take;
    const bool joined = p.take <= 64;
    p.chunk_bytes = (uint32_t)((joined ? 128 : 2 * p.take) + p.n) * 128;
    // two chunks a stage, which halves the waits, where three such stages fit (75 tokens of 4096 x 14336
    // 40.6 us, 41.2 with one; 96, which leave two, 42.1 and 43.8)
    const uint32_t rest = 16384 + 1024 + 512, room = 232448 - rest;
    const int chunks = (d + kK - 1) / kK;
    p.per = room / (2 * p.chunk_bytes) >= 3 && chunks > 1 ? 2 : 1;
    p.steps = (chunks + p.per - 1) / p.per;
    p.load_bytes = (uint32_t)p.per * (2 * p.take + p.n) * 128;
    p.stages = std::max(2, std::min(16, (int)(room / (p.per * p.chunk_bytes))));
    p.columns = 32;
    while (p.columns < (joined ? 1u : 2u) * p.n)
        p.columns *= 2;
    if (!tensor_map_2d(&p.X, X, d, p.T, (uint64_t)ldx * 2, kK, p.n) ||
        !tensor_map_2d(&p.Wg, Wg, d, p.f, (uint64_t)d * 2, kK, p.take, true) ||
        !tensor_map_2d(&p.Wu, Wu, d, p.f, (uint64_t)d * 2, kK, p.take, true))
        return cudaErrorInvalidValue;
    const uint32_t smem = (uint32_t)p.stages * p.per * p.chunk_bytes + rest;
    const auto kernel = joined ? k_glu_few<true> : k_glu_few<false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
    if (e != cudaSuccess)
        return e;
    count_launch();
    e = launch_dependent(kernel, dim3(std::min(p.tiles, sms)), dim3(kFewThreads), smem, s, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace
}  // namespace tc

cudaError_t take_unclaimed(unsigned int *word)
{
    const unsigned int none = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(word, tc::g_unclaimed, sizeof none);
    return e == cudaSuccess && *word ? cudaMemcpyToSymbol(tc::g_unclaimed, &none, sizeof none) : e;
}
cudaError_t unclaimed_timeout(cudaStream_t s)
{
    count_launch();
    tc::k_unclaimed_timeout<<<1, 32, 0, s>>>();
    return cudaGetLastError();
}

cudaError_t glu_fwd(const void *X, int64_t ldx, const void *Wg, const void *Wu, int64_t T, int d, int f, int act,
                    void *G, void *U, void *H, unsigned int *err, cudaStream_t s)
{
    using namespace tc;
    typedef __nv_bfloat16 b16;
    const int sms = stream_sms(s);
    if (is_few(T, f, sms)) {
        FewParams p = {};
        p.T = (int)T;
        p.f = f;
        p.act = act;
        p.H = (b16 *)H;
        p.G = (b16 *)G;
        p.U = (b16 *)U;
        p.err = err;
        return launch_few(p, (const b16 *)X, ldx, (const b16 *)Wg, (const b16 *)Wu, d, sms, s);
    }
    GluParams p = {};
    p.rows = T;
    p.cols = f;
    p.chunks = (d + kK - 1) / kK;
    p.act = act;
    p.keep = G != nullptr;
    p.err = err;
    if (!out_map(&p.out[0], H, f, T, false) || (G && (!out_map(&p.out[1], G, f, T, false) ||
                                                       !out_map(&p.out[2], U, f, T, false))) ||
        !tensor_map_2d(&p.A[0], X, d, T, (uint64_t)ldx * 2, kK, kRows) ||
        !tensor_map_2d(&p.B[0], Wg, d, f, (uint64_t)d * 2, kK, 128) ||
        !tensor_map_2d(&p.B[1], Wu, d, f, (uint64_t)d * 2, kK, 128))
        return cudaErrorInvalidValue;
    return launch_products<GLU_FWD>(p, device_sms(), sms, s);
}

namespace tc {
namespace {

// The gradients' workspace: the parts of cut tiles, and behind them what is laid out anew, first for
// the one product, then for the other
struct Space {
    size_t parts, all;
};
Space space_of(int64_t T, int d, int f)
{
    const int64_t units = std::max(1, device_sms() / 2);
    const auto tiles = [](int64_t n) { return (n + 255) / 256; };
    const Cut dx = cut_of(tiles(T) * tiles(d), tiles(T), 2 * ((f + kK - 1) / kK), units);
    const Cut dw = cut_of(2 * tiles(f) * tiles(d), tiles(f), (T + kK - 1) / kK, units);
    const Laid l = laid_of(T, d, f, 1);
    Space w;
    w.parts = (size_t)std::max(dx.parts, dw.parts) * (256 * 256 * sizeof(float));
    w.all = w.parts + std::max(l.X ? l.x_bytes : 0, l.W ? 2 * l.w_bytes : 0);
    return w;
}

}  // namespace
}  // namespace tc

size_t glu_bwd_workspace(int64_t T, int d, int f) { return tc::space_of(T, d, f).all; }

cudaError_t glu_bwd(const void *dH, int64_t lddh, const void *X, int64_t ldx, const void *Wg, const void *Wu,
                    const void *G, const void *U, int64_t T, int d, int f, int act, void *dG, void *dU, void *dX,
                    sn_dtype grad_dt, void *dWg, void *dWu, bool accumulate, void *ws, unsigned int *err,
                    cudaStream_t s)
{
    using namespace tc;
    typedef __nv_bfloat16 b16;
    // (rows behind one another are one)
    const bool one = lddh == f;
    const GradArgs a{(const b16 *)dH, (const b16 *)G, (const b16 *)U, (b16 *)dG, (b16 *)dU, one ? 1 : T, lddh,
                     one ? T * (f / 8) : f / 8, act};
    const int all = device_sms(), sms = dX || dWg ? stream_sms(s) : all;
    const int64_t across = std::min<int64_t>((a.f8 + 255) / 256, 8 * all);
    count_launch();
    cudaError_t e = launch_dependent(k_glu_grad, dim3((unsigned)across, (unsigned)std::min<int64_t>(a.T, 65535)),
                                     dim3(256), 0, s, a);
    if (e == cudaSuccess)
        e = cudaGetLastError();
    const Laid l = laid_of(T, d, f, ldx);
    char *anew = l.X || l.W ? (char *)ws + space_of(T, d, f).parts : nullptr;
    if (e == cudaSuccess && dX) {
        int64_t ld = d;
        if (l.W) {
            e = lay(Wg, Wu, anew, anew + l.w_bytes, f, d, d, l.ld, s);
            if (e != cudaSuccess)
                return e;
            Wg = anew;
            Wu = anew + l.w_bytes;
            ld = l.ld;
        }
        GluParams p = {};
        p.rows = T;
        p.cols = d;
        p.chunks = (f + kK - 1) / kK;
        p.at[0] = dX;
        p.parts = (float *)ws;
        p.err = err;
        if (!out_map(&p.out[0], dX, d, T, false) || !tensor_map_2d(&p.A[0], dG, f, T, (uint64_t)f * 2, kK, kRows) ||
            !tensor_map_2d(&p.A[1], dU, f, T, (uint64_t)f * 2, kK, kRows) ||
            !tensor_map_2d(&p.B[0], Wg, d, f, (uint64_t)ld * 2, 64, kK) ||
            !tensor_map_2d(&p.B[1], Wu, d, f, (uint64_t)ld * 2, 64, kK))
            return cudaErrorInvalidValue;
        e = launch_products<GLU_DX>(p, all, sms, s);
    }
    if (e == cudaSuccess && dWg) {
        if (l.X) {
            e = lay(X, nullptr, anew, nullptr, T, d, ldx, l.ld, s);
            if (e != cudaSuccess)
                return e;
            X = anew;
            ldx = l.ld;
        }
        GluParams p = {};
        p.rows = f;
        p.cols = d;
        p.chunks = (T + kK - 1) / kK;
        p.at[0] = dWg;
        p.at[1] = dWu;
        p.parts = (float *)ws;
        p.out_f32 = grad_dt == SN_F32;
        p.add = accumulate;
        p.err = err;
        if (!out_map(&p.out[0], dWg, d, f, p.out_f32) || !out_map(&p.out[1], dWu, d, f, p.out_f32) ||
            !tensor_map_2d(&p.A[0], dG, f, T, (uint64_t)f * 2, 64, kK) ||
            !tensor_map_2d(&p.A[1], dU, f, T, (uint64_t)f * 2, 64, kK) ||
            !tensor_map_2d(&p.B[0], X, d, T, (uint64_t)ldx * 2, 64, kK))
            return cudaErrorInvalidValue;
        e = launch_products<GLU_DW>(p, all, sms, s);
    }
    return e;
}

}  // namespace sn
