// sn_norm.cuh — what the kernels that norm rows of a residual stream share (sn_rmsnorm.cu,
// sn_blocknorm.cu): the lanes of a row, sums over them, weights of either type, and rows whose
// squares leave fp32's range.
#pragma once

#include <algorithm>
#include <atomic>

#include "sn_vec.cuh"

namespace sn {
namespace {

// A row of d elements, in `nv` 16-byte pieces, is shared by G lanes: lane l has the pieces l,
// l + G, ... (at most C).  Narrow rows are a warp's each (S = 32: a block of 256 threads takes
// eight), wider ones a block's of G <= S threads, G a multiple of 32, so that no width leaves
// more than a few lanes without work.
// EXACT: G is S, and every lane has all its pieces: no bounds, and indices that are constants
// (codes of 65536 rows of 8192: 522 us, 569 with bounds; without a residual 16384 rows of 4096 41
// and 44).
template <int S, bool EXACT = false>
struct Shape {
    static constexpr int kThreads = S == 32 ? 256 : S;      // at most
    static constexpr int kRows = S == 32 ? 8 : 1;
    static __device__ __forceinline__ int lanes() { return S == 32 || EXACT ? S : (int)blockDim.x; }
};

// The sums (or maxima) of K values over the lanes of a row, in every lane.  `red`: 2 * K * 32
// floats that calls alternate between (`turn`), so one barrier a call is enough.
template <int S, int K, bool MAX, bool EXACT = false>
__device__ __forceinline__ void row_reduce(float (&v)[K], float *red, int &turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float x = __shfl_xor_sync(0xffffffffu, v[k], o);
            v[k] = MAX ? max_nan(v[k], x) : v[k] + x;
        }
    if (S == 32)
        return;
    const int warps = Shape<S, EXACT>::lanes() / 32;
    float *at = red + turn * (K * 32);
    turn ^= 1;
    // (lanes 1 to 3 of the last warp fill up to a multiple of four)
    const int slot = (int)threadIdx.x / 32 + (int)threadIdx.x % 32;
    if (threadIdx.x % 32 == 0 || (threadIdx.x % 32 < 4 && slot >= warps && slot < 32))
#pragma unroll
        for (int k = 0; k < K; ++k)
            at[k * 32 + slot] = threadIdx.x % 32 == 0 ? v[k] : 0.f;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < S / 32; w += 4) {
            if (!EXACT && w >= warps)
                break;
            const float4 x = *(const float4 *)(at + k * 32 + w);
            s = MAX ? make_float4(max_nan(s.x, x.x), max_nan(s.y, x.y), max_nan(s.z, x.z), max_nan(s.w, x.w))
                    : make_float4(s.x + x.x, s.y + x.y, s.z + x.z, s.w + x.w);
        }
        v[k] = MAX ? max_nan(max_nan(s.x, s.y), max_nan(s.z, s.w)) : (s.x + s.y) + (s.z + s.w);
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

// ---- rows whose squares leave fp32's range -----------------------------------------------
// A sum of squares is taken as it is where its mean (with eps) is from kLeast on, so that what
// squares below fp32's numbers lose is below 2^-49 of it, and where it did not overflow.  Other
// rows are taken again as h f, f = 2^-80 or 2^100: a finite row's mean of squares, with eps f^2
// beside it, is then a number, n is the same, and the reciprocal root is 1 / f of the row's.  A
// mean that still is none comes from an infinity or a NaN, and the row is NaN.
//
// The kernels below keep that off the other rows' way, each as its registers allow: the test is two
// comparisons with bounds that the host made, and what a scaled row takes is not kept beside what
// the others do (kept, it spilled: the gradient of 65536 rows of 8192 bf16 took 837 us, 605 now).
constexpr float kLeast = 0x1p-100f, kMost = 3.402823466e38f;

float least_sum(int d, float eps) { return std::max(0.f, (kLeast - eps) * (float)d); }
float most_sum(float eps) { return eps < 1e37f ? kMost / 2.f : 0.f; }

template <typename A>
__device__ __forceinline__ bool in_range(const A &a, float sum) { return sum >= a.least && sum <= a.most; }
template <typename A>
__device__ __forceinline__ float factor_of(const A &a, float sum) { return sum < a.least ? 0x1p100f : 0x1p-80f; }
__device__ __forceinline__ float root_of(float mean) { return mean <= kMost ? rsqrtf(mean) : NAN; }
// Threads of a block that walks a row by single elements
constexpr int kAnyThreads = 512;

// ---- launches ----------------------------------------------------------------------------------

// The lanes of a row of nv pieces: the fewest warps that hold it with `most` pieces a lane
int lanes_of(int nv, int most) { return std::max(1, (nv + 32 * most - 1) / (32 * most)) * 32; }

// Blocks of `threads` that are on an SM at once, asked for once for each kernel and size (a
// property of the code, the same on every GPU it runs on)
template <auto KERNEL>
int resident(int threads)
{
    static std::atomic<int> known[33];
    std::atomic<int> &slot = known[threads / 32];
    int n = slot.load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, threads, 0) != cudaSuccess)
            return 1;
        slot.store(n = std::max(n, 1), std::memory_order_relaxed);
    }
    return n;
}

template <typename K, typename A>
cudaError_t launch(K kernel, int64_t grid, int threads, const A &a, cudaStream_t s)
{
    count_launch();
    const cudaError_t e = launch_dependent(kernel, dim3((unsigned)grid), dim3(threads), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace
}  // namespace sn
