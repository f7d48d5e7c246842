// sn_grads.cu — the global gradient norm over a list of tensors, and clipping by it.
//
//   sumsq = sum over all tensors of g^2,  norm = sqrt(sumsq),
//   out = g * c,  c = max_norm / max(norm, max_norm)
//
// Bound by DRAM: 2 or 4 bytes read an element for the sum, the same again and as many
// written to clip (nothing where c = 1 in place).  The list is cut into chunks of kChunkBytes
// once, when its handle is made; both kernels walk the chunk table, so a list of
// hundreds of tensors of every size is one launch with the same work for every block.
//
// Measured, 1.74 billion bf16 gradients (3.5 GB): the sum 470 us (7.4 TB/s), clipping 1000 us (7.0
// TB/s); a list of 4 MB 6.2 and 5.5 us, launch and the last block's sum.
#include <algorithm>
#include <new>
#include <vector>

#include "sn_vec.cuh"

// One piece of a tensor.
struct sn_grad_chunk {
    const void *src;
    void *dst;
    int n;          // elements
    int flags;      // below
};

struct sn_grads {
    int device;
    int64_t chunks;
    int sms;
    void *mem;                 // the one device allocation that the pointers below lie in
    sn_grad_chunk *table;
    double *partial;           // one sum per block
    unsigned int *ticket;      // blocks that are done; 0 between calls
};

namespace sn {
namespace {

constexpr int kThreads = 256;
// 8 loads of 16 bytes a thread (bf16 chunks of half as much: 524 us for 3.5 GB, now 469)
constexpr int kChunkBytes = 32768;
constexpr int kPerSm = 8;
// Clipping, blocks an SM of a list with kMany chunks an SM or more: 3.5 GB of bf16 take 1000 us,
// 1024 with 8 (fewer rounds of the same blocks write in step).  Below that the blocks would not
// have the same number of chunks (0.34 GB: 108 us with 8, 115 with 32).
constexpr int kPerSmMany = 32, kMany = 128;
enum { SRC_BF16 = 1, DST_BF16 = 2, ALIGNED = 4, IN_PLACE = 8 };

// Squares below 2^-126 lose bits and above 2^128 overflow: a thread whose fp32 sum lies
// outside this range takes its elements again in fp64, so that the norm of any finite
// gradients is right.
constexpr float kLow = 0x1p-100f, kHigh = 0x1p126f;

template <typename T, int U>
__device__ __forceinline__ double square_sum(const uint4 (&v)[U])
{
    constexpr int N = Vec<T>::N;
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[N];
        Vec<T>::unpack(v[u], f);
#pragma unroll
        for (int i = 0; i < N; ++i)
            s = fmaf(f[i], f[i], s);
    }
    if (s >= kLow && s <= kHigh)
        return (double)s;
    double d = 0.0;
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
        float f[N];
        uint4 w = v[0];
#pragma unroll
        for (int k = 1; k < U; ++k)
            w = u == k ? v[k] : w;
        constexpr uint32_t kMagnitude = N == 8 ? 0x7FFF7FFFu : 0x7FFFFFFFu;
        if (((w.x | w.y | w.z | w.w) & kMagnitude) == 0)   // zeros: an embedding's unused rows
            continue;
        Vec<T>::unpack(w, f);
#pragma unroll
        for (int i = 0; i < N; ++i)
            d = fma((double)f[i], (double)f[i], d);
    }
    return d;
}

template <typename T>
__device__ __forceinline__ double chunk_sum(const sn_grad_chunk &c)
{
    constexpr int N = Vec<T>::N, U = 8;
    const T *src = (const T *)c.src;
    double s = 0.0;
    int done = 0;
    if (aligned16(src)) {
        const int nv = c.n / N;
        for (int i = threadIdx.x; i < nv; i += U * kThreads) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[u] = i + u * kThreads < nv ? __ldg((const uint4 *)src + i + u * kThreads)
                                             : make_uint4(0, 0, 0, 0);
            s += square_sum<T, U>(v);
        }
        done = nv * N;
    }
    for (int i = done + threadIdx.x; i < c.n; i += kThreads) {
        const double x = (double)Vec<T>::one(src[i]);
        s = fma(x, x, s);
    }
    return s;
}

// The sum of `s` over the block, in thread 0
__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double red[kThreads / 32];
    s = warp_sum(s);
    __syncthreads();
    if (threadIdx.x % 32 == 0)
        red[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kThreads / 32; ++w)
            s += red[w];
    return s;
}

// Every block sums its chunks in fp64; the block that is done last adds the blocks' sums in
// their order, whichever block that is, so the result is the same bits every time.
__global__ void __launch_bounds__(kThreads) k_sumsq(const sn_grad_chunk *__restrict__ table,
                                                     int64_t chunks, double *__restrict__ partial,
                                                     unsigned int *ticket, double *out, int accumulate)
{
    griddep_start();
    double s = 0.0;
    sn_grad_chunk next = {};
    if (blockIdx.x < chunks)
        next = table[blockIdx.x];
    for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const sn_grad_chunk c = next;
        if (i + gridDim.x < chunks)
            next = table[i + gridDim.x];
        s += c.flags & SRC_BF16 ? chunk_sum<__nv_bfloat16>(c) : chunk_sum<float>(c);
    }
    s = block_sum(s);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        partial[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last)
        return;
    __threadfence();
    s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads)
        s += __ldcg(partial + i);
    s = block_sum(s);
    if (threadIdx.x == 0) {
        *out = accumulate ? *out + s : s;
        *ticket = 0;
    }
}

// dst = src * pre * f; pre is 1, or 2^-126 for a factor below fp32's normal numbers, which would
// lose bits in one: such a list goes by single elements.
template <typename S, typename D>
__device__ __forceinline__ void scale_chunk(const sn_grad_chunk &c, float f, float pre)
{
    const S *src = (const S *)c.src;
    D *dst = (D *)c.dst;
    int done = 0;
    if ((c.flags & ALIGNED) && pre == 1.f) {
        constexpr int N = 8, U = sizeof(S) == 2 ? 4 : 2;  // 8 elements, 64 bytes of loads in flight
        const int nv = c.n / N;
        for (int i = threadIdx.x; i < nv; i += U * kThreads) {
            uint4 v[U][N / Vec<S>::N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < N / Vec<S>::N; ++j)
                    if (i + u * kThreads < nv)
                        v[u][j] = ((const uint4 *)src)[(i + u * kThreads) * (N / Vec<S>::N) + j];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kThreads < nv) {
                    float x[N];
#pragma unroll
                    for (int j = 0; j < N / Vec<S>::N; ++j)
                        Vec<S>::unpack(v[u][j], *(float(*)[Vec<S>::N])(x + j * Vec<S>::N));
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        x[k] *= f;
#pragma unroll
                    for (int j = 0; j < N / Vec<D>::N; ++j)
                        ((uint4 *)dst)[(i + u * kThreads) * (N / Vec<D>::N) + j] =
                            Vec<D>::pack(*(const float(*)[Vec<D>::N])(x + j * Vec<D>::N));
                }
        }
        done = nv * N;
    }
    for (int i = done + threadIdx.x; i < c.n; i += kThreads)
        dst[i] = Vec<D>::round(Vec<S>::one(src[i]) * pre * f);
}

// Three blocks an SM: 64 bytes of loads a thread in flight for either type fit 78 registers (two
// blocks of 123 registers: 3.5 GB of bf16 1104 us).
__global__ void __launch_bounds__(kThreads, 3) k_clip(const sn_grad_chunk *__restrict__ table,
                                                    int64_t chunks, const double *sumsq, float max_norm,
                                                    float *norm_out)
{
    griddep_start();
    const double norm = sqrt(*sumsq);
    // NaN stays NaN; an infinite norm gives 0
    const double factor = norm > (double)max_norm ? (double)max_norm / norm : norm == norm ? 1.0 : norm;
    // (in whole numbers: an fp64 comparison and product took 0.3 us of a short list's call)
    const int high = __double2hiint(factor);
    const bool small = high > 0 && high < (1023 - 126) << 20;          // 0 < factor < 2^-126
    const float pre = small ? 0x1p-126f : 1.f;
    const float f = (float)__hiloint2double(small ? high + (126 << 20) : high, __double2loint(factor));
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *norm_out = (float)norm;
    // from the list's end, whose elements the sum has left in L2
    sn_grad_chunk next = {};
    if (blockIdx.x < chunks)
        next = table[chunks - 1 - blockIdx.x];
    for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const sn_grad_chunk c = next;
        if (i + gridDim.x < chunks)
            next = table[chunks - 1 - i - gridDim.x];
        if (f == 1.f && (c.flags & IN_PLACE))
            continue;
        switch (c.flags & (SRC_BF16 | DST_BF16)) {
        case 0: scale_chunk<float, float>(c, f, pre); break;
        case SRC_BF16: scale_chunk<__nv_bfloat16, float>(c, f, pre); break;
        case DST_BF16: scale_chunk<float, __nv_bfloat16>(c, f, pre); break;
        default: scale_chunk<__nv_bfloat16, __nv_bfloat16>(c, f, pre); break;
        }
    }
}

int grid_of(const sn_grads &g, int per_sm)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(g.chunks, (int64_t)g.sms * per_sm));
}

}  // namespace

int device_sms()
{
    int dev = 0, sms = 1;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms;
}

cudaError_t grads_create(int n, const void *const *src, const sn_dtype *src_dt, const int64_t *count,
                         void *const *dst, const sn_dtype *dst_dt, sn_grads **out, cudaStream_t s)
{
    std::vector<sn_grad_chunk> table;
    for (int t = 0; t < n; ++t) {
        const int es = src_dt[t] == SN_BF16 ? 2 : 4, ed = dst_dt[t] == SN_BF16 ? 2 : 4;
        const char *p = (const char *)src[t];
        char *q = (char *)dst[t];
        const int flags = (src_dt[t] == SN_BF16 ? SRC_BF16 : 0) | (dst_dt[t] == SN_BF16 ? DST_BF16 : 0) |
                          ((((uintptr_t)p | (uintptr_t)q) & 15) == 0 ? ALIGNED : 0) |
                          (p == q ? IN_PLACE : 0);
        const int most = kChunkBytes / es;
        for (int64_t i = 0; i < count[t]; i += most)
            table.push_back({p + i * es, q + i * ed, (int)std::min<int64_t>(most, count[t] - i), flags});
    }
    sn_grads *g = new sn_grads();
    g->chunks = (int64_t)table.size();
    g->sms = device_sms();
    const size_t tb = (table.size() * sizeof(sn_grad_chunk) + 255) & ~(size_t)255;
    const size_t pb = ((size_t)g->sms * kPerSm * sizeof(double) + 255) & ~(size_t)255;
    cudaError_t e = cudaGetDevice(&g->device);
    if (e == cudaSuccess)
        e = cudaMalloc(&g->mem, tb + pb + 256);
    if (e == cudaSuccess) {
        g->table = (sn_grad_chunk *)g->mem;
        g->partial = (double *)((char *)g->mem + tb);
        g->ticket = (unsigned int *)((char *)g->mem + tb + pb);
        if (!table.empty())
            e = cudaMemcpyAsync(g->table, table.data(), table.size() * sizeof(sn_grad_chunk),
                                cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess)
            e = cudaMemsetAsync(g->ticket, 0, sizeof(unsigned int), s);
        if (e == cudaSuccess)
            e = cudaStreamSynchronize(s);
    }
    if (e != cudaSuccess) {
        cudaFree(g->mem);
        delete g;
        return e;
    }
    *out = g;
    return cudaSuccess;
}

cudaError_t grads_destroy(sn_grads *g)
{
    const cudaError_t e = cudaFree(g->mem);
    delete g;
    return e;
}

int grads_device(const sn_grads *g) { return g->device; }

cudaError_t grads_sumsq(const sn_grads &g, double *sumsq, bool accumulate, cudaStream_t s)
{
    count_launch();
    const cudaError_t e = launch_dependent(k_sumsq, dim3(grid_of(g, kPerSm)), dim3(kThreads), 0, s, g.table, g.chunks,
                                           g.partial, g.ticket, sumsq, (int)accumulate);
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t grads_clip(const sn_grads &g, const double *sumsq, float max_norm, float *norm, cudaStream_t s)
{
    const int per_sm = g.chunks >= (int64_t)kMany * g.sms ? kPerSmMany : kPerSm;
    count_launch();
    const cudaError_t e = launch_dependent(k_clip, dim3(grid_of(g, per_sm)), dim3(kThreads), 0, s, g.table, g.chunks,
                                           sumsq, max_norm, norm);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace sn
