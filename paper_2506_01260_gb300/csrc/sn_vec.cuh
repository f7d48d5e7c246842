// sn_vec.cuh — 16-byte pieces of bf16 and fp32 rows, and sums over the threads that share
// a row: what the step operators' kernels (embedding, norm, log probabilities, gradients)
// have in common.
#pragma once

#include "sn_internal.cuh"

namespace sn {

// N elements of T lie in 16 bytes; they are computed with as fp32.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float one(float x) { return x; }
    static __device__ __forceinline__ float round(float x) { return x; }
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                          __float_as_uint(f[3]));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *(const uint32_t *)&p;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// N consecutive elements as fp32 (16-byte aligned for fp32, N * 2 bytes for bf16)
template <int N>
__device__ __forceinline__ void load_floats(const float *p, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 v = __ldg((const float4 *)(p + i));
        f[i] = v.x;
        f[i + 1] = v.y;
        f[i + 2] = v.z;
        f[i + 3] = v.w;
    }
}
__device__ __forceinline__ void load_floats(const __nv_bfloat16 *p, float (&f)[8])
{
    Vec<__nv_bfloat16>::unpack(__ldg((const uint4 *)p), f);
}
__device__ __forceinline__ void load_floats(const __nv_bfloat16 *p, float (&f)[4])
{
    const uint2 v = __ldg((const uint2 *)p);
    f[0] = __uint_as_float(v.x << 16);
    f[1] = __uint_as_float(v.x & 0xFFFF0000u);
    f[2] = __uint_as_float(v.y << 16);
    f[3] = __uint_as_float(v.y & 0xFFFF0000u);
}

__device__ __forceinline__ bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

template <typename V>
__device__ __forceinline__ V warp_sum(V v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---- fp32 pairs: one instruction for two (the intrinsics on float2 compile to one; 64-bit
// integers through inline PTX took 2.5, moves among them) ------------------------------------
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// a 16-byte piece as pairs
__device__ __forceinline__ void unpack_pairs(uint4 v, float2 (&f)[2])
{
    f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
    f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ void unpack_pairs(uint4 v, float2 (&f)[4])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ uint4 pack_pairs(const float2 (&f)[2])
{
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x),
                      __float_as_uint(f[1].y));
}
__device__ __forceinline__ uint4 pack_pairs(const float2 (&f)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __float22bfloat162_rn(f[i]);
        w[i] = *(const uint32_t *)&p;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Asks for `bytes` (a multiple of 16) from a 16-byte boundary on to be brought into L2
__device__ __forceinline__ void prefetch_l2(const void *p, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

int device_sms();   // SMs of the current device

}  // namespace sn
