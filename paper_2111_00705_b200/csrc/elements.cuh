// Element types of the operators (binary32, bfloat16, binary16) and block-wide reductions in
// binary32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "operators.h"

namespace cdadam {

typedef __nv_bfloat16 bf16;
typedef __half f16;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(f16 v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 narrow<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ f16 narrow<f16>(float v) { return __float2half_rn(v); }

// Element i of a vector whose type is known at run time only (parameters).
__device__ __forceinline__ float any_at(const AnyVec &v, int64_t i)
{
    if (v.type == 0) return __ldg(static_cast<const float *>(v.p) + i);
    if (v.type == 1) return widen(__ldg(static_cast<const bf16 *>(v.p) + i));
    return widen(__ldg(static_cast<const f16 *>(v.p) + i));
}

constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Sum / maximum over a block of NT threads, the same value in every thread.  `sh`: NT / 32
// floats, free for reuse after the block's next barrier.
template <int NT>
__device__ __forceinline__ float block_sum_all(float v, float *sh)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < NT / 32 ? sh[lane] : 0.0f);
}
template <int NT>
__device__ __forceinline__ float block_max_all(float v, float *sh)
{
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_max(lane < NT / 32 ? sh[lane] : kNegInf);
}


// 2^x, relative error below 2^-22; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two binary32 operations in one instruction, each rounded to nearest.
__device__ __forceinline__ uint64_t bits64(float2 v)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 floats(uint64_t b)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(b));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits64(a)), "l"(bits64(b)));
    return floats(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits64(a)), "l"(bits64(b)));
    return floats(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits64(a)), "l"(bits64(b)), "l"(bits64(c)));
    return floats(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// The larger of two; NaN if either is NaN.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A 16-byte vector of T: n elements, widened to n / 2 pairs and narrowed back; `running` is the
// type in which a maximum is carried along (the 16-bit types keep it packed), `below` the largest
// value of T that is not above v, `at_least` raises every element to a bound (NaN stays NaN).
template <typename T> struct Vec;

template <> struct Vec<float> {
    static constexpr int n = 4;
    static constexpr bool wide_range = true;
    typedef float running;
    static __device__ __forceinline__ running lowest() { return kNegInf; }
    static __device__ __forceinline__ void wide(const uint4 &u, float2 (&f)[2])
    {
        f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[2])
    {
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    }
    static __device__ __forceinline__ running top(const uint4 &u)
    {
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
    static __device__ __forceinline__ running max(running a, running b) { return fmaxf(a, b); }
    static __device__ __forceinline__ float value(running a) { return a; }
    static __device__ __forceinline__ running below(float v) { return v; }
    static __device__ __forceinline__ uint4 at_least(const uint4 &u, running t)
    {
        return make_uint4(__float_as_uint(max_nan(__uint_as_float(u.x), t)), __float_as_uint(max_nan(__uint_as_float(u.y), t)),
                          __float_as_uint(max_nan(__uint_as_float(u.z), t)), __float_as_uint(max_nan(__uint_as_float(u.w), t)));
    }
};

template <> struct Vec<bf16> {
    static constexpr int n = 8;
    static constexpr bool wide_range = true;
    typedef __nv_bfloat162 running;
    static __device__ __forceinline__ __nv_bfloat162 two(uint32_t w) { return *reinterpret_cast<__nv_bfloat162 *>(&w); }
    static __device__ __forceinline__ running lowest() { return two(0xFF80FF80u); }
    static __device__ __forceinline__ float2 up(uint32_t w)
    {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ void wide(const uint4 &u, float2 (&f)[4])
    {
        f[0] = up(u.x); f[1] = up(u.y); f[2] = up(u.z); f[3] = up(u.w);
    }
    static __device__ __forceinline__ uint32_t down(float2 f)
    {
        __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
        return *reinterpret_cast<uint32_t *>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[4])
    {
        return make_uint4(down(f[0]), down(f[1]), down(f[2]), down(f[3]));
    }
    static __device__ __forceinline__ running max(running a, running b) { return __hmax2(a, b); }
    static __device__ __forceinline__ running top(const uint4 &u)
    {
        return __hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w)));
    }
    static __device__ __forceinline__ float value(running a) { return fmaxf(__low2float(a), __high2float(a)); }
    static __device__ __forceinline__ running below(float v) { return __bfloat162bfloat162(__float2bfloat16_rd(v)); }
    static __device__ __forceinline__ uint32_t word(__nv_bfloat162 h) { return *reinterpret_cast<uint32_t *>(&h); }
    static __device__ __forceinline__ uint4 at_least(const uint4 &u, running t)
    {
        return make_uint4(word(__hmax2_nan(two(u.x), t)), word(__hmax2_nan(two(u.y), t)), word(__hmax2_nan(two(u.z), t)),
                          word(__hmax2_nan(two(u.w), t)));
    }
};

template <> struct Vec<f16> {
    static constexpr int n = 8;
    static constexpr bool wide_range = false;   // -65504 is too near for "far below everything"
    typedef __half2 running;
    static __device__ __forceinline__ __half2 two(uint32_t w) { return *reinterpret_cast<__half2 *>(&w); }
    static __device__ __forceinline__ running lowest() { return two(0xFC00FC00u); }
    static __device__ __forceinline__ float2 up(uint32_t w) { return __half22float2(two(w)); }
    static __device__ __forceinline__ void wide(const uint4 &u, float2 (&f)[4])
    {
        f[0] = __half22float2(two(u.x)); f[1] = __half22float2(two(u.y));
        f[2] = __half22float2(two(u.z)); f[3] = __half22float2(two(u.w));
    }
    static __device__ __forceinline__ uint32_t down(float2 f)
    {
        __half2 h = __floats2half2_rn(f.x, f.y);
        return *reinterpret_cast<uint32_t *>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[4])
    {
        return make_uint4(down(f[0]), down(f[1]), down(f[2]), down(f[3]));
    }
    static __device__ __forceinline__ running max(running a, running b) { return __hmax2(a, b); }
    static __device__ __forceinline__ running top(const uint4 &u)
    {
        return __hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w)));
    }
    static __device__ __forceinline__ float value(running a) { return fmaxf(__low2float(a), __high2float(a)); }
    static __device__ __forceinline__ running below(float v) { return __half2half2(__float2half_rd(v)); }
    static __device__ __forceinline__ uint32_t word(__half2 h) { return *reinterpret_cast<uint32_t *>(&h); }
    static __device__ __forceinline__ uint4 at_least(const uint4 &u, running t)
    {
        return make_uint4(word(__hmax2_nan(two(u.x), t)), word(__hmax2_nan(two(u.y), t)), word(__hmax2_nan(two(u.z), t)),
                          word(__hmax2_nan(two(u.w), t)));
    }
};

// 1 / sqrt(v): the approximation and one Newton step, within 1 ulp or so and a third of the
// instructions of the correctly rounded quotient and root.  0 and infinity have no step to take (0
// times infinity): v = 0 gives infinity, a sum of squares that overflowed gives 0.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v);
    return r > 0.0f && r < 3e38f ? r * fmaf(-0.5f * r * v, r, 1.5f) : r;
}

// Element i of a gradient whose type is known at run time only; accumulate: added to what is there.
__device__ __forceinline__ void store_grad(void *p, int64_t i, int type, int accumulate, float v)
{
    if (type == 0) {
        float *q = static_cast<float *>(p) + i;
        *q = accumulate ? *q + v : v;
    } else if (type == 1) {
        bf16 *q = static_cast<bf16 *>(p) + i;
        *q = narrow<bf16>(accumulate ? widen(*q) + v : v);
    } else {
        f16 *q = static_cast<f16 *>(p) + i;
        *q = narrow<f16>(accumulate ? widen(*q) + v : v);
    }
}

template <typename T> __device__ __forceinline__ T minus_inf() { return narrow<T>(kNegInf); }

}  // namespace cdadam
