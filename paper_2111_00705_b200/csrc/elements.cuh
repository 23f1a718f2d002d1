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

}  // namespace cdadam
