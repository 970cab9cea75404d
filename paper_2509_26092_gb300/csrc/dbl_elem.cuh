// dbl_elem.cuh -- element types and block sums of the token operators (ln.cu, scan.cu, distill.cu), whose
// tensors are fp32 or the library's 16-bit format.
#pragma once

#include "dbl_internal.cuh"

namespace dbl {

inline bool elem_dtype_ok(int dtype) { return dtype == DBL_F32 || dtype == DBL_BF16; }
inline size_t elem_bytes(int dtype) { return dtype == DBL_F32 ? sizeof(float) : sizeof(act_t); }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

#if defined(__CUDACC__)
namespace dev {

__device__ __forceinline__ float elem_f(float v) { return v; }
__device__ __forceinline__ float elem_f(act_t v) { return act::to_f(v); }

template <class T>
__device__ __forceinline__ T elem_from(float v);
template <>
__device__ __forceinline__ float elem_from<float>(float v) { return v; }
template <>
__device__ __forceinline__ act_t elem_from<act_t>(float v) { return act::from_f(v); }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Sum (or maximum) over the block's threads, the same bits in all of them.  red: 32 floats of shared memory, free
// again after the call.
__device__ __forceinline__ float block_sum(float v, float* red)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += red[w];
    __syncthreads();
    return s;
}

__device__ __forceinline__ float block_max(float v, float* red)
{
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = red[0];
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) s = fmaxf(s, red[w]);
    __syncthreads();
    return s;
}

}  // namespace dev
#endif

}  // namespace dbl
