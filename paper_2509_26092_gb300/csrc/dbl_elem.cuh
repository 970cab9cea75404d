// dbl_elem.cuh -- element types and block sums of the token operators (ln.cu, scan.cu, distill.cu), whose
// tensors are fp32 or the library's 16-bit format.
#pragma once

#include "dbl_internal.cuh"

namespace dbl {

inline bool elem_dtype_ok(int dtype) { return dtype == DBL_F32 || dtype == DBL_BF16; }
inline size_t elem_bytes(int dtype) { return dtype == DBL_F32 ? sizeof(float) : sizeof(act_t); }
constexpr int kMaxColumns = (1 << 30) - 1;  // of a row: the kernels' indexes and twice this are 32-bit
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

#if defined(__CUDACC__)
// Lets KERNEL be launched with up to `bytes` of dynamic shared memory, the same for all its launches, and in clusters of
// more than eight blocks where asked.  Once per device.
template <auto KERNEL>
int allow_launch(size_t bytes, bool large_clusters, const char* what)
{
    static std::atomic<bool> done[64] = {};
    int dev = 0;
    int rc = cuda_check(cudaGetDevice(&dev), what);
    if (rc != DBL_OK || (dev >= 0 && dev < 64 && done[dev])) return rc;
    rc = cuda_check(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes), what);
    if (rc == DBL_OK && large_clusters)
        rc = cuda_check(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1), what);
    if (rc == DBL_OK && dev >= 0 && dev < 64) done[dev] = true;
    return rc;
}

// Clusters of S blocks that the device holds at a time, 0 where none; KERNEL's launches of S blocks have the same threads and
// shared memory, or these are their bounds.  Asked until the device has answered, once per device, after allow_launch.
template <auto KERNEL>
int clusters_held(int dev, int S, int threads, size_t smem)
{
    static std::atomic<int> known[64][17] = {};
    if (S > 1 && S > max_cluster()) return 0;
    const bool keep = dev >= 0 && dev < 64 && S <= 16;
    if (keep)
        if (const int k = known[dev][S]) return k - 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(S);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        n = 0;
    }
    if (keep && (e == cudaSuccess || e == cudaErrorInvalidClusterSize)) known[dev][S] = n + 1;  // its answer
    return n;
}

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

// From a 16-byte boundary to one, a multiple of 16 bytes; counted on the barrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, uintptr_t src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

// Waits for a phase, for what blocks of the cluster wrote before it too.  Bounded, like every wait of the library: a
// block that gives up says so in the status word and does not wait again.
__device__ __forceinline__ bool bounded_try(uint64_t* bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void bounded_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* status)
{
    if (bounded_try(bar, parity)) return;
    const uint64_t t0 = globaltimer();
    for (uint32_t i = 0; i < kWaitLimitPolls; ++i) {
        if (bounded_try(bar, parity)) return;
        if ((i & 63u) == 63u && (*abort || globaltimer() - t0 > kWaitLimitNs)) break;
    }
    *abort = 1;
    atomicExch(status, DBL_ERR_TIMEOUT);
}

// Stores to the shared memory of a block of the cluster, counted on a barrier of that block's.
__device__ __forceinline__ void st_async4(uint32_t addr, uint32_t bar, float4 v)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%2, %3, %4, %5}, [%1];" ::"r"(addr),
                 "r"(bar), "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)),
                 "r"(__float_as_uint(v.w))
                 : "memory");
}

__device__ __forceinline__ void st_async2(uint32_t addr, uint32_t bar, float2 v)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%2, %3}, [%1];" ::"r"(addr), "r"(bar),
                 "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y))
                 : "memory");
}

// The cluster's barrier in two steps, nothing written before it being read after it: who has waited knows that every block
// of the cluster has arrived, so that its shared memory is there to be written to.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// A block stays until the others no longer write to its shared memory (also where one has given up).
__device__ __forceinline__ void cluster_leave()
{
    cluster_arrive();
    cluster_wait();
}

// Before a block's end: one that gave up leaves the copies that it started some time to land.
__device__ __forceinline__ void linger(volatile int* abort)
{
    if (!*abort) return;
    const uint64_t t0 = globaltimer();
    for (uint32_t i = 0; i < kWaitLimitPolls && globaltimer() - t0 < kWaitLimitNs / 8; ++i) {}
}

}  // namespace dev

#endif

}  // namespace dbl
