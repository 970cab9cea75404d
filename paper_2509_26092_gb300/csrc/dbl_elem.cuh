// dbl_elem.cuh -- element types, launches, block sums and rows that begin anywhere, of the token operators (ln.cu, scan.cu,
// distill.cu, route.cu, exchange.cu, grouped.cu, dropout.cu), whose tensors are fp32 or the library's 16-bit format.
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

// Rows that begin at any element, in units of 16 bytes.  Unit u that is stored lies on a 16-byte boundary and holds the row's
// elements u*N - lead to u*N - lead + N - 1 (N = 16 / sizeof(T); `lead` of the first are before the row, and the last may
// reach past its end); what is read for it lies anywhere in memory, put together from the two units on boundaries that it
// covers, of which a lane loads one and takes the other from its neighbour.
template <class T>
struct RowOf {
    const uint4* base;         // the boundary at or before the row
    int c, units, low, high;   // units from the boundary that the row is in, and those that lie in the tensor as a whole
    int first;                 // the row's first element, from the boundary on
    int back;                  // 0 or -1: of unit 0 from the boundary
    uint32_t shift;            // bytes of a unit read from its boundary

    // row r of [rows, c] at stride ld
    __device__ __forceinline__ RowOf(const void* tensor, int64_t r, int64_t rows, int c, int64_t ld, int lead) : c(c)
    {
        const uintptr_t first_byte = reinterpret_cast<uintptr_t>(tensor), begin = first_byte + (size_t)(r * ld) * sizeof(T);
        const uintptr_t last = first_byte + ((size_t)(rows - 1) * ld + c) * sizeof(T);
        const int d = (int)(begin & 15u), from = d - lead * (int)sizeof(T);
        base = reinterpret_cast<const uint4*>(begin - d);
        units = (int)((d + (size_t)c * sizeof(T) + 15) / 16);
        low = begin - d < first_byte ? 1 : 0;
        high = (begin - d) + (size_t)units * 16 > last ? units - 1 : units;
        first = d / (int)sizeof(T);
        back = from >> 4;
        shift = (uint32_t)from & 15u;
    }
    // M units u, u + 32, .. of what is stored: all lanes of a warp, u growing by 1 from lane to lane.  All loads go out first.
    // The neighbour of lane 31 is lane 0 with the unit after; the last of those it loads for this alone.
    template <int M>
    __device__ __forceinline__ void load(int u, uint4 (&v)[M + 1]) const
    {
        u += back;
#pragma unroll
        for (int m = 0; m <= M; ++m) {
            const int at = u + 32 * m;
            v[m] = at >= low && at < high && (m < M || (threadIdx.x & 31) == 0) ? base[at] : make_uint4(0, 0, 0, 0);
        }
    }
    template <int M>
    __device__ __forceinline__ void join(int u, uint4 (&v)[M + 1]) const
    {
        u += back;
        if (low != 0 || high != units) {  // the tensor begins or ends in a unit of this row, which is read by elements
#pragma unroll
            for (int m = 0; m <= M; ++m) {
                const int at = u + 32 * m;
                if (at >= 0 && at < units && (at < low || at >= high)) v[m] = by_elements(at);
            }
        }
        if (shift == 0) return;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const bool after = (threadIdx.x & 31) == 0;
            const int to = (threadIdx.x + 1) & 31;
            uint32_t w[8] = {v[m].x, v[m].y, v[m].z, v[m].w};
            w[4] = __shfl_sync(0xffffffffu, after ? v[m + 1].x : v[m].x, to);
            w[5] = __shfl_sync(0xffffffffu, after ? v[m + 1].y : v[m].y, to);
            w[6] = __shfl_sync(0xffffffffu, after ? v[m + 1].z : v[m].z, to);
            w[7] = __shfl_sync(0xffffffffu, after ? v[m + 1].w : v[m].w, to);
            if (shift & 8) {
#pragma unroll
                for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
            }
            if (shift & 4) {
#pragma unroll
                for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
            }
            if (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (shift & 2) * 8);
            }
            v[m] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ __forceinline__ uint4 by_elements(int at) const
    {
        constexpr int N = 16 / (int)sizeof(T);
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = at * N + i - first;
            if (e < 0 || e >= c) continue;
            if constexpr (sizeof(T) == 2)
                w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(base)[at * N + i] << (16 * (i & 1));
            else
                w[i] = reinterpret_cast<const uint32_t*>(base)[at * N + i];
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// Elements `first` to last - 1 of a unit to the row's from e + first on, those that the row has, one by one.
template <class T>
__device__ __forceinline__ void store_part(T* row, int c, int e, uint4 v, int first, int last)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
        if (i < first || i >= last || e + i < 0 || e + i >= c) continue;
        if constexpr (sizeof(T) == 2)
            reinterpret_cast<uint16_t*>(row)[e + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        else
            reinterpret_cast<uint32_t*>(row)[e + i] = w[i];
    }
}

// A unit to the row's elements from e on, row + e being on a boundary.
template <class T>
__device__ __forceinline__ void store_unit(T* row, int c, int e, uint4 v)
{
    constexpr int N = 16 / (int)sizeof(T);
    if (e >= 0 && e + N <= c)
        *reinterpret_cast<uint4*>(row + e) = v;
    else
        store_part(row, c, e, v, 0, N);
}

// Elements of the unit on a boundary in which a row begins that come before it.
template <class T>
__device__ __forceinline__ int unit_lead(const T* row) { return (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)); }

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
