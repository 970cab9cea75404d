// distill.cu -- distillation loss against a teacher's largest logits, with the labels' cross-entropy, forward and
// backward in one call.
//
// With m the row's largest logit, the sums of exp((z - m)/T) (and of exp(z - m), for the label) give the logarithms of
// q, and the gradient is the same exponentials times a factor, but for the k classes of the teacher and the label's.
// Bound by memory as long as a row is read once: a block, or a cluster of blocks for a long row, brings its part of
// the row into shared memory by one bulk copy, passes over it there three times (maximum, sums, gradient), and the
// gradient goes back from the logits' place by another.  Blocks of a cluster exchange (maximum, sums) once.
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxThreads = 512;
constexpr int kMaxK = DBL_DISTILL_MAX_K;
constexpr int kMaxCluster = 16;
constexpr int kStream = 256;                 // threads of the kernel for rows that no cluster holds
constexpr size_t kPartBytes = 68 * 1024;     // of a row, to a block: three blocks on an SM
constexpr size_t kMaxPartBytes = 200 * 1024;
constexpr float kLog2e = 1.4426950408889634f;

__device__ int g_distill_status;

struct DistillArgs {
    const void* z;
    const float* top;
    const int32_t* cls;
    const int32_t* labels;
    const float* weight;
    const float* scale;
    float* row_loss;
    void* dz;
    int64_t rows, ld, ld_grad;
    int v, k;
    float tau, alpha;
};

__device__ __forceinline__ float exp2_ftz(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 exp2_2(float2 x) { return make_float2(exp2_ftz(x.x), exp2_ftz(x.y)); }
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// 16 bytes of logits, as pairs.
template <class T>
struct Unit {
    static constexpr int E = 16 / (int)sizeof(T), P = E / 2;
    static __device__ __forceinline__ void floats(float2 (&f)[P], uint4 r)
    {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (sizeof(T) == 2)
                f[i] = act::unpack2_u32(w[i]);
            else
                f[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        }
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[P])
    {
        uint4 r;
        uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (sizeof(T) == 2)
                w[i] = act::pack2_u32(f[i].x, f[i].y);
            else
                w[2 * i] = __float_as_uint(f[i].x), w[2 * i + 1] = __float_as_uint(f[i].y);
        }
        return r;
    }
    // running maximum of what the unit holds (in its own format: no rounding)
    static __device__ __forceinline__ void max(uint4& m, uint4 r)
    {
        uint32_t *a = reinterpret_cast<uint32_t*>(&m), *b = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2) {
                const act2_t v = __hmax2(*reinterpret_cast<act2_t*>(a + i), *reinterpret_cast<act2_t*>(b + i));
                a[i] = *reinterpret_cast<const uint32_t*>(&v);
            } else {
                a[i] = __float_as_uint(fmaxf(__uint_as_float(a[i]), __uint_as_float(b[i])));
            }
        }
    }
};

// The teacher's distribution of row r, by one warp: p[j] (0 where the entry is absent) and its class (or -1).
// Returns log(sum) + largest/T, so that log p = t/T less that; NaN where there is no entry.
__device__ __forceinline__ float teacher(const DistillArgs& a, int64_t r, float* p, int* cls, bool& some)
{
    const int lane = threadIdx.x & 31;
    const float inv_tau = 1.f / a.tau;
    float tm = -INFINITY;
    bool any = false;
    for (int j = lane; j < a.k; j += 32) {
        const int c = a.cls[r * a.k + j];
        const float t = a.top[r * a.k + j];
        const bool there = c >= 0 && c < a.v && t != -INFINITY && a.alpha > 0.f;  // a term of weight 0 is absent
        cls[j] = there ? c : -1;
        p[j] = t;
        if (there) any = true, tm = fmaxf(tm, t);
    }
    some = __any_sync(0xffffffffu, any);
    tm = warp_max(tm);
    float sum = 0.f;
    for (int j = lane; j < a.k; j += 32) {
        const float e = cls[j] >= 0 ? expf((p[j] - tm) * inv_tau) : 0.f;
        p[j] = e;
        sum += e;
    }
    sum = warp_sum(sum);
    const float inv = 1.f / sum;
    for (int j = lane; j < a.k; j += 32) p[j] = cls[j] >= 0 ? p[j] * inv : 0.f;
    return logf(sum) + tm * inv_tau;
}

// The first term of row r's loss over alpha*T^2, by one warp, from the logits z of the entries' classes.
__device__ __forceinline__ float divergence(const DistillArgs& a, int64_t r, const float* p, const int* cls, const float* zc, float log_t,
                                            float m, float log_q)
{
    const float inv_tau = 1.f / a.tau;
    float loss = 0.f;
    for (int j = threadIdx.x & 31; j < a.k; j += 32)
        if (cls[j] >= 0 && p[j] != 0.f)
            loss += p[j] * ((a.top[r * a.k + j] * inv_tau - log_t) - ((zc[j] - m) * inv_tau - log_q));
    return warp_sum(loss);
}

struct Smem {
    uint64_t full;
    int abort, some;
    float log_t, zl;
    float red[32];
    float2 red2[32];
    float4 part[kMaxCluster];  // (maximum, sum at T, sum at 1) of every block of the cluster
};

// and p, cls, the entries' logits and gradients ([k] each)
__host__ __device__ inline size_t head_bytes(int k) { return ((sizeof(Smem) + 15) / 16 * 16 + (size_t)k * 16 + 127) / 128 * 128; }

// One row, or a cluster's part of it, per block.
template <class T>
__global__ void __launch_bounds__(kMaxThreads, 3) distill_kernel(DistillArgs a)
{
    typedef Unit<T> U;
    constexpr int E = U::E, P = U::P;
    extern __shared__ __align__(128) char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    float* p = reinterpret_cast<float*>(smem_raw + (sizeof(Smem) + 15) / 16 * 16);
    int* cls = reinterpret_cast<int*>(p + a.k);
    float *zc = reinterpret_cast<float*>(cls + a.k), *fix = zc + a.k;
    const size_t head = head_bytes(a.k);
    uint4* units = reinterpret_cast<uint4*>(smem_raw + head);
    T* elems = reinterpret_cast<T*>(units);

    uint32_t nrank;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(nrank));
    const int S = (int)nrank, rank = (int)cluster_ctarank(), tid = threadIdx.x, threads = blockDim.x;
    const int64_t r = blockIdx.x / S;
    const T* z = static_cast<const T*>(a.z) + r * a.ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + r * a.ld_grad : nullptr;
    // the row in units of 16 bytes, from the boundary at or before its first element; this block's part of them
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(z), p1 = p0 + (size_t)a.v * sizeof(T);
    const int lead = (int)(p0 & 15) / (int)sizeof(T);
    const int all = (int)(((p1 + 15) >> 4) - (p0 >> 4)), per = (all + S - 1) / S;
    const int u0 = min(rank * per, all), n = min(per, all - u0);
    const int first = u0 * E - lead;  // the element that is elems[0]
    const int e0 = max(first, 0), e1 = min(first + n * E, a.v);
    const float w = a.weight ? a.weight[r] : 1.f / (float)a.rows;
    const int lab = a.labels && a.alpha < 1.f ? a.labels[r] : -1;
    const bool given = lab >= 0 && lab < a.v;

    grid_dependency_trigger();
    auto zeros = [&] {
        const T zero = elem_from<T>(0.f);
        const int mis = (int)(reinterpret_cast<uintptr_t>(dz + e0) & 15) / (int)sizeof(T), b0 = min(e0 + (mis ? E - mis : 0), e1);
        const int b1 = b0 + (e1 - b0) / E * E;
        for (int i = e0 + tid; i < b0; i += threads) dz[i] = zero;
        for (int i = b0 + tid * E; i < b1; i += threads * E) *reinterpret_cast<uint4*>(dz + i) = make_uint4(0, 0, 0, 0);
        for (int i = b1 + tid; i < e1; i += threads) dz[i] = zero;
    };
    if (w == 0.f) {
        if (rank == 0 && tid == 0) a.row_loss[r] = 0.f;
        if (dz) zeros();
        return;
    }
    // whole units by one bulk copy, the row's ends by elements (nothing where they are another row's)
    const int c0 = u0 == 0 && lead ? 1 : 0, c1 = n - (u0 + n == all && (p1 & 15) && n > c0 ? 1 : 0);
    if (tid == 0) {
        mbar_init(&sm.full, 1);
        sm.abort = 0;
        fence_mbar_init();
        const uint32_t bytes = (uint32_t)max(c1 - c0, 0) * 16;
        mbar_arrive_expect_tx(&sm.full, bytes);
        if (bytes) bulk_load(smem_u32(units + c0), (p0 & ~(uintptr_t)15) + (uintptr_t)(u0 + c0) * 16, bytes, &sm.full);
    }
    for (int i = tid; i < 2 * E; i += threads) {
        const int u = i < E ? 0 : c1, at = u * E + i % E;
        if (n > 0 && (i < E ? c0 == 1 : c1 < n)) {
            const int el = first + at;
            elems[at] = el >= 0 && el < a.v ? z[el] : elem_from<T>(-INFINITY);
        }
    }
    if (tid < 32) {
        bool some;
        const float log_t = teacher(a, r, p, cls, some);
        if (tid == 0) {
            sm.log_t = log_t, sm.some = some;
            sm.zl = given ? elem_f(z[lab]) : 0.f;
        }
        if (rank == 0)
            for (int j = tid; j < a.k; j += 32) zc[j] = cls[j] >= 0 ? elem_f(z[cls[j]]) : 0.f;
    }
    __syncthreads();
    const bool some = sm.some;
    bounded_wait(&sm.full, 0, &sm.abort, &g_distill_status);
    if (!some && !given) {
        linger(&sm.abort);
        if (rank == 0 && tid == 0) a.row_loss[r] = 0.f;
        if (dz) zeros();
        return;
    }
    // maximum
    const uint32_t lowest = sizeof(T) == 4 ? 0xff800000u : act::kF16 ? 0xfc00fc00u : 0xff80ff80u;  // minus infinity
    uint4 mx = make_uint4(lowest, lowest, lowest, lowest);
#pragma unroll 4
    for (int i = tid; i < n; i += threads) U::max(mx, units[i]);
    float2 f[P];
    U::floats(f, mx);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < P; ++i) m = fmaxf(m, fmaxf(f[i].x, f[i].y));
    m = block_max(m, sm.red);
    // sums; one kind of exponential where there is one term, or T = 1
    const bool two = some && given && a.tau != 1.f;
    const float cA = some ? kLog2e / a.tau : kLog2e;
    float2 sA = both(0.f), sB = both(0.f);
    if (m != -INFINITY) {  // otherwise nothing here
        const float2 nm = both(-m);
        if (two) {
#pragma unroll 2
            for (int i = tid; i < n; i += threads) {
                U::floats(f, units[i]);
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    const float2 d = __fadd2_rn(f[q], nm);
                    sA = __fadd2_rn(sA, exp2_2(__fmul2_rn(d, both(cA))));
                    sB = __fadd2_rn(sB, exp2_2(__fmul2_rn(d, both(kLog2e))));
                }
            }
        } else {
#pragma unroll 2
            for (int i = tid; i < n; i += threads) {
                U::floats(f, units[i]);
#pragma unroll
                for (int q = 0; q < P; ++q) sA = __fadd2_rn(sA, exp2_2(__fmul2_rn(__fadd2_rn(f[q], nm), both(cA))));
            }
        }
    }
    float tA = warp_sum(sA.x + sA.y), tB = warp_sum(sB.x + sB.y);
    if ((tid & 31) == 0) sm.red2[tid >> 5] = make_float2(tA, tB);
    __syncthreads();
    tA = tB = 0.f;
    for (int i = 0; i < threads >> 5; ++i) tA += sm.red2[i].x, tB += sm.red2[i].y;
    if (S > 1) {
        if (tid < S)
            st_cluster_v4(mapa_shared(smem_u32(&sm.part[rank]), tid), __float_as_uint(m), __float_as_uint(tA), __float_as_uint(tB), 0);
        // also: no block writes a gradient to the logits' place before the others have read what they need there
        cluster_sync_all();
        m = sm.part[0].x;
        for (int i = 1; i < S; ++i) m = fmaxf(m, sm.part[i].x);
        tA = tB = 0.f;
        for (int i = 0; i < S; ++i) {
            const float4 q = sm.part[i];
            tA += q.y * exp2_ftz((q.x - m) * cA);
            tB += q.z * exp2_ftz((q.x - m) * kLog2e);
        }
    }
    if (!two) tB = tA;
    if (rank == 0 && tid < 32) {
        float loss = some ? divergence(a, r, p, cls, zc, sm.log_t, m, logf(tA)) * (a.alpha * a.tau * a.tau) : 0.f;
        if (given) loss += (1.f - a.alpha) * (logf(tB) - (sm.zl - m));
        if (tid == 0) a.row_loss[r] = loss;
    }
    linger(&sm.abort);
    if (!dz) return;
    const float fw = a.scale ? w * *a.scale : w;
    const float gt = some ? fw * a.alpha * a.tau : 0.f, gl = given ? fw * (1.f - a.alpha) : 0.f;
    // exponentials' factors: the two terms', or both in one
    const float fA = two ? gt / tA : (gt + gl) / tA, fB = gl / tB;
    auto grad = [&](float2 v) {
        const float2 d = __fadd2_rn(v, both(-m));
        const float2 g = __fmul2_rn(exp2_2(__fmul2_rn(d, both(cA))), both(fA));
        return two ? __ffma2_rn(exp2_2(__fmul2_rn(d, both(kLog2e))), both(fB), g) : g;
    };
    // the classes of the teacher and the label, before their logits are overwritten
    auto fix_of = [&](int c, float pj) {
        const float g = grad(both(elem_f(elems[c - first]))).x;
        return g - gt * pj - (c == lab && given ? gl : 0.f);
    };
    for (int j = tid; j < a.k; j += threads) {
        if (cls[j] < e0 || cls[j] >= e1) continue;
        float pj = 0.f;
        for (int i = 0; i < a.k; ++i)
            if (cls[i] == cls[j]) pj += p[i];  // a class may be named again
        fix[j] = fix_of(cls[j], pj);
    }
    float fix_lab = 0.f;
    bool lab_here = given && tid == threads - 1 && lab >= e0 && lab < e1;
    if (lab_here) {
        float pj = 0.f;
        for (int i = 0; i < a.k; ++i)
            if (cls[i] == lab) pj += p[i];
        fix_lab = fix_of(lab, pj);
    }
    __syncthreads();
    if (two) {
#pragma unroll 2
        for (int i = tid; i < n; i += threads) {
            U::floats(f, units[i]);
#pragma unroll
            for (int q = 0; q < P; ++q) f[q] = grad(f[q]);
            units[i] = U::pack(f);
        }
    } else {
        const float2 nm = both(-m);
#pragma unroll 2
        for (int i = tid; i < n; i += threads) {
            U::floats(f, units[i]);
#pragma unroll
            for (int q = 0; q < P; ++q) f[q] = __fmul2_rn(exp2_2(__fmul2_rn(__fadd2_rn(f[q], nm), both(cA))), both(fA));
            units[i] = U::pack(f);
        }
    }
    __syncthreads();
    for (int j = tid; j < a.k; j += threads)
        if (cls[j] >= e0 && cls[j] < e1) elems[cls[j] - first] = elem_from<T>(fix[j]);
    if (lab_here) elems[lab - first] = elem_from<T>(fix_lab);
    const bool same = ((reinterpret_cast<uintptr_t>(dz) ^ p0) & 15) == 0;  // rows begin at the same place of a unit
    if (same) fence_async_shared();
    __syncthreads();
    if (!same) {
        for (int i = e0 + tid; i < e1; i += threads) dz[i] = elems[i - first];
        return;
    }
    if (tid == 0 && c1 > c0) {
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dz + first + c0 * E), "r"(smem_u32(units + c0)),
                     "r"((uint32_t)(c1 - c0) * 16)
                     : "memory");
        bulk_commit();
    }
    for (int i = e0 + tid; i < min(first + c0 * E, e1); i += threads) dz[i] = elems[i - first];
    for (int i = max(first + c1 * E, e0) + tid; i < e1; i += threads) dz[i] = elems[i - first];
    if (tid == 0) bulk_wait_read();
}

// Rows that no cluster holds in shared memory: one row per block, read three times.
template <class T>
__global__ void __launch_bounds__(kStream) distill_stream_kernel(DistillArgs a)
{
    __shared__ float red[32];
    __shared__ float p[kMaxK], zc[kMaxK];
    __shared__ int cls[kMaxK];
    __shared__ int some_s;
    __shared__ float log_ts;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + r * a.ld;
        T* dz = a.dz ? static_cast<T*>(a.dz) + r * a.ld_grad : nullptr;
        const float w = a.weight ? a.weight[r] : 1.f / (float)a.rows;
        const int lab = a.labels && a.alpha < 1.f ? a.labels[r] : -1;
        const bool given = lab >= 0 && lab < a.v;
        if (threadIdx.x < 32) {
            bool some;
            const float log_t = teacher(a, r, p, cls, some);
            for (int j = threadIdx.x; j < a.k; j += 32) zc[j] = cls[j] >= 0 ? elem_f(z[cls[j]]) : 0.f;
            if (threadIdx.x == 0) some_s = some, log_ts = log_t;
        }
        __syncthreads();
        const bool some = some_s;
        if (w == 0.f || (!some && !given)) {
            if (threadIdx.x == 0) a.row_loss[r] = 0.f;
            if (dz)
                for (int i = threadIdx.x; i < a.v; i += kStream) dz[i] = elem_from<T>(0.f);
            __syncthreads();
            continue;
        }
        float m = -INFINITY;
        for (int i = threadIdx.x; i < a.v; i += kStream) m = fmaxf(m, elem_f(z[i]));
        m = block_max(m, red);
        const float cA = kLog2e / a.tau;
        float sA[4] = {0.f, 0.f, 0.f, 0.f}, sB[4] = {0.f, 0.f, 0.f, 0.f};  // chains of a fourth of a thread's terms
        for (int i = threadIdx.x; i < a.v; i += 4 * kStream)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i + q * kStream < a.v) {
                    const float d = elem_f(z[i + q * kStream]) - m;
                    sA[q] += exp2_ftz(d * cA);
                    sB[q] += exp2_ftz(d * kLog2e);
                }
        const float tA = block_sum((sA[0] + sA[1]) + (sA[2] + sA[3]), red), tB = block_sum((sB[0] + sB[1]) + (sB[2] + sB[3]), red);
        const float zl = given ? elem_f(z[lab]) : 0.f;
        if (threadIdx.x < 32) {
            float loss = some ? divergence(a, r, p, cls, zc, log_ts, m, logf(tA)) * (a.alpha * a.tau * a.tau) : 0.f;
            if (given) loss += (1.f - a.alpha) * (logf(tB) - (zl - m));
            if (threadIdx.x == 0) a.row_loss[r] = loss;
        }
        __syncthreads();
        if (!dz) continue;
        const float fw = a.scale ? w * *a.scale : w;
        const float gt = some ? fw * a.alpha * a.tau : 0.f, gl = given ? fw * (1.f - a.alpha) : 0.f;
        const float fA = gt / tA, fB = gl / tB;
        auto grad = [&](float v) {
            float g = 0.f;
            if (some) g = fA * exp2_ftz((v - m) * cA);
            if (given) g = fmaf(fB, exp2_ftz((v - m) * kLog2e), g);
            return g;
        };
        for (int i = threadIdx.x; i < a.v; i += kStream) dz[i] = elem_from<T>(grad(elem_f(z[i])));
        __syncthreads();
        for (int j = threadIdx.x; j < a.k; j += kStream) {
            if (cls[j] < 0) continue;
            float pj = 0.f;
            for (int i = 0; i < a.k; ++i)
                if (cls[i] == cls[j]) pj += p[i];
            dz[cls[j]] = elem_from<T>(grad(zc[j]) - gt * pj - (cls[j] == lab && given ? gl : 0.f));
        }
        if (given && threadIdx.x == 0) {
            float pj = 0.f;
            for (int i = 0; i < a.k; ++i)
                if (cls[i] == lab) pj += p[i];
            if (pj == 0.f) dz[lab] = elem_from<T>(grad(zl) - gl);  // not among the entries (or of no weight there)
        }
        __syncthreads();
    }
}

// loss = sum of weight*row_loss, in one block and a fixed order
__global__ void __launch_bounds__(1024) distill_loss_kernel(const float* row_loss, const float* weight, int64_t rows,
                                                           float* loss)
{
    __shared__ float red[32];
    grid_dependency_wait();
    float s = 0.f;
    for (int64_t r = threadIdx.x; r < rows; r += 1024) s += weight ? weight[r] * row_loss[r] : row_loss[r];
    s = block_sum(s, red);
    if (threadIdx.x == 0) *loss = weight ? s : s / (float)rows;
}

template <class T>
int launch(const DistillArgs& a, cudaStream_t st, const char* what)
{
    constexpr auto kernel = distill_kernel<T>;
    const size_t head = head_bytes(a.k);
    const size_t row = ((size_t)a.v * sizeof(T) + 15) / 16 * 16 + 16;
    auto part = [&](int S) { return (row / 16 + S - 1) / S * 16; };
    // as many blocks to a row as bring three on an SM, and for few rows, as fill the SMs with parts of 8 KB and more
    int S = 1;
    while (S < kMaxCluster && part(S) > kPartBytes) S *= 2;
    while (S < kMaxCluster && a.rows * S * 2 <= sm_count() && part(2 * S) >= 8192) S *= 2;
    while (S > 1 && !cluster_held<kernel>(S, kMaxThreads, kMaxPartBytes + head_bytes(kMaxK))) S /= 2;
    if (part(S) > kMaxPartBytes) {
        distill_stream_kernel<T><<<(int)std::min<int64_t>(a.rows, 1 << 20), kStream, 0, st>>>(a);
        return launch_check(what);
    }
    if (a.rows * S > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^31 blocks", what);
    const size_t smem = head + part(S);
    int threads = 64;  // four units of 16 bytes a thread and pass, or more
    while (threads < kMaxThreads && (size_t)threads * 64 < part(S)) threads *= 2;
    int rc = cuda_check(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem), what);
    if (rc == DBL_OK && S > 8)
        rc = cuda_check(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1), what);
    if (rc != DBL_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(a.rows * S));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, a);
    rc = launch_check(what);
    return err == cudaSuccess ? rc : cuda_check(err, what);
}

}  // namespace

namespace dbl {

int distill_device_status(int* status) { return take_status(g_distill_status, status); }

}  // namespace dbl

extern "C" int dbl_distill_fwd_bwd(const dbl_distill_shape* s, const void* logits, const float* teacher_logits,
                                   const int32_t* teacher_classes, const int32_t* labels, const float* row_weight,
                                   const float* loss_scale, float* row_loss, float* loss, void* dlogits, void* stream)
{
    const char* w = "distill_fwd_bwd";
    if (!s || s->rows < 0 || s->classes <= 0 || s->k < 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0, classes <= 0 or k < 0", w);
    if (s->k > kMaxK) return set_error(DBL_ERR_UNSUPPORTED, "%s: k = %d, at most %d", w, s->k, kMaxK);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", w);
    if (!(s->temperature > 0.f) || isinf(s->temperature) || !(s->alpha >= 0.f && s->alpha <= 1.f))
        return set_error(DBL_ERR_INVALID, "%s: temperature must be finite and > 0, alpha in [0, 1]", w);
    if ((s->ld && s->ld < s->classes) || (s->ld_grad && s->ld_grad < s->classes))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", w);
    if (s->k > 0 && (!teacher_logits || !teacher_classes))
        return set_error(DBL_ERR_INVALID, "%s: k > 0 needs the teacher's logits and classes", w);
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(logits, e) || !aligned_to(dlogits, e) || !aligned_to(teacher_logits, 4) ||
        !aligned_to(teacher_classes, 4) || !aligned_to(labels, 4) || !aligned_to(row_weight, 4) ||
        !aligned_to(loss_scale, 4) || !aligned_to(row_loss, 4) || !aligned_to(loss, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    DistillArgs a = {logits, teacher_logits, teacher_classes, labels, row_weight, loss_scale, row_loss, dlogits, s->rows,
                     s->ld ? s->ld : s->classes, s->ld_grad ? s->ld_grad : s->classes, s->classes, s->k, s->temperature,
                     s->alpha};
    if (logits && dlogits == logits && a.ld != a.ld_grad)
        return set_error(DBL_ERR_INVALID, "%s: a gradient in the logits' place needs their row stride", w);
    cudaStream_t st = as_stream(stream);
    if (s->rows == 0) {
        if (!loss) return DBL_OK;
        return cuda_check(cudaMemsetAsync(loss, 0, sizeof(float), st), w);
    }
    if (!logits || !row_loss) return set_error(DBL_ERR_INVALID, "%s: logits and row_loss must not be NULL", w);
    int rc = s->dtype == DBL_F32 ? launch<float>(a, st, w) : launch<act_t>(a, st, w);
    if (rc != DBL_OK || !loss) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(1024);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, distill_loss_kernel, (const float*)row_loss, row_weight, s->rows, loss);
    rc = launch_check("distill_fwd_bwd loss");
    return err == cudaSuccess ? rc : cuda_check(err, "distill_fwd_bwd loss");
}
