// distill.cu -- distillation loss against a teacher's largest logits, with the labels' cross-entropy, forward and
// backward in one call.
//
// With m the row's largest logit, the sums of exp((z - m)/T) (and of exp(z - m), for the label) give the logarithms of
// q, and the gradient is the same exponentials times a factor, but for the k classes of the teacher and the label's.
// Bound by memory as long as a row is read once: a block, or a cluster of blocks for a long row, brings its part of
// the row into shared memory by one bulk copy, passes over it there three times (maximum, sums, gradient), and the
// gradient goes back from the logits' place by another.  Blocks of a cluster exchange (maximum, sums) once.  Sums and
// probabilities are fp32; the gradient is rounded once, when it is stored.
//
// On a GB300 that copies 6.78 TB/s: 4096 x 32000 in bf16, labels and teacher, 105 us = 5.0 TB/s (three blocks on an SM
// in turns of load, passes and store; the exponentials' unit half busy, 17 instructions an element.  Four chunks of a row,
// loaded and stored on their own, 127 us: shorter loops).  9 x 131071 in fp16 12.5 us and 740 x 1000 in fp32 10.5 us:
// two launches and one row's chain of load, sums and store.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxThreads = 256;             // that pass over the row; a warp more takes the teacher's entries
constexpr int kFewK = 64;                    // and up to this many, looks for classes that are named twice; of more all
                                             // threads do, and bring them (4096 x 32000 in bf16, 100 entries: 120 us,
                                             // brought by the one warp 132; 1024: 245 us, all by the one warp 968)
constexpr int kMaxK = DBL_DISTILL_MAX_K;
constexpr int kMaxCluster = 16;
constexpr int kWarpRows = 4;                 // rows of a block, a warp each, where they have
constexpr size_t kWarpBytes = 12288 + 16, kWarpBytesFew = 4096 + 16;  // this many bytes at the most
constexpr int kWarpK = 128;                  // and the teacher this many entries
constexpr int kStream = 256;                 // threads of the kernel for rows that no cluster holds
constexpr size_t kPartBytes = 68 * 1024;     // of a row, to a block: three blocks on an SM
constexpr size_t kLargePartBytes = 106 * 1024;  // two
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
    float tau, alpha, one;  // one: the weight of a row where none are given
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

// What a row's group keeps in shared memory beside its logits: of the teacher's k entries the classes (-1: absent, and
// past the end to a multiple of 4), p, t/T, the student's logits, and their gradients.
struct Entries {
    int* cls;
    float *p, *lt, *zc, *fix;
    static __host__ __device__ size_t bytes(int k) { return (size_t)((k + 3) / 4 * 4) * 20; }
    __device__ __forceinline__ Entries(char* at, int k)
    {
        const int n = (k + 3) / 4 * 4;
        cls = reinterpret_cast<int*>(at);
        p = reinterpret_cast<float*>(cls + n), lt = p + n, zc = lt + n, fix = zc + n;
    }
};

// A lane's first entries of a row as they are in memory, asked for before anything else is known of the row.
struct Ahead {
    static constexpr int N = 2;
    int c[N];
    float t[N];
    __device__ __forceinline__ void ask(const DistillArgs& a, int64_t r)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = i * 32 + (threadIdx.x & 31);
            c[i] = j < a.k ? __ldg(a.cls + r * a.k + j) : -1;
            t[i] = j < a.k ? __ldg(a.top + r * a.k + j) : 0.f;
        }
    }
};

// Row r's entries, by a warp of which each lane has its first ones, or by `threads` threads that have none; z: the student's
// logits where those of the entries' classes are to be kept too.
template <class T>
__device__ __forceinline__ void load_entries(const DistillArgs& a, int64_t r, const T* z, const Entries& en, const Ahead* ahead,
                                             int tid, int threads)
{
    const float inv_tau = 1.f / a.tau;
    auto keep = [&](int j, int c, float t) {
        const bool there = c >= 0 && c < a.v && t != -INFINITY && a.alpha > 0.f;  // a term of weight 0 is absent
        en.cls[j] = there ? c : -1;
        en.lt[j] = t * inv_tau;
        if (z) en.zc[j] = there ? elem_f(z[c]) : 0.f;
    };
    const int end = (a.k + 3) / 4 * 4;
    if (ahead) {
#pragma unroll
        for (int i = 0; i < Ahead::N; ++i)
            if (i * 32 + tid < end) keep(i * 32 + tid, ahead->c[i], ahead->t[i]);
    }
#pragma unroll 4
    for (int j = (ahead ? Ahead::N * 32 : 0) + tid; j < end; j += threads)
        keep(j, j < a.k ? __ldg(a.cls + r * a.k + j) : -1, j < a.k ? __ldg(a.top + r * a.k + j) : 0.f);
}

// The teacher's distribution, by one warp.  log_t: log p = t/T less that.  False where there is no entry.
__device__ __forceinline__ bool teacher(const DistillArgs& a, const Entries& en, float& log_t)
{
    const int lane = threadIdx.x & 31;
    float tm = -INFINITY, sum = 0.f;
    bool any = false;
    for (int j = lane; j < a.k; j += 32)
        if (en.cls[j] >= 0) any = true, tm = fmaxf(tm, en.lt[j]);
    tm = warp_max(tm);
    for (int j = lane; j < a.k; j += 32) {
        const float e = en.cls[j] >= 0 ? expf(en.lt[j] - tm) : 0.f;
        en.p[j] = e;
        sum += e;
    }
    sum = warp_sum(sum);
    const float inv = 1.f / sum;
    for (int j = lane; j < a.k; j += 32) en.p[j] = en.cls[j] >= 0 ? en.p[j] * inv : 0.f;
    log_t = logf(sum) + tm;
    return __any_sync(0xffffffffu, any);
}

// Whether another entry names the class of entry j.
__device__ __forceinline__ bool again(const DistillArgs& a, const Entries& en, int j)
{
    const int c = en.cls[j];
    int count = 0;
#pragma unroll 4
    for (int i = 0; i < a.k; i += 4) {
        const int4 q = *reinterpret_cast<const int4*>(en.cls + i);
        count += (q.x == c) + (q.y == c) + (q.z == c) + (q.w == c);
    }
    return count > 1;
}

// The first term of a row's loss over alpha*T^2, by one warp.
__device__ __forceinline__ float divergence(const DistillArgs& a, const Entries& en, float log_t, float m, float log_q)
{
    const float inv_tau = 1.f / a.tau;
    float loss = 0.f;
    for (int j = threadIdx.x & 31; j < a.k; j += 32)
        if (en.cls[j] >= 0 && en.p[j] != 0.f) loss += en.p[j] * ((en.lt[j] - log_t) - ((en.zc[j] - m) * inv_tau - log_q));
    return warp_sum(loss);
}

// The whole probability of class c, which several entries may name.
__device__ __forceinline__ float named(const DistillArgs& a, const Entries& en, int c)
{
    float s = 0.f;
    for (int i = 0; i < a.k; i += 4) {
        const int4 q = *reinterpret_cast<const int4*>(en.cls + i);
        if (q.x == c) s += en.p[i];
        if (q.y == c) s += en.p[i + 1];
        if (q.z == c) s += en.p[i + 2];
        if (q.w == c) s += en.p[i + 3];
    }
    return s;
}

struct Smem {
    float4 part[kMaxCluster];            // (maximum, sum at T, sum at 1) of every block of the cluster
    float4 warp[kMaxThreads / 32];       // of every warp
    uint64_t full;
    int abort, some, named;  // named: an entry has the label's class
    float log_t;
};

__host__ __device__ inline size_t head_bytes(int k) { return ((sizeof(Smem) + 15) / 16 * 16 + Entries::bytes(k) + 127) / 128 * 128; }

// (maximum, sums) of the parts of a row as one.
__device__ __forceinline__ float4 join(const float4* part, int n, float cA)
{
    float4 t = make_float4(-INFINITY, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < n; ++i) t.x = fmaxf(t.x, part[i].x);
    const float m = t.x == -INFINITY ? 0.f : t.x;  // nothing but minus infinities: sums of 0, or NaN
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float4 q = part[i];
        t.y = fmaf(q.y, exp2_ftz((q.x - m) * cA), t.y);
        t.z = fmaf(q.z, exp2_ftz((q.x - m) * kLog2e), t.z);
    }
    return t;
}

// One row, or a cluster's part of it, per block; WARP: a row per warp.
template <class T, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxThreads + 32, WARP ? 10 : 3) distill_kernel(DistillArgs a, int bytes_of_group)
{
    typedef Unit<T> U;
    typedef typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type Bits;
    constexpr int E = U::E, P = U::P;
    extern __shared__ __align__(128) char smem_raw[];
    char* const base = smem_raw + (WARP ? (threadIdx.x >> 5) * bytes_of_group : 0);
    Smem& sm = *reinterpret_cast<Smem*>(base);
    const Entries en(base + (sizeof(Smem) + 15) / 16 * 16, a.k);
    uint4* units = reinterpret_cast<uint4*>(base + head_bytes(a.k));
    T* elems = reinterpret_cast<T*>(units);

    int S = 1, rank = 0;
    if (!WARP) {
        uint32_t n;
        asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
        S = (int)n, rank = (int)cluster_ctarank();
    }
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x - 32;
    const bool side = !WARP && tid >= threads;  // the warp beside those that pass over the row
    auto sync = [] {
        if (WARP)
            __syncwarp();
        else
            __syncthreads();
    };
    const int64_t r = WARP ? (int64_t)blockIdx.x * kWarpRows + (threadIdx.x >> 5) : S == 1 ? blockIdx.x : blockIdx.x / (unsigned)S;
    grid_dependency_trigger();
    if (r >= a.rows) return;
    Ahead ahead;
    if (WARP || side) ahead.ask(a, r);
    if (tid == 0) {
        mbar_init(&sm.full, 1);
        sm.abort = sm.named = 0;
        fence_mbar_init();
    }
    const T* z = static_cast<const T*>(a.z) + r * a.ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + r * a.ld_grad : nullptr;
    // the row in units of 16 bytes, from the boundary at or before its first element; this block's part of them
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(z), p1 = p0 + (size_t)a.v * sizeof(T);
    const int lead = (int)(p0 & 15) / (int)sizeof(T);
    const int all = (int)(((p1 + 15) >> 4) - (p0 >> 4)), per = S == 1 ? all : (int)((unsigned)(all + S - 1) / (unsigned)S);
    const int u0 = min(rank * per, all), n = min(per, all - u0);
    const int first = u0 * E - lead;  // the element that is elems[0]
    const int e0 = max(first, 0), e1 = min(first + n * E, a.v);
    const float w = a.weight ? __ldg(a.weight + r) : a.one;
    const int lab = a.labels && a.alpha < 1.f ? __ldg(a.labels + r) : -1;
    const float scale = a.scale ? __ldg(a.scale) : 1.f;
    const bool given = lab >= 0 && lab < a.v;

    auto zeros = [&] {
        const T zero = elem_from<T>(0.f);
        const int mis = (int)(reinterpret_cast<uintptr_t>(dz + e0) & 15) / (int)sizeof(T), b0 = min(e0 + (mis ? E - mis : 0), e1);
        const int b1 = b0 + (e1 - b0) / E * E, step = WARP ? 32 : blockDim.x;
        for (int i = e0 + tid; i < b0; i += step) dz[i] = zero;
        for (int i = b0 + tid * E; i < b1; i += step * E) *reinterpret_cast<uint4*>(dz + i) = make_uint4(0, 0, 0, 0);
        for (int i = b1 + tid; i < e1; i += step) dz[i] = zero;
    };
    if (w == 0.f) {
        if (rank == 0 && tid == 0) a.row_loss[r] = 0.f;
        if (dz) zeros();
        return;
    }
    // whole units by one bulk copy, the row's ends by elements (nothing where they are another row's)
    const int c0 = u0 == 0 && lead ? 1 : 0, c1 = n - (u0 + n == all && (p1 & 15) && n > c0 ? 1 : 0);
    if (tid == 0) {
        const uint32_t bytes = (uint32_t)max(c1 - c0, 0) * 16;
        mbar_arrive_expect_tx(&sm.full, bytes);
        if (bytes) bulk_load(smem_u32(units + c0), (p0 & ~(uintptr_t)15) + (uintptr_t)(u0 + c0) * 16, bytes, &sm.full);
    }
    if ((c0 || c1 < n) && tid < 2 * E && n > 0 && (tid < E ? c0 == 1 : c1 < n)) {
        const int at = (tid < E ? 0 : c1 * E) + tid % E, el = first + at;
        elems[at] = el >= 0 && el < a.v ? z[el] : elem_from<T>(-INFINITY);
    }
    float zl = given && !WARP ? elem_f(z[lab]) : 0.f;
    sync();
    if (!WARP && S > 1) cluster_arrive();  // here; w, and so the return above, is the same in all blocks of a row
    // while the row is on its way
    const bool many = a.k > kFewK;
    if (many && !WARP) {
        load_entries<T>(a, r, z, en, nullptr, tid, blockDim.x);
        sync();
    }
    if (WARP || side) {
        if (WARP || !many) load_entries<T>(a, r, WARP ? nullptr : z, en, &ahead, tid & 31, 32);
        __syncwarp();
        float log_t;
        const bool some = teacher(a, en, log_t);
        if ((tid & 31) == 0) sm.log_t = log_t, sm.some = some;
        for (int j = tid & 31; j < a.k; j += 32) en.fix[j] = !many && again(a, en, j) ? 1.f : 0.f;
    }
    // Two kinds of exponential where there may be two terms and T is not 1.
    const bool kl = a.k > 0 && a.alpha > 0.f, two = kl && given && a.tau != 1.f;
    const float cA = kl ? kLog2e / a.tau : kLog2e;
    float2 f[P];
    float4 t = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (!side) {
        bounded_wait(&sm.full, 0, &sm.abort, &g_distill_status);
        if (WARP) {  // the whole row is here
            for (int j = tid; j < a.k; j += 32) en.zc[j] = en.cls[j] >= 0 ? elem_f(elems[en.cls[j] - first]) : 0.f;
            if (given) zl = elem_f(elems[lab - first]);
        }
        const uint32_t lowest = sizeof(T) == 4 ? 0xff800000u : act::kF16 ? 0xfc00fc00u : 0xff80ff80u;  // minus infinity
        uint4 mx = make_uint4(lowest, lowest, lowest, lowest);
#pragma unroll 4
        for (int i = tid; i < n; i += threads) U::max(mx, units[i]);
        U::floats(f, mx);
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < P; ++i) m = fmaxf(m, fmaxf(f[i].x, f[i].y));
        m = warp_max(m);
        float2 sA = both(0.f), sB = both(0.f);
        const float2 nm = both(m == -INFINITY ? 0.f : -m);  // nothing but minus infinities: sums of 0
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
        t = make_float4(m, warp_sum(sA.x + sA.y), two ? warp_sum(sB.x + sB.y) : 0.f, 0.f);
        if (!WARP && (tid & 31) == 0) sm.warp[tid >> 5] = t;
    }
    sync();
    if (!WARP) {
        t = join(sm.warp, threads >> 5, cA);
        if (S > 1) {
            cluster_wait();  // a block's shared memory is stored to from afar once it has begun
            if (tid < S)
                st_cluster_v4(mapa_shared(smem_u32(&sm.part[rank]), tid), __float_as_uint(t.x), __float_as_uint(t.y), __float_as_uint(t.z), 0);
            // also: no block writes a gradient to the logits' place before the others have read what they need there
            cluster_sync_all();
            t = join(sm.part, S, cA);
        }
    }
    linger(&sm.abort);
    const bool some = sm.some;
    if (!some && !given) {
        if (rank == 0 && tid == 0) a.row_loss[r] = 0.f;
        if (dz) zeros();
        return;
    }
    const float m = t.x, bad = m == -INFINITY ? NAN : 0.f;  // no distribution
    const float tA = t.y + bad, tB = two ? t.z + bad : tA;
    if (rank == 0 && (WARP || side)) {
        float loss = some ? divergence(a, en, sm.log_t, m, logf(tA)) * (a.alpha * a.tau * a.tau) : 0.f;
        if (given) loss += (1.f - a.alpha) * (logf(tB) - (zl - m));
        if ((tid & 31) == 0) a.row_loss[r] = loss;
    }
    if (!dz) return;
    const float fw = w * scale;
    const float gt = some ? fw * a.alpha * a.tau : 0.f, gl = given ? fw * (1.f - a.alpha) : 0.f;
    // exponentials' factors: the two terms', or both in one
    const float fA = two ? gt / tA : (gt + gl) / tA, fB = gl / tB;
    auto grad = [&](float2 v) {
        const float2 d = __fadd2_rn(v, both(-m));
        const float2 g = __fmul2_rn(exp2_2(__fmul2_rn(d, both(cA))), both(fA));
        return two ? __ffma2_rn(exp2_2(__fmul2_rn(d, both(kLog2e))), both(fB), g) : g;
    };
    // Many entries find those of the same class through the class's place in the row, whose logit is kept and whose gradient
    // is written last: each leaves its number there, and who reads another's marks both.
    auto place = [&](int j) { return elems + (en.cls[j] - first); };
    auto here = [&](int j) { return en.cls[j] >= e0 && en.cls[j] < e1; };
    if (many) {
        if (!side)
            for (int j = tid; j < a.k; j += threads)
                if (here(j)) *reinterpret_cast<Bits*>(place(j)) = (Bits)j;
        sync();
        if (!side)
            for (int j = tid; j < a.k; j += threads)
                if (here(j)) {
                    const int other = (int)*reinterpret_cast<const Bits*>(place(j));
                    if (other != j) en.fix[other] = en.fix[j] = 1.f;
                }
        sync();
    }
    // the classes of the teacher and the label, from their logits as they were
    const bool lab_here = given && lab >= e0 && lab < e1 && tid == threads - 1;
    float fix_lab = 0.f;
    if (!side) {
        for (int j = tid; j < a.k; j += threads) {
            const int c = en.cls[j];
            if (!here(j)) continue;
            const float pj = en.fix[j] != 0.f ? named(a, en, c) : en.p[j];
            const bool label = given && c == lab;
            en.fix[j] = grad(both(en.zc[j])).x - gt * pj - (label ? gl : 0.f);
            if (label) sm.named = 1;
        }
        if (lab_here) fix_lab = grad(both(zl)).x - gl;
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
    }
    sync();
    if (!side) {
        for (int j = tid; j < a.k; j += threads)
            if (here(j)) *place(j) = elem_from<T>(en.fix[j]);
        if (lab_here && !sm.named) elems[lab - first] = elem_from<T>(fix_lab);
    }
    const bool same = ((reinterpret_cast<uintptr_t>(dz) ^ p0) & 15) == 0;  // rows begin at the same place of a unit
    if (same) fence_async_shared();
    sync();
    const int step = WARP ? 32 : blockDim.x;
    if (!same) {
        for (int i = e0 + tid; i < e1; i += step) dz[i] = elems[i - first];
        return;
    }
    if (tid == 0 && c1 > c0) {
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dz + first + c0 * E), "r"(smem_u32(units + c0)),
                     "r"((uint32_t)(c1 - c0) * 16)
                     : "memory");
        bulk_commit();
    }
    for (int i = e0 + tid; i < min(first + c0 * E, e1); i += step) dz[i] = elems[i - first];
    for (int i = max(first + c1 * E, e0) + tid; i < e1; i += step) dz[i] = elems[i - first];
    if (tid == 0) bulk_wait_read();
}

// Rows that no cluster holds in shared memory: one row per block, read three times.
template <class T>
__global__ void __launch_bounds__(kStream) distill_stream_kernel(DistillArgs a)
{
    __shared__ float red[32];
    __shared__ __align__(16) char entries[kMaxK * 20];
    const Entries en(entries, a.k);
    __shared__ int some_s;
    __shared__ float log_ts;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + r * a.ld;
        T* dz = a.dz ? static_cast<T*>(a.dz) + r * a.ld_grad : nullptr;
        const float w = a.weight ? a.weight[r] : a.one;
        const int lab = a.labels && a.alpha < 1.f ? a.labels[r] : -1;
        const bool given = lab >= 0 && lab < a.v;
        if (threadIdx.x < 32) {
            float log_t;
            Ahead ahead;
            ahead.ask(a, r);
            load_entries(a, r, z, en, &ahead, threadIdx.x, 32);
            __syncwarp();
            const bool some = teacher(a, en, log_t);
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
            float loss = some ? divergence(a, en, log_ts, m, logf(tA)) * (a.alpha * a.tau * a.tau) : 0.f;
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
            const int c = en.cls[j];
            if (c >= 0) dz[c] = elem_from<T>(grad(en.zc[j]) - gt * named(a, en, c) - (c == lab && given ? gl : 0.f));
        }
        if (given && threadIdx.x == 0) dz[lab] = elem_from<T>(grad(zl) - gt * named(a, en, lab) - gl);
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
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < rows; r += 1024) s += weight ? weight[r] * row_loss[r] : row_loss[r];
    s = block_sum(s, red);
    if (threadIdx.x == 0) *loss = weight ? s : s / (float)rows;
}

template <class T>
int launch(const DistillArgs& a, cudaStream_t st, const char* what)
{
    constexpr auto kernel = distill_kernel<T, false>;
    constexpr auto kernel_w = distill_kernel<T, true>;
    const size_t head = head_bytes(a.k);
    const size_t row = ((size_t)a.v * sizeof(T) + 15) / 16 * 16 + 16;
    auto part = [&](int S) { return (row / 16 + S - 1) / S * 16; };
    // Many rows go by the rows in flight on an SM: of short ones a warp each leaves most room (8000 x 5000 in bf16: 59 us
    // a warp each, 77 us a block each; 8000 x 8000 104 and 86 us).  Few go by the threads of each.
    if (row <= (a.rows >= 4 * sm_count() ? kWarpBytes : kWarpBytesFew) && a.k <= kWarpK) {
        const size_t group = (head + row + 127) / 128 * 128;
        const int64_t grid = (a.rows + kWarpRows - 1) / kWarpRows;
        if (grid > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^31 blocks", what);
        const int rc = allow_launch<kernel_w>(kWarpRows * (kWarpBytes + head_bytes(kWarpK) + 128), false, what);
        if (rc != DBL_OK) return rc;
        kernel_w<<<(unsigned)grid, 32 * kWarpRows, group * kWarpRows, st>>>(a, (int)group);
        return launch_check(what);
    }
    // As many blocks to a row as bring two on an SM: a cluster's blocks wait for one another, and three smaller parts on
    // an SM do not make up for that where there are many rows (4000 x 40000 in bf16: 196 us a block each, 224 us two;
    // 600 x 50257 44 and 50 us; 200 x 50257 26 and 24 us).  For few rows, as fill the SMs, with parts of 8 KB and more.
    int S = 1;
    while (S < kMaxCluster && part(S) > kLargePartBytes) S *= 2;
    while (S < kMaxCluster && part(S) > kPartBytes && a.rows * S * 2 <= 3 * sm_count()) S *= 2;
    while (S < kMaxCluster && a.rows * S * 2 <= sm_count() && part(2 * S) >= 8192) S *= 2;
    while (S > 1 && !cluster_held<kernel>(S, kMaxThreads + 32, kMaxPartBytes + head_bytes(kMaxK))) S /= 2;
    if (part(S) > kMaxPartBytes) {
        distill_stream_kernel<T><<<(int)std::min<int64_t>(a.rows, 1 << 20), kStream, 0, st>>>(a);
        return launch_check(what);
    }
    if (a.rows * S > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^31 blocks", what);
    const size_t smem = head + part(S);
    // 256 bytes of the part to a thread, so that registers allow more blocks on an SM (2673 x 15504 in bf16: 56 us, with
    // 64 bytes 69 us); 64 where there are few rows
    const size_t share = a.rows * S >= 2 * sm_count() ? 256 : 64;
    int threads = 64;
    while (threads < kMaxThreads && threads * share < part(S)) threads *= 2;
    int rc = allow_launch<kernel>(kMaxPartBytes + head_bytes(kMaxK), true, what);
    if (rc != DBL_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(a.rows * S));
    cfg.blockDim = dim3(threads + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, a, 0);
    rc = launch_check(what);
    return err == cudaSuccess ? rc : cuda_check(err, what);
}

}  // namespace

namespace dbl {

static int read_word(int* status) { return status_read(g_distill_status, status); }
static int clear_word() { return status_clear(g_distill_status); }
StatusWord distill_status_word() { return {read_word, clear_word}; }

}  // namespace dbl

extern "C" int dbl_distill_fwd_bwd(const dbl_distill_shape* s, const void* logits, const float* teacher_logits,
                                   const int32_t* teacher_classes, const int32_t* labels, const float* row_weight,
                                   const float* loss_scale, float* row_loss, float* loss, void* dlogits, void* stream)
{
    const char* w = "distill_fwd_bwd";
    if (!s || s->rows < 0 || s->classes <= 0 || s->k < 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0, classes <= 0 or k < 0", w);
    if (s->classes > kMaxColumns) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^30 classes or more", w);
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
                     s->alpha, s->rows > 0 ? 1.f / (float)s->rows : 0.f};
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
