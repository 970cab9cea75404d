// ln.cu -- layer norm over the last dimension, forward (with the residual addition before it) and backward (with
// the skip path's gradient and the sums over rows for gamma and beta).
//
// With mu and s = 1/sqrt(variance + eps) of a row and h = (x - mu)*s: y = h*gamma + beta; for g = dy*gamma,
// dx = s*(g - mean(g) - h*mean(g*h)) + dskip; dgamma = sum of dy*h over the rows, dbeta = sum of dy.  The variance is
// taken of the deviations from the mean, so that an offset of the row costs no digits.  Rows, sums and statistics are
// held in fp32; what is stored (the sum with the residual too) is rounded once, to the tensors' format.
//
// Bound by memory: a row is read once and written once.  A group of threads takes a row, 16 columns a thread, and goes
// on to another until there are none; a group's next rows are on their way into shared memory meanwhile, each by one
// bulk copy, so that what is in flight does not go by the registers (loads into registers a row ahead reached 0.4 of
// the copy rate).  Rows of up to 256 columns: several to a warp.  Rows of more than 8192: a cluster of blocks each.
//
// On a GB300 that copies 6.78 TB/s, bf16 but where said: forward with the residual, 32768 x 1024 in fp16 52 us =
// 5.1 TB/s (shared memory's latency between two sums over the row; 22 warps on an SM); 256 x 512 4.6 us, the launch.
// Backward with the skip gradient, 65536 x 2048 174 us = 6.2 TB/s; 10007 x 1537 in fp32 54 us = 3.4 TB/s (rows that
// begin at any word: 4-byte accesses, more than twice the instructions).  100000 x 64: 17.5 and 21 us.
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxGroup = 512;     // threads of a row
constexpr int kBlock = 256;        // threads of a block of several groups
constexpr int kMaxSplit = 8;       // blocks of a row
constexpr int kMaxDepth = 4;       // rows of a group on their way
constexpr int kWide = 256;         // threads of the kernels for rows wider than a group
constexpr int kShort = 256;        // columns of a short row, at the most
constexpr int kShortFwd = 3, kShortBwd = 2;  // blocks on an SM for them
constexpr int kSumThreads = 1024;
constexpr size_t kRingBytes = 200 * 1024;  // shared memory for them on an SM
constexpr size_t kMaxSmem = kRingBytes + 16 * 1024;

__device__ int g_ln_status;

struct LnArgs {
    const void *x, *res, *dy;
    const float *gamma, *beta;
    void *sum, *y;
    float *mean, *invstd;
    float* parts;
    int64_t rows, ld_in, ld_out;
    int c;
    float eps;
    int group, depth, slot;  // threads of a row, rows on their way, bytes of one in shared memory
    int part;                // columns of a block, where a cluster takes a row
    int batch;               // short rows at a time
};

// Loads that stay where they are written: the compiler moves others behind the wait for the row, where nothing hides them
// (backward of 65536 x 2048: 173 and 204 us; of 40000 x 1001 95 and 101).  Not for single fp32 columns, which take the
// registers for more addresses (10007 x 1537: 60 us, 54 where the compiler chooses).  v is left as it is where `there`
// does not hold.
__device__ __forceinline__ void ask(float4& v, const float* p, bool there)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %5, 0;\n\t@p ld.global.nc.v4.f32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "+f"(v.x), "+f"(v.y), "+f"(v.z), "+f"(v.w)
                 : "l"(p), "r"((int)there));
}
__device__ __forceinline__ void ask(float& v, const float* p, bool there)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p ld.global.nc.f32 %0, [%1];\n\t}" : "+f"(v) : "l"(p), "r"((int)there));
}

// This thread's columns of a row, in pairs: J accesses of 16 bytes where rows allow it (VEC; FULL: every thread has all
// of its columns), otherwise of 4 bytes.
template <class T, bool VEC, bool FULL, int N, int W = 32>
struct Cols {
    static constexpr int A = VEC ? 16 / (int)sizeof(T) : 2, J = N / A, P = A / 2;  // columns, accesses, pairs of one
    // first column of access j, and how far the second of its (first) pair is: single fp32 columns lie side by side in
    // a warp, 16-bit ones in a thread, which can store them at once in rows that begin at a word
    static constexpr bool ASIDE = !VEC && sizeof(T) == 4;
    static constexpr int MATE = ASIDE ? W : 1;
    static __device__ __forceinline__ int base(int g) { return (g & ~(W - 1)) * N + (g & (W - 1)) * (ASIDE ? 1 : A); }
    static __device__ __forceinline__ int col(int j, int g) { return base(g) + j * W * A; }
    static __device__ __forceinline__ float2 pair(const T* p) { return make_float2(elem_f(p[0]), elem_f(p[1])); }
    // access j of a row in shared memory that begins `off` elements after row; zeros past its end
    static __device__ __forceinline__ void read(float2* f, const char* row, int off, int c, int g, int j)
    {
        const int i = col(j, g);
        if constexpr (VEC) {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (FULL || i < c) r = *reinterpret_cast<const uint4*>(row + i * sizeof(T));
            const T* p = reinterpret_cast<const T*>(&r);
#pragma unroll
            for (int k = 0; k < P; ++k) f[k] = pair(p + 2 * k);
        } else {
            const T* p = reinterpret_cast<const T*>(row) + off + i;
            f[0] = make_float2(i < c ? elem_f(p[0]) : 0.f, i + MATE < c ? elem_f(p[MATE]) : 0.f);
        }
    }
    // all accesses; 16-bit pairs in one where the row begins at a word
    static __device__ __forceinline__ void read_all(float2* f, const char* row, int off, int c, int g)
    {
        if (!VEC && sizeof(T) == 2 && off % 2 == 0) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int i = col(j, g);
                uint32_t v = 0;
                if (i < c) v = reinterpret_cast<const uint32_t*>(row)[(off + i) / 2];
                f[j] = act::unpack2_u32(v);
                if (i + 1 >= c) f[j].y = 0.f;  // another row's
            }
        } else {
#pragma unroll
            for (int j = 0; j < J; ++j) read(f + j * P, row, off, c, g, j);
        }
    }
    static __device__ __forceinline__ void write_all(T* row, const float2* f, int c, int g)
    {
        if (!VEC && sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(row) & 3) == 0) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int i = col(j, g);
                if (i + 1 < c)
                    *reinterpret_cast<uint32_t*>(row + i) = act::pack2_u32(f[j].x, f[j].y);
                else if (i < c)
                    row[i] = elem_from<T>(f[j].x);
            }
        } else {
#pragma unroll
            for (int j = 0; j < J; ++j) write(row, f + j * P, c, g, j);
        }
    }
    static __device__ __forceinline__ void write(T* row, const float2* f, int c, int g, int j)
    {
        const int i = col(j, g);
        if constexpr (VEC) {
            uint4 o;
            T* p = reinterpret_cast<T*>(&o);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if constexpr (sizeof(T) == 2)
                    reinterpret_cast<uint32_t*>(&o)[k] = act::pack2_u32(f[k].x, f[k].y);
                else
                    p[2 * k] = f[k].x, p[2 * k + 1] = f[k].y;
            }
            if (FULL || i < c) *reinterpret_cast<uint4*>(row + i) = o;
        } else {
            if (sizeof(T) == 2 && i + 1 < c && (reinterpret_cast<uintptr_t>(row) & 3) == 0) {
                *reinterpret_cast<uint32_t*>(row + i) = act::pack2_u32(f[0].x, f[0].y);
            } else {
                if (i < c) row[i] = elem_from<T>(f[0].x);
                if (i + MATE < c) row[i + MATE] = elem_from<T>(f[0].y);
            }
        }
    }
    // parameters of the same columns (`other` where there are none, and past the row's end)
    static __device__ __forceinline__ void param(float2* f, const float* p, float other, int c, int g, int j)
    {
        const int i = col(j, g);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            if constexpr (VEC) {
                if (k % 2 == 0) {
                    float4 q = make_float4(other, other, other, other);
                    ask(q, p + i + 2 * k, p && (FULL || i < c));
                    f[k] = make_float2(q.x, q.y), f[k + 1] = make_float2(q.z, q.w);
                }
            } else {
                f[k] = make_float2(other, other);
                if constexpr (!ASIDE) {
                    ask(f[k].x, p + i, p && i < c);
                    ask(f[k].y, p + i + MATE, p && i + MATE < c);
                } else if (p) {
                    if (i < c) f[k].x = __ldg(p + i);
                    if (i + MATE < c) f[k].y = __ldg(p + i + MATE);
                }
            }
        }
    }
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// What one bulk copy brings of `len` elements at p, of a tensor that goes from `first` to before `end`: all from the 16-byte
// boundary at or before them to the one at or after them, or where that would leave the tensor, the 16-byte units within.
struct Span {
    uintptr_t lo;
    uint32_t bytes, skip;  // skip: from the boundary at or before the first element
    int head, tail;        // elements before the span, and the first one after it
};
template <class T>
__device__ __forceinline__ Span span_of(const T* first, const T* end, const T* p, int len)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p), e = b + len * sizeof(T);
    uintptr_t lo = b & ~(uintptr_t)15, hi = (e + 15) & ~(uintptr_t)15;
    Span s = {lo, 0, 0, 0, len};
    if (lo < reinterpret_cast<uintptr_t>(first) || hi > reinterpret_cast<uintptr_t>(end)) {
        lo = (b + 15) & ~(uintptr_t)15, hi = e & ~(uintptr_t)15;
        if (hi < lo) hi = lo;
        s.skip = (uint32_t)(lo - s.lo), s.lo = lo;
        s.head = min(len, (int)((lo - b) / sizeof(T))), s.tail = max(s.head, (int)((hi - b) / sizeof(T)));
    }
    s.bytes = (uint32_t)(hi - lo);
    return s;
}

// A block's groups: their places, barriers and rows in shared memory.
template <class T, bool VEC, int TENSORS>
struct Groups {
    int G, g, id, n, warp, warps, depth, slot, c;
    uint64_t* bars;  // of this group, one per row on its way
    float2* red;     // of this group: [2][warps]
    char* ring;      // of this group: [depth][TENSORS][slot]
    int* abort;
    int64_t rows, ld;
    unsigned phase;

    static __host__ __device__ size_t head(int warps) { return 128 + (size_t)warps * (kMaxDepth * sizeof(uint64_t) + 4 * sizeof(float2)); }

    __device__ __forceinline__ void set(const LnArgs& a, char* smem)
    {
        G = a.group, g = threadIdx.x % G, id = threadIdx.x / G, n = blockDim.x / G, warp = g >> 5, warps = G >> 5;
        depth = a.depth, slot = a.slot, c = a.c, rows = a.rows, ld = a.ld_in, phase = 0;
        const int all = blockDim.x >> 5;
        abort = reinterpret_cast<int*>(smem);
        bars = reinterpret_cast<uint64_t*>(smem + 128) + id * kMaxDepth;
        red = reinterpret_cast<float2*>(smem + 128 + (size_t)all * kMaxDepth * sizeof(uint64_t)) + id * warps * 4;
        ring = smem + (head(all) + 127) / 128 * 128 + (size_t)id * depth * TENSORS * slot;
        if (threadIdx.x == 0) *abort = 0;
        if (g == 0) {
            for (int k = 0; k < depth; ++k) mbar_init(&bars[k], 1);
            fence_mbar_init();
        }
        __syncthreads();
    }
    __device__ __forceinline__ void sync() const
    {
        if (warps == 1)
            __syncwarp();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(G) : "memory");
    }
    // One thread's work: row r of every tensor into place k.
    __device__ __forceinline__ void fetch(const T* const (&from)[TENSORS], int k, int64_t r) const
    {
        char* const to = ring + (size_t)k * TENSORS * slot;
        if constexpr (VEC) {
            const uint32_t bytes = c * sizeof(T);
            mbar_arrive_expect_tx(&bars[k], (from[TENSORS - 1] ? TENSORS : TENSORS - 1) * bytes);
#pragma unroll
            for (int t = 0; t < TENSORS; ++t)
                if (t < TENSORS - 1 || from[t]) bulk_load(smem_u32(to + t * slot), reinterpret_cast<uintptr_t>(from[t] + r * ld), bytes, &bars[k]);
        } else {
            Span sp[TENSORS];
            uint32_t sum = 0;
#pragma unroll
            for (int t = 0; t < TENSORS; ++t) sp[t] = span(from[t], r), sum += sp[t].bytes;
            mbar_arrive_expect_tx(&bars[k], sum);
#pragma unroll
            for (int t = 0; t < TENSORS; ++t)
                if (sp[t].bytes) bulk_load(smem_u32(to + t * slot) + sp[t].skip, sp[t].lo, sp[t].bytes, &bars[k]);
        }
    }
    __device__ __forceinline__ Span span(const T* from, int64_t r) const
    {
        if (!from) return {0, 0, 0, 0, c};
        return span_of(from, from + (rows - 1) * ld + c, from + r * ld, c);
    }
    // elements from the 16-byte boundary to a row's first one
    __device__ __forceinline__ int offset(const T* from, int64_t r) const
    {
        if constexpr (VEC) return 0;
        constexpr uint32_t E = 16 / sizeof(T);
        return (int)(((uint32_t)reinterpret_cast<uintptr_t>(from) / sizeof(T) + (uint32_t)r * (uint32_t)ld) % E);
    }
    __device__ __forceinline__ const char* row(int k, int t) const { return ring + ((size_t)k * TENSORS + t) * slot; }
    __device__ __forceinline__ void wait(const T* const (&from)[TENSORS], int k, int64_t r)
    {
        bounded_wait(&bars[k], phase >> k & 1, abort, &g_ln_status);
        phase ^= 1u << k;
        if (VEC || (r >= 16 && r < rows - 16)) return;  // of 16 rows the 16 bytes before or after are the tensor's
        // rows at the tensor's ends: what the bulk copy has left out, fewer elements than a warp has lanes
        T v[TENSORS];
        int at[TENSORS];
#pragma unroll
        for (int t = 0; t < TENSORS; ++t) {
            const Span s = span(from[t], r);
            at[t] = !from[t] ? c : g < s.head ? g : s.tail + g - s.head;
            if (at[t] < c) v[t] = from[t][r * ld + at[t]];
        }
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
            if (at[t] < c) (reinterpret_cast<T*>(ring + ((size_t)k * TENSORS + t) * slot) + offset(from[t], r))[at[t]] = v[t];
        fence_async_shared();  // before a later row's bulk copy to the same place
        sync();
    }
    // Sums over the group, the same bits in all its threads; which: 0 or 1, not the same twice in a row.
    __device__ __forceinline__ float2 total(float2 v, int which) const
    {
        v = make_float2(warp_sum(v.x), warp_sum(v.y));
        if (warps == 1) return v;
        float2* p = red + which * warps;
        if ((threadIdx.x & 31) == 0) p[warp] = v;
        sync();
        v = (threadIdx.x & 31) < warps ? p[threadIdx.x & 31] : make_float2(0.f, 0.f);
        return make_float2(warp_sum(v.x), warp_sum(v.y));
    }
    __device__ __forceinline__ float total(float v, int which) const
    {
        v = warp_sum(v);
        if (warps == 1) return v;
        float2* p = red + which * warps;
        if ((threadIdx.x & 31) == 0) p[warp].x = v;
        sync();
        return warp_sum((threadIdx.x & 31) < warps ? p[threadIdx.x & 31].x : 0.f);
    }
};

// What the blocks of a cluster, each with its columns of a row, tell one another of it: a pair of sums, stored into every
// block's slot of the sender, by turns in two places.  Who has all pairs of row n+1 knows that all blocks have read
// those of row n: a block sends after its threads have met, and they have read by then.
struct Exchange {
    uint64_t bar[2];
    float2 slot[2][kMaxSplit];

    __device__ __forceinline__ void init()
    {
        if (threadIdx.x == 0) {
            mbar_init(&bar[0], 1);
            mbar_init(&bar[1], 1);
            fence_mbar_init();
        }
        cluster_sync_all();
    }
    // v: the block's, the same in all its threads; returns the blocks' pairs in their order
    __device__ __forceinline__ const float2* all(float2 v, int which, uint32_t parity, int S, int rank, int* abort)
    {
        if (threadIdx.x == 0) mbar_arrive_expect_tx(&bar[which], S * sizeof(float2));
        if ((int)threadIdx.x < S)
            st_async2(mapa_shared(smem_u32(&slot[which][rank]), threadIdx.x), mapa_shared(smem_u32(&bar[which]), threadIdx.x), v);
        bounded_wait(&bar[which], parity, abort, &g_ln_status);
        return slot[which];
    }
};

// A cluster's columns of a row: the arguments with this block's part of every tensor.
template <class T>
__device__ __forceinline__ void take_part(LnArgs& a, int rank)
{
    const int skip = rank * a.part;
    a.c = min(a.part, a.c - skip);
    a.x = static_cast<const T*>(a.x) + skip, a.y = static_cast<T*>(a.y) + skip;
    if (a.res) a.res = static_cast<const T*>(a.res) + skip;
    if (a.dy) a.dy = static_cast<const T*>(a.dy) + skip;
    if (a.sum) a.sum = static_cast<T*>(a.sum) + skip;
    if (a.gamma) a.gamma += skip;
    if (a.beta) a.beta += skip;
    if (a.parts) a.parts += skip;
}

template <class T, bool VEC, bool FULL, int N, int THREADS, int BLOCKS, bool SPLIT>
__global__ void __launch_bounds__(THREADS, BLOCKS) ln_fwd_kernel(LnArgs a)
{
    typedef Cols<T, VEC, FULL, N> C;
    constexpr int P = C::P;
    extern __shared__ __align__(128) char smem[];
    __shared__ Exchange ex;
    const int c = a.c, S = SPLIT ? (a.c + a.part - 1) / a.part : 1, rank = SPLIT ? (int)cluster_ctarank() : 0;
    if (SPLIT) {
        take_part<T>(a, rank);
        ex.init();
    }
    Groups<T, VEC, 2> w;
    w.set(a, smem);
    const T* const from[2] = {static_cast<const T*>(a.x), static_cast<const T*>(a.res)};
    const int g = w.g;
    const int64_t hop = (int64_t)gridDim.x / S * w.n;
    int64_t r = (int64_t)blockIdx.x / S * w.n + w.id;
    if (g == 0)
        for (int k = 0; k < w.depth; ++k)
            if (r + k * hop < a.rows) w.fetch(from, k, r + k * hop);
    float2 ga[N / 2], be[N / 2];  // from row to row
#pragma unroll
    for (int j = 0; j < C::J; ++j) {
        C::param(ga + j * P, a.gamma, 1.f, a.c, g, j);
        C::param(be + j * P, a.beta, 0.f, a.c, g, j);
    }
    const float inv_c = 1.f / a.c;
    int par = 0;
    uint32_t turn = 0;  // of the exchange's two places
    for (int k = 0; r < a.rows; r += hop, k = k + 1 == w.depth ? 0 : k + 1, turn ^= par, par ^= 1) {
        float2 v[N / 2], s = both(0.f);
        w.wait(from, k, r);
        const int off = w.offset(from[0], r), off_r = w.offset(from[1], r);
        C::read_all(v, w.row(k, 0), off, a.c, g);
        if (a.res) {
            float2 u[N / 2];
            C::read_all(u, w.row(k, 1), off_r, a.c, g);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[i] = __fadd2_rn(v[i], u[i]);
        }
        if (a.sum) C::write_all(static_cast<T*>(a.sum) + r * a.ld_out, v, a.c, g);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) s = __fadd2_rn(s, v[i]);
        float mean = w.total(s.x + s.y, 0) * inv_c;
        if (w.warps == 1) __syncwarp();
        if (g == 0 && r + w.depth * hop < a.rows) w.fetch(from, k, r + w.depth * hop);  // the group has read the place
        s = both(0.f);
#pragma unroll
        for (int j = 0; j < C::J; ++j) {
            const int i0 = C::col(j, g);
#pragma unroll
            for (int i = j * P; i < (j + 1) * P; ++i) {
                v[i] = __fadd2_rn(v[i], both(-mean));
                if (VEC) {
                    if (FULL || i0 < a.c) s = __ffma2_rn(v[i], v[i], s);
                } else {
                    if (i0 < a.c) s.x = fmaf(v[i].x, v[i].x, s.x);
                    if (i0 + C::MATE < a.c) s.y = fmaf(v[i].y, v[i].y, s.y);
                }
            }
        }
        float var = w.total(s.x + s.y, 1) * inv_c;
        if (SPLIT) {  // the parts' means and variances as one: that of the means is added to those of the parts
            const float2* p = ex.all(make_float2(mean, var), par, turn, S, rank, w.abort);
            auto share = [&](int k) { return (float)min(a.part, c - k * a.part) / c; };
            float whole = 0.f;
            for (int k = 0; k < S; ++k) whole = fmaf(p[k].x, share(k), whole);
            var = 0.f;
            for (int k = 0; k < S; ++k) {
                const float d = p[k].x - whole;
                var = fmaf(fmaf(d, d, p[k].y), share(k), var);
            }
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[i] = __fadd2_rn(v[i], both(mean - whole));
            mean = whole;
        }
        const float inv = 1.f / sqrtf(var + a.eps);
#pragma unroll
        for (int j = 0; j < C::J; ++j) {
            float2* f = v + j * P;
#pragma unroll
            for (int i = 0; i < P; ++i) f[i] = __ffma2_rn(__fmul2_rn(f[i], both(inv)), ga[j * P + i], be[j * P + i]);
        }
        C::write_all(static_cast<T*>(a.y) + r * a.ld_out, v, a.c, g);
        if (g == 0 && rank == 0 && a.mean) {
            a.mean[r] = mean;
            a.invstd[r] = inv;
        }
    }
    linger(w.abort);
    if (SPLIT) cluster_leave();
}

// x: the normalised tensor, res: dskip, y: dx.  The row stays in registers between its two passes.  A thread also adds up dy*xhat and dy of its columns over the rows
// that its group takes; a block leaves these sums in parts[block][2][c].
template <class T, bool VEC, bool FULL, int N, int THREADS, int BLOCKS, bool SPLIT>
__global__ void __launch_bounds__(THREADS, BLOCKS) ln_bwd_kernel(LnArgs a)
{
    typedef Cols<T, VEC, FULL, N> C;
    constexpr int P = C::P;
    extern __shared__ __align__(128) char smem[];
    __shared__ Exchange ex;
    const int c = a.c, S = SPLIT ? (a.c + a.part - 1) / a.part : 1, rank = SPLIT ? (int)cluster_ctarank() : 0;
    if (SPLIT) {
        take_part<T>(a, rank);
        ex.init();
    }
    Groups<T, VEC, 3> w;
    w.set(a, smem);
    const T* const from[3] = {static_cast<const T*>(a.x), static_cast<const T*>(a.dy), static_cast<const T*>(a.res)};
    const int g = w.g;
    const int64_t team = blockIdx.x / S, hop = (int64_t)gridDim.x / S * w.n;
    int64_t r = team * w.n + w.id;
    float mean = 0.f, inv = 0.f;
    if (r < a.rows) {
        if (g == 0)
            for (int k = 0; k < w.depth; ++k)
                if (r + k * hop < a.rows) w.fetch(from, k, r + k * hop);
        mean = a.mean[r], inv = a.invstd[r];
    }
    grid_dependency_trigger();
    float2 dg[N / 2], db[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) dg[i] = db[i] = both(0.f);
    const float inv_c = 1.f / c;
    bool first = true;
    int par = 0;
    uint32_t turn = 0;  // of the exchange's two places
    for (int k = 0; r < a.rows; r += hop, k = k + 1 == w.depth ? 0 : k + 1, turn ^= par, par ^= 1) {
        float2 h[N / 2], d[N / 2], ga[N / 2], tx = both(0.f), ty = tx;
#pragma unroll
        for (int j = 0; j < C::J; ++j) C::param(ga + j * P, a.gamma, 1.f, a.c, g, j);  // back before the row is
        w.wait(from, k, r);
        const int off_x = w.offset(from[0], r), off_d = w.offset(from[1], r);
        const float is = inv, mu = mean;
        if (r + hop < a.rows) mean = a.mean[r + hop], inv = a.invstd[r + hop];
#pragma unroll
        for (int j = 0; j < C::J; ++j) {
            C::read(h + j * P, w.row(k, 0), off_x, a.c, g, j);
            C::read(d + j * P, w.row(k, 1), off_d, a.c, g, j);
#pragma unroll
            for (int q = 0; q < P; ++q) {  // past the row's end d is 0
                const int i = j * P + q;
                h[i] = __fmul2_rn(__fadd2_rn(h[i], both(-mu)), both(is));
                dg[i] = __ffma2_rn(d[i], h[i], dg[i]);
                db[i] = __fadd2_rn(db[i], d[i]);
                d[i] = __fmul2_rn(d[i], ga[i]);
                tx = __fadd2_rn(tx, d[i]);
                ty = __ffma2_rn(d[i], h[i], ty);
            }
        }
        float2 t = w.total(make_float2(tx.x + tx.y, ty.x + ty.y), par);
        if (SPLIT) {
            const float2* p = ex.all(t, par, turn, S, rank, w.abort);
            t = p[0];
            for (int i = 1; i < S; ++i) t = __fadd2_rn(t, p[i]);
        }
        if (w.warps == 1) __syncwarp();
        // the row before this one has been read by all of the group: its place is free
        if (g == 0 && !first && r + (w.depth - 1) * hop < a.rows) w.fetch(from, (k ? k : w.depth) - 1, r + (w.depth - 1) * hop);
        first = false;
        tx = both(-t.x * inv_c * is), ty = both(-t.y * inv_c * is);
        const int off_s = w.offset(from[2], r);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) d[i] = __ffma2_rn(h[i], ty, __ffma2_rn(d[i], both(is), tx));
#pragma unroll
        for (int j = 0; j < C::J; ++j) {
            if (a.res) {
                float2 u[P];
                C::read(u, w.row(k, 2), off_s, a.c, g, j);
#pragma unroll
                for (int q = 0; q < P; ++q) d[j * P + q] = __fadd2_rn(d[j * P + q], u[q]);
            }
            C::write(static_cast<T*>(a.y) + r * a.ld_out, d + j * P, a.c, g, j);
        }
    }
    linger(w.abort);
    if (SPLIT) cluster_leave();
    if (!a.parts) return;
    // groups of one block: through shared memory, all rows being done
    float* out = a.parts + team * 2 * c;
    float* sums = reinterpret_cast<float*>(w.ring - (size_t)w.id * w.depth * 3 * w.slot);
    if (w.n > 1) {
        __syncthreads();
        out = sums + w.id * 2 * a.c;
    }
#pragma unroll
    for (int j = 0; j < C::J; ++j)
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int i = C::col(j, g) + 2 * q, m = i + C::MATE;
            if (i < a.c) out[i] = dg[j * P + q].x, out[c + i] = db[j * P + q].x;
            if (m < a.c) out[m] = dg[j * P + q].y, out[c + m] = db[j * P + q].y;
        }
    if (w.n == 1) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.c; i += blockDim.x) {
        float t = 0.f;
        for (int k = 0; k < w.n; ++k) t += sums[k * 2 * a.c + i];
        a.parts[(int64_t)blockIdx.x * 2 * a.c + i] = t;
    }
}

// Short rows that lie one after another: W lanes take a row, a warp 32/W of them at a time; `batch` of them on their way in
// one bulk copy, two such places to a warp.
template <class T, bool VEC, int W, int TENSORS>
struct Batches {
    static constexpr int AT_ONCE = 32 / W;
    int batch, slot, pitch, c;
    int64_t rows;
    uint64_t* bars;
    char* ring;  // of this warp
    int* abort;
    unsigned phase;

    static __host__ __device__ size_t head() { return 128 + kBlock / 32 * 2 * sizeof(uint64_t); }

    __device__ __forceinline__ void set(const LnArgs& a, char* smem)
    {
        batch = a.batch, slot = a.slot, pitch = (a.res ? TENSORS : TENSORS - 1) * slot, c = a.c, rows = a.rows, phase = 0;
        const int warp = threadIdx.x >> 5;
        abort = reinterpret_cast<int*>(smem);
        bars = reinterpret_cast<uint64_t*>(smem + 128) + warp * 2;
        ring = smem + (head() + 127) / 128 * 128 + (size_t)warp * 2 * pitch;
        if (threadIdx.x == 0) *abort = 0;
        if ((threadIdx.x & 31) == 0) {
            mbar_init(&bars[0], 1);
            mbar_init(&bars[1], 1);
            fence_mbar_init();
        }
        __syncthreads();
    }
    __device__ __forceinline__ int count(int64_t r) const { return (int)min((int64_t)batch, rows - r); }
    __device__ __forceinline__ Span span(const T* from, int64_t r) const
    {
        if (!from) return {0, 0, 0, 0, 0};
        return span_of(from, from + rows * c, from + r * c, count(r) * c);
    }
    // One lane's work: the rows from r into place k.
    __device__ __forceinline__ void fetch(const T* const (&from)[TENSORS], int k, int64_t r) const
    {
        Span sp[TENSORS];
        uint32_t sum = 0;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t) sp[t] = span(from[t], r), sum += sp[t].bytes;
        mbar_arrive_expect_tx(&bars[k], sum);
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
            if (sp[t].bytes) bulk_load(smem_u32(ring + (size_t)k * pitch + t * slot) + sp[t].skip, sp[t].lo, sp[t].bytes, &bars[k]);
    }
    __device__ __forceinline__ const char* place(int k, int t) const { return ring + (size_t)k * pitch + t * slot; }
    // elements from the 16-byte boundary to the first one of row r
    __device__ __forceinline__ int offset(const T* from, int64_t r) const
    {
        return VEC ? 0 : (int)((reinterpret_cast<uintptr_t>(from + r * c) & 15) / sizeof(T));
    }
    __device__ __forceinline__ void wait(const T* const (&from)[TENSORS], int k, int64_t r)
    {
        bounded_wait(&bars[k], phase >> k & 1, abort, &g_ln_status);
        phase ^= 1u << k;
        if (VEC || (r > 16 && r + batch + 16 < rows)) return;
        T v[TENSORS];
        int at[TENSORS];
        const int lane = threadIdx.x & 31, len = count(r) * c;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t) {
            const Span s = span(from[t], r);
            at[t] = !from[t] ? len : lane < s.head ? lane : s.tail + lane - s.head;
            if (at[t] < len) v[t] = from[t][r * c + at[t]];
        }
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
            if (at[t] < len) (reinterpret_cast<T*>(ring + (size_t)k * pitch + t * slot) + offset(from[t], r))[at[t]] = v[t];
        fence_async_shared();
        __syncwarp();
    }
    static __device__ __forceinline__ float total(float v)
    {
#pragma unroll
        for (int o = W / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
};

template <class T, bool VEC, int W>
__global__ void __launch_bounds__(kBlock, kShortFwd) ln_fwd_short_kernel(LnArgs a)
{
    typedef Cols<T, VEC, false, 8, W> C;
    constexpr int P = C::P;
    extern __shared__ __align__(128) char smem[];
    Batches<T, VEC, W, 2> w;
    w.set(a, smem);
    const T* const from[2] = {static_cast<const T*>(a.x), static_cast<const T*>(a.res)};
    const int lane = threadIdx.x & 31, g = lane % W, sub = lane / W;
    const int64_t hop = (int64_t)gridDim.x * (kBlock / 32) * a.batch;
    int64_t r = ((int64_t)blockIdx.x * (kBlock / 32) + (threadIdx.x >> 5)) * a.batch;
    if (lane == 0)
        for (int k = 0; k < 2; ++k)
            if (r + k * hop < a.rows) w.fetch(from, k, r + k * hop);
    float2 ga[4], be[4];
#pragma unroll
    for (int j = 0; j < C::J; ++j) {
        C::param(ga + j * P, a.gamma, 1.f, a.c, g, j);
        C::param(be + j * P, a.beta, 0.f, a.c, g, j);
    }
    const float inv_c = 1.f / a.c;
    for (int k = 0; r < a.rows; r += hop, k ^= 1) {
        const int n = w.count(r);
        w.wait(from, k, r);
        const int off = w.offset(from[0], r), off_r = w.offset(from[1], r);
#pragma unroll 2
        for (int i = sub; i < a.batch; i += w.AT_ONCE) {  // a whole number of times; rows past the last are not stored
            if (i - sub >= n) break;
            const int64_t row = r + i;
            const int skip = i * a.c, bytes = VEC ? skip * (int)sizeof(T) : 0;
            float2 v[4], s = both(0.f);
#pragma unroll
            for (int j = 0; j < C::J; ++j) {
                C::read(v + j * P, w.place(k, 0) + bytes, off + skip, a.c, g, j);
                if (a.res) {
                    float2 u[P];
                    C::read(u, w.place(k, 1) + bytes, off_r + skip, a.c, g, j);
#pragma unroll
                    for (int q = 0; q < P; ++q) v[j * P + q] = __fadd2_rn(v[j * P + q], u[q]);
                }
                if (a.sum && i < n) C::write(static_cast<T*>(a.sum) + row * a.ld_out, v + j * P, a.c, g, j);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) s = __fadd2_rn(s, v[q]);
            const float mean = w.total(s.x + s.y) * inv_c;
            s = both(0.f);
#pragma unroll
            for (int j = 0; j < C::J; ++j) {
                const int i0 = C::col(j, g);
#pragma unroll
                for (int q = j * P; q < (j + 1) * P; ++q) {
                    v[q] = __fadd2_rn(v[q], both(-mean));
                    if (VEC) {
                        if (i0 < a.c) s = __ffma2_rn(v[q], v[q], s);
                    } else {
                        if (i0 < a.c) s.x = fmaf(v[q].x, v[q].x, s.x);
                        if (i0 + C::MATE < a.c) s.y = fmaf(v[q].y, v[q].y, s.y);
                    }
                }
            }
            const float inv = 1.f / sqrtf(fmaf(w.total(s.x + s.y), inv_c, a.eps));
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __ffma2_rn(__fmul2_rn(v[q], both(inv)), ga[q], be[q]);
            if (i < n) {
#pragma unroll
                for (int j = 0; j < C::J; ++j) C::write(static_cast<T*>(a.y) + row * a.ld_out, v + j * P, a.c, g, j);
                if (g == 0 && a.mean) {
                    a.mean[row] = mean;
                    a.invstd[row] = inv;
                }
            }
        }
        __syncwarp();
        if (lane == 0 && r + 2 * hop < a.rows) w.fetch(from, k, r + 2 * hop);
    }
    linger(w.abort);
}

template <class T, bool VEC, int W>
__global__ void __launch_bounds__(kBlock, kShortBwd) ln_bwd_short_kernel(LnArgs a)
{
    typedef Cols<T, VEC, false, 8, W> C;
    constexpr int P = C::P;
    extern __shared__ __align__(128) char smem[];
    Batches<T, VEC, W, 3> w;
    w.set(a, smem);
    const T* const from[3] = {static_cast<const T*>(a.x), static_cast<const T*>(a.dy), static_cast<const T*>(a.res)};
    const int lane = threadIdx.x & 31, g = lane % W, sub = lane / W;
    const int64_t hop = (int64_t)gridDim.x * (kBlock / 32) * a.batch;
    int64_t r = ((int64_t)blockIdx.x * (kBlock / 32) + (threadIdx.x >> 5)) * a.batch;
    if (lane == 0)
        for (int k = 0; k < 2; ++k)
            if (r + k * hop < a.rows) w.fetch(from, k, r + k * hop);
    // a batch's statistics, a row's in its lane, asked for a batch ahead
    float mean = 0.f, inv = 0.f;
    auto ask = [&](int64_t r) {
        const bool there = lane < a.batch && r + lane < a.rows;
        mean = there ? a.mean[r + lane] : 0.f, inv = there ? a.invstd[r + lane] : 0.f;
    };
    ask(r);
    grid_dependency_trigger();
    float2 ga[4], dg[4], db[4];
#pragma unroll
    for (int j = 0; j < C::J; ++j) C::param(ga + j * P, a.gamma, 1.f, a.c, g, j);
#pragma unroll
    for (int q = 0; q < 4; ++q) dg[q] = db[q] = both(0.f);
    const float inv_c = 1.f / a.c;
    for (int k = 0; r < a.rows; r += hop, k ^= 1) {
        const int n = w.count(r);
        w.wait(from, k, r);
        const int off_x = w.offset(from[0], r), off_d = w.offset(from[1], r), off_s = w.offset(from[2], r);
        const float mu_all = mean, is_all = inv;
        ask(r + hop);
#pragma unroll 2
        for (int i = sub; i < a.batch; i += w.AT_ONCE) {
            if (i - sub >= n) break;
            const int skip = i * a.c, bytes = VEC ? skip * (int)sizeof(T) : 0;
            const float mu = __shfl_sync(0xffffffffu, mu_all, i), is = __shfl_sync(0xffffffffu, is_all, i);
            float2 h[4], d[4], tx = both(0.f), ty = tx;
#pragma unroll
            for (int j = 0; j < C::J; ++j) {
                C::read(h + j * P, w.place(k, 0) + bytes, off_x + skip, a.c, g, j);
                C::read(d + j * P, w.place(k, 1) + bytes, off_d + skip, a.c, g, j);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {  // past the row's end d is 0
                if (i >= n) h[q] = d[q] = both(0.f);
                h[q] = __fmul2_rn(__fadd2_rn(h[q], both(-mu)), both(is));
                dg[q] = __ffma2_rn(d[q], h[q], dg[q]);
                db[q] = __fadd2_rn(db[q], d[q]);
                d[q] = __fmul2_rn(d[q], ga[q]);
                tx = __fadd2_rn(tx, d[q]);
                ty = __ffma2_rn(d[q], h[q], ty);
            }
            tx = both(-w.total(tx.x + tx.y) * inv_c * is), ty = both(-w.total(ty.x + ty.y) * inv_c * is);
#pragma unroll
            for (int j = 0; j < C::J; ++j) {
                float2 u[P];
#pragma unroll
                for (int q = 0; q < P; ++q) u[q] = __ffma2_rn(h[j * P + q], ty, __ffma2_rn(d[j * P + q], both(is), tx));
                if (a.res) {
                    float2 e[P];
                    C::read(e, w.place(k, 2) + bytes, off_s + skip, a.c, g, j);
#pragma unroll
                    for (int q = 0; q < P; ++q) u[q] = __fadd2_rn(u[q], e[q]);
                }
                if (i < n) C::write(static_cast<T*>(a.y) + (r + i) * a.ld_out, u, a.c, g, j);
            }
        }
        __syncwarp();
        if (lane == 0 && r + 2 * hop < a.rows) w.fetch(from, k, r + 2 * hop);
    }
    linger(w.abort);
    if (!a.parts) return;
    // the sums of a warp's rows at a time, then of the block's warps
    float* sums = reinterpret_cast<float*>(smem + (w.head() + 127) / 128 * 128);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < C::J; ++j)
#pragma unroll
        for (int q = 0; q < P; ++q) {
            float2 x = dg[j * P + q], y = db[j * P + q];
#pragma unroll
            for (int o = W; o < 32; o <<= 1) {
                x.x += __shfl_xor_sync(0xffffffffu, x.x, o), x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
                y.x += __shfl_xor_sync(0xffffffffu, y.x, o), y.y += __shfl_xor_sync(0xffffffffu, y.y, o);
            }
            const int i = C::col(j, g) + 2 * q, m = i + C::MATE;
            float* to = sums + (threadIdx.x >> 5) * 2 * a.c;
            if (sub == 0 && i < a.c) to[i] = x.x, to[a.c + i] = y.x;
            if (sub == 0 && m < a.c) to[m] = x.y, to[a.c + m] = y.y;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.c; i += kBlock) {
        float t = 0.f;
        for (int k = 0; k < kBlock / 32; ++k) t += sums[k * 2 * a.c + i];
        a.parts[(int64_t)blockIdx.x * 2 * a.c + i] = t;
    }
}

// Rows of more columns than a block holds: a block per row, which it reads once per step (from L2 but for the first).
template <class T>
__global__ void __launch_bounds__(kWide) ln_fwd_wide_kernel(LnArgs a)
{
    __shared__ float red[32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ld_in;
        const T* res = a.res ? static_cast<const T*>(a.res) + r * a.ld_in : nullptr;
        auto at = [&](int i) { return res ? elem_f(x[i]) + elem_f(res[i]) : elem_f(x[i]); };
        float s = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kWide) s += at(i);
        const float mean = block_sum(s, red) / a.c;
        s = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kWide) {
            const float d = at(i) - mean;
            s = fmaf(d, d, s);
        }
        const float inv = 1.f / sqrtf(block_sum(s, red) / a.c + a.eps);
        for (int i = threadIdx.x; i < a.c; i += kWide) {
            const float v = at(i), h = (v - mean) * inv;
            if (a.sum) static_cast<T*>(a.sum)[r * a.ld_out + i] = elem_from<T>(v);
            static_cast<T*>(a.y)[r * a.ld_out + i] = elem_from<T>(fmaf(h, a.gamma ? a.gamma[i] : 1.f,
                                                                        a.beta ? a.beta[i] : 0.f));
        }
        if (threadIdx.x == 0 && a.mean) {
            a.mean[r] = mean;
            a.invstd[r] = inv;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kWide) ln_bwd_wide_kernel(LnArgs a)
{
    __shared__ float red[32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ld_in;
        const T* dy = static_cast<const T*>(a.dy) + r * a.ld_in;
        const float mean = a.mean[r], inv = a.invstd[r];
        float s0 = 0.f, s1 = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kWide) {
            const float g = elem_f(dy[i]) * (a.gamma ? a.gamma[i] : 1.f);
            s0 += g;
            s1 = fmaf(g, (elem_f(x[i]) - mean) * inv, s1);
        }
        s0 = block_sum(s0, red) / a.c;
        s1 = block_sum(s1, red) / a.c;
        for (int i = threadIdx.x; i < a.c; i += kWide) {
            const float g = elem_f(dy[i]) * (a.gamma ? a.gamma[i] : 1.f), h = (elem_f(x[i]) - mean) * inv;
            float d = inv * (g - s0 - h * s1);
            if (a.res) d += elem_f(static_cast<const T*>(a.res)[r * a.ld_in + i]);
            static_cast<T*>(a.y)[r * a.ld_out + i] = elem_from<T>(d);
        }
    }
}

// The column sums of such rows: a block of columns over a part of the rows.
template <class T>
__global__ void __launch_bounds__(kWide) ln_params_wide_kernel(LnArgs a)
{
    grid_dependency_trigger();
    const int i = blockIdx.x * kWide + threadIdx.x;
    if (i >= a.c) return;
    float dg = 0.f, db = 0.f;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float d = elem_f(static_cast<const T*>(a.dy)[r * a.ld_in + i]);
        const float h = (elem_f(static_cast<const T*>(a.x)[r * a.ld_in + i]) - a.mean[r]) * a.invstd[r];
        dg = fmaf(d, h, dg);
        db += d;
    }
    a.parts[(int64_t)blockIdx.y * 2 * a.c + i] = dg;
    a.parts[((int64_t)blockIdx.y * 2 + 1) * a.c + i] = db;
}

// Sums of the parts, 32 columns a block: 32 threads per column, each every 32nd part.
__global__ void __launch_bounds__(kSumThreads) ln_params_sum_kernel(const float* parts, int nparts, int c, float* dgamma,
                                                                   float* dbeta)
{
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;  // of 2*c
    grid_dependency_wait();
    float s = 0.f;
    if (i < 2 * c) {
#pragma unroll 8
        for (int p = w; p < nparts; p += 32) s += parts[(int64_t)p * 2 * c + i];
    }
    red[w][lane] = s;
    __syncthreads();
    s = warp_sum(red[lane][w]);
    const int o = blockIdx.x * 32 + w;
    if (lane == 0 && o < 2 * c) (o < c ? dgamma : dbeta - c)[o] = s;
}

int check(const dbl_ln_shape* s, const char* what)
{
    if (!s || s->rows < 0 || s->c <= 0) return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0 or c <= 0", what);
    if (s->c > kMaxColumns) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^30 columns or more", what);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", what);
    if ((s->ld_in && s->ld_in < s->c) || (s->ld_out && s->ld_out < s->c))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", what);
    if (!(s->eps >= 0.f) || isinf(s->eps)) return set_error(DBL_ERR_INVALID, "%s: eps must be finite and >= 0", what);
    return DBL_OK;
}

LnArgs args(const dbl_ln_shape* s)
{
    LnArgs a = {};
    a.rows = s->rows;
    a.c = s->c;
    a.eps = s->eps;
    a.ld_in = s->ld_in ? s->ld_in : s->c;
    a.ld_out = s->ld_out ? s->ld_out : s->c;
    return a;
}

// Whether every row of every tensor starts and ends at a multiple of 16 bytes.
bool vec_of(const LnArgs& a, size_t e)
{
    return a.c * e % 16 == 0 && a.ld_in * e % 16 == 0 && a.ld_out * e % 16 == 0 && aligned16(a.x) && aligned16(a.res) &&
           aligned16(a.dy) && aligned16(a.sum) && aligned16(a.y) && aligned16(a.gamma) && aligned16(a.beta);
}

// Groups, blocks and shared memory for c columns of a row, n to a thread, `tensors` rows to read, `resident` threads on
// an SM and `split` blocks of them to a row.
struct Plan {
    int threads, teams;  // of a block; blocks, or clusters of them
    size_t smem;
    int split;           // blocks of a cluster
};
Plan plan_of(LnArgs& a, int n, int c, int tensors, int resident, int split, size_t e)
{
    Plan p;
    a.group = ((c + n - 1) / n + 31) / 32 * 32;
    const int groups = std::max(1, kBlock / a.group);
    p.threads = a.group * groups;
    p.split = split;
    const int on_sm = std::max(1, resident / p.threads);
    a.slot = (int)((c * e + 16 + 127) / 128 * 128);
    a.depth = (int)std::min<size_t>(kMaxDepth, std::max<size_t>(2, kRingBytes / on_sm / ((size_t)groups * tensors * a.slot)));
    p.smem = (Groups<float, true, 1>::head(p.threads / 32) + 127) / 128 * 128 +
             std::max((size_t)groups * a.depth * tensors * a.slot, groups > 1 ? (size_t)groups * 2 * c * sizeof(float) : 0);
    p.teams = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + groups - 1) / groups, (int64_t)on_sm * sm_count() / split));
    return p;
}

// (100000 x 64 in bf16 with the residual: forward 17.5 us, backward 21; a row to a warp 36 and 46.)
bool is_short(const LnArgs& a) { return a.c <= kShort && a.ld_in == a.c; }
int lanes_of(const LnArgs& a) { return a.c <= 64 ? 8 : a.c <= 128 ? 16 : 32; }

// Short rows: as many to a place as fill an SM's shared memory with what is on its way of `tensors`, but no more than leave
// every warp some.
Plan short_plan(LnArgs& a, int tensors, int there, int on_sm, size_t e)
{
    const int at_once = 32 / lanes_of(a), warps = kBlock / 32;
    const size_t room = kRingBytes / on_sm / (warps * 2 * tensors) - 160;  // of a place, for one tensor
    const int64_t even = (a.rows + (int64_t)on_sm * sm_count() * warps * at_once - 1) / ((int64_t)on_sm * sm_count() * warps * at_once);
    const int64_t times = std::max<int64_t>(1, std::min<int64_t>({even, (int64_t)(room / (a.c * e * at_once)), 32 / at_once}));
    a.batch = (int)times * at_once;
    a.slot = (int)((a.batch * a.c * e + 32 + 127) / 128 * 128);
    Plan p;
    p.threads = kBlock;
    p.split = 1;
    p.smem = (Batches<float, true, 32, 1>::head() + 127) / 128 * 128 +
             std::max((size_t)warps * 2 * there * a.slot, (size_t)warps * 2 * a.c * sizeof(float));
    p.teams = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + (int64_t)a.batch * warps - 1) / ((int64_t)a.batch * warps), (int64_t)on_sm * sm_count()));
    return p;
}

// Rows of up to 16 columns for each of a group's threads, wider ones by clusters of such blocks (4000 x 16000 in bf16:
// forward 110 us, 136 with 32 columns to a thread; backward 138, 192 with 32, which spill; clusters of four blocks of half
// the columns 210 and 208: the exchange takes longer).
bool held(const LnArgs& a) { return a.c <= 16 * kMaxGroup * std::min(kMaxSplit, std::max(1, max_cluster())); }
Plan plan_wide(LnArgs& a, int tensors, size_t e)
{
    const int S = (a.c + 16 * kMaxGroup - 1) / (16 * kMaxGroup);
    a.part = ((a.c + S - 1) / S + 15) / 16 * 16;  // whole 16-byte units; the last block's may be fewer
    Plan p = plan_of(a, 16, std::min(a.part, a.c), tensors, kMaxGroup, S, e);
    int dev = 0;
    if (S > 1 && cudaGetDevice(&dev) == cudaSuccess) {
        // no more clusters than the device holds (15 of seven blocks, not 21: backward of 700 x 50000 122 and 167 us), by
        // one kernel for all, each of which takes an SM's registers
        constexpr auto kernel = ln_bwd_kernel<act_t, true, false, 16, kMaxGroup, 1, true>;
        const int fit = allow_launch<kernel>(kMaxSmem, false, "layer_norm") == DBL_OK ? clusters_held<kernel>(dev, S, kMaxGroup, kMaxSmem) : 0;
        if (fit) p.teams = std::min(p.teams, fit);
    } else if (S > 1) {
        (void)cudaGetLastError();
    }
    return p;
}

// The backward pass's blocks or clusters, each of which leaves a row of partial column sums.  By the sizes and by what the
// device holds, which the workspace's size goes by too: the pointers' alignment and which are given have no part in it.
Plan bwd_plan(LnArgs& a, size_t e)
{
    if (!held(a)) return {kWide, (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + 15) / 16, 64)), 0, 1};
    if (is_short(a)) return short_plan(a, 3, a.res ? 3 : 2, kShortBwd, e);
    if (a.c <= 16 * kBlock) return plan_of(a, 16, a.c, 3, 2 * kBlock, 1, e);
    return plan_wide(a, 3, e);
}

template <auto KERNEL>
int launch(const LnArgs& a, const Plan& p, cudaStream_t st, const char* what)
{
    const int rc = allow_launch<KERNEL>(kMaxSmem, false, what);
    if (rc != DBL_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = p.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(p.teams * p.split));
    cfg.blockDim = dim3(p.threads);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = p.split > 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, KERNEL, a);
    const int ran = launch_check(what);
    return err == cudaSuccess ? ran : cuda_check(err, what);
}

template <class T, bool VEC, int N, int THREADS, int BLOCKS, bool SPLIT>
int run_fwd_held(const LnArgs& a, const Plan& p, cudaStream_t st, const char* what)
{
    if (VEC && a.c == a.group * N * p.split) return launch<ln_fwd_kernel<T, VEC, VEC, N, THREADS, BLOCKS, SPLIT>>(a, p, st, what);
    return launch<ln_fwd_kernel<T, VEC, false, N, THREADS, BLOCKS, SPLIT>>(a, p, st, what);
}

template <class T, bool VEC>
int run_fwd(LnArgs a, cudaStream_t st)
{
    const char* what = "layer_norm_fwd";
    constexpr size_t e = sizeof(T);
    if (held(a)) {
        constexpr int B16 = VEC ? 3 : 2;
        if (is_short(a)) {
            const Plan p = short_plan(a, a.res ? 2 : 1, a.res ? 2 : 1, kShortFwd, e);
            if (a.c <= 64) return launch<ln_fwd_short_kernel<T, VEC, 8>>(a, p, st, what);
            if (a.c <= 128) return launch<ln_fwd_short_kernel<T, VEC, 16>>(a, p, st, what);
            return launch<ln_fwd_short_kernel<T, VEC, 32>>(a, p, st, what);
        }
        if (a.c <= 16 * kBlock) {
            const Plan p = plan_of(a, 16, a.c, 2, kBlock * B16, 1, e);
            return run_fwd_held<T, VEC, 16, kBlock, B16, false>(a, p, st, what);
        }
        const Plan p = plan_wide(a, 2, e);
        if (p.split == 1) return run_fwd_held<T, VEC, 16, kMaxGroup, 1, false>(a, p, st, what);
        return run_fwd_held<T, VEC, 16, kMaxGroup, 1, true>(a, p, st, what);
    }
    ln_fwd_wide_kernel<T><<<(int)std::min<int64_t>(a.rows, 1 << 20), kWide, 0, st>>>(a);
    return launch_check(what);
}

template <class T, bool VEC, int N, int THREADS, int BLOCKS, bool SPLIT>
int run_bwd_held(const LnArgs& a, const Plan& p, cudaStream_t st, const char* what)
{
    if (VEC && a.c == a.group * N * p.split) return launch<ln_bwd_kernel<T, VEC, VEC, N, THREADS, BLOCKS, SPLIT>>(a, p, st, what);
    return launch<ln_bwd_kernel<T, VEC, false, N, THREADS, BLOCKS, SPLIT>>(a, p, st, what);
}

template <class T, bool VEC>
int run_bwd(const LnArgs& a, const Plan& p, cudaStream_t st)
{
    const char* what = "layer_norm_bwd";
    if (a.rows == 0) return DBL_OK;
    if (held(a)) {
        if (is_short(a)) {
            if (a.c <= 64) return launch<ln_bwd_short_kernel<T, VEC, 8>>(a, p, st, what);
            if (a.c <= 128) return launch<ln_bwd_short_kernel<T, VEC, 16>>(a, p, st, what);
            return launch<ln_bwd_short_kernel<T, VEC, 32>>(a, p, st, what);
        }
        if (a.c <= 16 * kBlock) return run_bwd_held<T, VEC, 16, kBlock, 2, false>(a, p, st, what);
        if (p.split == 1) return run_bwd_held<T, VEC, 16, kMaxGroup, 1, false>(a, p, st, what);
        return run_bwd_held<T, VEC, 16, kMaxGroup, 1, true>(a, p, st, what);
    }
    ln_bwd_wide_kernel<T><<<(int)std::min<int64_t>(a.rows, 1 << 20), kWide, 0, st>>>(a);
    const int rc = launch_check(what);
    if (rc != DBL_OK || !a.parts) return rc;
    ln_params_wide_kernel<T><<<dim3((a.c + kWide - 1) / kWide, p.teams), kWide, 0, st>>>(a);
    return launch_check(what);
}

}  // namespace

namespace dbl {

static int read_word(int* status) { return status_read(g_ln_status, status); }
static int clear_word() { return status_clear(g_ln_status); }
StatusWord ln_status_word() { return {read_word, clear_word}; }

}  // namespace dbl

extern "C" {

int dbl_layer_norm_fwd(const dbl_ln_shape* s, const void* x, const void* res, const float* gamma, const float* beta,
                       void* sum, void* y, float* save_mean, float* save_invstd, void* stream)
{
    int rc = check(s, "layer_norm_fwd");
    if (rc != DBL_OK) return rc;
    if (!x || !y) return set_error(DBL_ERR_INVALID, "layer_norm_fwd: x and y must not be NULL");
    if (!save_mean != !save_invstd) return set_error(DBL_ERR_INVALID, "layer_norm_fwd: save_mean and save_invstd go together");
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(x, e) || !aligned_to(res, e) || !aligned_to(sum, e) || !aligned_to(y, e) || !aligned_to(gamma, 4) ||
        !aligned_to(beta, 4) || !aligned_to(save_mean, 4) || !aligned_to(save_invstd, 4))
        return set_error(DBL_ERR_INVALID, "layer_norm_fwd: a pointer is not aligned to its element type");
    if (s->rows == 0) return DBL_OK;
    LnArgs a = args(s);
    a.x = x, a.res = res, a.gamma = gamma, a.beta = beta, a.sum = sum, a.y = y, a.mean = save_mean, a.invstd = save_invstd;
    cudaStream_t st = as_stream(stream);
    if (s->dtype == DBL_F32) return vec_of(a, e) ? run_fwd<float, true>(a, st) : run_fwd<float, false>(a, st);
    return vec_of(a, e) ? run_fwd<act_t, true>(a, st) : run_fwd<act_t, false>(a, st);
}

size_t dbl_layer_norm_workspace_bytes(const dbl_ln_shape* s)
{
    if (check(s, "layer_norm_workspace_bytes") != DBL_OK) return 0;
    LnArgs a = args(s);
    return (size_t)bwd_plan(a, elem_bytes(s->dtype)).teams * 2 * s->c * sizeof(float);
}

int dbl_layer_norm_bwd(const dbl_ln_shape* s, const void* dy, const void* dskip, const void* x, const float* gamma,
                       const float* save_mean, const float* save_invstd, void* dx, float* dgamma, float* dbeta,
                       void* ws, size_t ws_bytes, void* stream)
{
    int rc = check(s, "layer_norm_bwd");
    if (rc != DBL_OK) return rc;
    if (!dy || !x || !save_mean || !save_invstd || !dx)
        return set_error(DBL_ERR_INVALID, "layer_norm_bwd: dy, x, save_mean, save_invstd and dx must not be NULL");
    if (!dgamma != !dbeta) return set_error(DBL_ERR_INVALID, "layer_norm_bwd: dgamma and dbeta go together");
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(dy, e) || !aligned_to(dskip, e) || !aligned_to(x, e) || !aligned_to(dx, e) || !aligned_to(gamma, 4) ||
        !aligned_to(save_mean, 4) || !aligned_to(save_invstd, 4) || !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4))
        return set_error(DBL_ERR_INVALID, "layer_norm_bwd: a pointer is not aligned to its element type");
    LnArgs a = args(s);
    a.x = x, a.res = dskip, a.dy = dy, a.gamma = gamma, a.y = dx, a.parts = dgamma ? static_cast<float*>(ws) : nullptr;
    a.mean = const_cast<float*>(save_mean), a.invstd = const_cast<float*>(save_invstd);
    const Plan p = bwd_plan(a, e);
    if (dgamma) {
        if (!ws || ws_bytes < (size_t)p.teams * 2 * s->c * sizeof(float))
            return set_error(DBL_ERR_WORKSPACE, "layer_norm_bwd: workspace too small");
        if (!aligned16(ws)) return set_error(DBL_ERR_INVALID, "layer_norm_bwd: workspace must be 16-byte aligned");
    }
    cudaStream_t st = as_stream(stream);
    if (s->dtype == DBL_F32)
        rc = vec_of(a, e) ? run_bwd<float, true>(a, p, st) : run_bwd<float, false>(a, p, st);
    else
        rc = vec_of(a, e) ? run_bwd<act_t, true>(a, p, st) : run_bwd<act_t, false>(a, p, st);
    if (rc != DBL_OK || !dgamma) return rc;
    // its launch overlaps the end of the kernel before it
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)((2 * (int64_t)s->c + 31) / 32));
    cfg.blockDim = dim3(kSumThreads);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, ln_params_sum_kernel, (const float*)a.parts, s->rows ? p.teams : 0, s->c,
                                               dgamma, dbeta);
    rc = launch_check("layer_norm_bwd sums");
    return err == cudaSuccess ? rc : cuda_check(err, "layer_norm_bwd sums");
}

}  // extern "C"
