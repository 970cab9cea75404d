// scan.cu -- gated linear recurrence along a sequence, h_i = a_i*h_{i-1} + (1 - a_i)*x_i with a = 1/(1 + exp(-gate)),
// forward and backward.
//
// Steps compose: two of them, or two runs of them, with (product of the gates, state from zero) = (p1, h1) and (p2, h2)
// are one with (p1*p2, p2*h1 + h2).  So a sequence is cut into runs that are scanned at the same time from zero, their
// pairs are combined, and every state is its run's plus its product times the state before the run.  Backward the same
// with G_i = dh_i + a_{i+1}*G_{i+1}; dx = (1 - a)*G, dgate = G*(h_{i-1} - x)*a*(1 - a).  1 - a is taken of exp, not by
// subtraction.  States, products and sums are fp32; a state per DBL_SCAN_CHUNK steps is kept for the backward pass in
// fp32, the outputs are rounded once.
//
// Bound by memory where there are sequences enough, otherwise by the chain of parts: exchange of the pairs, state for
// the next part.  On a GB300 that copies 6.78 TB/s, bf16 but where said: backward of 8 x 8192 x 1024 124 us = 5.4 TB/s;
// forward of 1 x 65536 x 512 63 us = 3.2 TB/s, 22 parts one after another at 2.8 us each; of 185 x 196 x 256 in fp16 24 us =
// 2.4 TB/s, 740 blocks in three rounds; one token of 64 x 512 4.5 us, the launch; backward of 12 x 3001 x 393 with
// lengths 73 us = 1.4 TB/s (rows that begin anywhere: 190 instructions a step of 64 channels, 77 where TMA brings them).
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kThreads = 256;
constexpr int kChunk = DBL_SCAN_CHUNK;
constexpr int kShort = 16;        // steps up to which a thread takes its channels' whole sequence
constexpr int kMaxCluster = 16;

struct ScanArgs {
    const void *x, *gate, *dh;
    const float* h0;      // backward: dh_last
    const int32_t* lengths;
    void *h;              // backward: dx
    void *dgate;
    float *last;          // backward: dh0
    float *states;
    int64_t ld_x, ld_h;
    int n, t, c;
    int groups;           // blocks of channels (2 * lanes each) of a sequence
    bool pairs;           // channels 2j and 2j + 1 exist and are aligned as a pair in every row
};

__device__ __forceinline__ float exp2_ftz(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float rcp_ftz(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float min_nan(float x, float y)
{
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}

// A product of gates, none of which is 0, held above 0 where fp32 would round it there: with an infinite state it has to
// give infinity, as the steps do one after another, not NaN.  (A finite state times 2^-149 is 2^-21 at the most.)
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float2 at_least(float2 p, float2 least)
{
    float2 q;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(q.x) : "f"(p.x), "f"(least.x));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(q.y) : "f"(p.y), "f"(least.y));
    return q;
}
__device__ __forceinline__ bool finite2(float2 v) { return fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY; }

// a = sigma(z) and na = 1 - a of two channels, neither by subtraction: a = 1/(1 + e), na = e*a with e = exp(-z), held to
// 2^126 so that no product is infinity times 0 (a is 2^-126 at the least, for z < -87).  z = +inf gives 1 and 0 exactly;
// e below 2^-126 counts as 0 (z > 87).  The exponent -z*log2(e) is one rounded product, so e is off by up to
// (1.5*|z| + 4)*2^-24 of itself, and so is the smaller one of a and na; the larger one by a few units of 2^-24.  (The
// product's remainder would cost two instructions and more a channel; what 16-bit outputs are rounded by is 2^-9.)
__device__ __forceinline__ void gates2(float2 z, float2& a, float2& na)
{
    const float2 t = __fmul2_rn(z, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    const float2 e = make_float2(exp2_ftz(min_nan(t.x, 126.f)), exp2_ftz(min_nan(t.y, 126.f)));
    const float2 d = __fadd2_rn(e, make_float2(1.f, 1.f));
    a = make_float2(rcp_ftz(d.x), rcp_ftz(d.y));
    na = __fmul2_rn(e, a);
}

__device__ __forceinline__ int length_of(const ScanArgs& a, int64_t b)
{
    return a.lengths ? min(max(a.lengths[b], 0), a.t) : a.t;
}

// Two neighbouring channels of one step: as stored, as floats.  VEC: one aligned access for both (an even number of
// channels); otherwise the second may not exist (`two`).
template <class T>
struct Pair;
template <>
struct Pair<float> {
    typedef float2 raw;
    static __device__ __forceinline__ float2 floats(raw r) { return r; }
    static __device__ __forceinline__ raw pack(float2 v) { return v; }
    static __device__ __forceinline__ raw join(float a, float b) { return make_float2(a, b); }
    static __device__ __forceinline__ float first(raw r) { return r.x; }
    static __device__ __forceinline__ float second(raw r) { return r.y; }
};
template <>
struct Pair<act_t> {
    typedef uint32_t raw;
    static __device__ __forceinline__ float2 floats(raw r) { return act::unpack2_u32(r); }
    static __device__ __forceinline__ raw pack(float2 v) { return act::pack2_u32(v.x, v.y); }
    static __device__ __forceinline__ raw join(act_t a, act_t b)
    {
        return (uint32_t) * reinterpret_cast<uint16_t*>(&a) | (uint32_t) * reinterpret_cast<uint16_t*>(&b) << 16;
    }
    static __device__ __forceinline__ act_t first(raw r)
    {
        const uint16_t v = (uint16_t)r;
        return *reinterpret_cast<const act_t*>(&v);
    }
    static __device__ __forceinline__ act_t second(raw r)
    {
        const uint16_t v = (uint16_t)(r >> 16);
        return *reinterpret_cast<const act_t*>(&v);
    }
};

template <class T, bool VEC>
__device__ __forceinline__ typename Pair<T>::raw ld_pair(const T* p, bool two)
{
    if constexpr (VEC) return *reinterpret_cast<const typename Pair<T>::raw*>(p);
    return Pair<T>::join(p[0], two ? p[1] : elem_from<T>(0.f));
}

template <class T, bool VEC>
__device__ __forceinline__ void st_pair(T* p, float2 v, bool two)
{
    const typename Pair<T>::raw r = Pair<T>::pack(v);
    if constexpr (VEC) {
        *reinterpret_cast<typename Pair<T>::raw*>(p) = r;
    } else {
        p[0] = Pair<T>::first(r);
        if (two) p[1] = Pair<T>::second(r);
    }
}

template <class T>
__device__ __forceinline__ void st_any(T* p, float2 v, bool two, bool pairs)
{
    if (pairs)
        st_pair<T, true>(p, v, two);
    else
        st_pair<T, false>(p, v, two);
}

__device__ __forceinline__ float2 ld_state(const float* p, bool two)
{
    return p ? make_float2(p[0], two ? p[1] : 0.f) : make_float2(0.f, 0.f);
}

__device__ __forceinline__ void st_state(float* p, float2 v, bool two)
{
    p[0] = v.x;
    if (two) p[1] = v.y;
}

// Short sequences (single tokens among them): a thread takes two channels through all steps.
template <class T, bool VEC>
__global__ void __launch_bounds__(128) scan_fwd_short_kernel(ScanArgs a)
{
    const int pairs = (a.c + 1) / 2;
    const int64_t id = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (id >= (int64_t)a.n * pairs) return;
    const int64_t b = id / pairs;
    const int ch = 2 * (int)(id - b * pairs), len = length_of(a, b);
    const bool two = ch + 1 < a.c;
    const T* x = static_cast<const T*>(a.x) + b * a.t * a.ld_x + ch;
    const T* z = static_cast<const T*>(a.gate) + b * a.t * a.ld_x + ch;
    T* out = static_cast<T*>(a.h) + b * a.t * a.ld_h + ch;
    float2 h = ld_state(a.h0 ? a.h0 + b * a.c + ch : nullptr, two);
    if (a.states) st_state(a.states + b * a.c + ch, h, two);  // one chunk
#pragma unroll 4
    for (int i = 0; i < a.t; ++i) {
        float2 o = make_float2(0.f, 0.f);
        if (i < len) {
            float2 s, r;
            gates2(Pair<T>::floats(ld_pair<T, VEC>(z + i * a.ld_x, two)), s, r);
            o = h = __ffma2_rn(s, h, __fmul2_rn(r, Pair<T>::floats(ld_pair<T, VEC>(x + i * a.ld_x, two))));
        }
        st_pair<T, VEC>(out + i * a.ld_h, o, two);
    }
    if (a.last) st_state(a.last + b * a.c + ch, h, two);
}

template <class T, bool VEC>
__global__ void __launch_bounds__(128) scan_bwd_short_kernel(ScanArgs a)
{
    const int pairs = (a.c + 1) / 2;
    const int64_t id = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (id >= (int64_t)a.n * pairs) return;
    const int64_t b = id / pairs;
    const int ch = 2 * (int)(id - b * pairs), len = length_of(a, b);
    const bool two = ch + 1 < a.c;
    const T* x = static_cast<const T*>(a.x) + b * a.t * a.ld_x + ch;
    const T* z = static_cast<const T*>(a.gate) + b * a.t * a.ld_x + ch;
    const T* dh = static_cast<const T*>(a.dh) + b * a.t * a.ld_h + ch;
    T* dx = static_cast<T*>(a.h) + b * a.t * a.ld_x + ch;
    T* dz = static_cast<T*>(a.dgate) + b * a.t * a.ld_x + ch;
    float2 q = ld_state(a.h0 ? a.h0 + b * a.c + ch : nullptr, two);
    float2 h = ld_state(a.states + b * a.c + ch, two);
    float2 s[kShort], r[kShort], d[kShort];
#pragma unroll
    for (int i = 0; i < kShort; ++i) {
        s[i] = make_float2(1.f, 1.f), r[i] = d[i] = make_float2(0.f, 0.f);
        if (i < len) {
            gates2(Pair<T>::floats(ld_pair<T, VEC>(z + i * a.ld_x, two)), s[i], r[i]);
            const float2 v = Pair<T>::floats(ld_pair<T, VEC>(x + i * a.ld_x, two));
            d[i] = make_float2(h.x - v.x, h.y - v.y);
            h = __ffma2_rn(s[i], h, __fmul2_rn(r[i], v));
        }
    }
#pragma unroll
    for (int i = kShort - 1; i >= 0; --i) {
        if (i >= a.t) continue;
        float2 vx = make_float2(0.f, 0.f), vz = vx;
        if (i < len) {
            const float2 g = __fadd2_rn(Pair<T>::floats(ld_pair<T, VEC>(dh + i * a.ld_h, two)), q);
            vx = __fmul2_rn(r[i], g);
            q = __fmul2_rn(s[i], g);
            vz = __fmul2_rn(__fmul2_rn(vx, s[i]), d[i]);
        }
        st_pair<T, VEC>(dx + i * a.ld_x, vx, two);
        st_pair<T, VEC>(dz + i * a.ld_x, vz, two);
    }
    if (a.last) st_state(a.last + b * a.c + ch, q, two);
}

// ---------------------------------------------------------------------------- staging
// A warp's consecutive steps of its channels, copied ahead into shared memory of the warp's own, so that no other
// warp is waited for.  ALIGNED, where every row starts at a multiple of 16 bytes: one tensor copy (TMA) of a box of
// channels and steps, clipped at the tensor's ends, and the outputs go back the same way.  Otherwise the lanes copy the
// rows in chunks of 16 bytes (a bulk copy for each row, which a lane at a time issues, took 2750 cycles of a warp for
// 24 rows where these take 1600; words put together from two lanes' halves cost more than two stores of 16 bits).
__device__ __forceinline__ void tma_store_3d(const void* tmap, const void* src, int32_t c0, int32_t c1, int32_t c2)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(tmap)),
                 "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, uintptr_t src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

constexpr int kBlock = 8;  // steps worked on at once

template <class T, bool ALIGNED, int LANES, int R>
struct Stage {
    typedef typename Pair<T>::raw raw;
    static constexpr int SUBS = 32 / LANES, ROWS = R * SUBS;  // threads one after another in a warp, steps of a warp
    static constexpr int ROW_BYTES = 2 * LANES * (int)sizeof(T), E = 16 / (int)sizeof(T);
    static constexpr int PITCH = ROW_BYTES + (ALIGNED ? 0 : 16);
    static constexpr int BYTES = (ROWS * PITCH + 127) / 128 * 128;  // one tensor, one warp

    // Not ALIGNED: rows [0, n) of the warp, row 0 at g (its first channel), ch channels from there to the row's end, of a
    // tensor [lo, hi): in chunks of 16 bytes, a row from the boundary at or before its first element to the one at or
    // after its last.  By elements where that would leave the tensor, or pass 32 bits.
    static __device__ __forceinline__ void load(char* dst, const T* g, int64_t ld, int n, int ch, uintptr_t lo, uintptr_t hi)
    {
        constexpr int CHUNKS = PITCH / 16, COPIES = (ROWS * CHUNKS + 31) / 32;
        const int lane = threadIdx.x & 31, seg = min(ch, 2 * LANES) * (int)sizeof(T);
        const uintptr_t p = reinterpret_cast<uintptr_t>(g), base = p & ~(uintptr_t)15;
        if (base >= lo && ((reinterpret_cast<uintptr_t>(g + (n - 1) * ld) + seg + 15) & ~(uintptr_t)15) <= hi && ld < (1 << 24)) {
            const int b = (int)(p & 15), pitch = (int)ld * (int)sizeof(T);
            const uint32_t to = smem_u32(dst);
#pragma unroll
            for (int j = 0; j < COPIES; ++j) {
                const int q = lane + 32 * j, row = q / CHUNKS, at = q % CHUNKS * 16, off = b + row * pitch;
                if (row < n && at < (off & 15) + seg) cp_async16(to + row * PITCH + at, base + (uint32_t)((off & ~15) + at));
            }
        } else {
            for (int r = 0; r < n; ++r, g += ld, dst += PITCH)
                for (int i = lane; i < min(ch, 2 * LANES); i += 32) reinterpret_cast<T*>(dst)[offset(g) + i] = g[i];
        }
    }

    // rows [n, ROWS): a word of `v` everywhere
    static __device__ __forceinline__ void fill(char* st, int n, uint32_t v)
    {
        for (int w = n * (PITCH / 4) + (threadIdx.x & 31); w < ROWS * (PITCH / 4); w += 32) reinterpret_cast<uint32_t*>(st)[w] = v;
    }

    // elements from the 16-byte boundary to the row's first; of the rows after it, with m = ld % E
    static __device__ __forceinline__ int offset(const T* row) { return ALIGNED ? 0 : (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)); }
    static __device__ __forceinline__ int offset(int first, int m, int i) { return ALIGNED ? 0 : (first + m * i) & (E - 1); }

    // the two channels of this thread's row, which begins `off` elements in
    static __device__ __forceinline__ float2 pair(const char* row, int lane, int off)
    {
        if constexpr (ALIGNED) {
            return Pair<T>::floats(reinterpret_cast<const raw*>(row)[lane]);
        } else if constexpr (sizeof(T) == 4) {
            const float* p = reinterpret_cast<const float*>(row) + off + 2 * lane;
            return make_float2(p[0], p[1]);
        } else {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(row) + (off >> 1) + lane;
            return Pair<T>::floats(off & 1 ? __funnelshift_r(w[0], w[1], 16) : w[0]);
        }
    }
    static __device__ __forceinline__ void put(char* row, int lane, float2 v) { reinterpret_cast<raw*>(row)[lane] = Pair<T>::pack(v); }
};

// A pair of +infinity: a gate that is open, 1 and 0 exactly.
template <class T>
__device__ __forceinline__ constexpr uint32_t open_gate()
{
    return sizeof(T) == 4 ? 0x7f800000u : act::kF16 ? 0x7c007c00u : 0x7f807f80u;
}

// What a block of the kernels below works on.
struct Place {
    int S, rank, warp, lane, sub, subs, wsub, ch0, ch, len, chunks;
    int64_t b;
    bool one, two;
    template <int LANES>
    __device__ __forceinline__ void set(const ScanArgs& a)
    {
        uint32_t n;
        asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
        S = (int)n, rank = (int)cluster_ctarank();
        warp = threadIdx.x >> 5, lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, subs = blockDim.x / LANES;
        wsub = sub % (32 / LANES);
        const int64_t col = blockIdx.x / S;
        b = col / a.groups;
        ch0 = (int)(col - b * a.groups) * LANES * 2, ch = ch0 + 2 * lane;
        one = ch < a.c, two = ch + 1 < a.c;
        len = length_of(a, b);
        chunks = (a.t + kChunk - 1) / kChunk;
    }
};

__device__ __forceinline__ float2 step2(float4 pair, float2 h) { return __ffma2_rn(make_float2(pair.x, pair.y), h, make_float2(pair.z, pair.w)); }

// Exchange between the blocks of a cluster.  Stores to another block's shared memory that count themselves on that
// block's mbarrier, so that nobody waits but for the data: a barrier of the cluster would also wait for the blocks'
// stores to global memory.  Each block sends its pair to those that come after it in the scan's direction, and the last
// one sends the state for the next part to all, which they wait for before they send a pair.  Two places of each by
// turns: who has the state of part n knows that the last block has every block's pair of part n-1, which a block sends
// when it has read what it was sent of part n-2.
__device__ int g_scan_status;

struct Links {
    uint64_t pairs[2], carry[2];
    uint64_t full[kThreads / 32][2];  // a warp's stages
    int abort;
};

// Tensor maps of what is read and written, [n][t][c] each (ALIGNED).
struct Maps {
    CUtensorMap x, z, dh, h, dz;  // h: dx in the backward pass
};

__device__ __forceinline__ void link_wait(uint64_t* bar, uint32_t parity, int* abort) { bounded_wait(bar, parity, abort, &g_scan_status); }

// Barriers ready, and every block's shared memory there before it is written from afar.
__device__ __forceinline__ void links_init(Links& l, int S)
{
    if (threadIdx.x == 0) {
        for (int k = 0; k < 2; ++k) {
            mbar_init(&l.pairs[k], 1);
            mbar_init(&l.carry[k], 1);
            for (int i = 0; i < (int)blockDim.x / 32; ++i) mbar_init(&l.full[i][k], 1);
        }
        l.abort = 0;
        fence_mbar_init();
    }
    if (S > 1)
        cluster_sync_all();
    else
        __syncthreads();
}

// Longer sequences.  A cluster takes one block of 2*LANES channels of a sequence, its blocks of threads consecutive
// parts of it at a time; in a block each LANES threads take R consecutive steps of all the channels, a thread two
// channels.  A thread scans its steps from a zero state and keeps, for each, that state and the product of the gates
// up to it: with the state h before them, the state after a step is state + product*h.  The threads' and the blocks'
// last pairs (product, state) are combined through shared memory, the last thread's state goes on to the cluster's
// next part.  So each element is read and written once, and the sums' order depends on the sizes, the alignment and the
// device (how many clusters it holds) alone.  Steps past
// a length are given open gates, which leave the state as it is.
template <class T, bool ALIGNED, int LANES, int R>
struct FwdSmem {
    typedef Stage<T, ALIGNED, LANES, R> St;
    typedef char Stages[2][2][St::BYTES];  // of a warp: two parts of x and gate; before this struct
    float4 agg[2][kThreads / LANES][LANES];
    float2 carry[2][LANES];
    Links links;
    alignas(16) float4 slot[1];  // [2][cluster][LANES]
};

template <class T, bool ALIGNED, int LANES, int R, int BLOCKS>
__global__ void __launch_bounds__(kThreads, BLOCKS) scan_fwd_kernel(ScanArgs a, const __grid_constant__ Maps maps)
{
    typedef FwdSmem<T, ALIGNED, LANES, R> Smem;
    typedef typename Smem::St St;
    extern __shared__ __align__(128) char smem_raw[];
    typename Smem::Stages* const stages = reinterpret_cast<typename Smem::Stages*>(smem_raw);
    Smem& sm = *reinterpret_cast<Smem*>(stages + blockDim.x / 32);
    Place w;
    w.set<LANES>(a);
    const int tile = w.subs * R, step = tile * w.S, lane = w.lane, ch = a.c - w.ch0;
    int row = w.rank * tile + w.warp * St::ROWS;  // the warp's first step
    const int64_t row0 = w.b * a.t + row;
    const T* x = static_cast<const T*>(a.x) + row0 * a.ld_x + w.ch0;
    const T* z = static_cast<const T*>(a.gate) + row0 * a.ld_x + w.ch0;
    T* out = static_cast<T*>(a.h) + row0 * a.ld_h + w.ch0;
    const int64_t hop = step * a.ld_x, hop_h = step * a.ld_h;
    char(*stage)[2][St::BYTES] = stages[w.warp];
    uint64_t* full = sm.links.full[w.warp];
    const int mx = (int)(a.ld_x % St::E), o0 = w.wsub * R;
    const uintptr_t x_lo = reinterpret_cast<uintptr_t>(a.x), z_lo = reinterpret_cast<uintptr_t>(a.gate);
    const uintptr_t x_size = (((int64_t)a.n * a.t - 1) * a.ld_x + a.c) * sizeof(T);
    auto fetch = [&](int ring, int ahead) {  // the warp's rows `ahead` parts on (0 or 1)
        const int n = min(w.len - row - ahead * step, St::ROWS);
        if (n <= 0) return;
        if constexpr (ALIGNED) {
            if ((threadIdx.x & 31) == 0) {
                bulk_wait_read();  // the output that lay in this stage
                mbar_arrive_expect_tx(&full[ring], 2 * St::ROWS * St::ROW_BYTES);
                tma_load_3d(stage[ring][0], &maps.x, &full[ring], w.ch0, row + ahead * step, (int)w.b);
                tma_load_3d(stage[ring][1], &maps.z, &full[ring], w.ch0, row + ahead * step, (int)w.b);
            }
        } else {
            St::load(stage[ring][0], x + ahead * hop, a.ld_x, n, ch, x_lo, x_lo + x_size);
            St::load(stage[ring][1], z + ahead * hop, a.ld_x, n, ch, z_lo, z_lo + x_size);
        }
    };
    links_init(sm.links, w.S);
    fetch(0, 0);
    const bool last = w.sub == w.subs - 1;
    float2 end = make_float2(0.f, 0.f);
    if (last) {
        if (w.one) end = ld_state(a.h0 ? a.h0 + w.b * a.c + w.ch : nullptr, w.two);
        sm.carry[0][lane] = end;
    }
    float* keep = a.states ? a.states + (w.b * w.chunks + (row + o0) / kChunk) * a.c + w.ch : nullptr;
    const bool keeper = a.states && (row + o0) % kChunk == 0 && w.one;
    int par = 0, turn = 0, phase = 0;
    const int parts_end = w.len > 0 ? (int)min((int64_t)a.t, ((int64_t)(w.len - 1) / step + 1) * step) : 0;
    for (int at = 0; at < parts_end; at += step, turn += par, par ^= 1) {
        if (w.S > 1 && threadIdx.x == 0) {
            mbar_arrive_expect_tx(&sm.links.pairs[par], w.rank * LANES * sizeof(float4));
            if (a.t - at > step) mbar_arrive_expect_tx(&sm.links.carry[par ^ 1], LANES * sizeof(float2));
        }
        const int live = max(0, min(w.len - row, St::ROWS));
        char *sx = stage[par][0], *sz = stage[par][1];
        if (live > 0) {
            if constexpr (ALIGNED) {
                link_wait(&full[par], phase >> par & 1, &sm.links.abort);
                phase ^= 1 << par;
            } else {
                cp_wait();
                __syncwarp();
            }
        }
        if (live < St::ROWS) {
            __syncwarp();
            St::fill(sx, live, 0);
            St::fill(sz, live, open_gate<T>());
            __syncwarp();
        }
        const int ox = St::offset(x + o0 * a.ld_x), oz = St::offset(z + o0 * a.ld_x);
        const char *rx = sx + o0 * St::PITCH, *rz = sz + o0 * St::PITCH;
        float2 h[R], p[R];
        float2 hh = make_float2(0.f, 0.f), pp = make_float2(1.f, 1.f);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float2 s, r;
            gates2(St::pair(rz + i * St::PITCH, lane, St::offset(oz, mx, i)), s, r);
            h[i] = hh = __ffma2_rn(s, hh, __fmul2_rn(r, St::pair(rx + i * St::PITCH, lane, St::offset(ox, mx, i))));
            p[i] = pp = __fmul2_rn(pp, s);
        }
        p[R - 1] = at_least(pp, make_float2(kLeast, kLeast));
        sm.agg[par][w.sub][lane] = make_float4(p[R - 1].x, p[R - 1].y, hh.x, hh.y);
        if (a.t - at > step) fetch(par ^ 1, 1);
        __syncthreads();
        float2 in;
        if (w.S > 1) {
            if (at > 0) link_wait(&sm.links.carry[par], par ? turn & 1 : (turn & 1) ^ 1, &sm.links.abort);
            if (w.rank + 1 + w.sub < w.S) {  // the block's pair, to the blocks after it
                float2 ph = make_float2(0.f, 0.f), pb = make_float2(1.f, 1.f);
#pragma unroll 8
                for (int k = 0; k < w.subs; ++k) {
                    const float4 v = sm.agg[par][k][lane];
                    ph = step2(v, ph);
                    pb = __fmul2_rn(pb, make_float2(v.x, v.y));
                }
                pb = at_least(pb, make_float2(kLeast, kLeast));
                const uint32_t to = smem_u32(&sm.slot[(par * w.S + w.rank) * LANES + lane]), bar = smem_u32(&sm.links.pairs[par]);
                for (int k = w.rank + 1 + w.sub; k < w.S; k += w.subs)
                    st_async4(mapa_shared(to, k), mapa_shared(bar, k), make_float4(pb.x, pb.y, ph.x, ph.y));
            }
            link_wait(&sm.links.pairs[par], turn & 1, &sm.links.abort);
            in = sm.carry[par][lane];
#pragma unroll 8
            for (int k = 0; k < w.rank; ++k) in = step2(sm.slot[(par * w.S + k) * LANES + lane], in);
        } else {
            in = sm.carry[par][lane];
        }
#pragma unroll 8
        for (int k = 0; k < w.sub; ++k) in = step2(sm.agg[par][k][lane], in);
        if (last) {
            end = __ffma2_rn(p[R - 1], in, h[R - 1]);
            if (w.rank == w.S - 1 && a.t - at > step) {
                if (w.S == 1) {
                    sm.carry[par ^ 1][lane] = end;
                } else {
#pragma unroll 4
                    for (int k = 0; k < w.S; ++k)
                        st_async2(mapa_shared(smem_u32(&sm.carry[par ^ 1][lane]), k),
                                  mapa_shared(smem_u32(&sm.links.carry[par ^ 1]), k), end);
                }
            }
        }
        if (keeper && row + o0 < a.t) st_state(keep, in, w.two);
        const int rows = max(0, min(a.t - row, St::ROWS));
        // An infinite state's products of gates do not become 0; a finite one beside it keeps its bits.  In a branch of its own
        // (185 x 196 x 256: 18.8 us, 18.5 without; held at every step 19.1, by a loop that computes them again 19.3.)
        const bool known = finite2(in);
        auto least = [&] { return make_float2(fabsf(in.x) < INFINITY ? 0.f : kLeast, fabsf(in.y) < INFINITY ? 0.f : kLeast); };
        if constexpr (ALIGNED) {
            // through the stage of x, which the warp has read
            if (known) {
#pragma unroll
                for (int i = 0; i < R; ++i) St::put(sx + (o0 + i) * St::PITCH, lane, __ffma2_rn(p[i], in, h[i]));
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) St::put(sx + (o0 + i) * St::PITCH, lane, __ffma2_rn(at_least(p[i], least()), in, h[i]));
            }
            if (live < St::ROWS) {
                __syncwarp();
                St::fill(sx, live, 0);
            }
            fence_async_shared();
            __syncwarp();
            if ((threadIdx.x & 31) == 0 && rows > 0) {
                tma_store_3d(&maps.h, sx, w.ch0, row, (int)w.b);
                bulk_commit();
            }
        } else {
            T* g = out + o0 * a.ld_h + 2 * lane;
            auto put = [&](int i, float2 v) {
                if (w.one && o0 + i < rows) st_any(g, o0 + i < live ? v : make_float2(0.f, 0.f), w.two, a.pairs);
                g += a.ld_h;
            };
            if (known) {
#pragma unroll
                for (int i = 0; i < R; ++i) put(i, __ffma2_rn(p[i], in, h[i]));
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) put(i, __ffma2_rn(at_least(p[i], least()), in, h[i]));
            }
            __syncwarp();
        }
        row += step;
        if (!ALIGNED) x += hop, z += hop, out += hop_h;
        if (a.states) keep += (int64_t)(step / kChunk) * a.c;
    }
    if (parts_end < a.t) {  // parts after the sequence's end: its last state, and zeros
        __syncthreads();
        if (w.S > 1 && parts_end > 0) link_wait(&sm.links.carry[par], par ? turn & 1 : (turn & 1) ^ 1, &sm.links.abort);
        const float2 in = sm.carry[par][lane];
        if (a.states && w.one)
            for (int j = parts_end / kChunk + w.rank * w.subs + w.sub; j < w.chunks; j += w.S * w.subs)
                st_state(a.states + (w.b * w.chunks + j) * a.c + w.ch, in, w.two);
        if (w.one)
            for (int64_t i = (int64_t)parts_end + w.rank * w.subs + w.sub; i < a.t; i += w.S * w.subs)
                st_any(static_cast<T*>(a.h) + (w.b * a.t + i) * a.ld_h + w.ch, make_float2(0.f, 0.f), w.two, a.pairs);
    }
    if (ALIGNED) bulk_wait_read();
    linger(&sm.links.abort);
    if (w.S > 1) cluster_leave();
    if (a.last && last && w.one && w.rank == w.S - 1) st_state(a.last + w.b * a.c + w.ch, end, w.two);
}

// Backward: the same split.  What step i hands to the step before it is q_i = a_i*G_i, G_i = dh_i + q_{i+1}: over a
// thread's steps q = product*q' + sum of a_1...a_i * dh_i, so that the first pass runs forward for both recurrences.
// The states are recomputed from the forward pass's kept ones, of which the threads of a chunk share one; for the
// second pass, which goes back through the steps in blocks, the first leaves product and state at the blocks' starts.
template <class T, bool ALIGNED, int LANES, int R>
struct BwdSmem {
    typedef Stage<T, ALIGNED, LANES, R> St;
    typedef char Stages[2][3][St::BYTES];  // of a warp: two parts of x, gate and dh; before this struct
    float4 agg[2][kThreads / LANES][LANES];
    float2 aggq[2][kThreads / LANES][LANES];
    float2 carry[2][LANES];
    Links links;
    alignas(16) float4 slot[1];  // [2][cluster][LANES]
};

template <class T, bool ALIGNED, int LANES, int R, int BLOCKS>
__global__ void __launch_bounds__(kThreads, BLOCKS) scan_bwd_kernel(ScanArgs a, const __grid_constant__ Maps maps)
{
    typedef BwdSmem<T, ALIGNED, LANES, R> Smem;
    typedef typename Smem::St St;
    constexpr int SHARE = kChunk / R, NB = R / kBlock;
    extern __shared__ __align__(128) char smem_raw[];
    typename Smem::Stages* const stages = reinterpret_cast<typename Smem::Stages*>(smem_raw);
    Smem& sm = *reinterpret_cast<Smem*>(stages + blockDim.x / 32);
    Place w;
    w.set<LANES>(a);
    const int tile = w.subs * R, step = tile * w.S, lane = w.lane, ch = a.c - w.ch0;
    const int top = w.len > 0 ? (w.len - 1) / step * step : -step;  // the last part with a step of the sequence; -step: none
    int64_t row = (int64_t)top + w.rank * tile + w.warp * St::ROWS;
    const int64_t row0 = w.b * a.t + row;
    const T* x = static_cast<const T*>(a.x) + row0 * a.ld_x + w.ch0;
    const T* z = static_cast<const T*>(a.gate) + row0 * a.ld_x + w.ch0;
    const T* dh = static_cast<const T*>(a.dh) + row0 * a.ld_h + w.ch0;
    T* dx = static_cast<T*>(a.h) + row0 * a.ld_x + w.ch0;
    T* dz = static_cast<T*>(a.dgate) + row0 * a.ld_x + w.ch0;
    const int64_t hop = step * a.ld_x, hop_h = step * a.ld_h;
    char(*stage)[3][St::BYTES] = stages[w.warp];
    uint64_t* full = sm.links.full[w.warp];
    const int mx = (int)(a.ld_x % St::E), mh = (int)(a.ld_h % St::E), o0 = w.wsub * R;
    const uintptr_t x_lo = reinterpret_cast<uintptr_t>(a.x), z_lo = reinterpret_cast<uintptr_t>(a.gate);
    const uintptr_t x_size = (((int64_t)a.n * a.t - 1) * a.ld_x + a.c) * sizeof(T);
    const uintptr_t d_lo = reinterpret_cast<uintptr_t>(a.dh), d_size = (((int64_t)a.n * a.t - 1) * a.ld_h + a.c) * sizeof(T);
    auto fetch = [&](int ring, int back) {  // the warp's rows `back` parts before (0 or 1)
        const int64_t from = row - back * step;
        const int n = (int)min(w.len - from, (int64_t)St::ROWS);
        if (n <= 0) return;
        if constexpr (ALIGNED) {
            if ((threadIdx.x & 31) == 0) {
                bulk_wait_read();
                mbar_arrive_expect_tx(&full[ring], 3 * St::ROWS * St::ROW_BYTES);
                tma_load_3d(stage[ring][0], &maps.x, &full[ring], w.ch0, (int)from, (int)w.b);
                tma_load_3d(stage[ring][1], &maps.z, &full[ring], w.ch0, (int)from, (int)w.b);
                tma_load_3d(stage[ring][2], &maps.dh, &full[ring], w.ch0, (int)from, (int)w.b);
            }
        } else {
            St::load(stage[ring][0], x - back * hop, a.ld_x, n, ch, x_lo, x_lo + x_size);
            St::load(stage[ring][1], z - back * hop, a.ld_x, n, ch, z_lo, z_lo + x_size);
            St::load(stage[ring][2], dh - back * hop_h, a.ld_h, n, ch, d_lo, d_lo + d_size);
        }
    };
    const float* kept = a.states + (w.b * w.chunks + (row + o0) / kChunk) * a.c + w.ch;
    links_init(sm.links, w.S);
    if (top >= 0) fetch(0, 0);
    float2 start = make_float2(0.f, 0.f);  // the state before this thread's chunk
    if (top >= 0 && w.one && row + o0 < a.t) start = ld_state(kept, w.two);
    for (int64_t i = (int64_t)top + step + w.rank * w.subs + w.sub; i < a.t; i += w.S * w.subs)  // the parts after that one
        if (w.one) {
            const int64_t at = (w.b * a.t + i) * a.ld_x + w.ch;
            st_any(static_cast<T*>(a.h) + at, make_float2(0.f, 0.f), w.two, a.pairs);
            st_any(static_cast<T*>(a.dgate) + at, make_float2(0.f, 0.f), w.two, a.pairs);
        }
    const bool last = w.sub == 0;
    float2 end = make_float2(0.f, 0.f);
    if (last) {
        if (w.one) end = ld_state(a.h0 ? a.h0 + w.b * a.c + w.ch : nullptr, w.two);
        sm.carry[0][lane] = end;
    }
    int par = 0, turn = 0, phase = 0;
    for (int at = top; at >= 0; at -= step, turn += par, par ^= 1) {
        if (w.S > 1 && threadIdx.x == 0) {
            mbar_arrive_expect_tx(&sm.links.pairs[par], (w.S - 1 - w.rank) * LANES * sizeof(float4));
            if (at > 0) mbar_arrive_expect_tx(&sm.links.carry[par ^ 1], LANES * sizeof(float2));
        }
        const int live = (int)max((int64_t)0, min(w.len - row, (int64_t)St::ROWS));
        char *sx = stage[par][0], *sz = stage[par][1], *sd = stage[par][2];
        if (live > 0) {
            if constexpr (ALIGNED) {
                link_wait(&full[par], phase >> par & 1, &sm.links.abort);
                phase ^= 1 << par;
            } else {
                cp_wait();
                __syncwarp();
            }
        }
        if (live < St::ROWS) {
            __syncwarp();
            St::fill(sx, live, 0);
            St::fill(sz, live, open_gate<T>());
            St::fill(sd, live, 0);
            __syncwarp();
        }
        const int ox = St::offset(x + o0 * a.ld_x), oz = St::offset(z + o0 * a.ld_x), od = St::offset(dh + o0 * a.ld_h);
        char *rx = sx + o0 * St::PITCH, *rz = sz + o0 * St::PITCH;
        const char* rd = sd + o0 * St::PITCH;
        float2 hh = make_float2(0.f, 0.f), pp = make_float2(1.f, 1.f), qq = make_float2(0.f, 0.f);
        float4 mark[NB];  // (product, state) before block k
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            mark[k] = make_float4(pp.x, pp.y, hh.x, hh.y);
#pragma unroll
            for (int i = k * kBlock; i < (k + 1) * kBlock; ++i) {
                float2 s, r;
                gates2(St::pair(rz + i * St::PITCH, lane, St::offset(oz, mx, i)), s, r);
                hh = __ffma2_rn(s, hh, __fmul2_rn(r, St::pair(rx + i * St::PITCH, lane, St::offset(ox, mx, i))));
                pp = __fmul2_rn(pp, s);
                qq = __ffma2_rn(pp, St::pair(rd + i * St::PITCH, lane, St::offset(od, mh, i)), qq);
            }
        }
        sm.agg[par][w.sub][lane] = make_float4(pp.x, pp.y, hh.x, hh.y);
        sm.aggq[par][w.sub][lane] = qq;
        float2 h = start;
        if (at > 0) {
            fetch(par ^ 1, 1);
            kept -= (int64_t)(step / kChunk) * a.c;
            if (w.one) start = ld_state(kept, w.two);
        }
        __syncthreads();
        float2 q;
        if (w.S > 1) {
            if (at < top) link_wait(&sm.links.carry[par], par ? turn & 1 : (turn & 1) ^ 1, &sm.links.abort);
            if (w.sub < w.rank) {  // the block's pair, to the blocks before it
                float2 qb = make_float2(0.f, 0.f), pb = make_float2(1.f, 1.f);
#pragma unroll 8
                for (int k = w.subs - 1; k >= 0; --k) {
                    const float4 u = sm.agg[par][k][lane];
                    qb = __ffma2_rn(make_float2(u.x, u.y), qb, sm.aggq[par][k][lane]);
                    pb = __fmul2_rn(pb, make_float2(u.x, u.y));
                }
                const uint32_t to = smem_u32(&sm.slot[(par * w.S + w.rank) * LANES + lane]), bar = smem_u32(&sm.links.pairs[par]);
                for (int k = w.sub; k < w.rank; k += w.subs)
                    st_async4(mapa_shared(to, k), mapa_shared(bar, k), make_float4(pb.x, pb.y, qb.x, qb.y));
            }
            link_wait(&sm.links.pairs[par], turn & 1, &sm.links.abort);
            q = sm.carry[par][lane];
#pragma unroll 8
            for (int k = w.S - 1; k > w.rank; --k) q = step2(sm.slot[(par * w.S + k) * LANES + lane], q);
        } else {
            q = sm.carry[par][lane];
        }
#pragma unroll 8
        for (int k = w.subs - 1; k > w.sub; --k) {
            const float4 u = sm.agg[par][k][lane];
            q = __ffma2_rn(make_float2(u.x, u.y), q, sm.aggq[par][k][lane]);
        }
        for (int k = w.sub & ~(SHARE - 1); k < w.sub; ++k) h = step2(sm.agg[par][k][lane], h);  // this chunk's
        if (last) {
            end = __ffma2_rn(pp, q, qq);
            if (w.rank == 0 && at > 0) {
                if (w.S == 1) {
                    sm.carry[par ^ 1][lane] = end;
                } else {
#pragma unroll 4
                    for (int k = 0; k < w.S; ++k)
                        st_async2(mapa_shared(smem_u32(&sm.carry[par ^ 1][lane]), k),
                                  mapa_shared(smem_u32(&sm.links.carry[par ^ 1]), k), end);
                }
            }
        }
        const int rows = (int)max((int64_t)0, min(a.t - row, (int64_t)St::ROWS));
        T *gx = dx + o0 * a.ld_x + 2 * lane, *gz = dz + o0 * a.ld_x + 2 * lane;
#pragma unroll
        for (int k = NB - 1; k >= 0; --k) {
            float2 u = step2(mark[k], h), s[kBlock], r[kBlock], v[kBlock];
#pragma unroll
            for (int i = 0; i < kBlock; ++i) {  // v: (the state before the step less x)*(1 - a)
                const int n = k * kBlock + i, o = n * St::PITCH;
                gates2(St::pair(rz + o, lane, St::offset(oz, mx, n)), s[i], r[i]);
                const float2 xi = St::pair(rx + o, lane, St::offset(ox, mx, n));
                v[i] = __fmul2_rn(__ffma2_rn(xi, make_float2(-1.f, -1.f), u), r[i]);
                u = __ffma2_rn(s[i], u, __fmul2_rn(r[i], xi));
            }
#pragma unroll
            for (int i = kBlock - 1; i >= 0; --i) {
                const int n = k * kBlock + i, o = n * St::PITCH;
                const float2 g = __fadd2_rn(St::pair(rd + o, lane, St::offset(od, mh, n)), q);
                float2 vx = __fmul2_rn(r[i], g);
                q = __fmul2_rn(s[i], g);
                float2 vz = __fmul2_rn(q, v[i]);
                if constexpr (ALIGNED) {
                    St::put(rx + o, lane, vx);
                    St::put(rz + o, lane, vz);
                } else {
                    if (o0 + n >= live) vx = vz = make_float2(0.f, 0.f);
                    if (w.one && o0 + n < rows) {
                        st_any(gx + n * a.ld_x, vx, w.two, a.pairs);
                        st_any(gz + n * a.ld_x, vz, w.two, a.pairs);
                    }
                }
            }
        }
        if constexpr (ALIGNED) {
            if (live < St::ROWS) {
                __syncwarp();
                St::fill(sx, live, 0);
                St::fill(sz, live, 0);
            }
            fence_async_shared();
            __syncwarp();
            if ((threadIdx.x & 31) == 0 && rows > 0) {
                tma_store_3d(&maps.h, sx, w.ch0, (int)row, (int)w.b);
                tma_store_3d(&maps.dz, sz, w.ch0, (int)row, (int)w.b);
                bulk_commit();
            }
        } else {
            __syncwarp();
            x -= hop, z -= hop, dh -= hop_h, dx -= hop, dz -= hop;
        }
        row -= step;
    }
    if (ALIGNED) bulk_wait_read();
    linger(&sm.links.abort);
    if (w.S > 1) cluster_leave();
    if (a.last && last && w.one && w.rank == 0) st_state(a.last + w.b * a.c + w.ch, end, w.two);
}

// A sequence without steps: the state (or its gradient) passes through.
__global__ void __launch_bounds__(kThreads) scan_copy_kernel(const float* from, float* to, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.f;
}

int check(const dbl_scan_shape* s, const char* what)
{
    if (!s || s->n < 0 || s->t < 0 || s->c <= 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, n < 0, t < 0 or c <= 0", what);
    if (s->t > (1 << 30)) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^30 steps", what);
    if (s->c > kMaxColumns) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^30 channels or more", what);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", what);
    if ((s->ld_x && s->ld_x < s->c) || (s->ld_h && s->ld_h < s->c))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", what);
    return DBL_OK;
}

ScanArgs args(const dbl_scan_shape* s)
{
    ScanArgs a = {};
    a.n = s->n, a.t = s->t, a.c = s->c;
    a.ld_x = s->ld_x ? s->ld_x : s->c;
    a.ld_h = s->ld_h ? s->ld_h : s->c;
    return a;
}

template <class T, bool ALIGNED, int LANES, int R, int BLOCKS, bool BWD>
constexpr auto kernel_of()
{
    if constexpr (BWD)
        return scan_bwd_kernel<T, ALIGNED, LANES, R, BLOCKS>;
    else
        return scan_fwd_kernel<T, ALIGNED, LANES, R, BLOCKS>;
}

// [n][t][c] at row stride ld, in boxes of `cols` channels and `rows` steps.
template <class T>
int encode(CUtensorMap* m, const void* p, const ScanArgs& a, int64_t ld, int cols, int rows, const char* what)
{
    const PFN_encodeTiled fn = encode_tiled();
    if (!fn) return set_error(DBL_ERR_CUDA, "%s: cuTensorMapEncodeTiled unavailable from the driver", what);
    const CUtensorMapDataType dt = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : act::kF16    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                  : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const cuuint64_t dims[3] = {(cuuint64_t)a.c, (cuuint64_t)a.t, (cuuint64_t)a.n};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * sizeof(T), (cuuint64_t)ld * sizeof(T) * a.t};
    const cuuint32_t box[3] = {(cuuint32_t)cols, (cuuint32_t)rows, 1}, one[3] = {1, 1, 1};
    const CUresult r = fn(m, dt, 3, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DBL_OK : set_error(DBL_ERR_CUDA, "%s: tensor map (%d)", what, (int)r);
}

template <class T, bool ALIGNED, int LANES, int R, bool BWD>
size_t smem_of(int S, int warps)
{
    typedef FwdSmem<T, ALIGNED, LANES, R> Fwd;
    typedef BwdSmem<T, ALIGNED, LANES, R> Bwd;
    return (BWD ? sizeof(Bwd) + warps * sizeof(typename Bwd::Stages) : sizeof(Fwd) + warps * sizeof(typename Fwd::Stages)) +
           (S > 1 ? sizeof(float4) * 2 * S * LANES : 0);
}

// How a launch is split, and about how long it takes, in fourths of what a part takes without an exchange.
struct Split {
    int subs, S;
    int64_t cols, cost;
};

// Blocks of a cluster: the fewest parts one after another.  How many clusters the device holds at a time depends on where
// they fit, and one more waits until another is done (152 SMs hold 14 clusters of 16 blocks, 23 of 12, 36 of 8, 74 of 4 and
// 152 of 2, two blocks on an SM: forward, 1 x 65536 x 512, 16 clusters of 16 blocks 83 us, of 12 63 us).  It is asked for
// blocks of 256 threads, also where a short sequence's have fewer and more of them fit.  An exchange takes
// a part a fourth longer (185 x 196 x 256: no exchange 24 us, clusters of two 30), a cluster's start takes about a part,
// and rows of fewer channels are slower to bring (8 lanes and 32: forward, 4 x 8192 x 1024 54 and 46 us, backward 98 and
// 69; 16 lanes and 32: backward, 15 x 1154 x 1660 87 and 82).
template <class T, bool ALIGNED, int LANES, int R, int BLOCKS, bool BWD>
int split_of(const ScanArgs& a, int dev, Split& best, const char* what)
{
    constexpr auto kernel = kernel_of<T, ALIGNED, LANES, R, BLOCKS, BWD>();
    const int rc = allow_launch<kernel>(smem_of<T, ALIGNED, LANES, R, BWD>(kMaxCluster, kThreads / 32), true, what);
    if (rc != DBL_OK) return rc;
    // parts of whole chunks, where there are several; whole warps
    int subs = std::min(kThreads / LANES, (a.t + R - 1) / R);
    const int unit = subs * R < a.t ? std::max(kChunk / R, 32 / LANES) : 32 / LANES;
    subs = (subs + unit - 1) / unit * unit;
    best = {subs, 0, (int64_t)a.n * ((a.c + 2 * LANES - 1) / (2 * LANES)), 0};
    for (int S = 1; S <= kMaxCluster; ++S) {
        int held = clusters_held<kernel>(dev, S, kThreads, smem_of<T, ALIGNED, LANES, R, BWD>(S, kThreads / 32));
        if (held == 0 && S > 1) continue;
        if (held == 0) held = sm_count();  // no answer: single blocks run all the same
        const int64_t parts = ((int64_t)a.t + (int64_t)subs * R * S - 1) / ((int64_t)subs * R * S);
        const int64_t cost = (best.cols + held - 1) / held * (parts + 1) * (S > 1 ? 5 : 4) * (LANES == 32 ? 10 : LANES == 16 ? 13 : 18);
        if (best.S == 0 || cost < best.cost) best.S = S, best.cost = cost;
        if (parts == 1) break;
    }
    return DBL_OK;
}

template <class T, bool ALIGNED, int LANES, int R, int BLOCKS, bool BWD>
int launch_tiles(ScanArgs a, const Split& sp, cudaStream_t st, const char* what)
{
    constexpr auto kernel = kernel_of<T, ALIGNED, LANES, R, BLOCKS, BWD>();
    typedef Stage<T, ALIGNED, LANES, R> St;
    a.groups = (a.c + 2 * LANES - 1) / (2 * LANES);
    const int S = sp.S, subs = sp.subs;
    if (sp.cols * S > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^31 blocks", what);
    Maps maps;
    int rc = DBL_OK;
    if (ALIGNED) {
        rc = encode<T>(&maps.x, a.x, a, a.ld_x, 2 * LANES, St::ROWS, what);
        if (rc == DBL_OK) rc = encode<T>(&maps.z, a.gate, a, a.ld_x, 2 * LANES, St::ROWS, what);
        if (rc == DBL_OK) rc = encode<T>(&maps.h, a.h, a, BWD ? a.ld_x : a.ld_h, 2 * LANES, St::ROWS, what);
        if (BWD && rc == DBL_OK) rc = encode<T>(&maps.dh, a.dh, a, a.ld_h, 2 * LANES, St::ROWS, what);
        if (BWD && rc == DBL_OK) rc = encode<T>(&maps.dz, a.dgate, a, a.ld_x, 2 * LANES, St::ROWS, what);
        if (rc != DBL_OK) return rc;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(sp.cols * S));
    cfg.blockDim = dim3(subs * LANES);
    cfg.dynamicSmemBytes = smem_of<T, ALIGNED, LANES, R, BWD>(S, subs * LANES / 32);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, a, maps);
    rc = launch_check(what);
    return err == cudaSuccess ? rc : cuda_check(err, what);
}

// Narrower blocks have more of them on a sequence at a time (1 x 65536 x 64, 8, 16 and 32 lanes: 30, 40 and 62 us, backward
// 40, 55 and 93); the widest that is as good.
template <class T, bool ALIGNED, int R, bool BWD>
int launch_lanes(const ScanArgs& a, cudaStream_t st, const char* what)
{
    Split s32, s16, s8;
    int dev = 0;
    int rc = cuda_check(cudaGetDevice(&dev), what);
    if (rc == DBL_OK) rc = split_of<T, ALIGNED, 32, R, 2, BWD>(a, dev, s32, what);
    if (rc == DBL_OK) rc = split_of<T, ALIGNED, 16, R, 2, BWD>(a, dev, s16, what);
    if (rc == DBL_OK) rc = split_of<T, ALIGNED, 8, R, 2, BWD>(a, dev, s8, what);
    if (rc != DBL_OK) return rc;
    if (s32.cost <= s16.cost && s32.cost <= s8.cost) return launch_tiles<T, ALIGNED, 32, R, 2, BWD>(a, s32, st, what);
    if (s16.cost <= s8.cost) return launch_tiles<T, ALIGNED, 16, R, 2, BWD>(a, s16, st, what);
    return launch_tiles<T, ALIGNED, 8, R, 2, BWD>(a, s8, st, what);
}

template <class T, bool BWD>
int launch(ScanArgs a, cudaStream_t st, const char* what)
{
    // whether every row of every tensor starts at a multiple of w bytes
    auto rows_at = [&](size_t w) {
        return a.ld_x * sizeof(T) % w == 0 && a.ld_h * sizeof(T) % w == 0 && aligned_to(a.x, w) && aligned_to(a.gate, w) &&
               aligned_to(a.h, w) && aligned_to(a.dh, w) && aligned_to(a.dgate, w);
    };
    a.pairs = a.c % 2 == 0 && rows_at(2 * sizeof(T));
    if (a.t <= kShort) {
        const int64_t grid = ((int64_t)a.n * ((a.c + 1) / 2) + 127) / 128;
        if (grid > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^31 blocks", what);
        const auto kernel = BWD ? (a.pairs ? scan_bwd_short_kernel<T, true> : scan_bwd_short_kernel<T, false>)
                                : (a.pairs ? scan_fwd_short_kernel<T, true> : scan_fwd_short_kernel<T, false>);
        kernel<<<(unsigned)grid, 128, 0, st>>>(a);
        return launch_check(what);
    }
    // 16 steps a thread halve the exchanges of 8 (forward, 1 x 65536 x 512: 83 and 122 us).  fp32 has room for 8, and so
    // have the backward pass's unaligned rows (12 x 3001 x 393: 73 us; 75 with 16, one block on an SM).
    constexpr int R = sizeof(T) == 2 ? 16 : 8, RU = BWD ? 8 : R;
    const bool aligned = rows_at(16);
    return aligned ? launch_lanes<T, true, R, BWD>(a, st, what) : launch_lanes<T, false, RU, BWD>(a, st, what);
}

int pass_through(const dbl_scan_shape* s, const float* from, float* to, cudaStream_t st)
{
    if (!to || from == to) return DBL_OK;
    const int64_t n = (int64_t)s->n * s->c, blocks = (n + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return set_error(DBL_ERR_UNSUPPORTED, "gated_scan: more than 2^31 blocks");
    scan_copy_kernel<<<(unsigned)blocks, kThreads, 0, st>>>(from, to, n);
    return launch_check("gated_scan");
}

}  // namespace

namespace dbl {

static int read_word(int* status) { return status_read(g_scan_status, status); }
static int clear_word() { return status_clear(g_scan_status); }
StatusWord scan_status_word() { return {read_word, clear_word}; }

}  // namespace dbl

extern "C" {

size_t dbl_gated_scan_states_bytes(const dbl_scan_shape* s)
{
    if (check(s, "gated_scan_states_bytes") != DBL_OK) return 0;
    return (size_t)s->n * ((s->t + (int64_t)kChunk - 1) / kChunk) * s->c * sizeof(float);
}

size_t dbl_gated_scan_workspace_bytes(const dbl_scan_shape*, int) { return 0; }

int dbl_gated_scan_fwd(const dbl_scan_shape* s, const void* x, const void* gate, const float* h0, const int32_t* lengths,
                       void* h, float* h_last, float* states, void*, size_t, void* stream)
{
    int rc = check(s, "gated_scan_fwd");
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(x, e) || !aligned_to(gate, e) || !aligned_to(h, e) || !aligned_to(h0, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(h_last, 4) || !aligned_to(states, 4))
        return set_error(DBL_ERR_INVALID, "gated_scan_fwd: a pointer is not aligned to its element type");
    if (s->n == 0) return DBL_OK;
    cudaStream_t st = as_stream(stream);
    if (s->t == 0) return pass_through(s, h0, h_last, st);
    if (!x || !gate || !h) return set_error(DBL_ERR_INVALID, "gated_scan_fwd: x, gate and h must not be NULL");
    ScanArgs a = args(s);
    a.x = x, a.gate = gate, a.h0 = h0, a.lengths = lengths, a.h = h, a.last = h_last, a.states = states;
    return s->dtype == DBL_F32 ? launch<float, false>(a, st, "gated_scan_fwd") : launch<act_t, false>(a, st, "gated_scan_fwd");
}

int dbl_gated_scan_bwd(const dbl_scan_shape* s, const void* dh, const float* dh_last, const void* x, const void* gate,
                       const float* states, const int32_t* lengths, void* dx, void* dgate, float* dh0, void*, size_t,
                       void* stream)
{
    int rc = check(s, "gated_scan_bwd");
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(x, e) || !aligned_to(gate, e) || !aligned_to(dh, e) || !aligned_to(dx, e) || !aligned_to(dgate, e) ||
        !aligned_to(dh_last, 4) || !aligned_to(lengths, 4) || !aligned_to(dh0, 4) || !aligned_to(states, 4))
        return set_error(DBL_ERR_INVALID, "gated_scan_bwd: a pointer is not aligned to its element type");
    if (s->n == 0) return DBL_OK;
    cudaStream_t st = as_stream(stream);
    if (s->t == 0) return pass_through(s, dh_last, dh0, st);
    if (!x || !gate || !dh || !states || !dx || !dgate)
        return set_error(DBL_ERR_INVALID, "gated_scan_bwd: dh, x, gate, states, dx and dgate must not be NULL");
    ScanArgs a = args(s);
    a.x = x, a.gate = gate, a.dh = dh, a.h0 = dh_last, a.lengths = lengths, a.h = dx, a.dgate = dgate, a.last = dh0;
    a.states = const_cast<float*>(states);
    return s->dtype == DBL_F32 ? launch<float, true>(a, st, "gated_scan_bwd") : launch<act_t, true>(a, st, "gated_scan_bwd");
}

}  // extern "C"
