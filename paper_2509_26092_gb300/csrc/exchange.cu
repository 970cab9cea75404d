// exchange.cu -- tokens to their experts' groups and back: rows copied to the slots of their entries, the weighted sum
// of the entries' rows, and the gradients of both.
//
// Bound by memory: every row is read once and written once, token by token, so that a token's own row is read once for all
// its entries.  From a graph: 16384 rows of 1024 to two entries 12.9 us (the rows partly in the L2; 14.9 at the copy rate),
// combine of 20011x2x1000 25.1 (22.2), its gradients of 32768x4x1024 90.7 (89.3).
#include <type_traits>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

struct ExchangeArgs {
    const void* a;         // x; grouped rows (combine); dout
    const void* b;         // res (combine); grouped rows (combine_bwd)
    const int32_t* slots;
    const float* weights;
    void* out;             // xg; out; dyg
    float* dweights;
    int64_t rows, grouped_rows, ld_rows, ld_grouped;
    int k, c;
};

__device__ __forceinline__ int64_t slot_of(const ExchangeArgs& a, int64_t entry)
{
    const int32_t s = a.slots[entry];
    return s >= 0 && s < a.grouped_rows ? s : -1;
}

// W bytes of a row: 16, 8 or 4, or one element.
template <class T, int W = 16>
struct Chunk {
    static constexpr int N = W / (int)sizeof(T), WORDS = W / 4;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (W == 16) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else if constexpr (W == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (W == 16)
            *reinterpret_cast<uint4*>(p) = vec();
        else if constexpr (W == 8)
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<uint32_t*>(p) = w[0];
    }
    __device__ __forceinline__ uint4 vec() const { return make_uint4(w[0], w[1 % WORDS], w[2 % WORDS], w[3 % WORDS]); }
    __device__ __forceinline__ void set(uint4 v) { w[0] = v.x, w[1 % WORDS] = v.y, w[2 % WORDS] = v.z, w[3 % WORDS] = v.w; }
    __device__ __forceinline__ void get(float (&f)[N]) const
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            if constexpr (sizeof(T) == 4) {
                f[i] = __uint_as_float(w[i]);
            } else {
                const float2 t = act::unpack2_u32(w[i]);
                f[2 * i] = t.x, f[2 * i + 1] = t.y;
            }
    }
    __device__ __forceinline__ void put(const float (&f)[N])
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            if constexpr (sizeof(T) == 4)
                w[i] = __float_as_uint(f[i]);
            else
                w[i] = act::pack2_u32(f[2 * i], f[2 * i + 1]);
    }
};

template <>
struct Chunk<act_t, 2> {
    static constexpr int N = 1;
    act_t v = elem_from<act_t>(0.f);

    __device__ __forceinline__ void load(const act_t* p) { v = *p; }
    __device__ __forceinline__ void store(act_t* p) const { *p = v; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = elem_f(v); }
    __device__ __forceinline__ void put(const float (&f)[1]) { v = elem_from<act_t>(f[0]); }
};

// A thread to a chunk of a row, rows_per_block rows to a block.
template <class T, int W>
__global__ void __launch_bounds__(256) expert_scatter_kernel(const ExchangeArgs a, int rows_per_block)
{
    using V = Chunk<T, W>;
    const unsigned chunks = (unsigned)a.c / V::N;
    const int64_t r0 = (int64_t)blockIdx.x * rows_per_block;
    const unsigned n = (unsigned)min((int64_t)rows_per_block, a.rows - r0) * chunks;
    for (unsigned i = threadIdx.x; i < n; i += 256) {
        const unsigned l = i / chunks, u = (i - l * chunks) * V::N;
        const int64_t r = r0 + l;
        V v;
        v.load(static_cast<const T*>(a.a) + r * a.ld_rows + u);
        for (int j = 0; j < a.k; ++j) {
            const int64_t s = slot_of(a, r * a.k + j);
            if (s >= 0) v.store(static_cast<T*>(a.out) + s * a.ld_grouped + u);
        }
    }
}

// G threads to a row, NC chunks of it to a thread at a time, two entries' rows and the residual's asked for together.
template <class T, int W, int G, int NC>
__global__ void __launch_bounds__(256) expert_combine_kernel(const ExchangeArgs a)
{
    static_assert(W > 2 || G <= 32, "rows go by single elements up to 255 of them");
    using V = Chunk<T, W>;
    const int chunks = a.c / V::N, g = threadIdx.x % G;
    const int64_t r = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (r >= a.rows) return;
    const T* res = a.b ? static_cast<const T*>(a.b) + r * a.ld_rows : nullptr;
    T* out = static_cast<T*>(a.out) + r * a.ld_rows;
    for (int c0 = g; c0 < chunks; c0 += G * NC) {
        V rv[NC];
        if (res) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
                if (c0 + i * G < chunks) rv[i].load(res + (c0 + i * G) * V::N);
        }
        float sum[NC][V::N] = {};
        for (int j0 = 0; j0 < a.k; j0 += 2) {
            V y[2][NC] = {};  // zeros where an entry is absent
            float w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool in = j0 + j < a.k;
                const int64_t s = in ? slot_of(a, r * a.k + j0 + j) : -1;
                w[j] = in ? (a.weights ? a.weights[r * a.k + j0 + j] : 1.f) : 0.f;
                if (s >= 0) {
                    const T* row = static_cast<const T*>(a.a) + s * a.ld_grouped;
#pragma unroll
                    for (int i = 0; i < NC; ++i)
                        if (c0 + i * G < chunks) y[j][i].load(row + (c0 + i * G) * V::N);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    float f[V::N];
                    y[j][i].get(f);
#pragma unroll
                    for (int e = 0; e < V::N; ++e) sum[i][e] = fmaf(w[j], f[e], sum[i][e]);
                }
        }
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (c0 + i * G < chunks) {
                if (res) {
                    float f[V::N];
                    rv[i].get(f);
#pragma unroll
                    for (int e = 0; e < V::N; ++e) sum[i][e] += f[e];
                }
                V o;
                o.put(sum[i]);
                o.store(out + (c0 + i * G) * V::N);
            }
    }
}

// G threads to a row, NC chunks of it to a thread, kept while the entries pass (NC = 0: any number, read again for each).
template <class T, int W, int G, int NC>
__global__ void __launch_bounds__(256) expert_combine_bwd_kernel(const ExchangeArgs a)
{
    static_assert(G <= 32 || G == 256, "the sum over a row is a warp's or the block's");
    static_assert(W > 2 || G <= 32, "rows go by single elements up to 255 of them");
    using V = Chunk<T, W>;
    constexpr int HELD = NC ? NC : 1;
    __shared__ float red[32];
    const int chunks = a.c / V::N, g = threadIdx.x % G;
    const int64_t r = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (G < 256 && (int64_t)blockIdx.x * (256 / G) + (threadIdx.x & ~31) / G >= a.rows) return;  // whole warps
    const bool live = r < a.rows;
    const T* d = static_cast<const T*>(a.a) + (live ? r : 0) * a.ld_rows;
    V held[HELD];
    if (NC && live) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (g + i * G < chunks) held[i].load(d + (g + i * G) * V::N);
    }
    for (int j = 0; j < a.k; ++j) {
        const int64_t s = live ? slot_of(a, r * a.k + j) : -1;
        float dot = 0.f;
        if (s >= 0) {
            const float w = a.weights ? a.weights[r * a.k + j] : 1.f;
            T* o = static_cast<T*>(a.out) + s * a.ld_grouped;
            const T* y = a.dweights ? static_cast<const T*>(a.b) + s * a.ld_grouped : nullptr;
            auto one = [&](const V& dv, const V& yv, int u) {
                float f[V::N];
                dv.get(f);
                if (y) {
                    float h[V::N];
                    yv.get(h);
#pragma unroll
                    for (int e = 0; e < V::N; ++e) dot = fmaf(f[e], h[e], dot);
                }
#pragma unroll
                for (int e = 0; e < V::N; ++e) f[e] *= w;
                V p;
                p.put(f);
                p.store(o + u);
            };
            if constexpr (NC > 0) {
                V yv[NC];
                if (y) {
#pragma unroll
                    for (int i = 0; i < NC; ++i)
                        if (g + i * G < chunks) yv[i].load(y + (g + i * G) * V::N);
                }
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (g + i * G < chunks) one(held[i], yv[i], (g + i * G) * V::N);
            } else {
                for (int i = g; i < chunks; i += G) {
                    V dv, yv;
                    dv.load(d + i * V::N);
                    if (y) yv.load(y + i * V::N);
                    one(dv, yv, i * V::N);
                }
            }
        }
        if (!a.dweights) continue;
        if constexpr (G == 256) {
            dot = block_sum(dot, red);
        } else {
#pragma unroll
            for (int o = G / 2; o; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        if (live && g == 0) a.dweights[r * a.k + j] = dot;
    }
}

// The same for long rows that begin anywhere: a warp to a part of a row, kPart units of it.
constexpr int kPart = 128;

template <class T>
__device__ __forceinline__ RowOf<T> token_row(const ExchangeArgs& a, const void* p, int64_t r, int lead)
{
    return {p, r, a.rows, a.c, a.ld_rows, lead};
}
template <class T>
__device__ __forceinline__ RowOf<T> grouped_row(const ExchangeArgs& a, const void* p, int64_t s, int lead)
{
    return {p, s, a.grouped_rows, a.c, a.ld_grouped, lead};
}

// M units to a thread at a time.
template <class T, int M>
__global__ void __launch_bounds__(256) expert_scatter_any_kernel(const ExchangeArgs a, int parts)
{
    static_assert(sizeof(T) == 2 || M == 4, "rows of fp32 come here with more than kShort units");
    constexpr int N = Chunk<T>::N;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = item / parts;
    const int part = (int)(item - r * parts);
    if (r >= a.rows) return;
    for (int j = 0; j < a.k; ++j) {
        const int64_t s = slot_of(a, r * a.k + j);
        if (s < 0) continue;
        T* o = static_cast<T*>(a.out) + s * a.ld_grouped;
        const int lead = unit_lead(o), units = (a.c + lead + N - 1) / N, end = min(units, (part + 1) * kPart);
        const RowOf<T> x = token_row<T>(a, a.a, r, lead);
        for (int u0 = part * kPart; u0 < end; u0 += 32 * M) {
            const int u = u0 + lane;
            uint4 v[M + 1];
            x.template load<M>(u, v);
            x.template join<M>(u, v);
#pragma unroll
            for (int m = 0; m < M; ++m)
                if (u + 32 * m < end) store_unit(o, a.c, (u + 32 * m) * N - lead, v[m]);
        }
    }
}

template <class T, int M>
__global__ void __launch_bounds__(256) expert_combine_any_kernel(const ExchangeArgs a, int parts)
{
    static_assert(sizeof(T) == 2, "rows of fp32 go by four bytes at the least");
    constexpr int N = Chunk<T>::N;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = item / parts;
    const int part = (int)(item - r * parts);
    if (r >= a.rows) return;
    T* o = static_cast<T*>(a.out) + r * a.ld_rows;
    const int lead = unit_lead(o), units = (a.c + lead + N - 1) / N, end = min(units, (part + 1) * kPart);
    for (int u0 = part * kPart; u0 < end; u0 += 32 * M) {
        const int u = u0 + lane;
        float sum[M][N] = {};
        auto add = [&](const RowOf<T>& row, float w) {
            uint4 v[M + 1];
            row.template load<M>(u, v);
            row.template join<M>(u, v);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                Chunk<T> y;
                float f[N];
                y.set(v[m]);
                y.get(f);
#pragma unroll
                for (int i = 0; i < N; ++i) sum[m][i] = fmaf(w, f[i], sum[m][i]);
            }
        };
        for (int j = 0; j < a.k; ++j) {
            const int64_t s = slot_of(a, r * a.k + j);
            const float w = a.weights ? a.weights[r * a.k + j] : 1.f;
            if (s >= 0) {
                add(grouped_row<T>(a, a.a, s, lead), w);
            } else {  // w*0, which is not 0 for every w
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[m][i] = fmaf(w, 0.f, sum[m][i]);
            }
        }
        if (a.b) add(token_row<T>(a, a.b, r, lead), 1.f);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            Chunk<T> t;
            t.put(sum[m]);
            if (u + 32 * m < end) store_unit(o, a.c, (u + 32 * m) * N - lead, t.vec());
        }
    }
}

// G threads to a row, M units to a thread at a time: eight rows of one warp to a block, or one row.
template <class T, int G, int M>
__global__ void __launch_bounds__(G == 32 ? 256 : G) expert_combine_bwd_any_kernel(const ExchangeArgs a)
{
    static_assert(sizeof(T) == 2 || G > 32, "rows of fp32 come here with more than 256 units");
    constexpr int N = Chunk<T>::N, R = G == 32 ? 8 : 1;
    __shared__ float red[32];
    const int lane = threadIdx.x & 31, warp = (threadIdx.x % G) >> 5;
    const int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / G;
    if (r >= a.rows) return;
    for (int j = 0; j < a.k; ++j) {
        const int64_t s = slot_of(a, r * a.k + j);
        float dot = 0.f;
        if (s >= 0) {
            const float w = a.weights ? a.weights[r * a.k + j] : 1.f;
            T* o = static_cast<T*>(a.out) + s * a.ld_grouped;
            const int lead = unit_lead(o), units = (a.c + lead + N - 1) / N;
            const RowOf<T> d = token_row<T>(a, a.a, r, lead), y = grouped_row<T>(a, a.dweights ? a.b : a.out, s, lead);
            for (int u0 = warp * 32 * M; u0 < units; u0 += G * M) {
                const int u = u0 + lane;
                uint4 dv[M + 1], yv[M + 1];
                d.template load<M>(u, dv);
                if (a.dweights) {
                    y.template load<M>(u, yv);
                    y.template join<M>(u, yv);
                }
                d.template join<M>(u, dv);
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const int e = (u + 32 * m) * N - lead;
                    Chunk<T> c;
                    float f[N], h[N];
                    c.set(dv[m]);
                    c.get(f);
                    if (a.dweights) {
                        c.set(yv[m]);
                        c.get(h);
                        if (e >= 0 && e + N <= a.c) {
#pragma unroll
                            for (int i = 0; i < N; ++i) dot = fmaf(f[i], h[i], dot);
                        } else {  // a row's first and last unit hold what is outside it
#pragma unroll
                            for (int i = 0; i < N; ++i)
                                if (e + i >= 0 && e + i < a.c) dot = fmaf(f[i], h[i], dot);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] *= w;
                    c.put(f);
                    if (u + 32 * m < units) store_unit(o, a.c, e, c.vec());
                }
            }
        }
        if (!a.dweights) continue;
        dot = G == 32 ? warp_sum(dot) : block_sum(dot, red);
        if (threadIdx.x % G == 0) a.dweights[r * a.k + j] = dot;
    }
}

int check(const dbl_exchange_shape* s, const char* w)
{
    if (!s || s->rows < 0 || s->k <= 0 || s->c <= 0 || s->grouped_rows < 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0, grouped_rows < 0, k <= 0 or c <= 0", w);
    if (s->c > kMaxColumns) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^30 channels or more", w);
    if (s->k > DBL_ROUTE_MAX_K) return set_error(DBL_ERR_UNSUPPORTED, "%s: k = %d, at most %d", w, s->k, DBL_ROUTE_MAX_K);
    if (s->rows > INT32_MAX / s->k) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^31 entries or more", w);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", w);
    if ((s->ld_rows && s->ld_rows < s->c) || (s->ld_grouped && s->ld_grouped < s->c))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", w);
    return DBL_OK;
}

ExchangeArgs args(const dbl_exchange_shape* s, const void* a, const void* b, const int32_t* slots, const float* weights,
                  void* out, float* dweights)
{
    return {a, b, slots, weights, out, dweights, s->rows, s->grouped_rows ? s->grouped_rows : s->rows * s->k,
            s->ld_rows ? s->ld_rows : s->c, s->ld_grouped ? s->ld_grouped : s->c, s->k, s->c};
}

// The bytes of a chunk: what the rows' addresses, strides and length have in common, 16 at most, an element at least; 0: long
// rows that begin at any element, in units put together.  (30000 rows of 70 elements, two entries: combine 17 us by units, as a
// warp has a row, 7 so; 8000 rows of 1001, four entries: scatter 32 us by elements, 15 by units, the gradients 68 and 39.)
// Where they have four bytes in common, of more than `four` units: 8000 rows of 1001 in fp32 scatter 39 us by four bytes, 28 by
// units, the gradients 56 and 59; 3000 rows of 4001 have 60 and 39, 136 and 84; and 8000 of 129, 32 units, 7.7 and 8.5, 6.8 and
// 15.  combine, which adds in registers, is never faster by units: 32 and 46, 49 and 65, 6.0 and 8.6.
// Where they have two bytes in common, from 256 columns on.  20000 rows of 129, 199 and 255 in bf16, two entries: scatter 10.0,
// 14.2 and 17.0 us by elements, 12.1, 12.2 and 13.5 by units; combine 9.3, 9.6 and 9.7, 16.4, 16.5 and 17.5; the gradients 8.1, 8.5
// and 9.1, 22.9, 22.9 and 24.9.  One border for the three, scatter's and long rows': at 257 and 511 combine takes 13.2 and 18.4 by
// elements, 17.5 and 27.6 by units, the gradients 13.3 and 20.5, 24.8 and 38.3.
int chunk_bytes(const ExchangeArgs& a, size_t e, size_t four)
{
    uintptr_t bits = reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.b) | reinterpret_cast<uintptr_t>(a.out);
    bits |= (uintptr_t)a.c * e | (uintptr_t)a.ld_rows * e | (uintptr_t)a.ld_grouped * e;
    if (bits & 3) return a.c < 256 ? 2 : 0;
    if (bits & 4) return a.c * e / 16 > four ? 0 : 4;
    return bits & 8 ? 8 : 16;
}

// f(bytes, as a value of their type)
template <class T, class F>
void with_bytes(int bytes, F f)
{
    if (bytes == 16)
        f(std::integral_constant<int, 16>());
    else if (bytes == 8)
        f(std::integral_constant<int, 8>());
    else if (bytes == 4)
        f(std::integral_constant<int, 4>());
    else if constexpr (sizeof(T) == 2)
        f(std::integral_constant<int, 2>());
}

// Units of a row that begins anywhere up to which a thread has two at a time, not four.  (combine, 20000 rows of 333 with two
// entries: 18 us with two, 27 with four; 8000 of 1001 with four 25.4 and 23.8, 3000 of 4001 with four 42 and 37; one unit at a
// time 20, 29 and 51.)
constexpr int kShort = 64;

// Parts of a row that begins anywhere, and the blocks of eight warps that take them.
template <class T>
int row_parts(const ExchangeArgs& a) { return ((a.c + 2 * (Chunk<T>::N - 1)) / Chunk<T>::N + kPart - 1) / kPart; }
unsigned part_blocks(const ExchangeArgs& a, int parts) { return (unsigned)((a.rows * parts + 7) / 8); }

// Rows of a block of the kernel that has a thread for a chunk: four chunks to a thread where there are many rows, one where
// there are few.
int block_rows(const ExchangeArgs& a, int chunks)
{
    const int64_t all = a.rows * chunks;
    const int per = all >= (int64_t)sm_count() * 8 * 1024 ? 1024 : 256;
    return chunks >= per ? 1 : per / chunks;
}

template <class T>
void launch_scatter(const ExchangeArgs& a, cudaStream_t st)
{
    const int bytes = chunk_bytes(a, sizeof(T), kShort);
    if (bytes == 0) {
        const int parts = row_parts<T>(a);
        if constexpr (sizeof(T) == 2)
            if (a.c / Chunk<T>::N <= kShort) {
                expert_scatter_any_kernel<T, 2><<<part_blocks(a, parts), 256, 0, st>>>(a, parts);
                return;
            }
        expert_scatter_any_kernel<T, 4><<<part_blocks(a, parts), 256, 0, st>>>(a, parts);
        return;
    }
    with_bytes<T>(bytes, [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int rpb = block_rows(a, a.c / Chunk<T, W>::N);
        expert_scatter_kernel<T, W><<<(unsigned)((a.rows + rpb - 1) / rpb), 256, 0, st>>>(a, rpb);
    });
}

// Threads to a row and chunks to a thread at a time of the forward pass.  More chunks of 16 bytes leave too few warps on an SM:
// 20011 rows of 1000 with two entries 25.1 us with two, 27.8 with four (127 registers); 8000 of 512 in fp32 with eight 27 and 33.
// Chunks of 8 bytes are the same (20000 of 1204 in bf16, two entries, 43 us with 256 threads to a row, 74 with 64 and eight
// each).  Chunks of 4 want many to a thread: 8000 of 1001 in fp32, four entries, 32 us with 128 threads to a row and eight each,
// 50 with 256 and one; 8000 of 1002 in bf16 17 with 64 and eight, 19 with 128 and four, 26 with 256 and one; 20000 of 333 in
// fp32, two entries, 17.5 with 64 and six, 47 with 256 and one.
template <class T>
void launch_combine(const ExchangeArgs& a, cudaStream_t st)
{
    const int bytes = chunk_bytes(a, sizeof(T), SIZE_MAX);
    if constexpr (sizeof(T) == 2)
        if (bytes == 0) {
            const int parts = row_parts<T>(a);
            if (a.c / Chunk<T>::N > kShort)
                expert_combine_any_kernel<T, 4><<<part_blocks(a, parts), 256, 0, st>>>(a, parts);
            else
                expert_combine_any_kernel<T, 2><<<part_blocks(a, parts), 256, 0, st>>>(a, parts);
            return;
        }
    with_bytes<T>(bytes, [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int chunks = a.c / Chunk<T, W>::N;
        auto run = [&](auto g, auto nc) {
            constexpr int G = decltype(g)::value, NC = decltype(nc)::value;
            expert_combine_kernel<T, W, G, NC><<<(unsigned)((a.rows + 256 / G - 1) / (256 / G)), 256, 0, st>>>(a);
        };
#define DBL_I(n) std::integral_constant<int, n>()
        if (chunks <= 8) return run(DBL_I(8), DBL_I(1));
        if (chunks <= 32) return run(DBL_I(32), DBL_I(1));
        if (chunks <= 64) return run(DBL_I(32), DBL_I(2));
        if (chunks <= 256) return run(DBL_I(32), DBL_I(W == 16 ? 2 : 4));
        if constexpr (W == 4) {
            if (chunks <= 384) return run(DBL_I(64), DBL_I(6));
            if (chunks <= 512) return run(DBL_I(64), DBL_I(8));
            if (chunks <= 768) return run(DBL_I(256), DBL_I(3));
            run(DBL_I(128), DBL_I(8));
        } else if constexpr (W > 4) {
            run(DBL_I(256), DBL_I(1));
        }
#undef DBL_I
    });
}

template <class T>
void launch_combine_bwd(const ExchangeArgs& a, cudaStream_t st)
{
    const int bytes = chunk_bytes(a, sizeof(T), 256);
    if (bytes == 0) {
        // a row to a warp, or to a block of two or eight: 8000 rows of 1001, four entries, 43 us with a warp, 39 with two
        const int units = a.c / Chunk<T>::N;
        if (units > 512)
            expert_combine_bwd_any_kernel<T, 256, 2><<<(unsigned)a.rows, 256, 0, st>>>(a);
        else if (sizeof(T) == 4 || units > 96)
            expert_combine_bwd_any_kernel<T, 64, 2><<<(unsigned)a.rows, 64, 0, st>>>(a);
        else if constexpr (sizeof(T) == 2)
            expert_combine_bwd_any_kernel<T, 32, 2><<<(unsigned)((a.rows + 7) / 8), 256, 0, st>>>(a);
        return;
    }
    with_bytes<T>(bytes, [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int chunks = a.c / Chunk<T, W>::N;
        auto run = [&](auto g, auto nc) {
            constexpr int G = decltype(g)::value, NC = decltype(nc)::value;
            expert_combine_bwd_kernel<T, W, G, NC><<<(unsigned)((a.rows + 256 / G - 1) / (256 / G)), 256, 0, st>>>(a);
        };
#define DBL_I(n) std::integral_constant<int, n>()
        if (chunks <= 8) return run(DBL_I(8), DBL_I(1));
        if (chunks <= 16) return run(DBL_I(8), DBL_I(2));
        if (chunks <= 32) return run(DBL_I(32), DBL_I(1));
        if (chunks <= 64) return run(DBL_I(32), DBL_I(2));
        if (chunks <= 128) return run(DBL_I(32), DBL_I(4));
        if (chunks <= 256) return run(DBL_I(32), DBL_I(8));
        if constexpr (W > 2) {
            if (chunks <= 512) return run(DBL_I(W < 16 ? 32 : 256), DBL_I(W < 16 ? 16 : 2));
            if (chunks <= 1024) return run(DBL_I(256), DBL_I(4));
            run(DBL_I(256), DBL_I(0));
        }
#undef DBL_I
    });
}

}  // namespace

extern "C" int dbl_expert_scatter(const dbl_exchange_shape* s, const void* x, const int32_t* slots, void* xg, void* stream)
{
    const char* w = "expert_scatter";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(x, e) || !aligned_to(xg, e) || !aligned_to(slots, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (s->rows == 0) return DBL_OK;
    if (!x || !slots || !xg) return set_error(DBL_ERR_INVALID, "%s: x, slots and xg must not be NULL", w);
    const ExchangeArgs a = args(s, x, nullptr, slots, nullptr, xg, nullptr);
    cudaStream_t st = as_stream(stream);
    s->dtype == DBL_F32 ? launch_scatter<float>(a, st) : launch_scatter<act_t>(a, st);
    return launch_check(w);
}

extern "C" int dbl_expert_combine(const dbl_exchange_shape* s, const void* yg, const int32_t* slots, const float* weights,
                                  const void* res, void* out, void* stream)
{
    const char* w = "expert_combine";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(yg, e) || !aligned_to(res, e) || !aligned_to(out, e) || !aligned_to(slots, 4) || !aligned_to(weights, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (s->rows == 0) return DBL_OK;
    if (!yg || !slots || !out) return set_error(DBL_ERR_INVALID, "%s: yg, slots and out must not be NULL", w);
    const ExchangeArgs a = args(s, yg, res, slots, weights, out, nullptr);
    cudaStream_t st = as_stream(stream);
    s->dtype == DBL_F32 ? launch_combine<float>(a, st) : launch_combine<act_t>(a, st);
    return launch_check(w);
}

extern "C" int dbl_expert_combine_bwd(const dbl_exchange_shape* s, const void* dout, const void* yg, const int32_t* slots,
                                      const float* weights, void* dyg, float* dweights, void* stream)
{
    const char* w = "expert_combine_bwd";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(dout, e) || !aligned_to(yg, e) || !aligned_to(dyg, e) || !aligned_to(slots, 4) ||
        !aligned_to(weights, 4) || !aligned_to(dweights, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (s->rows == 0) return DBL_OK;
    if (!dout || !slots || !dyg || (dweights && !yg))
        return set_error(DBL_ERR_INVALID, "%s: dout, slots and dyg must not be NULL, nor yg with dweights", w);
    const ExchangeArgs a = args(s, dout, yg, slots, weights, dyg, dweights);
    cudaStream_t st = as_stream(stream);
    s->dtype == DBL_F32 ? launch_combine_bwd<float>(a, st) : launch_combine_bwd<act_t>(a, st);
    return launch_check(w);
}
