// exchange.cu -- tokens to their experts' groups and back: rows copied to the slots of their entries, the weighted sum
// of the entries' rows, and the gradients of both.
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

// VB bytes of a row, the most that all rows' addresses and lengths allow: 16, or 8, 4, 2.
template <class T, int VB>
struct Chunk {
    static constexpr int N = VB / (int)sizeof(T);
    static constexpr int W = VB < 4 ? 1 : VB / 4;
    uint32_t w[W];

    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (VB == 16) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else if constexpr (VB == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        } else if constexpr (VB == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (VB == 16)
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (VB == 8)
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else if constexpr (VB == 4)
            *reinterpret_cast<uint32_t*>(p) = w[0];
        else
            *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
    __device__ __forceinline__ void get(float (&f)[N]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(w[i]);
        } else if constexpr (VB == 2) {
            f[0] = act::unpack2_u32(w[0]).x;
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 v = act::unpack2_u32(w[i]);
                f[2 * i] = v.x, f[2 * i + 1] = v.y;
            }
        }
    }
    __device__ __forceinline__ void put(const float (&f)[N])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
        } else if constexpr (VB == 2) {
            w[0] = act::pack2_u32(f[0], 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = act::pack2_u32(f[2 * i], f[2 * i + 1]);
        }
    }
};

// A thread to a chunk of a row, rows_per_block rows to a block.
template <class T, int VB>
__global__ void __launch_bounds__(256) expert_scatter_kernel(const ExchangeArgs a, int rows_per_block)
{
    using V = Chunk<T, VB>;
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
template <class T, int VB, int G, int NC>
__global__ void __launch_bounds__(256) expert_combine_kernel(const ExchangeArgs a)
{
    using V = Chunk<T, VB>;
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
            V y[2][NC] = {};
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
template <class T, int VB, int G, int NC>
__global__ void __launch_bounds__(256) expert_combine_bwd_kernel(const ExchangeArgs a)
{
    using V = Chunk<T, VB>;
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

// The bytes of a chunk: what the rows' addresses, strides and length have in common.
int chunk_bytes(const ExchangeArgs& a, size_t e)
{
    uintptr_t bits = reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.b) | reinterpret_cast<uintptr_t>(a.out);
    bits |= (uintptr_t)a.c * e | (uintptr_t)a.ld_rows * e | (uintptr_t)a.ld_grouped * e;
    return bits & 1 ? 1 : bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16;
}

// f(element type, chunk bytes), both as values of their types.
template <class F>
void with_chunks(int dtype, int bytes, F f)
{
    if (dtype == DBL_F32) {
        if (bytes == 16) f(0.f, std::integral_constant<int, 16>());
        else if (bytes == 8) f(0.f, std::integral_constant<int, 8>());
        else f(0.f, std::integral_constant<int, 4>());
    } else {
        if (bytes == 16) f(act_t(), std::integral_constant<int, 16>());
        else if (bytes == 8) f(act_t(), std::integral_constant<int, 8>());
        else if (bytes == 4) f(act_t(), std::integral_constant<int, 4>());
        else f(act_t(), std::integral_constant<int, 2>());
    }
}

// Rows of a block of the kernels that have a thread for a chunk: four chunks to a thread where there are many rows, one where
// there are few.
int block_rows(const ExchangeArgs& a, int chunks)
{
    const int64_t all = a.rows * chunks;
    const int per = all >= (int64_t)sm_count() * 8 * 1024 ? 1024 : 256;
    return chunks >= per ? 1 : per / chunks;
}

// Threads to a row and chunks to a thread of the forward pass: rows of up to 8, 32, 64, 128 chunks are held at once.
template <class T, int VB>
void launch_combine(const ExchangeArgs& a, cudaStream_t st)
{
    const int chunks = a.c / Chunk<T, VB>::N;
    auto run = [&](auto g, auto nc) {
        constexpr int G = decltype(g)::value, NC = decltype(nc)::value;
        expert_combine_kernel<T, VB, G, NC><<<(unsigned)((a.rows + 256 / G - 1) / (256 / G)), 256, 0, st>>>(a);
    };
#define DBL_I(n) std::integral_constant<int, n>()
    if (chunks <= 8) return run(DBL_I(8), DBL_I(1));
    if (chunks <= 32) return run(DBL_I(32), DBL_I(1));
    if (chunks <= 64) return run(DBL_I(32), DBL_I(2));
    if (chunks <= 256) return run(DBL_I(32), DBL_I(4));
    run(DBL_I(256), DBL_I(2));
#undef DBL_I
}

template <class T, int VB>
void launch_combine_bwd(const ExchangeArgs& a, cudaStream_t st)
{
    const int chunks = a.c / Chunk<T, VB>::N;
    auto run = [&](auto g, auto nc) {
        constexpr int G = decltype(g)::value, NC = decltype(nc)::value;
        expert_combine_bwd_kernel<T, VB, G, NC><<<(unsigned)((a.rows + 256 / G - 1) / (256 / G)), 256, 0, st>>>(a);
    };
#define DBL_I(n) std::integral_constant<int, n>()
    if (VB < 16 && chunks > 32) return chunks > 512 ? run(DBL_I(256), DBL_I(0)) : run(DBL_I(32), DBL_I(0));
    if (chunks <= 8) return run(DBL_I(8), DBL_I(1));
    if (chunks <= 16) return run(DBL_I(8), DBL_I(2));
    if (chunks <= 32) return run(DBL_I(32), DBL_I(1));
    if (chunks <= 64) return run(DBL_I(32), DBL_I(2));
    if (chunks <= 128) return run(DBL_I(32), DBL_I(4));
    if (chunks <= 512) return run(DBL_I(256), DBL_I(2));
    if (chunks <= 1024) return run(DBL_I(256), DBL_I(4));
    run(DBL_I(256), DBL_I(0));
#undef DBL_I
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
    with_chunks(s->dtype, chunk_bytes(a, e), [&](auto type, auto bytes) {
        using V = Chunk<decltype(type), decltype(bytes)::value>;
        const int rpb = block_rows(a, a.c / V::N);
        expert_scatter_kernel<decltype(type), decltype(bytes)::value><<<(unsigned)((a.rows + rpb - 1) / rpb), 256, 0, st>>>(a, rpb);
    });
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
    with_chunks(s->dtype, chunk_bytes(a, e), [&](auto type, auto bytes) { launch_combine<decltype(type), decltype(bytes)::value>(a, st); });
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
    with_chunks(s->dtype, chunk_bytes(a, e), [&](auto type, auto bytes) { launch_combine_bwd<decltype(type), decltype(bytes)::value>(a, st); });
    return launch_check(w);
}
