// dropout.cu -- dropout over tokens with the residual addition, the mask drawn from a counter-based generator
// (Philox4x32-10: Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).
//
// Bound by memory while a thread has two blocks of the generator for 16 bytes of 16-bit values: 65536 rows of 2048 with the residual
// 127 us (119 at the copy rate; 0.66 of the issue slots used, the multiplications' pipe the second most frequent stall).  Ten
// rounds of Philox4x64 for the same words would take four times the 32-bit multiplications.
#include <math.h>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

struct DropArgs {
    const void* x;
    const void* res;
    void* y;
    const uint64_t* step;
    int64_t rows, ld_in, ld_out;
    int c;
    uint32_t key0, key1, threshold;
    float scale;
};

// The four words of one block: ten rounds of two 32 x 32 -> 64 bit products.
__device__ __forceinline__ void philox(uint64_t block, uint64_t step, uint32_t k0, uint32_t k1, uint32_t (&w)[4])
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

template <class T>
__device__ __forceinline__ float dropped(const DropArgs& a, uint32_t word, float x, float res)
{
    return fmaf(word >= a.threshold ? x : 0.f, a.scale, res);
}

// Sixteen bytes of row r from channel `col` on, a multiple of four: two blocks of the generator, fp32 one.
template <class T>
__device__ __forceinline__ uint4 unit(const DropArgs& a, uint64_t step, int64_t r, unsigned col, uint4 xv, uint4 rv)
{
    constexpr int N = 16 / (int)sizeof(T);
    const uint32_t x[4] = {xv.x, xv.y, xv.z, xv.w}, res[4] = {rv.x, rv.y, rv.z, rv.w};
    const uint64_t first = (uint64_t)r * (((unsigned)a.c + 3) / 4) + col / 4;
    uint32_t y[4];
#pragma unroll
    for (int b = 0; b < N / 4; ++b) {
        uint32_t w[4];
        philox(first + b, step, a.key0, a.key1, w);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = __float_as_uint(dropped<T>(a, w[e], __uint_as_float(x[e]), __uint_as_float(res[e])));
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 f = act::unpack2_u32(x[2 * b + e]), g = act::unpack2_u32(res[2 * b + e]);
                y[2 * b + e] = act::pack2_u32(dropped<T>(a, w[2 * e], f.x, g.x), dropped<T>(a, w[2 * e + 1], f.y, g.y));
            }
        }
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

// Rows of a multiple of 16 bytes at 16-byte addresses: a unit to a thread, rows_per_block rows to a block.
template <class T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a, int rows_per_block)
{
    constexpr int N = 16 / (int)sizeof(T);
    const unsigned units = (unsigned)a.c / N;
    const int64_t r0 = (int64_t)blockIdx.x * rows_per_block;
    const unsigned n = (unsigned)min((int64_t)rows_per_block, a.rows - r0) * units;
    const uint64_t step = *a.step;
    for (unsigned i = threadIdx.x; i < n; i += 256) {
        const unsigned l = i / units, col = (i - l * units) * N;
        const int64_t r = r0 + l, in = r * a.ld_in + col;
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.x) + in);
        uint4 res = make_uint4(0, 0, 0, 0);
        if (a.res) res = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.res) + in);
        *reinterpret_cast<uint4*>(static_cast<T*>(a.y) + r * a.ld_out + col) = unit<T>(a, step, r, col, x, res);
    }
}

// Eight bytes in accesses of W.
template <int W>
__device__ __forceinline__ uint2 load8(const void* p)
{
    if (W == 8) return *static_cast<const uint2*>(p);
    return make_uint2(static_cast<const uint32_t*>(p)[0], static_cast<const uint32_t*>(p)[1]);
}
template <int W>
__device__ __forceinline__ void store8(void* p, uint2 v)
{
    if (W == 8)
        *static_cast<uint2*>(p) = v;
    else
        static_cast<uint32_t*>(p)[0] = v.x, static_cast<uint32_t*>(p)[1] = v.y;
}

// Rows of any length and alignment: a block of the generator, four channels, to a thread.  60000 rows of 1001 with the residual
// 89 us; units on boundaries put together by shuffles 145, a choice of accesses for each row 107.
template <class T, int W>
__global__ void __launch_bounds__(256) dropout_any_kernel(const DropArgs a, int rows_per_block)
{
    static_assert(sizeof(T) == 2 || W == 4, "wider accesses are pairs of 16-bit values");
    const unsigned per = ((unsigned)a.c + 3) / 4;
    const int64_t r0 = (int64_t)blockIdx.x * rows_per_block;
    const unsigned n = (unsigned)min((int64_t)rows_per_block, a.rows - r0) * per;
    const uint64_t step = *a.step;
    for (unsigned i = threadIdx.x; i < n; i += 256) {
        const unsigned l = i / per, col = (i - l * per) * 4, left = (unsigned)a.c - col;
        const int64_t r = r0 + l, in = r * a.ld_in + col;
        const T *x = static_cast<const T*>(a.x) + in, *res = static_cast<const T*>(a.res) + in;
        T* y = static_cast<T*>(a.y) + r * a.ld_out + col;
        uint32_t w[4];
        if (W > (int)sizeof(T) && left >= 4) {
            const uint2 xv = load8<W>(x), rv = a.res ? load8<W>(res) : make_uint2(0, 0);
            philox((uint64_t)r * per + col / 4, step, a.key0, a.key1, w);
            const float2 x0 = act::unpack2_u32(xv.x), x1 = act::unpack2_u32(xv.y);
            const float2 g0 = act::unpack2_u32(rv.x), g1 = act::unpack2_u32(rv.y);
            store8<W>(y, make_uint2(act::pack2_u32(dropped<T>(a, w[0], x0.x, g0.x), dropped<T>(a, w[1], x0.y, g0.y)),
                                    act::pack2_u32(dropped<T>(a, w[2], x1.x, g1.x), dropped<T>(a, w[3], x1.y, g1.y))));
            continue;
        }
        float f[4], g[4];
#pragma unroll
        for (unsigned e = 0; e < 4; ++e) {
            f[e] = e < left ? elem_f(x[e]) : 0.f;
            g[e] = e < left && a.res ? elem_f(res[e]) : 0.f;
        }
        philox((uint64_t)r * per + col / 4, step, a.key0, a.key1, w);
#pragma unroll
        for (unsigned e = 0; e < 4; ++e)
            if (e < left) y[e] = elem_from<T>(dropped<T>(a, w[e], f[e], g[e]));
    }
}

__global__ void dropout_advance_kernel(unsigned long long* step) { *step += 1; }

template <class T>
int launch(const DropArgs& a, cudaStream_t st, const char* what)
{
    uintptr_t bits = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.res) | reinterpret_cast<uintptr_t>(a.y);
    bits |= (uintptr_t)(a.ld_in | a.ld_out | a.c) * sizeof(T);
    const bool wide = (bits & 15) == 0;
    const int64_t units = wide ? a.c / (16 / (int)sizeof(T)) : (a.c + 3) / 4;
    const int per = a.rows * units >= (int64_t)sm_count() * 8 * 1024 ? 1024 : 256;  // four units to a thread, or one
    const int rpb = units >= per ? 1 : (int)(per / units);
    const unsigned blocks = (unsigned)((a.rows + rpb - 1) / rpb);
    if (wide)
        dropout_kernel<T><<<blocks, 256, 0, st>>>(a, rpb);
    else if (sizeof(T) == 4 || (bits & 3))
        dropout_any_kernel<T, (int)sizeof(T)><<<blocks, 256, 0, st>>>(a, rpb);
    else if (bits & 7)
        dropout_any_kernel<T, 4><<<blocks, 256, 0, st>>>(a, rpb);
    else if constexpr (sizeof(T) == 2)
        dropout_any_kernel<T, 8><<<blocks, 256, 0, st>>>(a, rpb);
    return launch_check(what);
}

}  // namespace

extern "C" int dbl_dropout_residual(const dbl_dropout_shape* s, const void* x, const void* res, const uint64_t* step,
                                    void* y, void* stream)
{
    const char* w = "dropout_residual";
    if (!s || s->rows < 0 || s->c <= 0) return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0 or c <= 0", w);
    if (s->c > kMaxColumns) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^30 channels or more", w);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", w);
    if (!(s->rate >= 0.f && s->rate < 1.f)) return set_error(DBL_ERR_INVALID, "%s: rate must be in [0, 1)", w);
    if ((s->ld_in && s->ld_in < s->c) || (s->ld_out && s->ld_out < s->c))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", w);
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(x, e) || !aligned_to(res, e) || !aligned_to(y, e) || !aligned_to(step, 8))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (s->rows == 0) return DBL_OK;
    if (!x || !y || !step) return set_error(DBL_ERR_INVALID, "%s: x, y and step must not be NULL", w);
    const int64_t ld_in = s->ld_in ? s->ld_in : s->c, ld_out = s->ld_out ? s->ld_out : s->c;
    if ((y == x || y == res) && ld_in != ld_out)
        return set_error(DBL_ERR_INVALID, "%s: an output in an input's place needs its row stride", w);
    const DropArgs a = {x, res, y, step, s->rows, ld_in, ld_out, s->c, (uint32_t)s->seed, (uint32_t)(s->seed >> 32),
                        (uint32_t)floor((double)s->rate * 4294967296.0), (float)(1.0 / (1.0 - (double)s->rate))};
    cudaStream_t st = as_stream(stream);
    return s->dtype == DBL_F32 ? launch<float>(a, st, w) : launch<act_t>(a, st, w);
}

extern "C" int dbl_dropout_advance(uint64_t* step, void* stream)
{
    if (!step || !aligned_to(step, 8)) return set_error(DBL_ERR_INVALID, "dropout_advance: step is NULL or not aligned to 8 bytes");
    dropout_advance_kernel<<<1, 1, 0, as_stream(stream)>>>(reinterpret_cast<unsigned long long*>(step));
    return launch_check("dropout_advance");
}
