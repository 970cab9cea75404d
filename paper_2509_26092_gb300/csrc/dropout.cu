// dropout.cu -- dropout over tokens with the residual addition, the mask drawn from a counter-based generator
// (Philox4x32-10: Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).
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

// One block of four channels to a thread, element by element.
template <class T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a)
{
    const int per = (a.c + 3) / 4;
    const int64_t total = a.rows * per;
    const uint64_t step = *a.step;
    for (int64_t b = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; b < total; b += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = b / per;
        const int col = (int)(b - row * per) * 4;
        uint32_t w[4];
        philox((uint64_t)b, step, a.key0, a.key1, w);
        const T* x = static_cast<const T*>(a.x) + row * a.ld_in + col;
        const T* res = a.res ? static_cast<const T*>(a.res) + row * a.ld_in + col : nullptr;
        T* y = static_cast<T*>(a.y) + row * a.ld_out + col;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < a.c) {
                const float v = w[i] >= a.threshold ? elem_f(x[i]) : 0.f;
                y[i] = elem_from<T>(fmaf(v, a.scale, res ? elem_f(res[i]) : 0.f));
            }
    }
}

__global__ void dropout_advance_kernel(unsigned long long* step) { *step += 1; }

template <class T>
int launch(const DropArgs& a, cudaStream_t st, const char* what)
{
    const int64_t total = a.rows * ((a.c + 3) / 4), cap = (int64_t)sm_count() * 8;
    int64_t blocks = (total + 255) / 256;
    if (blocks > cap) blocks = cap;
    dropout_kernel<T><<<(unsigned)blocks, 256, 0, st>>>(a);
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
