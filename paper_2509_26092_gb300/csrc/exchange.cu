// exchange.cu -- tokens to their experts' groups and back: rows copied to the slots of their entries, the weighted sum
// of the entries' rows, and the gradients of both.
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

// A block to a token.
template <class T>
__global__ void __launch_bounds__(256) expert_scatter_kernel(const ExchangeArgs a)
{
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.a) + r * a.ld_rows;
        for (int j = 0; j < a.k; ++j) {
            const int64_t s = slot_of(a, r * a.k + j);
            if (s < 0) continue;
            T* o = static_cast<T*>(a.out) + s * a.ld_grouped;
            for (int i = threadIdx.x; i < a.c; i += blockDim.x) o[i] = x[i];
        }
    }
}

template <class T>
__global__ void __launch_bounds__(256) expert_combine_kernel(const ExchangeArgs a)
{
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        T* o = static_cast<T*>(a.out) + r * a.ld_rows;
        const T* res = a.b ? static_cast<const T*>(a.b) + r * a.ld_rows : nullptr;
        for (int i = threadIdx.x; i < a.c; i += blockDim.x) {
            float sum = 0.f;
            for (int j = 0; j < a.k; ++j) {
                const int64_t s = slot_of(a, r * a.k + j);
                const float w = a.weights ? a.weights[r * a.k + j] : 1.f;
                sum = fmaf(w, s < 0 ? 0.f : elem_f(static_cast<const T*>(a.a)[s * a.ld_grouped + i]), sum);
            }
            o[i] = elem_from<T>(res ? sum + elem_f(res[i]) : sum);
        }
    }
}

template <class T>
__global__ void __launch_bounds__(256) expert_combine_bwd_kernel(const ExchangeArgs a)
{
    __shared__ float red[32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* d = static_cast<const T*>(a.a) + r * a.ld_rows;
        for (int j = 0; j < a.k; ++j) {
            const int64_t s = slot_of(a, r * a.k + j);
            const float w = a.weights ? a.weights[r * a.k + j] : 1.f;
            float dot = 0.f;
            if (s >= 0) {
                T* o = static_cast<T*>(a.out) + s * a.ld_grouped;
                const T* y = a.dweights ? static_cast<const T*>(a.b) + s * a.ld_grouped : nullptr;
                for (int i = threadIdx.x; i < a.c; i += blockDim.x) {
                    const float v = elem_f(d[i]);
                    if (y) dot = fmaf(v, elem_f(y[i]), dot);
                    o[i] = elem_from<T>(w * v);
                }
            }
            if (!a.dweights) continue;
            dot = block_sum(dot, red);
            if (threadIdx.x == 0) a.dweights[r * a.k + j] = dot;
        }
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

unsigned grid_for(int64_t rows)
{
    const int64_t cap = (int64_t)sm_count() * 8;
    return (unsigned)(rows < cap ? rows : cap);
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
    if (s->dtype == DBL_F32)
        expert_scatter_kernel<float><<<grid_for(s->rows), 256, 0, st>>>(a);
    else
        expert_scatter_kernel<act_t><<<grid_for(s->rows), 256, 0, st>>>(a);
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
    if (s->dtype == DBL_F32)
        expert_combine_kernel<float><<<grid_for(s->rows), 256, 0, st>>>(a);
    else
        expert_combine_kernel<act_t><<<grid_for(s->rows), 256, 0, st>>>(a);
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
    if (s->dtype == DBL_F32)
        expert_combine_bwd_kernel<float><<<grid_for(s->rows), 256, 0, st>>>(a);
    else
        expert_combine_bwd_kernel<act_t><<<grid_for(s->rows), 256, 0, st>>>(a);
    return launch_check(w);
}
