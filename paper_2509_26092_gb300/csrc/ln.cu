// ln.cu -- layer norm over the last dimension, forward (with the residual addition before it) and backward (with
// the skip path's gradient and the sums over rows for gamma and beta).
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kThreads = 256;
constexpr int kMaxParts = 304;  // blocks of rows whose column sums are kept apart

struct LnArgs {
    const void *x, *res, *dy;
    const float *gamma, *beta;
    void *sum, *y;
    float *mean, *invstd;
    int64_t rows, ld_in, ld_out;
    int c;
    float eps;
};

// One row per block, read once per step.
template <class T>
__global__ void __launch_bounds__(kThreads) ln_fwd_kernel(LnArgs a)
{
    __shared__ float red[32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ld_in;
        const T* res = a.res ? static_cast<const T*>(a.res) + r * a.ld_in : nullptr;
        auto at = [&](int i) { return res ? elem_f(x[i]) + elem_f(res[i]) : elem_f(x[i]); };
        float s = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kThreads) s += at(i);
        const float mean = block_sum(s, red) / a.c;
        s = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kThreads) {
            const float d = at(i) - mean;
            s = fmaf(d, d, s);
        }
        const float inv = 1.f / sqrtf(block_sum(s, red) / a.c + a.eps);
        for (int i = threadIdx.x; i < a.c; i += kThreads) {
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

// x: the normalised tensor, res: dskip, y: dx
template <class T>
__global__ void __launch_bounds__(kThreads) ln_bwd_kernel(LnArgs a)
{
    __shared__ float red[32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ld_in;
        const T* dy = static_cast<const T*>(a.dy) + r * a.ld_in;
        const float mean = a.mean[r], inv = a.invstd[r];
        float s0 = 0.f, s1 = 0.f;
        for (int i = threadIdx.x; i < a.c; i += kThreads) {
            const float g = elem_f(dy[i]) * (a.gamma ? a.gamma[i] : 1.f);
            s0 += g;
            s1 = fmaf(g, (elem_f(x[i]) - mean) * inv, s1);
        }
        s0 = block_sum(s0, red) / a.c;
        s1 = block_sum(s1, red) / a.c;
        for (int i = threadIdx.x; i < a.c; i += kThreads) {
            const float g = elem_f(dy[i]) * (a.gamma ? a.gamma[i] : 1.f), h = (elem_f(x[i]) - mean) * inv;
            float d = inv * (g - s0 - h * s1);
            if (a.res) d += elem_f(static_cast<const T*>(a.res)[r * a.ld_in + i]);
            static_cast<T*>(a.y)[r * a.ld_out + i] = elem_from<T>(d);
        }
    }
}

// parts[block][2][c]: each block's sums of dy*xhat and of dy over its rows
template <class T>
__global__ void __launch_bounds__(kThreads) ln_params_kernel(LnArgs a, float* parts)
{
    for (int i = threadIdx.x; i < a.c; i += kThreads) {
        float dg = 0.f, db = 0.f;
        for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
            const float d = elem_f(static_cast<const T*>(a.dy)[r * a.ld_in + i]);
            const float h = (elem_f(static_cast<const T*>(a.x)[r * a.ld_in + i]) - a.mean[r]) * a.invstd[r];
            dg = fmaf(d, h, dg);
            db += d;
        }
        parts[(int64_t)blockIdx.x * 2 * a.c + i] = dg;
        parts[((int64_t)blockIdx.x * 2 + 1) * a.c + i] = db;
    }
}

__global__ void __launch_bounds__(kThreads) ln_params_sum_kernel(const float* parts, int nparts, int c, float* dgamma,
                                                                float* dbeta)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= 2 * (int64_t)c) return;
    float s = 0.f;
    for (int p = 0; p < nparts; ++p) s += parts[(int64_t)p * 2 * c + i];
    (i < c ? dgamma : dbeta - c)[i] = s;
}

int check(const dbl_ln_shape* s, const char* what)
{
    if (!s || s->rows < 0 || s->c <= 0) return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0 or c <= 0", what);
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

int parts_of(const dbl_ln_shape* s) { return (int)std::min<int64_t>(std::max<int64_t>(s->rows, 1), kMaxParts); }

}  // namespace

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
    const int grid = (int)std::min<int64_t>(s->rows, 1 << 20);
    if (s->dtype == DBL_F32)
        ln_fwd_kernel<float><<<grid, kThreads, 0, as_stream(stream)>>>(a);
    else
        ln_fwd_kernel<act_t><<<grid, kThreads, 0, as_stream(stream)>>>(a);
    return launch_check("layer_norm_fwd");
}

size_t dbl_layer_norm_workspace_bytes(const dbl_ln_shape* s)
{
    if (check(s, "layer_norm_workspace_bytes") != DBL_OK) return 0;
    return (size_t)parts_of(s) * 2 * s->c * sizeof(float);
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
    if (dgamma) {
        if (!ws || ws_bytes < dbl_layer_norm_workspace_bytes(s))
            return set_error(DBL_ERR_WORKSPACE, "layer_norm_bwd: workspace too small");
        if (!aligned16(ws)) return set_error(DBL_ERR_INVALID, "layer_norm_bwd: workspace must be 16-byte aligned");
    }
    cudaStream_t st = as_stream(stream);
    LnArgs a = args(s);
    a.x = x, a.res = dskip, a.dy = dy, a.gamma = gamma, a.y = dx;
    a.mean = const_cast<float*>(save_mean), a.invstd = const_cast<float*>(save_invstd);
    if (s->rows > 0) {
        const int grid = (int)std::min<int64_t>(s->rows, 1 << 20);
        if (s->dtype == DBL_F32)
            ln_bwd_kernel<float><<<grid, kThreads, 0, st>>>(a);
        else
            ln_bwd_kernel<act_t><<<grid, kThreads, 0, st>>>(a);
        rc = launch_check("layer_norm_bwd");
    }
    if (rc != DBL_OK || !dgamma) return rc;
    const int np = parts_of(s);
    float* parts = static_cast<float*>(ws);
    if (s->dtype == DBL_F32)
        ln_params_kernel<float><<<np, kThreads, 0, st>>>(a, parts);
    else
        ln_params_kernel<act_t><<<np, kThreads, 0, st>>>(a, parts);
    rc = launch_check("layer_norm_bwd");
    if (rc != DBL_OK) return rc;
    ln_params_sum_kernel<<<(int)((2 * (int64_t)s->c + kThreads - 1) / kThreads), kThreads, 0, st>>>(parts, np, s->c, dgamma,
                                                                                                dbeta);
    return launch_check("layer_norm_bwd sums");
}

}  // extern "C"
