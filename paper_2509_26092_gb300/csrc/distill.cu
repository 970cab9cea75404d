// distill.cu -- distillation loss against a teacher's largest logits, with the labels' cross-entropy, forward and
// backward in one call.
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kThreads = 256;
constexpr int kMaxK = DBL_DISTILL_MAX_K;

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

// One row per block; three passes over its logits: the maximum, the sums of exponentials, the gradient.
template <class T>
__global__ void __launch_bounds__(kThreads) distill_kernel(DistillArgs a)
{
    __shared__ float red[32];
    __shared__ float p[kMaxK];
    __shared__ int cls[kMaxK];
    const float inv_tau = 1.f / a.tau;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + r * a.ld;
        T* dz = a.dz ? static_cast<T*>(a.dz) + r * a.ld_grad : nullptr;
        const float w = a.weight ? a.weight[r] : 1.f / (float)a.rows;
        const int lab = a.labels && a.alpha < 1.f ? a.labels[r] : -1;  // a term of weight 0 is absent
        const bool given = lab >= 0 && lab < a.v;
        // the teacher's distribution
        float tm = -INFINITY;
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            const int c = a.cls[r * a.k + j];
            const float t = a.top[r * a.k + j];
            const bool there = c >= 0 && c < a.v && t != -INFINITY && a.alpha > 0.f;
            cls[j] = there ? c : -1;
            p[j] = there ? t : -INFINITY;
            if (there) tm = fmaxf(tm, t);
        }
        const bool some = __syncthreads_or([&] {
            for (int j = threadIdx.x; j < a.k; j += kThreads)
                if (cls[j] >= 0) return 1;
            return 0;
        }());
        if (w == 0.f || (!some && !given)) {
            if (threadIdx.x == 0) a.row_loss[r] = 0.f;
            if (dz)
                for (int i = threadIdx.x; i < a.v; i += kThreads) dz[i] = elem_from<T>(0.f);
            __syncthreads();
            continue;
        }
        tm = block_max(tm, red);
        float ts = 0.f;
        for (int j = threadIdx.x; j < a.k; j += kThreads) ts += cls[j] >= 0 ? expf((p[j] - tm) * inv_tau) : 0.f;
        ts = block_sum(ts, red);
        const float log_ts = logf(ts);
        // the student's
        float m = -INFINITY;
        for (int i = threadIdx.x; i < a.v; i += kThreads) m = fmaxf(m, elem_f(z[i]));
        m = block_max(m, red);
        float s1 = 0.f, st = 0.f;
        for (int i = threadIdx.x; i < a.v; i += kThreads) {
            const float d = elem_f(z[i]) - m;
            st += __expf(d * inv_tau);
            s1 += __expf(d);
        }
        s1 = block_sum(s1, red);
        st = block_sum(st, red);
        const float log_st = logf(st);
        float loss = 0.f;
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            if (cls[j] < 0) continue;
            const float lp = (p[j] - tm) * inv_tau - log_ts, pj = expf(lp);
            if (pj != 0.f) loss += pj * (lp - ((elem_f(z[cls[j]]) - m) * inv_tau - log_st));
        }
        loss = block_sum(loss, red) * (a.alpha * a.tau * a.tau);
        if (given) loss += (1.f - a.alpha) * (logf(s1) - (elem_f(z[lab]) - m));
        if (threadIdx.x == 0) a.row_loss[r] = loss;
        if (!dz) continue;
        const float f = a.scale ? w * *a.scale : w;
        const float ft = some ? f * a.alpha * a.tau / st : 0.f, f1 = given ? f * (1.f - a.alpha) / s1 : 0.f;
        auto grad = [&](float d) {
            float g = 0.f;
            if (some) g = ft * __expf(d * inv_tau);
            if (given) g = fmaf(f1, __expf(d), g);
            return g;
        };
        // entries of the teacher's and the label: their gradients are taken before the row may be overwritten
        float fix[kMaxK / kThreads], fix_lab = 0.f;
#pragma unroll
        for (int q = 0; q < kMaxK / kThreads; ++q) {
            const int j = threadIdx.x + q * kThreads;
            fix[q] = 0.f;
            if (j >= a.k || cls[j] < 0) continue;
            float pj = 0.f;
            for (int i = 0; i < a.k; ++i)
                if (cls[i] == cls[j]) pj += expf((p[i] - tm) * inv_tau - log_ts);
            fix[q] = grad(elem_f(z[cls[j]]) - m) - f * a.alpha * a.tau * pj - (cls[j] == lab ? f * (1.f - a.alpha) : 0.f);
        }
        bool lab_apart = given;
        for (int i = 0; i < a.k && lab_apart; ++i) lab_apart = cls[i] != lab;
        if (lab_apart) fix_lab = grad(elem_f(z[lab]) - m) - f * (1.f - a.alpha);
        __syncthreads();
        for (int i = threadIdx.x; i < a.v; i += kThreads) dz[i] = elem_from<T>(grad(elem_f(z[i]) - m));
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kMaxK / kThreads; ++q) {
            const int j = threadIdx.x + q * kThreads;
            if (j < a.k && cls[j] >= 0) dz[cls[j]] = elem_from<T>(fix[q]);
        }
        if (lab_apart && threadIdx.x == 0) dz[lab] = elem_from<T>(fix_lab);
        __syncthreads();
    }
}

// loss = sum of weight*row_loss, in one block and a fixed order
__global__ void __launch_bounds__(1024) distill_loss_kernel(const float* row_loss, const float* weight, int64_t rows,
                                                           float* loss)
{
    __shared__ float red[32];
    float s = 0.f;
    for (int64_t r = threadIdx.x; r < rows; r += 1024) s += weight ? weight[r] * row_loss[r] : row_loss[r];
    s = block_sum(s, red);
    if (threadIdx.x == 0) *loss = weight ? s : s / (float)rows;
}

}  // namespace

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
    const int grid = (int)std::min<int64_t>(s->rows, 1 << 20);
    if (s->dtype == DBL_F32)
        distill_kernel<float><<<grid, kThreads, 0, st>>>(a);
    else
        distill_kernel<act_t><<<grid, kThreads, 0, st>>>(a);
    int rc = launch_check(w);
    if (rc != DBL_OK || !loss) return rc;
    distill_loss_kernel<<<1, 1024, 0, st>>>(row_loss, row_weight, s->rows, loss);
    return launch_check("distill_fwd_bwd loss");
}
