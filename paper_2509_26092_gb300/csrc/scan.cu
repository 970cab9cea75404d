// scan.cu -- gated linear recurrence along a sequence, h_i = a_i*h_{i-1} + (1 - a_i)*x_i with a = 1/(1 + exp(-gate)),
// forward and backward.
#include <math.h>

#include <algorithm>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kThreads = 128;
constexpr int kChunk = DBL_SCAN_CHUNK;

struct ScanArgs {
    const void *x, *gate, *dh;
    const float *h0;      // backward: dh_last
    const int32_t* lengths;
    void *h;              // backward: dx
    void *dgate;
    float *last;          // backward: dh0
    float *states;
    int64_t ld_x, ld_h;
    int n, t, c;
};

// a = sigma(z) and 1 - a, both to full relative precision: with e = exp(-|z|) the larger is 1/(1 + e), the
// smaller e/(1 + e).
__device__ __forceinline__ void gates(float z, float& a, float& na)
{
    const float e = __expf(-fabsf(z));
    const float big = __fdividef(1.f, 1.f + e), small = e * big;
    a = z >= 0.f ? big : small;
    na = z >= 0.f ? small : big;
}

__device__ __forceinline__ int length_of(const ScanArgs& a, int64_t b)
{
    return a.lengths ? min(max(a.lengths[b], 0), a.t) : a.t;
}

// One thread per channel of a sequence, step by step.
template <class T>
__global__ void __launch_bounds__(kThreads) scan_fwd_kernel(ScanArgs a)
{
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= (int64_t)a.n * a.c) return;
    const int64_t b = id / a.c;
    const int ch = (int)(id - b * a.c), len = length_of(a, b);
    const int chunks = (a.t + kChunk - 1) / kChunk;
    float h = a.h0 ? a.h0[id] : 0.f;
    for (int i = 0; i < a.t; ++i) {
        if (a.states && i % kChunk == 0) a.states[(b * chunks + i / kChunk) * a.c + ch] = h;
        const int64_t row = b * a.t + i;
        float out = 0.f;
        if (i < len) {
            float s, r;
            gates(elem_f(static_cast<const T*>(a.gate)[row * a.ld_x + ch]), s, r);
            out = h = fmaf(s, h, r * elem_f(static_cast<const T*>(a.x)[row * a.ld_x + ch]));
        }
        static_cast<T*>(a.h)[row * a.ld_h + ch] = elem_from<T>(out);
    }
    if (a.last) a.last[id] = h;
}

template <class T>
__global__ void __launch_bounds__(kThreads) scan_bwd_kernel(ScanArgs a)
{
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= (int64_t)a.n * a.c) return;
    const int64_t b = id / a.c;
    const int ch = (int)(id - b * a.c), len = length_of(a, b);
    const int chunks = (a.t + kChunk - 1) / kChunk;
    const T *x = static_cast<const T*>(a.x) + b * a.t * a.ld_x + ch, *z = static_cast<const T*>(a.gate) + b * a.t * a.ld_x + ch;
    T *dx = static_cast<T*>(a.h) + b * a.t * a.ld_x + ch, *dz = static_cast<T*>(a.dgate) + b * a.t * a.ld_x + ch;
    const T* dh = static_cast<const T*>(a.dh) + b * a.t * a.ld_h + ch;
    float q = a.h0 ? a.h0[id] : 0.f;  // a_{i+1} * G_{i+1}, what reaches h_i from the steps after it
    for (int j = chunks - 1; j >= 0; --j) {
        const int lo = j * kChunk, hi = min(lo + kChunk, a.t);
        float prev[kChunk];
        float h = a.states[(b * chunks + j) * a.c + ch];
        for (int i = lo; i < min(hi, len); ++i) {
            float s, r;
            prev[i - lo] = h;
            gates(elem_f(z[i * a.ld_x]), s, r);
            h = fmaf(s, h, r * elem_f(x[i * a.ld_x]));
        }
        for (int i = hi - 1; i >= lo; --i) {
            float vx = 0.f, vz = 0.f;
            if (i < len) {
                float s, r;
                gates(elem_f(z[i * a.ld_x]), s, r);
                const float g = elem_f(dh[i * a.ld_h]) + q;
                vx = r * g;
                vz = vx * (prev[i - lo] - elem_f(x[i * a.ld_x])) * s;
                q = s * g;
            }
            dx[i * a.ld_x] = elem_from<T>(vx);
            dz[i * a.ld_x] = elem_from<T>(vz);
        }
    }
    if (a.last) a.last[id] = q;
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

int64_t blocks_of(const dbl_scan_shape* s) { return ((int64_t)s->n * s->c + kThreads - 1) / kThreads; }

int pass_through(const dbl_scan_shape* s, const float* from, float* to, cudaStream_t st)
{
    if (!to || from == to) return DBL_OK;
    scan_copy_kernel<<<(unsigned)blocks_of(s), kThreads, 0, st>>>(from, to, (int64_t)s->n * s->c);
    return launch_check("gated_scan");
}

}  // namespace

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
    if (s->dtype == DBL_F32)
        scan_fwd_kernel<float><<<(unsigned)blocks_of(s), kThreads, 0, st>>>(a);
    else
        scan_fwd_kernel<act_t><<<(unsigned)blocks_of(s), kThreads, 0, st>>>(a);
    return launch_check("gated_scan_fwd");
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
    if (s->dtype == DBL_F32)
        scan_bwd_kernel<float><<<(unsigned)blocks_of(s), kThreads, 0, st>>>(a);
    else
        scan_bwd_kernel<act_t><<<(unsigned)blocks_of(s), kThreads, 0, st>>>(a);
    return launch_check("gated_scan_bwd");
}

}  // extern "C"
