// grouped.cu -- matrix products of each group's rows with the group's own weights (a layer of experts): forward, data
// gradient and weight gradient, the groups' bounds on the device.
#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxGroups = DBL_GROUPED_MAX_GROUPS;

struct GroupedArgs {
    const act_t* a;     // x; dy; x
    const act_t* b;     // w; w; dy
    const act_t* mask;  // dgrad, or nullptr
    void* out;          // y; dx; dw
    const int32_t* offsets;
    int64_t rows, ld_in, ld_out;
    int groups, n_in, n_out, relu, accumulate;
};

// The groups' bounds into off[0..groups], in order and inside the tensors whatever the device memory holds.  By one warp.
__device__ __forceinline__ void load_offsets(const int32_t* offsets, int groups, int64_t rows, int* off, int lane)
{
    int before = 0;
    for (int i0 = 0; i0 <= groups; i0 += 32) {
        const int i = i0 + lane;
        int v = i <= groups ? offsets[i] : 0;
        v = max(0, (int)min((int64_t)v, rows));
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v = max(v, u);
        }
        v = max(v, before);
        if (i <= groups) off[i] = v;
        before = __shfl_sync(0xffffffffu, v, 31);
    }
}

constexpr int kTile = 64, kStep = 16;

// 64 x 64 outputs to a block, 4 x 4 to a thread, on the CUDA cores.  PASS 0: rows of x and of w_e; 1: rows of dy, columns of
// w_e; 2: columns of dy and of x, over the group's rows.
template <int PASS>
__global__ void __launch_bounds__(256) grouped_kernel(const GroupedArgs a)
{
    __shared__ int off[kMaxGroups + 1];
    __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
    if (threadIdx.x < 32) load_offsets(a.offsets, a.groups, a.rows, off, threadIdx.x);
    __syncthreads();
    int group = 0, row0 = 0, row1 = 0;
    if (PASS == 2) {
        group = blockIdx.z;
        row0 = off[group], row1 = off[group + 1];
    } else {
        int tile = blockIdx.y;
        for (; group < a.groups; ++group) {
            const int n = (off[group + 1] - off[group] + kTile - 1) / kTile;
            if (tile < n) break;
            tile -= n;
        }
        if (group == a.groups) return;
        row0 = off[group] + tile * kTile;
        row1 = off[group + 1];
    }
    const int col0 = blockIdx.x * kTile, out0 = blockIdx.y * kTile;  // out0: wgrad's rows
    const int depth = PASS == 0 ? a.n_in : PASS == 1 ? a.n_out : row1 - row0;
    const act_t* w = a.b + (PASS == 2 ? 0 : (int64_t)group * a.n_out * a.n_in);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < depth; k0 += kStep) {
        for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
            const int m = PASS == 2 ? i % kTile : i / kStep, k = PASS == 2 ? i / kTile : i % kStep;
            float v = 0.f;
            if (k0 + k < depth) {
                if (PASS == 0 && row0 + m < row1) v = elem_f(a.a[(int64_t)(row0 + m) * a.ld_in + k0 + k]);
                if (PASS == 1 && row0 + m < row1) v = elem_f(a.a[(int64_t)(row0 + m) * a.ld_out + k0 + k]);
                if (PASS == 2 && out0 + m < a.n_out) v = elem_f(a.b[(int64_t)(row0 + k0 + k) * a.ld_out + out0 + m]);
            }
            sa[k][m] = v;
            const int n = PASS == 0 ? i / kStep : i % kTile, l = PASS == 0 ? i % kStep : i / kTile;
            v = 0.f;
            if (k0 + l < depth) {
                if (PASS == 0 && col0 + n < a.n_out) v = elem_f(w[(int64_t)(col0 + n) * a.n_in + k0 + l]);
                if (PASS == 1 && col0 + n < a.n_in) v = elem_f(w[(int64_t)(k0 + l) * a.n_in + col0 + n]);
                if (PASS == 2 && col0 + n < a.n_in) v = elem_f(a.a[(int64_t)(row0 + k0 + l) * a.ld_in + col0 + n]);
            }
            sb[l][n] = v;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kStep; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = ty + 16 * i, n = col0 + tx + 16 * j;
            float v = acc[i][j];
            if (PASS == 2) {
                if (out0 + m >= a.n_out || n >= a.n_in) continue;
                float* o = static_cast<float*>(a.out) + ((int64_t)group * a.n_out + out0 + m) * a.n_in + n;
                *o = a.accumulate ? *o + v : v;
                continue;
            }
            if (row0 + m >= row1 || n >= (PASS == 0 ? a.n_out : a.n_in)) continue;
            const int64_t ld = PASS == 0 ? a.ld_out : a.ld_in;
            const int64_t at = (int64_t)(row0 + m) * ld + n;
            if (PASS == 0 && a.relu && v < 0.f) v = 0.f;
            if (PASS == 1 && a.mask && !(elem_f(a.mask[at]) > 0.f)) v = 0.f;
            static_cast<act_t*>(a.out)[at] = elem_from<act_t>(v);
        }
}

int check(const dbl_grouped_shape* s, const char* w)
{
    if (!s || s->rows < 0 || s->groups <= 0 || s->n_in <= 0 || s->n_out <= 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0, groups <= 0, n_in <= 0 or n_out <= 0", w);
    if (s->groups > kMaxGroups) return set_error(DBL_ERR_UNSUPPORTED, "%s: %d groups, at most %d", w, s->groups, kMaxGroups);
    if (s->rows > 1 << 30) return set_error(DBL_ERR_UNSUPPORTED, "%s: more than 2^30 rows", w);
    if (s->n_in >= 1 << 24 || s->n_out >= 1 << 24) return set_error(DBL_ERR_UNSUPPORTED, "%s: rows of 2^24 columns or more", w);
    if (s->n_in % 8 || s->n_out % 8) return set_error(DBL_ERR_INVALID, "%s: n_in and n_out must be multiples of 8", w);
    if ((s->ld_in && s->ld_in < s->n_in) || (s->ld_out && s->ld_out < s->n_out))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", w);
    if (s->ld_in % 8 || s->ld_out % 8) return set_error(DBL_ERR_INVALID, "%s: row strides must be multiples of 8", w);
    return DBL_OK;
}

template <int PASS>
int run(const dbl_grouped_shape* s, const void* a, const void* b, const int32_t* offsets, const void* mask, void* out,
        int accumulate, void* stream, const char* w)
{
    const GroupedArgs g = {static_cast<const act_t*>(a), static_cast<const act_t*>(b), static_cast<const act_t*>(mask), out,
                           offsets, s->rows, s->ld_in ? s->ld_in : s->n_in, s->ld_out ? s->ld_out : s->n_out, s->groups,
                           s->n_in, s->n_out, s->relu != 0, accumulate};
    const int cols = PASS == 0 ? s->n_out : s->n_in;
    const dim3 grid((cols + kTile - 1) / kTile,
                    PASS == 2 ? (s->n_out + kTile - 1) / kTile : (unsigned)(s->rows / kTile + s->groups),
                    PASS == 2 ? s->groups : 1);
    grouped_kernel<PASS><<<grid, 256, 0, as_stream(stream)>>>(g);
    return launch_check(w);
}

}  // namespace

extern "C" size_t dbl_grouped_workspace_bytes(const dbl_grouped_shape* s, int pass)
{
    (void)pass;
    (void)check(s, "grouped_workspace_bytes");
    return 0;
}

extern "C" int dbl_grouped_fwd(const dbl_grouped_shape* s, const void* x, const void* wt, const int32_t* offsets, void* y,
                               void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_fwd";
    (void)ws, (void)ws_bytes;
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned16(x) || !aligned16(wt) || !aligned16(y) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a tensor is not 16-byte aligned, or offsets not to 4 bytes", w);
    if (s->rows == 0) return DBL_OK;
    if (!x || !wt || !offsets || !y) return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    return run<0>(s, x, wt, offsets, nullptr, y, 0, stream, w);
}

extern "C" int dbl_grouped_dgrad(const dbl_grouped_shape* s, const void* dy, const void* wt, const int32_t* offsets,
                                 const void* mask, void* dx, void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_dgrad";
    (void)ws, (void)ws_bytes;
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned16(dy) || !aligned16(wt) || !aligned16(mask) || !aligned16(dx) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a tensor is not 16-byte aligned, or offsets not to 4 bytes", w);
    if (s->rows == 0) return DBL_OK;
    if (!dy || !wt || !offsets || !dx) return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    return run<1>(s, dy, wt, offsets, mask, dx, 0, stream, w);
}

extern "C" int dbl_grouped_wgrad(const dbl_grouped_shape* s, const void* x, const void* dy, const int32_t* offsets, float* dw,
                                 int accumulate, void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_wgrad";
    (void)ws, (void)ws_bytes;
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned16(x) || !aligned16(dy) || !aligned16(dw) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a tensor is not 16-byte aligned, or offsets not to 4 bytes", w);
    if (!dw) return set_error(DBL_ERR_INVALID, "%s: dw must not be NULL", w);
    if (s->rows == 0) {
        if (accumulate) return DBL_OK;
        return cuda_check(cudaMemsetAsync(dw, 0, (size_t)s->groups * s->n_in * s->n_out * sizeof(float), as_stream(stream)), w);
    }
    if (!x || !dy || !offsets) return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    return run<2>(s, x, dy, offsets, nullptr, dw, accumulate != 0, stream, w);
}
