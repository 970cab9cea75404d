// route.cu -- the router of a layer of experts: the k experts of every token and their weights, the tokens' places
// grouped by expert, and the gradient of the logits.
#include <math.h>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxExperts = DBL_ROUTE_MAX_EXPERTS, kMaxK = DBL_ROUTE_MAX_K;
constexpr int kMaxBlocks = 256;  // that count entries; the workspace holds one count for each block and expert

struct RouteArgs {
    const void* logits;
    const float* bias;
    const float* row_weight;
    int32_t* chosen;
    float* weights;
    int32_t* slots;
    int32_t* offsets;
    int32_t* counts;  // [blocks][experts]
    int64_t rows, ld;
    int experts, k, normalise, rows_per_block;
};

// A number that orders keys as integers, 0 for those that are never chosen.
__device__ __forceinline__ uint32_t rank_of(float key)
{
    if (!(key > -INFINITY)) return 0u;  // -infinity and NaN
    const uint32_t u = __float_as_uint(key + 0.f);  // -0 as 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// A warp to a row; every lane has the experts lane, lane + 32, ...
template <class T>
__device__ __forceinline__ void choose_row(const RouteArgs& a, int64_t r, int lane, int32_t* chosen, float* weights)
{
    const T* z = static_cast<const T*>(a.logits) + r * a.ld;
    const bool dead = a.row_weight && a.row_weight[r] == 0.f;
    float peak = -INFINITY, sum = 0.f;
    bool bad = false;
    if (!dead) {
        for (int e = lane; e < a.experts; e += 32) {
            const float v = elem_f(z[e]);
            bad |= !(v < INFINITY);
            peak = fmaxf(peak, v);
        }
        peak = warp_max(peak);
        bad = __any_sync(0xffffffffu, bad);
        if (!a.normalise && !bad && peak > -INFINITY) {
            for (int e = lane; e < a.experts; e += 32) sum += expf(elem_f(z[e]) - peak);
            sum = warp_sum(sum);
        }
    }
    if (dead || bad) {
        for (int j = lane; j < a.k; j += 32) {
            chosen[j] = -1;
            weights[j] = dead ? 0.f : NAN;
        }
        return;
    }
    uint32_t last = 0xffffffffu;
    int last_e = -1, mine = -1;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = 0;
        int best_e = a.experts;
        for (int e = lane; e < a.experts; e += 32) {
            const uint32_t v = rank_of(elem_f(z[e]) + (a.bias ? a.bias[e] : 0.f));
            const bool after = v < last || (v == last && e > last_e);  // what was chosen before comes before in this order
            if (after && v > best) best = v, best_e = e;
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        const int e = (int)__reduce_min_sync(0xffffffffu, best == top && top ? (unsigned)best_e : (unsigned)a.experts);
        if (top == 0) break;
        last = top;
        last_e = e;
        if (lane == j) mine = e;
    }
    const float v = mine >= 0 ? elem_f(z[mine]) : -INFINITY;
    if (a.normalise) {
        peak = warp_max(v);
        sum = warp_sum(mine >= 0 ? expf(v - peak) : 0.f);
    }
    if (lane < a.k) {
        chosen[lane] = mine;
        weights[lane] = mine >= 0 ? expf(v - peak) / sum : 0.f;
    }
}

// Counts the entries of each expert in the block's rows.
template <class T>
__global__ void __launch_bounds__(256) route_choose_kernel(const RouteArgs a)
{
    __shared__ int count[kMaxExperts];
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) count[e] = 0;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
    for (int64_t r = r0 + warp; r < r1; r += blockDim.x / 32) {
        choose_row<T>(a, r, lane, a.chosen + r * a.k, a.weights + r * a.k);
        __syncwarp();
        const int e = lane < a.k ? a.chosen[r * a.k + lane] : -1;
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) a.counts[blockIdx.x * a.experts + e] = count[e];
}

// Gives every entry its place: the entries of smaller experts, those of the same expert in the blocks before, and those
// before it in this block.
__global__ void __launch_bounds__(256) route_place_kernel(const RouteArgs a)
{
    __shared__ int at[kMaxExperts];          // the next place of an expert's entry
    __shared__ int part[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int running = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 256) {
        const int e = e0 + threadIdx.x;
        int before = 0, all = 0;
        if (e < a.experts)
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int n = a.counts[b * a.experts + e];
                if (b < (int)blockIdx.x) before += n;
                all += n;
            }
        int sum = all;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) part[warp] = sum;
        __syncthreads();
        int base = running;
        for (int w = 0; w < warp; ++w) base += part[w];
        const int end = base + sum;
        if (e < a.experts) {
            at[e] = end - all + before;
            if (blockIdx.x == 0) {
                if (e == 0) a.offsets[0] = 0;
                a.offsets[e + 1] = end;
            }
        }
        for (int w = 0; w < 8; ++w) running += part[w];
        __syncthreads();
    }
    if (warp) return;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
    for (int64_t i0 = r0 * a.k; i0 < r1 * a.k; i0 += 32) {
        const bool in = i0 + lane < r1 * a.k;
        const int e = in ? a.chosen[i0 + lane] : -1;
        const uint32_t same = __match_any_sync(0xffffffffu, e);
        const int rank = __popc(same & ((1u << lane) - 1));
        const int place = e >= 0 ? at[e] + rank : -1;
        __syncwarp();
        if (e >= 0 && rank == 0) at[e] += __popc(same);
        __syncwarp();
        if (in) a.slots[i0 + lane] = place;
    }
}

// A warp to a row: first what every expert gets, then the entries' experts.
template <class T>
__global__ void __launch_bounds__(256) route_bwd_kernel(const void* logits, const int32_t* chosen, const float* weights,
                                                        const float* dweights, void* dlogits, int64_t rows, int experts,
                                                        int k, int normalise, int64_t ld, int64_t ld_grad)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t r = (int64_t)blockIdx.x * 8 + warp; r < rows; r += (int64_t)gridDim.x * 8) {
        const T* z = static_cast<const T*>(logits) + r * ld;
        T* dz = static_cast<T*>(dlogits) + r * ld_grad;
        int e = lane < k ? chosen[r * k + lane] : -1;
        if (e >= experts) e = -1;
        const float w = lane < k ? weights[r * k + lane] : 0.f;
        const bool nan = __any_sync(0xffffffffu, isnan(w)), some = __any_sync(0xffffffffu, e >= 0);
        const float wd = e >= 0 ? w * dweights[r * k + lane] : 0.f;
        const float d = warp_sum(wd);
        if (nan || !some || normalise) {
            const T fill = elem_from<T>(nan ? NAN : 0.f);
            for (int i = lane; i < experts; i += 32) dz[i] = fill;
            if (nan || !some) continue;
        }
        float peak = -INFINITY, sum = 0.f;
        if (!normalise) {
            for (int i = lane; i < experts; i += 32) peak = fmaxf(peak, elem_f(z[i]));
            peak = warp_max(peak);
            for (int i = lane; i < experts; i += 32) sum += expf(elem_f(z[i]) - peak);
            sum = warp_sum(sum);
            for (int i = lane; i < experts; i += 32) dz[i] = elem_from<T>(-d * (expf(elem_f(z[i]) - peak) / sum));
        }
        float total = 0.f;  // of the row's entries of this lane's expert
        for (int i = 0; i < k; ++i) {
            const int other = __shfl_sync(0xffffffffu, e, i);
            const float v = __shfl_sync(0xffffffffu, normalise ? wd - w * d : wd, i);
            if (other == e) total += v;
        }
        __syncwarp();
        if (e >= 0) dz[e] = elem_from<T>(normalise ? total : total - d * (expf(elem_f(z[e]) - peak) / sum));
    }
}

int check(const dbl_route_shape* s, const char* w)
{
    if (!s || s->rows < 0 || s->experts <= 0 || s->k <= 0)
        return set_error(DBL_ERR_INVALID, "%s: null shape, rows < 0, experts <= 0 or k <= 0", w);
    if (s->k > s->experts) return set_error(DBL_ERR_INVALID, "%s: k = %d of %d experts", w, s->k, s->experts);
    if (s->experts > kMaxExperts || s->k > kMaxK)
        return set_error(DBL_ERR_UNSUPPORTED, "%s: at most %d experts and k = %d", w, kMaxExperts, kMaxK);
    if (s->rows > INT32_MAX / s->k) return set_error(DBL_ERR_UNSUPPORTED, "%s: 2^31 entries or more", w);
    if (!elem_dtype_ok(s->dtype)) return set_error(DBL_ERR_INVALID, "%s: dtype must be DBL_F32 or DBL_BF16", w);
    if ((s->ld && s->ld < s->experts) || (s->ld_grad && s->ld_grad < s->experts))
        return set_error(DBL_ERR_INVALID, "%s: a row stride is shorter than a row", w);
    return DBL_OK;
}

// Rows of a block, and how many blocks there are.
int plan_blocks(const dbl_route_shape* s, int* rows_per_block)
{
    int64_t per = (s->rows + kMaxBlocks - 1) / kMaxBlocks;
    if (per < 16) per = 16;
    *rows_per_block = (int)per;
    return (int)((s->rows + per - 1) / per);
}

}  // namespace

extern "C" size_t dbl_route_workspace_bytes(const dbl_route_shape* s)
{
    if (check(s, "route_workspace_bytes") != DBL_OK) return 0;
    int per;
    return (size_t)plan_blocks(s, &per) * s->experts * sizeof(int32_t);
}

extern "C" int dbl_route_fwd(const dbl_route_shape* s, const void* logits, const float* select_bias, const float* row_weight,
                             int32_t* chosen, float* weights, int32_t* slots, int32_t* offsets, void* ws, size_t ws_bytes,
                             void* stream)
{
    const char* w = "route_fwd";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned_to(logits, elem_bytes(s->dtype)) || !aligned_to(select_bias, 4) || !aligned_to(row_weight, 4) ||
        !aligned_to(chosen, 4) || !aligned_to(weights, 4) || !aligned_to(slots, 4) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (!offsets) return set_error(DBL_ERR_INVALID, "%s: offsets must not be NULL", w);
    cudaStream_t st = as_stream(stream);
    if (s->rows == 0) return cuda_check(cudaMemsetAsync(offsets, 0, (s->experts + 1) * sizeof(int32_t), st), w);
    if (!logits || !chosen || !weights || !slots)
        return set_error(DBL_ERR_INVALID, "%s: logits, chosen, weights and slots must not be NULL", w);
    if (ws_bytes < dbl_route_workspace_bytes(s) || !ws) return set_error(DBL_ERR_WORKSPACE, "%s: workspace too small", w);
    if (!aligned16(ws)) return set_error(DBL_ERR_INVALID, "%s: the workspace is not 16-byte aligned", w);
    int per;
    const int blocks = plan_blocks(s, &per);
    const RouteArgs a = {logits, select_bias, row_weight, chosen, weights, slots, offsets, static_cast<int32_t*>(ws), s->rows,
                         s->ld ? s->ld : s->experts, s->experts, s->k, s->normalise != 0, per};
    if (s->dtype == DBL_F32)
        route_choose_kernel<float><<<blocks, 256, 0, st>>>(a);
    else
        route_choose_kernel<act_t><<<blocks, 256, 0, st>>>(a);
    if ((rc = launch_check(w)) != DBL_OK) return rc;
    route_place_kernel<<<blocks, 256, 0, st>>>(a);
    return launch_check("route_fwd place");
}

extern "C" int dbl_route_bwd(const dbl_route_shape* s, const void* logits, const int32_t* chosen, const float* weights,
                             const float* dweights, void* dlogits, void* stream)
{
    const char* w = "route_bwd";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    const size_t e = elem_bytes(s->dtype);
    if (!aligned_to(logits, e) || !aligned_to(dlogits, e) || !aligned_to(chosen, 4) || !aligned_to(weights, 4) ||
        !aligned_to(dweights, 4))
        return set_error(DBL_ERR_INVALID, "%s: a pointer is not aligned to its element type", w);
    if (s->rows == 0) return DBL_OK;
    if ((!logits && !s->normalise) || !chosen || !weights || !dweights || !dlogits)
        return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    const int64_t cap = (int64_t)sm_count() * 8, need = (s->rows + 7) / 8;
    const unsigned blocks = (unsigned)(need < cap ? need : cap);
    const int64_t ld = s->ld ? s->ld : s->experts, ld_grad = s->ld_grad ? s->ld_grad : s->experts;
    cudaStream_t st = as_stream(stream);
    if (s->dtype == DBL_F32)
        route_bwd_kernel<float><<<blocks, 256, 0, st>>>(logits, chosen, weights, dweights, dlogits, s->rows, s->experts, s->k,
                                                        s->normalise != 0, ld, ld_grad);
    else
        route_bwd_kernel<act_t><<<blocks, 256, 0, st>>>(logits, chosen, weights, dweights, dlogits, s->rows, s->experts, s->k,
                                                        s->normalise != 0, ld, ld_grad);
    return launch_check(w);
}
