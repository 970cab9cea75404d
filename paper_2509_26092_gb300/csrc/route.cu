// route.cu -- the router of a layer of experts: the k experts of every token and their weights, the tokens' places
// grouped by expert, and the gradient of the logits.
//
// The bytes are few (65536 tokens over 128 experts 23 MB, 3.4 us); what bounds the router is the selection's instructions and
// the launches' latency.  The places are a counting sort without atomics on memory: a bit for each row in its expert's set gives
// the places in a block, a second launch (one for few rows) adds what the blocks before and the smaller experts have.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxExperts = DBL_ROUTE_MAX_EXPERTS, kMaxK = DBL_ROUTE_MAX_K;
constexpr int kMaxBlocks = 256;    // of the forward pass; the workspace holds one count for each block and expert
constexpr int kOneBlockRows = 256;  // up to here one block chooses and places
constexpr int kManyRows = 64;       // of a block: from here a thread takes a row

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
    const uint32_t u = __float_as_uint(key + 0.f);  // -0 as 0
    const uint32_t r = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
    return key > -INFINITY ? r : 0u;  // not -infinity, not NaN
}

// A warp to a row, EPL experts to a lane, neighbours in a lane, so that the lowest lane has the lowest of equal experts.
// Returns this lane's entry's expert (lane j < k: entry j) or -1, and its weight.
template <class T, int EPL>
__device__ __forceinline__ int choose_row(const RouteArgs& a, int64_t r, int lane, const float (&bias)[EPL], float& weight)
{
    const T* z = static_cast<const T*>(a.logits) + r * a.ld;
    const int e0 = lane * EPL;
    weight = 0.f;
    if (a.row_weight && a.row_weight[r] == 0.f) return -1;
    float v[EPL];
    if (sizeof(T) == 2 && EPL % 2 == 0 && (reinterpret_cast<uintptr_t>(z) & 3) == 0) {
#pragma unroll
        for (int i = 0; i < EPL; i += 2)
            if (e0 + i + 1 < a.experts) {
                const float2 f = act::unpack2_u32(*reinterpret_cast<const uint32_t*>(z + e0 + i));
                v[i] = f.x, v[i + 1] = f.y;
            } else {
                v[i] = e0 + i < a.experts ? elem_f(z[e0 + i]) : -INFINITY;
                v[i + 1] = -INFINITY;
            }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) v[i] = e0 + i < a.experts ? elem_f(z[e0 + i]) : -INFINITY;
    }
    bool bad = false;  // NaN or +infinity in the row
    uint32_t key[EPL], top = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        bad |= !(v[i] < INFINITY);
        top = max(top, rank_of(v[i]));
        key[i] = rank_of(v[i] + bias[i]);
    }
    if (__any_sync(0xffffffffu, bad)) {
        weight = NAN;
        return -1;
    }
    top = __reduce_max_sync(0xffffffffu, top);
    float peak = __uint_as_float(top ^ ((top & 0x80000000u) ? 0x80000000u : 0xffffffffu)), sum = 0.f;
    if (!a.normalise && top) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) sum += expf(v[i] - peak);
        sum = warp_sum(sum);
    }
    // the lane's experts, largest first
    uint32_t at = 0;  // EPL <= 4: where key[i] came from, four bits each
    if constexpr (EPL <= 4) {
        int from[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) from[i] = i;
#pragma unroll
        for (int pass = 0; pass < EPL - 1; ++pass)
#pragma unroll
            for (int i = 0; i + 1 < EPL - pass; ++i) {
                const bool swap = key[i + 1] > key[i];
                const uint32_t k0 = swap ? key[i + 1] : key[i], k1 = swap ? key[i] : key[i + 1];
                const int f0 = swap ? from[i + 1] : from[i], f1 = swap ? from[i] : from[i + 1];
                key[i] = k0, key[i + 1] = k1, from[i] = f0, from[i + 1] = f1;
            }
#pragma unroll
        for (int i = 0; i < EPL; ++i) at |= (uint32_t)from[i] << (4 * i);
    }
    uint32_t best = 0;
    int where = 0;
    auto scan = [&]() {
        best = 0;
#pragma unroll
        for (int i = 0; i < EPL; ++i)
            if (key[i] > best) best = key[i], where = i;
    };
    if constexpr (EPL > 4) scan();
    int mine = -1;
    for (int j = 0; j < a.k; ++j) {
        if constexpr (EPL <= 4) best = key[0], where = at & 15;
        const uint32_t most = __reduce_max_sync(0xffffffffu, best);
        if (most == 0) break;
        const int from = __ffs(__ballot_sync(0xffffffffu, best == most)) - 1;
        const int e = __shfl_sync(0xffffffffu, e0 + where, from);
        if (lane == j) mine = e;
        if (lane == from) {
            if constexpr (EPL <= 4) {
#pragma unroll
                for (int i = 0; i + 1 < EPL; ++i) key[i] = key[i + 1];
                key[EPL - 1] = 0;
                at >>= 4;
            } else {
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    if (i == where) key[i] = 0;
                scan();
            }
        }
    }
    const float logit = mine >= 0 ? elem_f(z[mine]) : -INFINITY;
    if (a.normalise) {
        peak = warp_max(logit);
        sum = warp_sum(mine >= 0 ? expf(logit - peak) : 0.f);
    }
    if (mine >= 0) weight = expf(logit - peak) / sum;
    return mine;
}

// Gives the entries of rows r0 .. r1 - 1 their places among the block's entries of the same expert, in order, counted from
// base[e], kPlaceRows rows at a time: a bit for each row in its expert's set; before a row are those of the words before and
// the bits before.  sets: 2 * experts * kPlaceRows / 32 words of shared memory.
constexpr int kPlaceRows = 128, kPlaceWords = kPlaceRows / 32;

__device__ __forceinline__ void place(const RouteArgs& a, int64_t r0, int64_t r1, int* base, uint32_t* sets)
{
    uint32_t* before = sets + a.experts * kPlaceWords;
    for (int64_t t0 = r0; t0 < r1; t0 += kPlaceRows) {
        const int n = (int)min((int64_t)kPlaceRows, r1 - t0) * a.k;
        const int32_t* chosen = a.chosen + t0 * a.k;
        for (int i = threadIdx.x; i < a.experts * kPlaceWords; i += blockDim.x) sets[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int e = chosen[i], row = i / a.k;
            if (e >= 0) atomicOr(&sets[e * kPlaceWords + row / 32], 1u << (row & 31));
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
            int at = base[e];
#pragma unroll
            for (int w = 0; w < kPlaceWords; ++w) {
                before[e * kPlaceWords + w] = (uint32_t)at;
                at += __popc(sets[e * kPlaceWords + w]);
            }
            base[e] = at;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int e = chosen[i], row = i / a.k, at = e * kPlaceWords + row / 32;
            a.slots[t0 * a.k + i] = e >= 0 ? (int)before[at] + __popc(sets[at] & ((1u << (row & 31)) - 1)) : -1;
        }
        __syncthreads();
    }
}

// Exclusive sums of total[0 .. experts) into base, added to what is there, and the groups' bounds; by all threads.
__device__ __forceinline__ void bounds(const RouteArgs& a, const int* total, int* base, int* part, bool write)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    int running = 0;
    for (int first = 0; first < a.experts; first += blockDim.x) {
        const int e = first + threadIdx.x;
        const int n = e < a.experts ? total[e] : 0;
        int sum = n;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) part[warp] = sum;
        __syncthreads();
        int before = running;
        for (int w = 0; w < min(warps, (a.experts - first + 31) / 32); ++w) {
            if (w < warp) before += part[w];
            running += part[w];
        }
        if (e < a.experts) {
            base[e] += before + sum - n;
            if (write) {
                if (e == 0) a.offsets[0] = 0;
                a.offsets[e + 1] = before + sum;
            }
        }
        __syncthreads();
    }
}

template <int EPL>
constexpr int choose_threads() { return EPL <= 8 ? 1024 : 512; }

// Chooses the block's rows' experts and counts the entries of each; where there is one block, it places them too.
template <class T, int EPL>
__global__ void __launch_bounds__(choose_threads<EPL>()) route_choose_kernel(const RouteArgs a)
{
    extern __shared__ uint32_t sets[];
    __shared__ int total[kMaxExperts], base[kMaxExperts], part[32];
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) total[e] = base[e] = 0;
    __syncthreads();
    grid_dependency_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
    float bias[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) bias[i] = a.bias && lane * EPL + i < a.experts ? a.bias[lane * EPL + i] : 0.f;
    for (int64_t r = r0 + warp; r < r1; r += blockDim.x / 32) {
        float weight;
        const int e = choose_row<T, EPL>(a, r, lane, bias, weight);
        if (lane < a.k) {
            a.chosen[r * a.k + lane] = e;
            a.weights[r * a.k + lane] = weight;
            if (e >= 0) atomicAdd(&total[e], 1);
        }
    }
    __syncthreads();
    // its entries' places in the block, or, where it is the only one, among all
    if (gridDim.x > 1)
        for (int e = threadIdx.x; e < a.experts; e += blockDim.x) a.counts[(int64_t)blockIdx.x * a.experts + e] = total[e];
    else
        bounds(a, total, base, part, true);
    place(a, r0, r1, base, sets);
}

// exp(x) for x <= 0, off by (1.5*|x| + 4)*2^-24 of it, and 0 below 2^-126: for sums that are divided by.  Two instructions where
// expf has several, for every expert of every row; the kernel for few rows, whose time is latency, calls expf.  Weights of 65536
// rows of 128 are 6.6e-8 off from 64 bits, with expf in fp32 operations 5.6e-8.
__device__ __forceinline__ float exp_near(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.44269504f));
    return r;
}

// The steps of a bitonic sort's runs of RUN, from STEP on: falling order where RUN is all.
template <int RUN, int STEP>
__device__ __forceinline__ void fall(float (&m)[16])
{
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if ((j ^ STEP) > j) {
            const float hi = fmaxf(m[j], m[j ^ STEP]), lo = fminf(m[j], m[j ^ STEP]);
            m[j] = (j & RUN) ? lo : hi;
            m[j ^ STEP] = (j & RUN) ? hi : lo;
        }
    if constexpr (STEP > 1) fall<RUN, STEP / 2>(m);
}

constexpr int kManyExperts = 512;
constexpr int kTileThreads = 512, kTileBytes = 160 * 1024;

// The same where there are many rows: a thread to a row, its logits in shared memory.  The row's experts form 16 classes,
// every 16th expert one; the k-th largest of the classes' maxima is a bound that at least k experts reach and few others
// (about 11 of 128 for k = 8), so that few enter the sorted list of KT.  160 instructions of a warp to a row where a warp to
// a row takes 400: 65536 rows of 128 with k = 8 21.5 us from a graph, both launches (47 before; 2 or 4 threads to a row, whose lists
// are merged, 26).  KT: k or more.  N: elements of 16 bytes.
template <class T, int KT, bool BIAS>
__global__ void __launch_bounds__(kTileThreads) route_choose_many_kernel(const RouteArgs a, int tile, int pitch)
{
    constexpr int N = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int total[kManyExperts];
    __shared__ __align__(16) float bias[BIAS ? kManyExperts : 1];  // read by 16 bytes
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) total[e] = 0;
    grid_dependency_trigger();
    const int padded = (a.experts + 15) / 16 * 16;
    if (BIAS)
        for (int e = threadIdx.x; e < padded; e += blockDim.x) bias[e] = e < a.experts ? a.bias[e] : 0.f;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
    const T* z0 = static_cast<const T*>(a.logits);
    const bool quads = ((reinterpret_cast<uintptr_t>(a.chosen) | reinterpret_cast<uintptr_t>(a.weights) |
                         reinterpret_cast<uintptr_t>(a.slots)) & 15) == 0;
    const bool wide = ((reinterpret_cast<uintptr_t>(z0) | (uintptr_t)a.ld * sizeof(T) | (uintptr_t)a.experts * sizeof(T)) & 15) == 0;
    for (int64_t t0 = r0; t0 < r1; t0 += tile) {
        const int n = (int)min((int64_t)tile, r1 - t0);
        __syncthreads();
        if (wide) {
            const int per = a.experts / N;
            for (int i = threadIdx.x; i < n * per; i += kTileThreads) {
                const int l = i / per, u = i - l * per;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem + l * pitch + u * 16)),
                             "l"(z0 + (t0 + l) * a.ld + u * N)
                             : "memory");
            }
        } else {
            for (int i = threadIdx.x; i < n * a.experts; i += kTileThreads) {
                const int l = i / a.experts, u = i - l * a.experts;
                reinterpret_cast<T*>(smem + l * pitch)[u] = z0[(t0 + l) * a.ld + u];
            }
        }
        const int64_t r = t0 + threadIdx.x;
        const bool dead = (int)threadIdx.x < n && a.row_weight && a.row_weight[r] == 0.f;
        const int tail = padded - a.experts;
        for (int i = threadIdx.x; i < n * tail; i += kTileThreads)
            reinterpret_cast<T*>(smem + i / tail * pitch)[a.experts + i % tail] = elem_from<T>(-INFINITY);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        const uint8_t* row = smem + min((int)threadIdx.x, n - 1) * pitch;
        // sixteen logits from i on, and their keys
        auto load16 = [&](int i, float (&v)[16], float (&key)[16]) {
#pragma unroll
            for (int q = 0; q < 16 / N; ++q) {
                const uint4 u = *reinterpret_cast<const uint4*>(row + (i + q * N) * (int)sizeof(T));
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (N == 8) {
                        const float2 f = act::unpack2_u32(w[j]);
                        v[q * 8 + 2 * j] = f.x, v[q * 8 + 2 * j + 1] = f.y;
                    } else {
                        v[q * 4 + j] = __uint_as_float(w[j]);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
                if (BIAS) b = *reinterpret_cast<const float4*>(bias + i + 4 * q);
                key[4 * q] = BIAS ? v[4 * q] + b.x : v[4 * q];
                key[4 * q + 1] = BIAS ? v[4 * q + 1] + b.y : v[4 * q + 1];
                key[4 * q + 2] = BIAS ? v[4 * q + 2] + b.z : v[4 * q + 2];
                key[4 * q + 3] = BIAS ? v[4 * q + 3] + b.w : v[4 * q + 3];
            }
        };
        float peak = -INFINITY, m[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) m[j] = -INFINITY;
        for (int i = 0; i < padded; i += 16) {
            float v[16], key[16];
            load16(i, v, key);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                asm("max.NaN.f32 %0, %0, %1;" : "+f"(peak) : "f"(v[j]));
                m[j] = fmaxf(m[j], key[j]);
            }
        }
        const bool none = dead || !(peak < INFINITY) || (int)threadIdx.x >= n;
        // the classes' maxima in falling order, then the bound
        fall<2, 1>(m);
        fall<4, 2>(m);
        fall<8, 4>(m);
        fall<16, 8>(m);
#pragma unroll
        for (int half = 8; half; half /= 2)
#pragma unroll
            for (int j = 0; j < half; ++j) m[j] = (a.k - 1 & half) ? m[j + half] : m[j];
        const float bound = fmaxf(m[0], -FLT_MAX);  // the k-th; -infinity is never chosen
        float top[KT];
        int id[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) top[j] = -INFINITY, id[j] = -1;
        float sum = 0.f;
        for (int i0 = 0; i0 < padded; i0 += 64) {
            uint64_t reach = 0;
            for (int i = i0; i < min(padded, i0 + 64); i += 16) {
                float v[16], key[16];
                load16(i, v, key);
                uint32_t bits = 0;
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (key[j] >= bound) bits |= 1u << j;
                if (!a.normalise) {
#pragma unroll
                    for (int j = 0; j < 16; j += 2) s0 += exp_near(v[j] - peak), s1 += exp_near(v[j + 1] - peak);
                    sum += s0 + s1;
                }
                reach |= (uint64_t)bits << (i - i0);
            }
            if (none) reach = 0;
            while (reach) {
                const int e = i0 + __ffsll((long long)reach) - 1;
                reach &= reach - 1;
                const float key = elem_f(reinterpret_cast<const T*>(row)[e]) + (BIAS ? bias[e] : 0.f);
                bool after[KT];  // what the list has there comes after this one: of equals the first stays before
#pragma unroll
                for (int j = 0; j < KT; ++j) after[j] = key > top[j];
#pragma unroll
                for (int j = KT - 1; j >= 0; --j) {
                    const bool moves = j > 0 && after[j ? j - 1 : 0];
                    top[j] = after[j] ? (moves ? top[j ? j - 1 : 0] : key) : top[j];
                    id[j] = after[j] ? (moves ? id[j ? j - 1 : 0] : e) : id[j];
                }
            }
        }
        float over = peak;
        if (a.normalise) {
            over = -INFINITY;
#pragma unroll
            for (int j = 0; j < KT; ++j)
                if (j < a.k && id[j] >= 0) over = fmaxf(over, elem_f(reinterpret_cast<const T*>(row)[id[j]]));
        }
        float weight[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            weight[j] = j < a.k && id[j] >= 0 ? expf(elem_f(reinterpret_cast<const T*>(row)[id[j]]) - over) : 0.f;
            if (a.normalise) sum += weight[j];
        }
        const float empty = none && !dead ? NAN : 0.f;
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            weight[j] = id[j] >= 0 && j < a.k ? weight[j] / sum : empty;
            if (j >= a.k) id[j] = -1;
        }
        // Places: a bit for each row in its expert's set; before a row are those of the tiles before, of the words before and
        // the bits before.
        __syncthreads();  // the logits are done with
        const int words = (n + 31) / 32;
        uint32_t* set = reinterpret_cast<uint32_t*>(smem);
        int* before = reinterpret_cast<int*>(smem) + a.experts * words;
        for (int i = threadIdx.x; i < a.experts * words; i += kTileThreads) set[i] = 0;
        __syncthreads();
        const int word = (int)threadIdx.x / 32;
        const uint32_t bit = 1u << (threadIdx.x & 31);
#pragma unroll
        for (int j = 0; j < KT; ++j)
            if (id[j] >= 0) atomicOr(&set[id[j] * words + word], bit);
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += kTileThreads) {
            int at = total[e];
            for (int w = 0; w < words; ++w) {
                before[e * words + w] = at;
                at += __popc(set[e * words + w]);
            }
            total[e] = at;
        }
        __syncthreads();
        if ((int)threadIdx.x >= n) continue;
        int slot[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j)
            slot[j] = id[j] >= 0 ? before[id[j] * words + word] + __popc(set[id[j] * words + word] & (bit - 1)) : -1;
        int32_t *c = a.chosen + r * a.k, *s = a.slots + r * a.k;
        float* w = a.weights + r * a.k;
        if (KT % 4 == 0 && a.k == KT && quads) {
#pragma unroll
            for (int j = 0; j + 3 < KT; j += 4) {
                *reinterpret_cast<int4*>(c + j) = make_int4(id[j], id[j + 1], id[j + 2], id[j + 3]);
                *reinterpret_cast<float4*>(w + j) = make_float4(weight[j], weight[j + 1], weight[j + 2], weight[j + 3]);
                *reinterpret_cast<int4*>(s + j) = make_int4(slot[j], slot[j + 1], slot[j + 2], slot[j + 3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < KT; ++j)
                if (j < a.k) c[j] = id[j], w[j] = weight[j], s[j] = slot[j];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) a.counts[(int64_t)blockIdx.x * a.experts + e] = total[e];
}

// Places in the block become places among all: after the entries of smaller experts and those of the same expert in the blocks
// before.  Threads share an expert's counts where there are more threads than experts.
__global__ void __launch_bounds__(1024) route_place_kernel(const RouteArgs a)
{
    __shared__ int total[kMaxExperts], base[kMaxExperts], part[32];
    for (int e = threadIdx.x; e < a.experts; e += 1024) total[e] = base[e] = 0;
    __syncthreads();
    grid_dependency_wait();
    const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
    const int64_t i0 = r0 * a.k + threadIdx.x, i1 = r1 * a.k;
    constexpr int AHEAD = 4;  // entries of a thread that are asked for before the sums
    int mine[AHEAD], at[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
        mine[q] = i0 + 1024 * q < i1 ? a.chosen[i0 + 1024 * q] : -1;
        at[q] = i0 + 1024 * q < i1 ? a.slots[i0 + 1024 * q] : 0;
    }
    const int shares = max(1, 1024 / a.experts), blocks = (int)gridDim.x;
    const int share = (int)threadIdx.x / a.experts, e = (int)threadIdx.x % a.experts;
    if (share < shares) {
        int before = 0, all = 0;
        constexpr int LOADS = 20;  // asked for at a time, in turns where there are more; 152 blocks and 128 experts take one
        for (int b0 = share; b0 < blocks; b0 += LOADS * shares) {
            int n[LOADS];
#pragma unroll
            for (int q = 0; q < LOADS; ++q) n[q] = b0 + q * shares < blocks ? a.counts[(int64_t)(b0 + q * shares) * a.experts + e] : 0;
#pragma unroll
            for (int q = 0; q < LOADS; ++q) {
                all += n[q];
                if (b0 + q * shares < (int)blockIdx.x) before += n[q];
            }
        }
        atomicAdd(&total[e], all);
        atomicAdd(&base[e], before);
    }
    __syncthreads();
    bounds(a, total, base, part, blockIdx.x == 0);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
        if (mine[q] >= 0) a.slots[i0 + 1024 * q] = at[q] + base[mine[q]];
    for (int64_t i = i0 + 1024 * AHEAD; i < i1; i += 1024) {
        const int c = a.chosen[i];
        if (c >= 0) a.slots[i] += base[c];
    }
}

// What a lane has of a row: entry `lane`, and every 32nd expert's logit.
template <int EPL>
struct RouteRow {
    int e;
    float w, dw, z[EPL];
};

// A warp to a row, the next one's loads on their way: first what every expert gets, then the entries' experts.
template <class T, int EPL>
__global__ void __launch_bounds__(256) route_bwd_kernel(const void* logits, const int32_t* chosen, const float* weights,
                                                        const float* dweights, void* dlogits, int64_t rows, int experts,
                                                        int k, int normalise, int64_t ld, int64_t ld_grad)
{
    const int lane = threadIdx.x & 31;
    const auto load = [&](int64_t r) {
        RouteRow<EPL> n;
        const bool in = r < rows && lane < k;
        n.e = in ? chosen[r * k + lane] : -1;
        n.w = in ? weights[r * k + lane] : 0.f;
        n.dw = in ? dweights[r * k + lane] : 0.f;
        if (!normalise) {
            const T* z = static_cast<const T*>(logits) + (r < rows ? r : 0) * ld;
#pragma unroll
            for (int i = 0; i < EPL; ++i) n.z[i] = lane + 32 * i < experts ? elem_f(z[lane + 32 * i]) : -INFINITY;
        }
        return n;
    };
    const int64_t step = (int64_t)gridDim.x * 8;
    int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (r >= rows) return;
    for (RouteRow<EPL> row = load(r), next; r < rows; r += step, row = next) {
        next = load(r + step);
        T* dz = static_cast<T*>(dlogits) + r * ld_grad;
        const int e = row.e < experts ? row.e : -1;
        const bool nan = __any_sync(0xffffffffu, isnan(row.w)), some = __any_sync(0xffffffffu, e >= 0);
        const float wd = e >= 0 ? row.w * row.dw : 0.f, d = warp_sum(wd);
        float peak = -INFINITY, sum = 0.f, scale = 0.f;
        if (nan || !some || normalise) {
            const T fill = elem_from<T>(nan ? NAN : 0.f);
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if (lane + 32 * i < experts) dz[lane + 32 * i] = fill;
            if (nan || !some) continue;
        } else {
#pragma unroll
            for (int i = 0; i < EPL; ++i) peak = fmaxf(peak, row.z[i]);
            peak = warp_max(peak);
#pragma unroll
            for (int i = 0; i < EPL; ++i) sum += row.z[i] = expf(row.z[i] - peak);
            scale = -d / warp_sum(sum);
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if (lane + 32 * i < experts) dz[lane + 32 * i] = elem_from<T>(row.z[i] * scale);
        }
        const float mine = normalise ? wd - row.w * d : wd;
        float term = 0.f;  // of the row's entries of this lane's expert: one, where no expert is named twice
        for (int i = 0; i < k; ++i) {
            const int other = __shfl_sync(0xffffffffu, e, i);
            const float t = __shfl_sync(0xffffffffu, mine, i);
            if (other == e) term += t;
        }
        if (!normalise) {  // its expert's exponential, from the lane that has it
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                const float q = __shfl_sync(0xffffffffu, row.z[i], e & 31);
                if (e >> 5 == i) p = q;
            }
            term = fmaf(p, scale, term);
        }
        __syncwarp();  // after the row's stores
        if (e >= 0) dz[e] = elem_from<T>(term);
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
    if (s->rows <= kOneBlockRows) {
        *rows_per_block = kOneBlockRows;
        return 1;
    }
    const int most = sm_count() < kMaxBlocks ? sm_count() : kMaxBlocks;
    int64_t per = (s->rows + most - 1) / most;
    if (per < 32) per = 32;
    *rows_per_block = (int)per;
    return (int)((s->rows + per - 1) / per);
}

// f(experts to a lane, as a value of its type)
template <class F>
int with_lanes(int experts, F f)
{
    if (experts <= 32) return f(std::integral_constant<int, 1>());
    if (experts <= 64) return f(std::integral_constant<int, 2>());
    if (experts <= 128) return f(std::integral_constant<int, 4>());
    if (experts <= 256) return f(std::integral_constant<int, 8>());
    if (experts <= 512) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

template <class T, int KT, bool BIAS>
int launch_many(const RouteArgs& a, int blocks, cudaStream_t st, const char* what)
{
    const int rc = allow_launch<route_choose_many_kernel<T, KT, BIAS>>(kTileBytes, false, what);
    if (rc != DBL_OK) return rc;
    const int pitch = (a.experts + 15) / 16 * 16 * (int)sizeof(T) + 16;  // an odd number of 16 bytes: rows in different banks
    int tile = kTileBytes / pitch / 32 * 32;
    if (tile > kTileThreads) tile = kTileThreads;
    if (tile > a.rows_per_block) tile = a.rows_per_block;
    const int sets = a.experts * ((tile + 31) / 32) * 2 * (int)sizeof(int);
    route_choose_many_kernel<T, KT, BIAS><<<blocks, kTileThreads, tile * pitch > sets ? tile * pitch : sets, st>>>(a, tile, pitch);
    return launch_check(what);
}

template <class T>
int launch_fwd(const RouteArgs& a, int blocks, cudaStream_t st, const char* what)
{
    const bool many = blocks > 1 && a.rows_per_block >= kManyRows && a.experts <= kManyExperts && a.k <= 16;
    int rc;
    if (many) {
        const auto go = [&](auto kt) {
            constexpr int KT = decltype(kt)::value;
            return a.bias ? launch_many<T, KT, true>(a, blocks, st, what) : launch_many<T, KT, false>(a, blocks, st, what);
        };
        rc = a.k <= 2 ? go(std::integral_constant<int, 2>()) : a.k <= 4 ? go(std::integral_constant<int, 4>())
             : a.k <= 8 ? go(std::integral_constant<int, 8>()) : go(std::integral_constant<int, 16>());
    } else {
        rc = with_lanes(a.experts, [&](auto epl) {
            constexpr int EPL = decltype(epl)::value, threads = choose_threads<EPL>();
            route_choose_kernel<T, EPL><<<blocks, threads, 2 * kPlaceWords * a.experts * sizeof(uint32_t), st>>>(a);
            return launch_check(what);
        });
    }
    if (rc != DBL_OK || blocks == 1) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(1024);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, route_place_kernel, a);
    rc = launch_check("route_fwd place");
    return err == cudaSuccess ? rc : cuda_check(err, "route_fwd place");
}

}  // namespace

extern "C" size_t dbl_route_workspace_bytes(const dbl_route_shape* s)
{
    if (check(s, "route_workspace_bytes") != DBL_OK) return 0;
    int per;
    const int blocks = plan_blocks(s, &per);
    return blocks > 1 ? (size_t)blocks * s->experts * sizeof(int32_t) : 0;
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
    const size_t need = dbl_route_workspace_bytes(s);
    if (need && (!ws || ws_bytes < need)) return set_error(DBL_ERR_WORKSPACE, "%s: workspace too small", w);
    if (!aligned16(ws)) return set_error(DBL_ERR_INVALID, "%s: the workspace is not 16-byte aligned", w);
    int per;
    const int blocks = plan_blocks(s, &per);
    const RouteArgs a = {logits, select_bias, row_weight, chosen, weights, slots, offsets, static_cast<int32_t*>(ws), s->rows,
                         s->ld ? s->ld : s->experts, s->experts, s->k, s->normalise != 0, per};
    return s->dtype == DBL_F32 ? launch_fwd<float>(a, blocks, st, w) : launch_fwd<act_t>(a, blocks, st, w);
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
    return with_lanes(s->experts, [&](auto epl) {
        constexpr int EPL = decltype(epl)::value;
        if (s->dtype == DBL_F32)
            route_bwd_kernel<float, EPL><<<blocks, 256, 0, st>>>(logits, chosen, weights, dweights, dlogits, s->rows, s->experts,
                                                                 s->k, s->normalise != 0, ld, ld_grad);
        else
            route_bwd_kernel<act_t, EPL><<<blocks, 256, 0, st>>>(logits, chosen, weights, dweights, dlogits, s->rows, s->experts,
                                                                 s->k, s->normalise != 0, ld, ld_grad);
        return launch_check(w);
    });
}
