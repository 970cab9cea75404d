// grouped.cu -- matrix products of each group's rows with the group's own weights (a layer of experts): forward, data
// gradient and weight gradient, the groups' bounds on the device.
#include "dbl_elem.cuh"

namespace {

using namespace dbl;
using namespace dbl::dev;

constexpr int kMaxGroups = DBL_GROUPED_MAX_GROUPS;

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

__device__ int g_grouped_status;  // DBL_OK or DBL_ERR_TIMEOUT, read by dbl_device_status()

__device__ __forceinline__ void report_timeout(volatile int* abort)
{
    *abort = 1;
    atomicExch(&g_grouped_status, DBL_ERR_TIMEOUT);
}

enum : int { kFwd = 0, kDgrad = 1, kWgrad = 2 };

// A tile is a CTA pair's: 256 of the features that the weights have (fwd: n_out, dgrad: n_in) for up to 256 tokens of a group,
// or 256 x 256 of a weight gradient.  The features are the MMA's M, 128 in each CTA, and the tokens its N, as many as there are
// to the next multiple of 32: a group's last tokens cost what they are, and a group of a few costs the reading of its
// weights.  (With the tokens as M, in blocks of 256: 122 rows over 8 groups of 512x2048 9.2 us, 65536 over 64 groups of
// different lengths 352.)  64 elements of the reduction to a stage; each CTA stages its own features and half of the tokens,
// and holds its features of the result in TMEM.
struct Cfg {
    static constexpr int A_BYTES = 128 * 64 * 2, B_BYTES = 128 * 64 * 2;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STAGES = 6;
    static constexpr int EPI = 8, PROD = 2, MMA_WARP = EPI + PROD;
    static constexpr int SMEM = STAGES * STAGE_BYTES + EPI * 2048 + 1024;
    static constexpr int NB = 2;  // accumulators of 256 columns: all of TMEM
    static constexpr int THREADS = 32 * (EPI + PROD + 1);
    static_assert(SMEM >= 117 * 1024, "one CTA on an SM: each takes all of TMEM before a cluster barrier");
};

// The weight gradient's reductions are cut into chains of this many stages, whose sums are added in registers: the tensor
// cores cut the digits of a sum below those of its largest term at every step of 16.  Error of dw against 64 bits, 65536 rows of
// normal numbers: 5.1e-7 with chains of 8, 7.5e-7 with 12, 1.0e-6 with 16 (fp32 on the CUDA cores 3.7e-7); of numbers above 0:
// 9.1e-7, 1.3e-6, 2.2e-6.  In fp16, whose products have more digits to lose, 6.5e-7 and above 0 2.8e-6; without chains 8192 rows
// are 9.1e-6 and 3.5e-5 off, in fp16 9.7e-6 and 5.3e-5.  Reading an accumulator stops the tensor cores for some 300 cycles: 32768 rows over 16 groups of
// 1024x4096 206, 200, 198 us.
constexpr int kChain = 8;

struct MmaArgs {
    const act_t* mask;  // dgrad, or nullptr
    void* out;
    const int32_t* offsets;
    int64_t rows, ld;   // ld: of out and mask
    int groups, n_in, n_out, relu, accumulate;
    int features;       // of the result (fwd, dgrad)
    int depth;          // of the reduction (fwd, dgrad)
    int blocks_a, blocks_b;  // blocks of 256 features; wgrad: of n_in and n_out
    int parts;          // of a tile's reduction; more than 1: out holds fp32 sums [parts][rows][features], [parts][dw]
};

struct Tile {
    int group, a0, b0;  // a0: the first of 256 features (wgrad: of n_in); b0: the first row (wgrad: of 256 of n_out)
    int n;              // the MMA's N
    int k0, k1;         // stages of the reduction
    int part;
    int row0, row1;     // of the group
};

// The tiles of a CTA pair, every nunits-th in the order of group, block of rows (wgrad: of n_in), block of features (of
// n_out): the features of some rows run at the same time, so that x is read once however long the group is.  Counted on, as
// every role of the kernel would divide for every tile.
template <int PASS>
struct Walk {
    int group, outer, inner, step_outer, step_inner;

    // a tile's parts are neighbours
    __device__ __forceinline__ static int inners(const MmaArgs& p) { return (PASS == kWgrad ? p.blocks_b : p.blocks_a) * p.parts; }
    __device__ __forceinline__ Walk(const MmaArgs& p, const int* first, int unit0, int nunits)
        : group(0), outer(unit0 / inners(p)), inner(unit0 % inners(p)), step_outer(nunits / inners(p)),
          step_inner(nunits % inners(p))
    {
        settle(p, first);
    }
    __device__ __forceinline__ void settle(const MmaArgs& p, const int* first)
    {
        for (; group < p.groups; ++group) {
            const int blocks = PASS == kWgrad ? p.blocks_a : first[group + 1] - first[group];
            if (outer < blocks) return;
            outer -= blocks;
        }
    }
    __device__ __forceinline__ void next(const MmaArgs& p, const int* first)
    {
        outer += step_outer;
        if ((inner += step_inner) >= inners(p)) inner -= inners(p), ++outer;
        settle(p, first);
    }
    __device__ __forceinline__ bool there(const MmaArgs& p) const { return group < p.groups; }
    __device__ __forceinline__ Tile tile(const MmaArgs& p, const int* off) const
    {
        Tile c;
        c.group = group;
        c.row0 = off[group];
        c.row1 = off[group + 1];
        const int block = p.parts > 1 ? inner / p.parts : inner;
        c.part = inner - block * p.parts;
        c.a0 = (PASS == kWgrad ? outer : block) * 256;
        c.b0 = PASS == kWgrad ? block * 256 : c.row0 + outer * 256;
        c.n = PASS == kWgrad ? 256 : min(256, (c.row1 - c.b0 + 31) / 32 * 32);
        const int kb = ((PASS == kWgrad ? c.row1 - c.row0 : p.depth) + 63) / 64;
        c.k0 = p.parts > 1 ? (int)((int64_t)kb * c.part / p.parts) : 0;
        c.k1 = p.parts > 1 ? (int)((int64_t)kb * (c.part + 1) / p.parts) : kb;
        return c;
    }
};

// The larger of each half and 0; NaN stays.
__device__ __forceinline__ uint32_t relu2(uint32_t v)
{
    uint32_t r;
    asm("max.NaN." DBL_ACT_X2 " %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0u));
    return r;
}

// v where the half of h is above 0, else 0.
__device__ __forceinline__ uint32_t pass2(uint32_t v, uint32_t h)
{
    return v & __hgt2_mask(*reinterpret_cast<const act2_t*>(&h), act::pack2(0.f, 0.f));
}

// Four 8 x 8 matrices, each column of one to 16 bytes of shared memory: lane l gives column l % 8 of matrix l / 8 its address.
__device__ __forceinline__ void store_columns(uint32_t addr, uint32_t m0, uint32_t m1, uint32_t m2, uint32_t m3)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(m0), "r"(m1), "r"(m2),
                 "r"(m3)
                 : "memory");
}

// tmA: fwd, dgrad: the weights, wgrad: x; tmB: the tokens in boxes of 128, wgrad: dy; tmC: the tokens in boxes of 16.
// The launch may begin before the kernel before it has ended (122 rows over 8 groups of 512x2048 in a loop of calls 10.2 -> 8.8 us).
template <int PASS>
__global__ void __launch_bounds__(Cfg::THREADS, 1)
    grouped_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const __grid_constant__ CUtensorMap tmC, const MmaArgs p)
{
    using C = Cfg;
    constexpr int STAGES = C::STAGES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES], accf_bar[C::NB], acce_bar[C::NB], drain_bar;
    __shared__ __align__(8) uint64_t tail_bar[C::PROD], peer_bar[STAGES];  // wgrad, the last rows of a group
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    __shared__ int off[kMaxGroups + 1], first[kMaxGroups + 1];  // first: row blocks of the groups before

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sgen = smem_raw + (sbase - smem_u32(smem_raw));
    const int rank = (int)cluster_ctarank();
    const int unit0 = blockIdx.x / 2, nunits = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], 1);
            mbar_init(&peer_bar[s], 1);
        }
        for (int b = 0; b < C::NB; ++b) {
            mbar_init(&accf_bar[b], 1);
            mbar_init(&acce_bar[b], C::EPI * 2);
        }
        for (int b = 0; b < C::PROD; ++b) mbar_init(&tail_bar[b], 1);
        mbar_init(&drain_bar, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp >= C::EPI && warp < C::MMA_WARP && lane == 0) {
        tma_prefetch_desc(&tmA);
        tma_prefetch_desc(&tmB);
    }
    if (warp == C::MMA_WARP) {
        tmem_alloc_cg<2>(&tmem_slot, C::NB * 256);
        tmem_relinquish_cg<2>();
    }
    if (warp == 0) {
        grid_dependency_wait();  // what is above may overlap the kernel before; memory only after it
        load_offsets(p.offsets, p.groups, p.rows, off, lane);
        __syncwarp();
        if (PASS != kWgrad) {
            int before = 0;
            for (int i0 = 0; i0 < p.groups; i0 += 32) {
                const int i = i0 + lane;
                int v = i < p.groups ? (off[i + 1] - off[i] + 255) / 256 : 0;
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += u;
                }
                if (i < p.groups) first[i + 1] = before + v;
                before += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) first[0] = 0;
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;
    Walk<PASS> walk(p, first, unit0, nunits);

    if (warp >= C::EPI && warp < C::MMA_WARP) {
        // ------------------------------------------------------------------ TMA producers (whole warp, one lane issues)
        const int prod = warp - C::EPI;
        int it = 0, last_it = -1, tails = 0;
        bool failed = false;
        for (; walk.there(p) && !failed; walk.next(p, first)) {
            const Tile tc = walk.tile(p, off);
            for (int k = tc.k0; k < tc.k1; ++k, ++it) {
                if (it % C::PROD != prod) continue;
                const int s = it % STAGES;
                const uint32_t ok = mbar_wait_warp(&empty_bar[s], ((it / STAGES) & 1) ^ 1, &abort_flag);
                if (__any_sync(0xffffffffu, ok == 0u)) {
                    failed = true;
                    break;
                }
                uint8_t* sa = sgen + s * C::STAGE_BYTES;
                uint8_t* sb = sa + C::A_BYTES;
                const uint32_t fb0 = mapa_shared(smem_u32(&full_bar[s]), 0);
                const int acol = tc.a0 + rank * 128;
                if constexpr (PASS == kWgrad) {
                    // the last rows of a group: what is behind them in the last 16 is of another group, or of none, and may be
                    // NaN, so it is made 0 in both operands before the pair's MMAs may start
                    const int row = tc.row0 + k * 64, valid = tc.row1 - row;
                    const bool tail = valid < 64 && (valid & 15);
                    const uint32_t bar = tail ? mapa_shared(smem_u32(&tail_bar[prod]), rank) : fb0;
                    if (tail)
                        mbar_arrive_expect_tx_elect(&tail_bar[prod], C::STAGE_BYTES);
                    else if (rank == 0)
                        mbar_arrive_expect_tx_elect(&full_bar[s], 2 * C::STAGE_BYTES);
                    const int bcol = tc.b0 + rank * 128;
                    for (int j = 0; j < 2; ++j) tma_load_2d_cg<2>(sa + j * 8192, &tmA, bar, acol + 64 * j, row);
                    for (int j = 0; j < 2; ++j) tma_load_2d_cg<2>(sb + j * 8192, &tmB, bar, bcol + 64 * j, row);
                    if (tail) {
                        const uint32_t landed = mbar_wait_warp(&tail_bar[prod], tails & 1, &abort_flag);
                        ++tails;
                        if (__any_sync(0xffffffffu, landed == 0u)) {
                            failed = true;
                            break;
                        }
                        const int from = valid * 128, to = (valid + 15) / 16 * 2048;  // a row has 128 bytes of an atom of 64 columns
                        for (int j = 0; j < C::STAGE_BYTES / 8192; ++j)
                            for (int i = from + lane * 16; i < to; i += 512)
                                *reinterpret_cast<uint4*>(sa + j * 8192 + i) = make_uint4(0, 0, 0, 0);
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(rank == 0 ? fb0 : mapa_shared(smem_u32(&peer_bar[s]), 0));
                        __syncwarp();
                    }
                } else {
                    const int half = tc.n / 2, row = tc.b0 + rank * half;  // this CTA's tokens
                    if (rank == 0) mbar_arrive_expect_tx_elect(&full_bar[s], 2 * (C::A_BYTES + half * 128));
                    if constexpr (PASS == kFwd)
                        tma_load_3d_cg<2>(sa, &tmA, fb0, k * 64, acol, tc.group);
                    else
                        for (int j = 0; j < 2; ++j) tma_load_3d_cg<2>(sa + j * 8192, &tmA, fb0, acol + 64 * j, k * 64, tc.group);
                    if (half == 128)
                        tma_load_2d_cg<2>(sb, &tmB, fb0, k * 64, row);
                    else
                        for (int j = 0; j < half; j += 16) tma_load_2d_cg<2>(sb + j * 128, &tmC, fb0, k * 64, row + j);
                }
                last_it = it;
            }
        }
        if (failed) {
            if (lane == 0) report_timeout(&abort_flag);
            if (rank == 0) {
                // let copies this producer issued land before the CTA's shared memory goes away
                for (int i = last_it; i >= 0 && i > last_it - STAGES * C::PROD; i -= C::PROD)
                    (void)mbar_drain_warp(&full_bar[i % STAGES], (i / STAGES) & 1);
            } else {
                // rank 1's copies complete on rank 0's barriers: give them a fixed time instead
                const uint64_t t0 = globaltimer();
                while (globaltimer() - t0 < 1000000ull) {
                }
            }
        }
    } else if (warp == C::MMA_WARP) {
        // ------------------------------------------------------------------ MMA issuer (rank 0: whole warp, one lane issues)
        // K-major operands: rows of 128 bytes, 32 bytes a step of 16.  MN-major ones: atoms of 64 columns, 8 KB apart, 16
        // rows of 128 bytes a step.
        constexpr bool a_mn = PASS != kFwd, b_mn = PASS == kWgrad;
        const uint64_t dA = smem_desc(0, a_mn ? 8192 : 16, 1024, kSwizzle128B);
        const uint64_t dB = smem_desc(0, b_mn ? 8192 : 16, 1024, kSwizzle128B);
        constexpr uint64_t a_step = a_mn ? 2048 / 16 : 2, b_step = b_mn ? 2048 / 16 : 2;
        bool failed = false;
        uint32_t peers = 0;  // bit s: the phase of peer_bar[s]
        auto wait_full = [&](int i, bool tail) -> bool {
            const int s = i % STAGES;
            uint32_t ok = mbar_wait_warp(&full_bar[s], (i / STAGES) & 1, &abort_flag);
            if (tail) {
                if (ok) ok = mbar_wait_warp(&peer_bar[s], peers >> s & 1, &abort_flag);
                if (ok) ok = (uint32_t)bounded_try(&peer_bar[s], peers >> s & 1);  // at once: the peer's zeros acquired
                peers ^= 1u << s;
            }
            return !__any_sync(0xffffffffu, ok == 0u);
        };
        int it = 0, lt = 0;
        for (; walk.there(p) && rank == 0 && !failed; walk.next(p, first)) {
            const Tile tc = walk.tile(p, off);
            const int chain = PASS == kWgrad ? kChain : tc.k1 - tc.k0;
            const bool tail = PASS == kWgrad && ((tc.row1 - tc.row0) & 15);
            const int length = PASS == kWgrad ? tc.row1 - tc.row0 : p.depth;
            const uint32_t idesc = idesc_act(256, tc.n, a_mn, b_mn);
            for (int k0 = tc.k0; k0 < tc.k1 && !failed; k0 += chain, ++lt) {
                const int buf = lt % C::NB, k1 = min(tc.k1, k0 + chain);
                const uint32_t free = mbar_wait_warp(&acce_bar[buf], ((lt / C::NB) & 1) ^ 1, &abort_flag);
                if (__any_sync(0xffffffffu, free == 0u)) {
                    failed = true;
                    break;
                }
                const uint32_t d = tmem + (uint32_t)(buf * 256);
                for (int k = k0; k < k1; ++k, ++it) {
                    if (!wait_full(it, tail && length - k * 64 < 64)) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const int s = it % STAGES;
                    const uint32_t sa = sbase + s * C::STAGE_BYTES;
                    const uint64_t ad = dA | (uint64_t)((sa >> 4) & 0x3FFFu);
                    const uint64_t bd = dB | (uint64_t)(((sa + C::A_BYTES) >> 4) & 0x3FFFu);
                    const int left = length - k * 64;
                    if (left > 48)
                        mma_act_x4_elect_cg<2>(d, ad, a_step, bd, b_step, idesc, k > k0 ? 1u : 0u);
                    else  // the steps of 16 that hold something
                        for (int j = 0; j < (left + 15) / 16; ++j)
                            mma_act_elect_cg<2>(d, ad + j * a_step, bd + j * b_step, idesc, (k > k0 || j > 0) ? 1u : 0u);
                    mma_commit_elect_cg<2>(&empty_bar[s], 3);
                }
                mma_commit_elect_cg<2>(&accf_bar[buf], 3);
            }
        }
        if (failed && lane == 0) report_timeout(&abort_flag);
        if (rank == 0) {
            // every MMA issued above completes before the accumulators are freed
            mma_commit_elect_cg<2>(&drain_bar, 1);
            (void)mbar_drain_warp(&drain_bar, 0);
        }
    } else {
        // ------------------------------------------------------------------ epilogue (warps 0 .. EPI-1)
        constexpr int CW = 128;  // wgrad: columns that one warp drains
        const int quarter = warp & 3, part = warp >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        [[maybe_unused]] uint4* stage = reinterpret_cast<uint4*>(sgen + STAGES * C::STAGE_BYTES) + warp * 128;  // 2 KB
        int lt = 0;
        bool failed = false;
        auto wait_acc = [&](int buf) -> bool {
            const uint32_t ok = mbar_wait_warp(&accf_bar[buf], (lt / C::NB) & 1, &abort_flag);
            if (__any_sync(0xffffffffu, ok == 0u)) {
                if (lane == 0) report_timeout(&abort_flag);
                failed = true;
                return false;
            }
            tc_fence_after();
            return true;
        };
        auto release = [&](int buf) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&acce_bar[buf]), 0));
        };
        for (; walk.there(p) && !failed; walk.next(p, first)) {
            const Tile tc = walk.tile(p, off);
            if constexpr (PASS == kWgrad) {
                const int m = tc.a0 + rank * 128 + quarter * 32 + lane;  // this thread's row of the result
                const int n0 = tc.b0 + part * CW;
                float acc[CW];
#pragma unroll
                for (int i = 0; i < CW; ++i) acc[i] = 0.f;
                for (int k0 = tc.k0; k0 < tc.k1; k0 += kChain, ++lt) {
                    const int buf = lt % C::NB;
                    if (!wait_acc(buf)) break;
                    const uint32_t taddr = lanes + (uint32_t)(buf * 256 + part * CW);
#pragma unroll
                    for (int ch = 0; ch < CW / 16; ++ch) {
                        uint32_t v[16];
                        tmem_ld_32x32b_x16(taddr + ch * 16, v);
                        tmem_ld_wait_regs(v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[ch * 16 + i] += __uint_as_float(v[i]);
                    }
                    release(buf);
                }
                if (failed) break;
                // consecutive lanes hold consecutive columns of dw: each store is a line of 128 bytes
                if (m < p.n_in) {
                    float* o = static_cast<float*>(p.out) + (((int64_t)tc.part * p.groups + tc.group) * p.n_out + n0) * p.n_in + m;
                    const int left = p.n_out - n0;  // a multiple of 8
                    if (p.accumulate) {
#pragma unroll
                        for (int i0 = 0; i0 < CW; i0 += 8)
                            if (i0 < left) {
                                float before[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) before[i] = o[(int64_t)i * p.n_in];
#pragma unroll
                                for (int i = 0; i < 8; ++i, o += p.n_in) *o = before[i] + acc[i0 + i];
                            }
                    } else {
#pragma unroll
                        for (int i0 = 0; i0 < CW; i0 += 8)
                            if (i0 < left) {
#pragma unroll
                                for (int i = 0; i < 8; ++i, o += p.n_in) *o = acc[i0 + i];
                            }
                    }
                }
            } else {
                if (p.parts > 1) {
                    // fp32 sums of this part: consecutive lanes hold consecutive features
                    const int buf = lt % C::NB, f = tc.a0 + rank * 128 + quarter * 32 + lane;
                    if (!wait_acc(buf)) break;
                    float* o = static_cast<float*>(p.out) + ((int64_t)tc.part * p.rows + tc.b0) * p.features + f;
#pragma unroll 1
                    for (int ch = part; ch < tc.n / 32; ch += 2) {
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(lanes + (uint32_t)(buf * 256 + ch * 32), v);
                        tmem_ld_wait_regs(v);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (f < p.features && tc.b0 + ch * 32 + i < tc.row1)
                                o[(int64_t)(ch * 32 + i) * p.features] = __uint_as_float(v[i]);
                    }
                    release(buf);
                    ++lt;
                    continue;
                }
                // 32 features of 32 tokens at a time: pairs of tokens in a thread, turned through shared memory into 64 bytes of a
                // token's row for four lanes, so that a store meets 8 rows.  The two warps of the same features take turns.
                const int buf = lt % C::NB, chunks = tc.n / 32;
                const int q = lane % 4, col = tc.a0 + rank * 128 + quarter * 32 + q * 8;
                const int r0 = tc.b0 + lane / 4;
                const int64_t at = (int64_t)r0 * p.ld + col, down = 8 * p.ld;
                constexpr int MOST = PASS == kDgrad ? 4 : 1;
                uint4 gate[MOST][4];  // dgrad: the mask, read while the tensor cores are at work
                if constexpr (PASS == kDgrad) {
                    if (p.mask && col < p.features) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int row = (part + 2 * c) * 32 + 8 * i;
                                if (r0 + row < tc.row1) gate[c][i] = __ldg(reinterpret_cast<const uint4*>(p.mask + at + row * p.ld));
                            }
                    }
                }
                if (!wait_acc(buf)) break;
                act_t* o = static_cast<act_t*>(p.out) + at;
                const auto chunk = [&](int ch, const uint4 (&h)[4]) {
                    const uint32_t taddr = lanes + (uint32_t)(buf * 256 + ch * 32);
                    uint32_t lo[16], hi[16];
                    tmem_ld_16x256b_x4(taddr, lo);
                    tmem_ld_16x256b_x4(taddr + (16u << 16), hi);
                    tmem_ld_wait_regs(lo);
                    tmem_ld_wait_regs(hi);
                    __syncwarp();  // the chunk before has been read
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint32_t m[4];  // features 0-7, 8-15, 16-23, 24-31 of tokens 8g .. 8g + 7
#pragma unroll
                        for (int f = 0; f < 2; ++f) {
                            m[f] = act::pack2_u32(__uint_as_float(lo[4 * g + 2 * f]), __uint_as_float(lo[4 * g + 2 * f + 1]));
                            m[2 + f] = act::pack2_u32(__uint_as_float(hi[4 * g + 2 * f]), __uint_as_float(hi[4 * g + 2 * f + 1]));
                        }
                        if (PASS == kFwd && p.relu) {
#pragma unroll
                            for (int f = 0; f < 4; ++f) m[f] = relu2(m[f]);
                        }
                        const int token = 8 * g + lane % 8;
                        store_columns(smem_u32(stage + token * 4 + (lane / 8 ^ (token >> 1 & 3))), m[0], m[1], m[2], m[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int token = 8 * i + lane / 4;
                        uint4 pk = stage[token * 4 + (q ^ (token >> 1 & 3))];  // in any eight lanes, eight different 16 bytes
                        if (PASS == kDgrad && p.mask)
                            pk = make_uint4(pass2(pk.x, h[i].x), pass2(pk.y, h[i].y), pass2(pk.z, h[i].z), pass2(pk.w, h[i].w));
                        if (r0 + ch * 32 + 8 * i < tc.row1 && col < p.features)
                            *reinterpret_cast<uint4*>(o + ch * 32 * p.ld + i * down) = pk;
                    }
                };
                if constexpr (PASS == kDgrad) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (part + 2 * c < chunks) chunk(part + 2 * c, gate[c]);
                } else {
#pragma unroll 1
                    for (int ch = part; ch < chunks; ch += 2) chunk(ch, gate[0]);
                }
                release(buf);
                ++lt;
            }
        }
    }
    grid_dependency_trigger();  // the next kernel's CTAs may be placed as these leave
    tc_fence_before();
    __syncthreads();
    // neither CTA of a pair leaves while the other may still signal its barriers or read its TMEM
    cluster_sync_all();
    if (warp == C::MMA_WARP) {
        tc_fence_after();
        tmem_dealloc_cg<2>(tmem, C::NB * 256);
    }
}

// The sum of a result's parts, in their order.  fwd, dgrad: eight features of a row to a thread, the rows of all groups.
template <int PASS>
__global__ void __launch_bounds__(256) grouped_sum_kernel(const float* parts, const MmaArgs p)
{
    grid_dependency_wait();
    const int per = p.features / 8;
    // the groups are neighbours: from the first one's first row to the last one's end, clamped as load_offsets does
    int first = 0, last = 0;
    if (threadIdx.x < 32) {
        first = min((int64_t)max(p.offsets[0], 0), p.rows);
        for (int i = threadIdx.x; i <= p.groups; i += 32) last = max(last, (int)min((int64_t)max(p.offsets[i], 0), p.rows));
        last = __reduce_max_sync(0xffffffffu, last);
    }
    __shared__ int range[2];
    if (threadIdx.x == 0) range[0] = first, range[1] = last;
    __syncthreads();
    const int64_t total = (int64_t)(range[1] - range[0]) * per, slice = p.rows * p.features;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = range[0] + i / per;
        const int col = (int)(i % per) * 8;
        float f[8] = {};
        const float* src = parts + row * p.features + col;
#pragma unroll 4
        for (int k = 0; k < p.parts; ++k) {
            const float4 a = *reinterpret_cast<const float4*>(src + k * slice), b = *reinterpret_cast<const float4*>(src + k * slice + 4);
            f[0] += a.x, f[1] += a.y, f[2] += a.z, f[3] += a.w;
            f[4] += b.x, f[5] += b.y, f[6] += b.z, f[7] += b.w;
        }
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = act::pack2_u32(f[2 * j], f[2 * j + 1]);
            if (PASS == kFwd && p.relu) w[j] = relu2(w[j]);
        }
        const int64_t at = row * p.ld + col;
        if (PASS == kDgrad && p.mask) {
            const uint4 h = *reinterpret_cast<const uint4*>(p.mask + at);
            w[0] = pass2(w[0], h.x), w[1] = pass2(w[1], h.y), w[2] = pass2(w[2], h.z), w[3] = pass2(w[3], h.w);
        }
        *reinterpret_cast<uint4*>(static_cast<act_t*>(p.out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// wgrad: four elements to a thread.
__global__ void __launch_bounds__(256) grouped_sum_dw_kernel(const float* parts, float* dw, int64_t n, int count, int accumulate)
{
    grid_dependency_wait();
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        float4 f = accumulate ? *reinterpret_cast<const float4*>(dw + i) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < count; ++k) {
            const float4 a = *reinterpret_cast<const float4*>(parts + k * n + i);
            f.x += a.x, f.y += a.y, f.z += a.z, f.w += a.w;
        }
        *reinterpret_cast<float4*>(dw + i) = f;
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

int encode(CUtensorMap* m, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
           const cuuint32_t* box, const char* w)
{
    const auto fn = encode_tiled();
    if (!fn) return set_error(DBL_ERR_CUDA, "%s: cuTensorMapEncodeTiled unavailable from the driver", w);
    const cuuint32_t es[3] = {1, 1, 1};
    const CUresult r = fn(m, act::kF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
                          const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DBL_OK : set_error(DBL_ERR_CUDA, "%s: tensor map encode failed (%d)", w, (int)r);
}

// Rows of c columns, in boxes of 64 columns.
int encode_rows(CUtensorMap* m, const void* base, int64_t rows, int c, int64_t ld, int box_rows, const char* w)
{
    const cuuint64_t dims[2] = {(cuuint64_t)c, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * sizeof(act_t)};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return encode(m, base, 2, dims, strides, box, w);
}

int encode_weights(CUtensorMap* m, const void* base, const dbl_grouped_shape* s, int box_rows, const char* w)
{
    const cuuint64_t dims[3] = {(cuuint64_t)s->n_in, (cuuint64_t)s->n_out, (cuuint64_t)s->groups};
    const cuuint64_t strides[2] = {dims[0] * sizeof(act_t), dims[0] * dims[1] * sizeof(act_t)};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    return encode(m, base, 3, dims, strides, box, w);
}

template <int PASS>
int launch(const CUtensorMap (&maps)[3], const MmaArgs& p, int64_t most_tiles, cudaStream_t st, const char* w)
{
    using C = Cfg;
    int rc = allow_launch<grouped_kernel<PASS>>(C::SMEM, false, w);
    if (rc != DBL_OK) return rc;
    int dev = 0;
    if ((rc = cuda_check(cudaGetDevice(&dev), w)) != DBL_OK) return rc;
    int pairs = clusters_held<grouped_kernel<PASS>>(dev, 2, C::THREADS, C::SMEM);
    if (pairs < 1) pairs = sm_count() / 2;  // the device has not answered, or DBL_MAX_CLUSTER is 1: there is no other form
    if (pairs > most_tiles) pairs = (int)most_tiles;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * pairs);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, grouped_kernel<PASS>, maps[0], maps[1], maps[2], p);
    rc = launch_check(w);
    return err == cudaSuccess ? rc : cuda_check(err, w);
}

// Tiles of a pass, an upper bound for the forward pass and the data gradient: the blocks of rows are the device's to count.
int64_t tiles_of(const dbl_grouped_shape* s, int pass)
{
    const int64_t in = (s->n_in + 255) / 256, out = (s->n_out + 255) / 256;
    if (pass == kWgrad) return s->groups * in * out;
    return (s->rows < s->groups ? s->rows : s->rows / 256 + s->groups) * (pass == kFwd ? out : in);
}

// Elements of the result that a part has.
int64_t part_elements(const dbl_grouped_shape* s, int pass)
{
    return pass == kWgrad ? (int64_t)s->groups * s->n_out * s->n_in : s->rows * (pass == kFwd ? s->n_out : s->n_in);
}

// Parts of a tile's reduction, which a second launch adds, where there are few tiles.  fwd, dgrad: as many as fill the pairs, with
// eight stages each at least: 8 rows of one group of 4096x4096 21.2 us whole, 12.2 in parts.  wgrad: the least modelled time in
// us, a stage taking 0.3, an item's end 2, the second launch 3 and what it reads and the parts are written at 5 TB/s; the groups
// are taken as of the same length, so that one long group among empty ones stays whole.  65000 rows of one group of 512x512 307 us
// whole, 39 in parts, 40000 of two of 2048x256 111 and 46, 48000 rows of one of 664x3424 (42 tiles for 76 pairs) 236 and 208.
int parts_of(const dbl_grouped_shape* s, int pass)
{
    const int64_t tiles = tiles_of(s, pass), pairs = sm_count() / 2;
    if (tiles == 0) return 1;
    const int64_t depth = pass == kFwd ? s->n_in : pass == kDgrad ? s->n_out : s->rows / s->groups, stages = depth / 64;
    if (pass != kWgrad) {
        const int64_t most = pairs / tiles, parts = most < stages / 8 ? most : stages / 8;
        return parts > 1 ? (int)parts : 1;
    }
    const double bytes = 4.0 * (double)part_elements(s, pass);
    int best = 1;
    double least = 0.0;
    for (int n = 1; n <= pairs && (n == 1 || stages / n >= 8); ++n) {
        const double rounds = (double)((tiles * n + pairs - 1) / pairs);
        const double us = rounds * (0.3 * (double)stages / n + 2.0) + (n > 1 ? 3.0 + 2 * n * bytes / 5e6 : 0.0);
        if (n == 1 || us < least) least = us, best = n;
    }
    return best;
}

// a: fwd, dgrad: the tokens' rows (x, dy), wgrad: x; b: the weights, wgrad: dy.
template <int PASS>
int run(const dbl_grouped_shape* s, const void* a, const void* b, const int32_t* offsets, const void* mask, void* out,
        int accumulate, void* ws, size_t ws_bytes, void* stream, const char* w)
{
    const int parts = parts_of(s, PASS);
    const size_t need = dbl_grouped_workspace_bytes(s, PASS);
    if (need && (!ws || ws_bytes < need)) return set_error(DBL_ERR_WORKSPACE, "%s: workspace too small", w);
    if (!aligned16(ws)) return set_error(DBL_ERR_INVALID, "%s: the workspace is not 16-byte aligned", w);
    const int64_t ld_in = s->ld_in ? s->ld_in : s->n_in, ld_out = s->ld_out ? s->ld_out : s->n_out;
    MmaArgs p = {};
    p.mask = static_cast<const act_t*>(mask);
    p.out = parts > 1 ? ws : out;
    p.offsets = offsets;
    p.rows = s->rows;
    p.parts = parts;
    p.ld = PASS == kFwd ? ld_out : ld_in;
    p.groups = s->groups, p.n_in = s->n_in, p.n_out = s->n_out;
    p.relu = s->relu != 0, p.accumulate = accumulate && parts == 1;
    p.features = PASS == kDgrad ? s->n_in : s->n_out;
    p.depth = PASS == kFwd ? s->n_in : s->n_out;
    p.blocks_a = ((PASS == kWgrad ? s->n_in : p.features) + 255) / 256;
    p.blocks_b = (s->n_out + 255) / 256;
    CUtensorMap maps[3];
    int rc;
    if (PASS == kWgrad) {
        if ((rc = encode_rows(&maps[0], a, s->rows, s->n_in, ld_in, 64, w)) != DBL_OK) return rc;
        if ((rc = encode_rows(&maps[1], b, s->rows, s->n_out, ld_out, 64, w)) != DBL_OK) return rc;
        maps[2] = maps[1];
    } else {
        const int64_t ld = PASS == kFwd ? ld_in : ld_out;
        if ((rc = encode_weights(&maps[0], b, s, PASS == kFwd ? 128 : 64, w)) != DBL_OK) return rc;
        if ((rc = encode_rows(&maps[1], a, s->rows, p.depth, ld, 128, w)) != DBL_OK) return rc;
        if ((rc = encode_rows(&maps[2], a, s->rows, p.depth, ld, 16, w)) != DBL_OK) return rc;
    }
    cudaStream_t st = as_stream(stream);
    rc = launch<PASS>(maps, p, tiles_of(s, PASS) * parts, st, w);
    if (rc != DBL_OK || parts == 1) return rc;
    p.out = out;
    const int64_t items = part_elements(s, PASS) / (PASS == kWgrad ? 4 : 8), blocks = (items + 255) / 256, cap = (int64_t)sm_count() * 8;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(blocks < cap ? blocks : cap));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const float* sums = static_cast<const float*>(ws);
    cudaError_t err;
    if constexpr (PASS == kWgrad)
        err = cudaLaunchKernelEx(&cfg, grouped_sum_dw_kernel, sums, static_cast<float*>(out), part_elements(s, PASS), parts, accumulate);
    else
        err = cudaLaunchKernelEx(&cfg, grouped_sum_kernel<PASS>, sums, p);
    rc = launch_check("grouped sum");
    return err == cudaSuccess ? rc : cuda_check(err, "grouped sum");
}

}  // namespace

namespace dbl {

static int read_word(int* status) { return status_read(g_grouped_status, status); }
static int clear_word() { return status_clear(g_grouped_status); }
StatusWord grouped_status_word() { return {read_word, clear_word}; }

}  // namespace dbl

extern "C" size_t dbl_grouped_workspace_bytes(const dbl_grouped_shape* s, int pass)
{
    if (check(s, "grouped_workspace_bytes") != DBL_OK || pass < kFwd || pass > kWgrad || s->rows == 0) return 0;
    const int parts = parts_of(s, pass);
    return parts > 1 ? (size_t)parts * part_elements(s, pass) * sizeof(float) : 0;
}

extern "C" int dbl_grouped_fwd(const dbl_grouped_shape* s, const void* x, const void* wt, const int32_t* offsets, void* y,
                               void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_fwd";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned16(x) || !aligned16(wt) || !aligned16(y) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a tensor is not 16-byte aligned, or offsets not to 4 bytes", w);
    if (s->rows == 0) return DBL_OK;
    if (!x || !wt || !offsets || !y) return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    return run<kFwd>(s, x, wt, offsets, nullptr, y, 0, ws, ws_bytes, stream, w);
}

extern "C" int dbl_grouped_dgrad(const dbl_grouped_shape* s, const void* dy, const void* wt, const int32_t* offsets,
                                 const void* mask, void* dx, void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_dgrad";
    int rc = check(s, w);
    if (rc != DBL_OK) return rc;
    if (!aligned16(dy) || !aligned16(wt) || !aligned16(mask) || !aligned16(dx) || !aligned_to(offsets, 4))
        return set_error(DBL_ERR_INVALID, "%s: a tensor is not 16-byte aligned, or offsets not to 4 bytes", w);
    if (s->rows == 0) return DBL_OK;
    if (!dy || !wt || !offsets || !dx) return set_error(DBL_ERR_INVALID, "%s: a tensor is NULL", w);
    return run<kDgrad>(s, dy, wt, offsets, mask, dx, 0, ws, ws_bytes, stream, w);
}

extern "C" int dbl_grouped_wgrad(const dbl_grouped_shape* s, const void* x, const void* dy, const int32_t* offsets, float* dw,
                                 int accumulate, void* ws, size_t ws_bytes, void* stream)
{
    const char* w = "grouped_wgrad";
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
    return run<kWgrad>(s, x, dy, offsets, nullptr, dw, accumulate != 0, ws, ws_bytes, stream, w);
}
