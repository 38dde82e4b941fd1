// Matrix product of 8-bit integers with scales for each row and column (eoq_lin_fwd, eoq_lin_bwd):
//   out[m][n] = row_scale[m] * col_scale[n] * sum over k of A[m][k] * B[n][k]  (+ bias[n]).
// The same kernel serves the three passes of a linear layer, which differ in the axis that is contiguous in memory:
//   forward   A tokens [m][k], B weights [n][k]             both K-major
//   errors    A errors [m][k], B weights [k][n]             B MN-major
//   weights   A errors [k][m], B tokens [k][n]              both MN-major
// so that no operand is ever transposed.  Sums are int32 and exact; a reduction longer than int32 holds is split, and the parts are added in 64
// bits.  One product of scales and one addition per output remain: three roundings in fp32 and the one to the output's type.
//
// Bound: the tensor pipe (128 cycles for 128 x 256 x 32 a block) where tiles are full.  Persistent blocks walk tiles of 128 x kN, or pairs of blocks tiles of
// 256 x 256 as one (each loads half of either operand: 64 bytes a cycle and SM instead of 96 for tiles of 128 x 256).  Roles: sixteen epilogue warps, a warp for the
// tensor copies, one for the MMAs.  Accumulators in tensor memory, two of a pair, four otherwise, let tiles' epilogues run beside the next ones' MMAs: what an epilogue
// takes is mostly waiting (for scales, tensor memory, stores), so that blocks with several tiles give them to two or four groups of warps in turn.  The two products of a
// backward pass share a launch: alone, 64 and 256 tiles leave 74 pairs idle for an eighth of the time each.  All waits are bounded.
// In short runs, before the power limit lowers the clock: 8192 tokens, 4096 to 4096 channels 80 us, 3.4 POPS; 16,384 tokens, 1024 to 4096 46 us forward, 87 for the two products
// backward (87% of the tensor pipe's cycles); these two together take 142 in long ones.
#include "eoq_lin.cuh"
#include "eoq_pair.cuh"

namespace eoq {

namespace {

constexpr int kStageK = 128;                   // bytes of the reduction in a stage
constexpr int kUnit = 2048;                    // staging: 32 rows of 64 bytes
constexpr int kMaxSmem = 225 * 1024;           // of dynamic shared memory: some of a block's 227 KB are static

template <int kN, bool kPair>
struct GemmShape {
    static constexpr int kBlocks = kPair ? 2 : 1, kOwnN = kN / kBlocks;   // columns of B that a block loads
    static constexpr int kEpiWarps = 16, kLoadWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1, kThreads = 32 * (kEpiWarps + 2);
    static constexpr int kSums = kPair ? 2 : 4;                           // accumulators
    static constexpr int kLeastGroups = kPair || kN == 128 ? 1 : kN == 64 ? 2 : 4;   // so that no epilogue warp has less than a chunk
    static constexpr int kA = kTileM * kStageK, kB = kOwnN * kStageK, kStage = kA + kB, kUnits = kPair ? 1 : 2, kStaging = kUnits * kEpiWarps * kUnit;
    static constexpr int kFit = (kMaxSmem - 1024 - kStaging) / kStage, kStages = kFit < 8 ? kFit : 8;
    static constexpr int kBytes = kStages * kStage + kStaging + 1024;
    static constexpr uint32_t kColumns = kSums * kN;                      // of tensor memory
};

__device__ __forceinline__ void mma_i8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t leader)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader));
}
// kPair: the bytes are counted by the first block's barrier, whichever block loads
template <bool kPair>
__device__ __forceinline__ void load_tile(uint32_t dst, const void *map, uint32_t bar, int c0, int c1)
{
    if constexpr (kPair)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
            ::"r"(dst), "l"(map), "r"(ptx::cluster_addr(bar, 0)), "r"(c0), "r"(c1) : "memory");
    else
        ptx::tma_load_2d(dst, map, bar, c0, c1);
}
__device__ __forceinline__ void store_tile_2d(const void *map, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// two fp32 operations in one instruction, each rounded as it is alone
__device__ __forceinline__ uint64_t pair_of(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma_2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// 32 sums of a row with their scales (scaled_sum, two at a time).  `scales`: of the 32 columns, and their biases 128 bytes on.  kLarge: some row of the warp's has a large scale.
template <bool kLarge>
__device__ __forceinline__ void scale_row(uint32_t (&r)[32], float row_scale, uint32_t scales)
{
    const bool large = kLarge && large_scale(row_scale);
    const float first = large ? row_scale * kLessScale : row_scale;
    const uint64_t rs = pair_of(first, first);
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        uint64_t s[2], b[2];
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(s[0]), "=l"(s[1]) : "r"(scales + j * 4) : "memory");
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(b[0]), "=l"(b[1]) : "r"(scales + 128 + j * 4) : "memory");
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (large) {
                float s0, s1;
                asm("mov.b64 {%0, %1}, %2;" : "=f"(s0), "=f"(s1) : "l"(s[i]));
                s[i] = pair_of(more_scale(s0), more_scale(s1));
            }
            const uint64_t v = fma_2(mul_2(pair_of(__int2float_rn((int)r[j + 2 * i]), __int2float_rn((int)r[j + 2 * i + 1])), rs), s[i], b[i]);
            asm("mov.b64 {%0, %1}, %2;" : "=r"(r[j + 2 * i]), "=r"(r[j + 2 * i + 1]) : "l"(v));
        }
    }
}

// 64 bytes of a row to the lane's place in the staging: pieces of 16 bytes in the order that tensor copies expect of such rows.  kPart: which 16 of the 32 words (of
// 16-bit types: all of them, rounded).
template <int kType, int kPart>
__device__ __forceinline__ void stage_row(const uint32_t (&r)[32], uint32_t unit, int lane)
{
    const uint32_t row = unit + lane * 64, turn = (uint32_t)((lane >> 1) & 3) << 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kType == EOQ_F16) {
                const __half2 h = __floats2half2_rn(__uint_as_float(r[8 * j + 2 * i]), __uint_as_float(r[8 * j + 2 * i + 1]));
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else if constexpr (kType == EOQ_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[8 * j + 2 * i]), __uint_as_float(r[8 * j + 2 * i + 1]));
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                w[i] = r[16 * kPart + 4 * j + i];
            }
        }
        st_shared_v4(row + ((uint32_t)(j << 4) ^ turn), w[0], w[1], w[2], w[3]);
    }
}

// The staged rows to rows of the output that tensor copies cannot address: 32 columns of a row at a time, or 16 of two.
template <int kE>
__device__ __forceinline__ void store_rows(const LinProduct &a, uint32_t unit, size_t out_row, int rows, int col0, int lane)
{
    if constexpr (kE == 2) {
        const int col = col0 + lane;
        const bool in = col < a.n;
        char *to = reinterpret_cast<char *>(a.out) + out_row * a.out_pitch + (size_t)col * 2;
#pragma unroll 8
        for (int i = 0; i < rows; ++i, to += a.out_pitch) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(unit + i * 64 + (((lane >> 3) ^ ((i >> 1) & 3)) << 4) + (lane & 7) * 2) : "memory");
            if (in) *reinterpret_cast<uint16_t *>(to) = v;
        }
    } else {
        const int c = lane & 15, col = col0 + c;
        char *to = reinterpret_cast<char *>(a.out) + (out_row + (lane >> 4)) * a.out_pitch + (size_t)col * 4;
#pragma unroll 8
        for (int i = lane >> 4; i < rows; i += 2, to += 2 * a.out_pitch) {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(unit + i * 64 + (((c >> 2) ^ ((i >> 1) & 3)) << 4) + (c & 3) * 4) : "memory");
            if (col < a.n) *reinterpret_cast<uint32_t *>(to) = v;
        }
    }
}

// A warp's 32 rows and 32 columns of scaled sums to memory, by way of its kUnits of staging, one being filled and, of two, one on its way out.  (Of a pair's block there is
// one: stages of operands are worth more, six instead of four some 6% of the time.)
template <int kType, int kUnits>
__device__ __forceinline__ void write_chunk(const LinProduct &a, const CUtensorMap *map, const uint32_t (&r)[32], uint32_t staging, int &units, size_t out_row, int rows, int col0, int lane)
{
    constexpr int kE = kType == EOQ_F16 || kType == EOQ_BF16 ? 2 : 4;
    auto out = [&](int col) {
        const uint32_t unit = staging + units % kUnits * kUnit;
        if (a.tensor_store) {
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (col < a.n) store_tile_2d(map, unit, col, (int)out_row);
                store_commit();
            }
        } else {
            __syncwarp();
            store_rows<kE>(a, unit, out_row, rows, col, lane);
            if (lane == 0) store_commit();   // (an empty group: what is waited for counts one for each unit, and the unit before may be another product's, on its way out)
        }
        __syncwarp();
        ++units;
    };
    stage_row<kType, 0>(r, staging + units % kUnits * kUnit, lane);
    out(col0);
    if constexpr (kE == 4) {
        if (lane == 0) store_wait_read<kUnits - 1>();
        __syncwarp();
        stage_row<kType, 1>(r, staging + units % kUnits * kUnit, lane);
        out(col0 + 16);
    }
}

// The calling pair or block's units in turn: next(product, unit) is false behind the last one.  Those of the first product are dealt out one by one; where some
// blocks get one more than the others, those others take `catch_up` units of the second product in the meantime, then all take theirs in turn.
struct Turns {
    int me, me_light, all, own0, first1, catch_up, light, units1, round;
    __device__ __forceinline__ Turns(const LinGemmArgs &a, int me_, int all_) : me(me_), all(all_), round(0)
    {
        const int units0 = a.p[0].units, each = units0 / all, more = units0 - each * all;
        own0 = each + (me < more ? 1 : 0);
        light = all - more;
        catch_up = me >= more && more > 0 ? a.catch_up : 0;
        first1 = more > 0 ? a.catch_up * light : 0;
        units1 = a.count > 1 ? a.p[1].units : 0;
        me_light = me - more;
    }
    __device__ __forceinline__ bool next(int &product, int &unit)
    {
        const int r = round++, k = r - own0;
        product = k < 0 ? 0 : 1;
        unit = k < 0 ? me + r * all : k < catch_up ? k * light + me_light : first1 + (k - catch_up) * all + me;
        return k < 0 || unit < units1;
    }
};

struct Maps {
    CUtensorMap a[2], b[2], out[2];
};

template <int kN, bool kPair>
__global__ void __launch_bounds__((GemmShape<kN, kPair>::kThreads), 1) lin_gemm_kernel(const __grid_constant__ LinGemmArgs args, const __grid_constant__ Maps maps)
{
    using S = GemmShape<kN, kPair>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 2 * S::kSums + 1];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t abort_s;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
    const uint32_t staging = smem_base + S::kStages * S::kStage;
    // of a stage: copies landed (of a pair: in the first block), MMAs done.  Of an accumulator: complete; read.  All MMAs done.
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (S::kStages + s); };
    auto sums_bar = [&](int i) { return bar0 + 8u * (2 * S::kStages + i); };
    auto read_bar = [&](int i) { return bar0 + 8u * (2 * S::kStages + S::kSums + i); };
    const uint32_t drain_bar = bar0 + 8u * (2 * S::kStages + 2 * S::kSums);
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int i = 0; i < S::kSums; ++i) {
            ptx::mbar_init(sums_bar(i), 1);
            ptx::mbar_init(read_bar(i), S::kBlocks * (S::kEpiWarps / args.groups));
        }
        ptx::mbar_init(drain_bar, 1);
        abort_s = 0;
        ptx::fence_barrier_init();
        for (int i = 0; i < args.count; ++i) {
            ptx::prefetch_tensormap(&maps.a[i]);
            ptx::prefetch_tensormap(&maps.b[i]);
        }
    }
    if (warp == S::kMmaWarp) tmem_take<kPair>(ptx::smem_u32(&tmem_base_s), S::kColumns);
    const int rank = kPair ? blockIdx.x & 1 : 0;
    // A unit: a tile and a part of its reduction.  Tiles go in bands of kBand tiles of n, down m inside a band, so that what runs at a time
    // shares operands in the L2.
    auto place = [&](const LinProduct &p, int u, int &m0, int &n0, int &split) {
        constexpr int kBand = 8;
        const int tiles = p.m_tiles * p.n_tiles;
        split = u / tiles;
        const int t = u - split * tiles, per_band = kBand * p.m_tiles, band = t / per_band, in = t - band * per_band;
        const int width = min(kBand, p.n_tiles - band * kBand);
        const int mt = in / width;
        m0 = mt * S::kBlocks * kTileM + rank * kTileM;
        n0 = (band * kBand + in - mt * width) * kN;
    };
    auto stages_of = [&](const LinProduct &p, int split) { return min(p.stages_per_split, p.k_stages - split * p.stages_per_split); };
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (the other block's barriers are ready)
    else __syncthreads();
    ptx::tc_fence_after();
    ptx::grid_dep_wait();
    if (args.launch_early) ptx::grid_dep_launch();
    const uint32_t tmem_base = tmem_base_s;
    const RoleCtx ctx{&abort_s, args.dev};
    Turns turns(args, blockIdx.x / S::kBlocks, gridDim.x / S::kBlocks);
    int which, u;

    if (warp == S::kLoadWarp) {
        bool ok = true;
        int slot = 0, started = 0;
        uint32_t phase = 0;
        while (ok && turns.next(which, u)) {
            const LinProduct &p = args.p[which];
            const CUtensorMap *map_a = &maps.a[which], *map_b = &maps.b[which];
            const bool a_mn = p.a_mn, b_mn = p.b_mn;
            int m0, n0, split;
            place(p, u, m0, n0, split);
            const int n_own = n0 + rank * S::kOwnN, stages = stages_of(p, split), k_first = split * p.stages_per_split;
            const uint32_t bytes = S::kBlocks * (S::kB + p.a_rows * kStageK);
            for (int it = 0; it < stages; ++it) {
                if (!(ok = __all_sync(0xffffffffu, wait_bar(empty_bar(slot), phase ^ 1u, ctx)))) break;
                if (lane == 0) {
                    const uint32_t dst = smem_base + slot * S::kStage;
                    const int k = (k_first + it) * kStageK;
                    if (rank == 0) ptx::mbar_expect_tx(full_bar(slot), bytes);
                    load_tile<kPair>(dst, map_a, full_bar(slot), a_mn ? m0 : k, a_mn ? k : m0);
                    load_tile<kPair>(dst + S::kA, map_b, full_bar(slot), b_mn ? n_own : k, b_mn ? k : n_own);
                }
                __syncwarp();
                ++started;
                if (++slot == S::kStages) { slot = 0; phase ^= 1u; }
            }
        }
        // Nothing may be in flight towards this block's memory when it ends: after a wait that ran out, the bytes still to come are waited for (by the
        // block whose barriers count them), with a limit.
        if (!ok && lane == 0 && rank == 0)
            for (int it = started > S::kStages ? started - S::kStages : 0; it < started; ++it)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (ptx::mbar_try_wait(full_bar(it % S::kStages), (uint32_t)(it / S::kStages) & 1u)) break;
    } else if (warp == S::kMmaWarp) {
        if (rank == 0) {
            const uint32_t leader = elect_one();
            bool ok = true;
            int slot = 0, turn = 0;
            uint32_t phase = 0;
            for (; ok && turns.next(which, u); ++turn) {
                const LinProduct &p = args.p[which];
                const bool a_mn = p.a_mn, b_mn = p.b_mn;
                // K-major: rows of 128 bytes, groups of eight 1024 bytes apart, 32 bytes along the row to the next step of the reduction.  MN-major: a row of the
                // reduction is 128 (or kN) bytes, groups of eight rows lie behind one another, 32 rows to the next step.
                constexpr int kBMnRow = S::kOwnN < 128 ? S::kOwnN : 128;
                const uint32_t idesc = make_idesc_i8(S::kBlocks * kTileM, kN, a_mn, b_mn);
                const uint32_t a_step = a_mn ? 32 * 128 / 16 : 2, b_step = b_mn ? 32 * kBMnRow / 16 : 2;
                const uint32_t a_hi = smem_desc_hi(1024, 2), b_hi = b_mn ? smem_desc_hi(8 * kBMnRow, layout_type_for(kBMnRow)) : a_hi;
                const uint32_t a_lead = (S::kA >> 4) << 16, b_lead = (S::kB >> 4) << 16;
                const int stages = stages_of(p, u / (p.m_tiles * p.n_tiles)), acc = turn % S::kSums;
                const uint32_t d = tmem_base + acc * kN;
                if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(read_bar(acc), (turn / S::kSums & 1) ^ 1, ctx)))) break;
                ptx::tc_fence_after();
                for (int it = 0; it < stages; ++it) {
                    if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(full_bar(slot), phase, ctx)))) break;
                    ptx::tc_fence_after();
                    const uint32_t a16 = ((smem_base + slot * S::kStage) >> 4) | a_lead, b16 = ((smem_base + slot * S::kStage + S::kA) >> 4) | b_lead;
#pragma unroll
                    for (int k = 0; k < kStageK / 32; ++k) {
                        const uint64_t ad = smem_desc_join(a16 + k * a_step, a_hi), bd = smem_desc_join(b16 + k * b_step, b_hi);
                        const uint32_t more = (k | it) != 0 ? 1u : 0u;
                        if constexpr (kPair) mma_i8_pair(d, ad, bd, idesc, more, leader);
                        else ptx::mma_i8(d, ad, bd, idesc, more, leader);
                    }
                    commit_both<kPair>(empty_bar(slot), leader);
                    if (++slot == S::kStages) { slot = 0; phase ^= 1u; }
                }
                commit_both<kPair>(sums_bar(acc), leader);
            }
            commit_both<kPair>(drain_bar, leader);
            if (!ok)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (ptx::mbar_try_wait(drain_bar, 0)) break;
        }
    } else {
        const int group_warps = S::kEpiWarps / args.groups, quad = warp & 3, group = warp / group_warps, part = warp % group_warps / 4, warp_n = kN * 4 / group_warps;
        const uint32_t staging_w = staging + warp * S::kUnits * kUnit;
        int units = 0;
        for (int turn = 0; turns.next(which, u); ++turn) {
            if (turn % args.groups != group) continue;
            const LinProduct &p = args.p[which];
            const CUtensorMap *map_out = &maps.out[which];
            const int type = p.out_type;
            int m0, n0, split;
            place(p, u, m0, n0, split);
            const int acc = turn % S::kSums, row0 = m0 + quad * 32, first_col = n0 + part * warp_n, rows = min(32, p.m - row0);
            const int chunks = rows <= 0 || first_col >= p.n ? 0 : min(warp_n / 32, (p.n - first_col + 31) / 32);
            // the row's scale and the first columns' arrive beside the tile's MMAs, the next columns' beside the arithmetic
            float row_scale = 0.0f, s = 0.0f, b = 0.0f;
            auto fetch = [&](int c) {
                const int col = first_col + c * 32 + lane;
                s = c < chunks && col < p.n ? p.col_scale ? __ldg(p.col_scale + col) : 1.0f : 0.0f;
                b = c < chunks && col < p.n && p.bias ? __ldg(p.bias + col) : 0.0f;
            };
            if (type != EOQ_I32) {
                row_scale = lane < rows ? __ldg(p.row_scale + row0 + lane) : 0.0f;
                fetch(0);
            }
            if (!__all_sync(0xffffffffu, wait_bar<32>(sums_bar(acc), turn / S::kSums & 1, ctx))) break;
            ptx::tc_fence_after();
            const bool any_large = __any_sync(0xffffffffu, large_scale(row_scale));
            const size_t out_row = (size_t)split * p.split_rows + row0;
            const uint32_t t_row = tmem_base + acc * kN + part * warp_n + ((uint32_t)(quad * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                const int col0 = first_col + c * 32;
                uint32_t r[32];
                ptx::tmem_ld_32x32(t_row + c * 32, r);
                // what went out of the next unit before has been read by now
                if (lane == 0) store_wait_read<S::kUnits - 1>();
                __syncwarp();
                if (type != EOQ_I32) {
                    // (in the unit that is filled next)
                    const uint32_t scales = staging_w + units % S::kUnits * kUnit;
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + lane * 4), "f"(s) : "memory");
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + 128 + lane * 4), "f"(b) : "memory");
                    __syncwarp();
                    fetch(c + 1);
                }
                ptx::tmem_ld_wait();
                if (type != EOQ_I32) {
                    const uint32_t scales = staging_w + units % S::kUnits * kUnit;
                    if (any_large) scale_row<true>(r, row_scale, scales);
                    else scale_row<false>(r, row_scale, scales);
                    __syncwarp();
                }
                if (type == EOQ_BF16) write_chunk<EOQ_BF16, S::kUnits>(p, map_out, r, staging_w, units, out_row, rows, col0, lane);
                else if (type == EOQ_F16) write_chunk<EOQ_F16, S::kUnits>(p, map_out, r, staging_w, units, out_row, rows, col0, lane);
                else write_chunk<EOQ_F32, S::kUnits>(p, map_out, r, staging_w, units, out_row, rows, col0, lane);   // (words as they are)
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_first<kPair>(read_bar(acc));
        }
        if (lane == 0) store_wait_all();
    }
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (neither block ends while the other's MMAs, copies or arrivals may reach it)
    else __syncthreads();
    if (warp == S::kMmaWarp) {
        ptx::tc_fence_after();
        tmem_return<kPair>(tmem_base, S::kColumns);
    }
}

// The parts of a split reduction, which stand `pitch` words apart row by row and `split_rows` rows apart, added and scaled: four columns a thread.
template <bool kLong>
__global__ void __launch_bounds__(256) lin_join_kernel(const __grid_constant__ LinProduct a, const int32_t *__restrict__ part, size_t pitch)
{
    ptx::grid_dep_wait_launch_small();
    const int per_row = (a.n + 3) / 4;
    const size_t total = (size_t)a.m * per_row;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const size_t row = i / per_row;
        const int col = (int)(i - row * per_row) * 4;
        using Sum = typename std::conditional<kLong, long long, int>::type;
        Sum s[4] = {};
#pragma unroll 4
        for (int p = 0; p < a.splits; ++p) {
            const int4 v = __ldg(reinterpret_cast<const int4 *>(part + ((size_t)p * a.split_rows + row) * pitch + col));
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
        const float rs = __ldg(a.row_scale + row);
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = col + j < a.n;
            const float f = kLong ? __ll2float_rn((long long)s[j]) : __int2float_rn((int)s[j]);
            v[j] = scaled_sum(f, rs, in && a.col_scale ? __ldg(a.col_scale + col + j) : 1.0f, in && a.bias ? __ldg(a.bias + col + j) : 0.0f);
        }
        char *dst = reinterpret_cast<char *>(a.out) + row * a.out_pitch;
        auto put = [&](auto type) {
            using E = decltype(type);
            const Raw<4 * E::kSize> w = E::from_f32(v);
            if (col + 4 <= a.n && reinterpret_cast<uintptr_t>(dst + (size_t)col * E::kSize) % (4 * E::kSize) == 0) {
                store_raw(dst + (size_t)col * E::kSize, w);
            } else {
                for (int j = 0; j < 4 && col + j < a.n; ++j) {
                    const float one[1] = {v[j]};
                    store_raw(dst + (size_t)(col + j) * E::kSize, E::from_f32(one));
                }
            }
        };
        if (a.out_type == EOQ_F32) put(Elem<EOQ_F32>());
        else if (a.out_type == EOQ_F16) put(Elem<EOQ_F16>());
        else put(Elem<EOQ_BF16>());
    }
}

constexpr int kMostStages = 1023;   // of a part: 130,944 products of codes, at most 2^14 each, are an int32

// Bytes of `splits` parts of a product's sums, their rows and columns.
size_t partial_pitch(int n) { return ((size_t)n + 3) & ~(size_t)3; }
size_t parts_bytes(const LinProduct &p) { return p.splits > 1 ? sizeof(int32_t) * (size_t)p.splits * p.split_rows * partial_pitch(p.n) : 0; }

struct Plan {
    int tile_n;       // 32, 64, 128, or 256: a pair's
    int catch_up;
};

// Cycles of a stage of a tile of width 32 << w: its MMAs, or what a block's copies take, two cycles for a row of a tile, 4.5 where rows straddle lines of 128 bytes.
double stage_cycles(const LinProduct &p, int w)
{
    static const double kMma[4] = {230.0, 230.0, 280.0, 520.0};
    const int own_n = w == 3 ? 128 : 32 << w;
    auto lines = [](size_t pitch) { return pitch % 128 == 0 || 128 % pitch == 0 ? 1.0 : 2.25; };
    const double copies = 2.0 * ((p.a_mn || p.m >= 128 ? 128.0 : p.m) * lines(p.pitch_a) + (p.b_mn ? 128.0 : own_n) * lines(p.pitch_b));
    return copies > kMma[w] ? copies : kMma[w];
}

// Tiles and splits of the products of a launch, by a model of what takes how long: cycles of a stage, of a tile's epilogue, of a
// launch that joins parts.  The time of a launch is that of its busiest block.
Plan plan_of(LinProduct *p, int count)
{
    LinProduct best[2] = {};
    Plan plan = {};
    double best_time = 0.0;
    for (int w = 0; w < 4; ++w) {
        const int tile_n = 32 << w, blocks = tile_n == 256 ? 2 : 1, tile_m = blocks * kTileM;
        const int room = kPartSms / blocks;
        bool fits = true, wider = w == 0;
        for (int i = 0; i < count; ++i) {
            if (blocks == 2 && (p[i].m <= kTileM || p[i].n <= 128)) fits = false;
            if (p[i].n > tile_n / 2) wider = true;   // (some product has columns for tiles this wide)
        }
        if (!fits || !wider) continue;
        for (int fill = 0; fill <= 2; ++fill) {
            LinProduct q[2];
            double unit[2] = {}, join = 0.0;
            bool splits_any = fill == 0;
            for (int i = 0; i < count; ++i) {
                q[i] = p[i];
                q[i].m_tiles = (p[i].m + tile_m - 1) / tile_m;
                q[i].n_tiles = (p[i].n + tile_n - 1) / tile_n;
                q[i].split_rows = q[i].m_tiles * tile_m;
                const size_t tiles = (size_t)q[i].m_tiles * q[i].n_tiles, least = (q[i].k_stages + kMostStages - 1) / kMostStages;
                size_t splits = fill == 0 ? 1 : (size_t)fill * room / tiles;
                if (splits < least) splits = least;
                if (splits > (size_t)q[i].k_stages) splits = q[i].k_stages;
                q[i].stages_per_split = (int)((q[i].k_stages + splits - 1) / splits);
                q[i].splits = (q[i].k_stages + q[i].stages_per_split - 1) / q[i].stages_per_split;
                if (q[i].splits > 1) splits_any = true;
                q[i].units = (int)(tiles * q[i].splits);
                // A tile's epilogue takes 24 cycles a column beside the next tile's stages, of single blocks not quite beside them.
                const double stages = (double)q[i].stages_per_split * stage_cycles(q[i], w), epilogue = 24.0 * tile_n + (blocks == 2 ? 400.0 : 200.0 + 0.5 * stages);
                unit[i] = stages > epilogue ? stages : epilogue;
                if (q[i].splits > 1) join += 7000.0 + (double)q[i].splits * q[i].m * q[i].n * 4.0 * 2.0 / 2500.0;
            }
            if (!splits_any) continue;
            int catch_up = 0;
            double time;
            if (count == 1) {
                time = (double)((q[0].units + room - 1) / room) * unit[0];
            } else {
                // the product with the longer units goes first
                if (unit[1] > unit[0]) {
                    const LinProduct t = q[0];
                    q[0] = q[1];
                    q[1] = t;
                    const double d = unit[0];
                    unit[0] = unit[1];
                    unit[1] = d;
                }
                const int more = q[0].units % room, light = room - more;
                if (more > 0) catch_up = (int)(unit[0] / unit[1] + 0.5);
                if ((long long)catch_up * light > q[1].units) catch_up = (q[1].units + light - 1) / light;
                const long long left = q[1].units - (long long)catch_up * (more > 0 ? light : 0);
                const double whole = (double)(q[0].units / room) * unit[0] + (more > 0 ? unit[0] > catch_up * unit[1] ? unit[0] : catch_up * unit[1] : 0.0);
                time = whole + (left > 0 ? (double)((left + room - 1) / room) * unit[1] : 0.0);
            }
            time += 6000.0 + join;
            if (best_time == 0.0 || time < best_time) {
                best_time = time;
                for (int i = 0; i < count; ++i) best[i] = q[i];
                plan.tile_n = tile_n;
                plan.catch_up = catch_up;
            }
        }
    }
    for (int i = 0; i < count; ++i) p[i] = best[i];
    return plan;
}

template <int kN, bool kPair>
cudaError_t launch(LinGemmArgs a, cudaStream_t st)
{
    using S = GemmShape<kN, kPair>;
    Maps maps = {};
    size_t units = 0;
    for (int i = 0; i < a.count; ++i) {
        const LinProduct &p = a.p[i];
        const bool got =
            (p.a_mn ? tiled_map_of(&maps.a[i], p.a, 1, p.m, p.k, p.pitch_a, 128, kStageK, 128) : tiled_map_of(&maps.a[i], p.a, 1, p.k, p.m, p.pitch_a, kStageK, p.a_rows, 128)) &&
            (p.b_mn ? tiled_map_of(&maps.b[i], p.b, 1, p.n, p.k, p.pitch_b, S::kOwnN, kStageK, S::kOwnN)
                    : tiled_map_of(&maps.b[i], p.b, 1, p.k, p.n, p.pitch_b, kStageK, S::kOwnN, 128));
        if (!got) return cudaErrorInvalidValue;
        if (p.tensor_store) {
            const int e = p.out_type == EOQ_F16 || p.out_type == EOQ_BF16 ? 2 : 4;
            if (!tiled_map_of(&maps.out[i], p.out, e, p.n, p.out_type == EOQ_I32 ? (size_t)p.splits * p.split_rows : (size_t)p.m, p.out_pitch, 64 / e, 32, 64))
                return cudaErrorInvalidValue;
        }
        units += p.units;
    }
    static_assert(S::kBytes <= kMaxSmem && S::kStages >= 4, "shared memory of a block");
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)lin_gemm_kernel<kN, kPair>, S::kBytes, allowed);
    if (e != cudaSuccess) return e;
    const size_t room = a.sm_count / S::kBlocks;
    const unsigned grid = (unsigned)(units < room ? units : room) * S::kBlocks;
    a.groups = S::kLeastGroups;
    while (!kPair && a.groups < 4 && units >= 2 * a.groups * room) a.groups *= 2;
    return launch_chained_clusters(S::kBlocks, lin_gemm_kernel<kN, kPair>, dim3(grid), dim3(S::kThreads), S::kBytes, st, a, maps);
}

}  // namespace

// Products as a pass describes them, with tiles and splits.
static Plan planned(LinGemmArgs &a)
{
    for (int i = 0; i < a.count; ++i) a.p[i].k_stages = (int)((a.p[i].k + kStageK - 1) / kStageK);
    return plan_of(a.p, a.count);
}

size_t lin_gemm_workspace_bytes(LinGemmArgs a)
{
    planned(a);
    size_t bytes = 0;
    for (int i = 0; i < a.count; ++i) bytes += (parts_bytes(a.p[i]) + 255) / 256 * 256;
    return bytes;
}

cudaError_t launch_lin_gemm(LinGemmArgs a, void *workspace, int *launches, cudaStream_t st)
{
    const Plan plan = planned(a);
    a.catch_up = plan.catch_up;
    LinProduct whole[2];
    char *part = reinterpret_cast<char *>(workspace);
    for (int i = 0; i < a.count; ++i) {
        LinProduct &p = a.p[i];
        // Of few tokens, only their rows are brought in; what stands in the others of a tile is nobody's.  (16 tokens, 4096 to 4096: 18.6 us with boxes of 128 rows, most of them
        // behind the end.)
        p.a_rows = p.a_mn || p.m >= kTileM ? kTileM : (p.m + 7) / 8 * 8;
        // (a tensor copy writes whole pieces of 16 bytes at the end of a row, past the last column)
        p.tensor_store = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && p.out_pitch % 16 == 0 && (size_t)p.n * (p.out_type == EOQ_F32 ? 4 : 2) % 16 == 0;
        whole[i] = p;
        if (p.splits == 1) continue;
        p.out = part;
        part += (parts_bytes(p) + 255) / 256 * 256;
        p.out_type = EOQ_I32;
        p.out_pitch = partial_pitch(p.n) * 4;
        p.tensor_store = true;
        a.launch_early = true;
    }
    cudaError_t e = plan.tile_n == 32    ? launch<32, false>(a, st)
                    : plan.tile_n == 64  ? launch<64, false>(a, st)
                    : plan.tile_n == 128 ? launch<128, false>(a, st)
                                         : launch<256, true>(a, st);
    ++*launches;
    for (int i = 0; i < a.count && e == cudaSuccess; ++i) {
        const LinProduct &p = whole[i];
        if (p.splits == 1) continue;
        ++*launches;
        const size_t pieces = (size_t)p.m * ((p.n + 3) / 4), blocks = (pieces + 255) / 256, cap = 8 * (size_t)a.sm_count;
        const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
        const int32_t *from = reinterpret_cast<const int32_t *>(a.p[i].out);
        e = p.k_stages > kMostStages ? launch_chained(lin_join_kernel<true>, grid, dim3(256), 0, st, p, from, partial_pitch(p.n))
                                     : launch_chained(lin_join_kernel<false>, grid, dim3(256), 0, st, p, from, partial_pitch(p.n));
    }
    return e;
}

}  // namespace eoq
