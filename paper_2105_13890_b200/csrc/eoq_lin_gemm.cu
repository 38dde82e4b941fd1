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
// 256 x 256 as one (each loads half of either operand: 64 bytes a cycle and SM instead of 96 for tiles of 128 x 256).  Roles: eight epilogue warps, a
// warp for the tensor copies, one for the MMAs.  Two accumulators in tensor memory let a tile's epilogue run beside the next one's MMAs.
// All waits are bounded.
#include "eoq_lin.cuh"
#include "eoq_pair.cuh"

namespace eoq {

namespace {

constexpr int kEpiWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kThreads = 320;
constexpr int kStageK = 128;                   // bytes of the reduction in a stage
constexpr int kMaxSmem = 224 * 1024;           // of dynamic shared memory: some 2.3 KB are static
constexpr int kUnit = 2048, kStageBytes = 2 * kUnit;   // staging of an epilogue warp: twice 32 rows of 64 bytes, on their way out and being filled

enum Major { kBothK = 0, kBMn = 1, kBothMn = 2 };

template <int kN, bool kPair>
struct GemmShape {
    static constexpr int kBlocks = kPair ? 2 : 1, kOwnN = kN / kBlocks;   // columns of B that a block loads
    static constexpr int kA = kTileM * kStageK, kB = kOwnN * kStageK, kStage = kA + kB;
    static constexpr int kFit = (kMaxSmem - 1024 - kEpiWarps * kStageBytes) / kStage, kStages = kFit < 8 ? kFit : 8;
    static constexpr int kBytes = kStages * kStage + kEpiWarps * kStageBytes + 1024;
    static constexpr uint32_t kColumns = 2 * kN;                          // of tensor memory: two accumulators
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

// 32 sums of a row with their scales.  `scales`: of the 32 columns, and their biases 128 bytes on.
__device__ __forceinline__ void scale_row(uint32_t (&r)[32], float row_scale, uint32_t scales)
{
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        const int4 s = ptx::ld_shared_128(scales + j * 4), b = ptx::ld_shared_128(scales + 128 + j * 4);
        const int sv[4] = {s.x, s.y, s.z, s.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[j + i] = __float_as_uint(__fmaf_rn(__int2float_rn((int)r[j + i]) * row_scale, __int_as_float(sv[i]), __int_as_float(bv[i])));
    }
}

// 64 bytes of a row to the lane's place in a unit of staging: pieces of 16 bytes in the order that tensor copies expect of such rows.
__device__ __forceinline__ void stage_piece(uint32_t unit, int lane, int j, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    st_shared_v4(unit + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), a, b, c, d);
}
// kPart: which 16 of the 32 words (of 16-bit types: all of them, rounded)
template <int kPart>
__device__ __forceinline__ void stage_row(const uint32_t (&r)[32], int type, uint32_t unit, int lane)
{
    if (type == EOQ_F16 || type == EOQ_BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = __uint_as_float(r[8 * j + 2 * i]), hi = __uint_as_float(r[8 * j + 2 * i + 1]);
                if (type == EOQ_F16) {
                    const __half2 h = __floats2half2_rn(lo, hi);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
            }
            stage_piece(unit, lane, j, w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) stage_piece(unit, lane, j, r[16 * kPart + 4 * j], r[16 * kPart + 4 * j + 1], r[16 * kPart + 4 * j + 2], r[16 * kPart + 4 * j + 3]);
    }
}

// The staged rows to rows of the output that tensor copies cannot address: 32 columns of a row at a time, or 16 of two.
__device__ __forceinline__ void store_rows(const LinGemmArgs &a, uint32_t unit, size_t out_row, int rows, int col0, int lane)
{
    if (a.out_type == EOQ_F16 || a.out_type == EOQ_BF16) {
        const int col = col0 + lane;
        const bool in = col < a.n;
        for (int i = 0; i < rows; ++i) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(unit + i * 64 + (((lane >> 3) ^ ((i >> 1) & 3)) << 4) + (lane & 7) * 2) : "memory");
            if (in) *reinterpret_cast<uint16_t *>(reinterpret_cast<char *>(a.out) + (out_row + i) * a.out_pitch + (size_t)col * 2) = v;
        }
    } else {
        const int c = lane & 15, col = col0 + c;
        for (int i = lane >> 4; i < rows; i += 2) {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(unit + i * 64 + (((c >> 2) ^ ((i >> 1) & 3)) << 4) + (c & 3) * 4) : "memory");
            if (col < a.n) *reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(a.out) + (out_row + i) * a.out_pitch + (size_t)col * 4) = v;
        }
    }
}

template <int kMajor, int kN, bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
lin_gemm_kernel(const __grid_constant__ LinGemmArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_out)
{
    using S = GemmShape<kN, kPair>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 5];
    __shared__ __align__(16) float scales_s[kEpiWarps][64];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t abort_s;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
    const uint32_t staging = smem_base + S::kStages * S::kStage;
    // of a stage: copies landed (of a pair: in the first block), MMAs done.  Of an accumulator: complete; read.  All MMAs done.
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (S::kStages + s); };
    auto sums_bar = [&](int i) { return bar0 + 8u * (2 * S::kStages + i); };
    auto read_bar = [&](int i) { return bar0 + 8u * (2 * S::kStages + 2 + i); };
    const uint32_t drain_bar = bar0 + 8u * (2 * S::kStages + 4);
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(sums_bar(i), 1);
            ptx::mbar_init(read_bar(i), S::kBlocks * kEpiWarps);
        }
        ptx::mbar_init(drain_bar, 1);
        abort_s = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&map_a);
        ptx::prefetch_tensormap(&map_b);
        if (a.tensor_store) ptx::prefetch_tensormap(&map_out);
    }
    if (warp == kMmaWarp) tmem_take<kPair>(ptx::smem_u32(&tmem_base_s), S::kColumns);
    const int rank = kPair ? blockIdx.x & 1 : 0, first = blockIdx.x / S::kBlocks, step = gridDim.x / S::kBlocks;
    const int tiles = a.m_tiles * a.n_tiles, units = tiles * a.splits;
    // Unit u: a tile and a part of its reduction.  Tiles go in bands of kBand tiles of n, down m inside a band, so that what runs at a time
    // shares operands in the L2.
    auto place = [&](int u, int &m0, int &n0, int &split) {
        constexpr int kBand = 8;
        split = u / tiles;
        const int t = u - split * tiles, per_band = kBand * a.m_tiles, band = t / per_band, in = t - band * per_band;
        const int width = min(kBand, a.n_tiles - band * kBand);
        const int mt = in / width;
        m0 = mt * S::kBlocks * kTileM + rank * kTileM;
        n0 = (band * kBand + in - mt * width) * kN;
    };
    auto stages_of = [&](int split) { return min(a.stages_per_split, a.k_stages - split * a.stages_per_split); };
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (the other block's barriers are ready)
    else __syncthreads();
    ptx::tc_fence_after();
    ptx::grid_dep_wait();
    if (a.launch_early) ptx::grid_dep_launch();
    const uint32_t tmem_base = tmem_base_s;
    const RoleCtx ctx{&abort_s, a.dev};

    if (warp == kLoadWarp) {
        bool ok = true;
        int slot = 0, started = 0;
        uint32_t phase = 0;
        for (int u = first; u < units && ok; u += step) {
            int m0, n0, split;
            place(u, m0, n0, split);
            const int n_own = n0 + rank * S::kOwnN, stages = stages_of(split), k_first = split * a.stages_per_split;
            // Blocks that work side by side begin at different places of the reduction (integer sums do not mind): in step, all of them asked for the same rows of a few
            // tokens at once, and 16 tokens 4096 to 4096 took 16.8 us where 32 took 11.0.
            int at = kPair ? 0 : (int)((unsigned)u % (unsigned)stages);
            for (int it = 0; it < stages; ++it, at = at + 1 == stages ? 0 : at + 1) {
                if (!(ok = __all_sync(0xffffffffu, wait_bar(empty_bar(slot), phase ^ 1u, ctx)))) break;
                if (lane == 0) {
                    const uint32_t dst = smem_base + slot * S::kStage;
                    const int k = (k_first + at) * kStageK;
                    if (rank == 0) ptx::mbar_expect_tx(full_bar(slot), S::kBlocks * S::kStage);
                    if (kMajor == kBothMn) load_tile<kPair>(dst, &map_a, full_bar(slot), m0, k);
                    else load_tile<kPair>(dst, &map_a, full_bar(slot), k, m0);
                    if (kMajor == kBothK) load_tile<kPair>(dst + S::kA, &map_b, full_bar(slot), k, n_own);
                    else load_tile<kPair>(dst + S::kA, &map_b, full_bar(slot), n_own, k);
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
    } else if (warp == kMmaWarp) {
        if (rank == 0) {
            const uint32_t leader = elect_one();
            const uint32_t idesc = make_idesc_i8(S::kBlocks * kTileM, kN, kMajor == kBothMn, kMajor != kBothK);
            // K-major: rows of 128 bytes, groups of eight 1024 bytes apart, 32 bytes along the row to the next step of the reduction.  MN-major: a row of the
            // reduction is 128 (or kN) bytes, groups of eight rows lie behind one another, 32 rows to the next step.
            constexpr int kBRow = kMajor == kBothK ? 128 : S::kOwnN < 128 ? S::kOwnN : 128;
            constexpr uint32_t kAStep = kMajor == kBothMn ? 32 * 128 / 16 : 2, kBStep = kMajor == kBothK ? 2 : 32 * kBRow / 16;
            const uint32_t a_hi = smem_desc_hi(1024, 2), b_hi = smem_desc_hi(8 * kBRow, layout_type_for(kBRow));
            const uint32_t a_lead = (S::kA >> 4) << 16, b_lead = (S::kB >> 4) << 16;
            bool ok = true;
            int slot = 0, turn = 0;
            uint32_t phase = 0;
            for (int u = first; u < units && ok; u += step, ++turn) {
                const int stages = stages_of(u / tiles), acc = turn & 1;
                const uint32_t d = tmem_base + acc * kN;
                if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(read_bar(acc), ((turn >> 1) & 1) ^ 1, ctx)))) break;
                ptx::tc_fence_after();
                for (int it = 0; it < stages; ++it) {
                    if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(full_bar(slot), phase, ctx)))) break;
                    ptx::tc_fence_after();
                    const uint32_t a16 = ((smem_base + slot * S::kStage) >> 4) | a_lead, b16 = ((smem_base + slot * S::kStage + S::kA) >> 4) | b_lead;
#pragma unroll
                    for (int k = 0; k < kStageK / 32; ++k) {
                        const uint64_t ad = smem_desc_join(a16 + k * kAStep, a_hi), bd = smem_desc_join(b16 + k * kBStep, b_hi);
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
        const int quad = warp & 3, half = warp >> 2;
        constexpr int kHalfN = kN >= 64 ? kN / 2 : kN, kChunks = kHalfN / 32;   // columns of a warp (of 32, the second four warps have none)
        const bool narrow = a.out_type == EOQ_F16 || a.out_type == EOQ_BF16;
        const uint32_t scales = ptx::smem_u32(&scales_s[warp][0]), staging_w = staging + warp * kStageBytes;
        int turn = 0, units_out = 0;
        for (int u = first; u < units; u += step, ++turn) {
            int m0, n0, split;
            place(u, m0, n0, split);
            const int acc = turn & 1, row0 = m0 + quad * 32, row = row0 + lane, first_col = n0 + half * kHalfN;
            const bool mine = row0 < a.m && (kN >= 64 || half == 0);
            // scales and biases of the tile arrive beside its MMAs
            float row_scale = 0.0f, s[kChunks], b[kChunks];
            if (a.out_type != EOQ_I32) {
                row_scale = row < a.m ? __ldg(a.row_scale + row) : 0.0f;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int col = first_col + c * 32 + lane;
                    s[c] = mine && col < a.n ? a.col_scale ? __ldg(a.col_scale + col) : 1.0f : 0.0f;
                    b[c] = mine && col < a.n && a.bias ? __ldg(a.bias + col) : 0.0f;
                }
            }
            if (!__all_sync(0xffffffffu, wait_bar<32>(sums_bar(acc), (turn >> 1) & 1, ctx))) break;
            ptx::tc_fence_after();
            const size_t out_row = (size_t)split * a.split_rows + row0;
            const uint32_t t_row = tmem_base + acc * kN + half * kHalfN + ((uint32_t)(quad * 32) << 16);
            const int chunks = !mine || first_col >= a.n ? 0 : min(kChunks, (a.n - first_col + 31) / 32);
            // a unit of staging to memory
            auto out = [&](int col) {
                const uint32_t unit = staging_w + (units_out & 1) * kUnit;
                ++units_out;
                if (a.tensor_store) {
                    ptx::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        if (col < a.n) store_tile_2d(&map_out, unit, col, (int)out_row);
                        store_commit();
                        store_wait_read<1>();   // (the other unit is free)
                    }
                    __syncwarp();
                } else {
                    __syncwarp();
                    store_rows(a, unit, out_row, min(32, a.m - row0), col, lane);
                    __syncwarp();
                }
            };
            uint32_t r[2][32];
            if (chunks > 0) ptx::tmem_ld_32x32(t_row, r[0]);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                if (c >= chunks) break;
                ptx::tmem_ld_wait();
                if (c + 1 < chunks) ptx::tmem_ld_32x32(t_row + (c + 1) * 32, r[(c + 1) & 1]);   // (on its way beside this chunk's arithmetic)
                if (a.out_type != EOQ_I32) {
                    scales_s[warp][lane] = s[c];
                    scales_s[warp][32 + lane] = b[c];
                    __syncwarp();
                    scale_row(r[c & 1], row_scale, scales);
                }
                stage_row<0>(r[c & 1], a.out_type, staging_w + (units_out & 1) * kUnit, lane);
                out(first_col + c * 32);
                if (!narrow) {
                    stage_row<1>(r[c & 1], a.out_type, staging_w + (units_out & 1) * kUnit, lane);
                    out(first_col + c * 32 + 16);
                }
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_first<kPair>(read_bar(acc));
        }
        if (a.tensor_store && lane == 0) store_wait_all();
    }
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (neither block ends while the other's MMAs, copies or arrivals may reach it)
    else __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after();
        tmem_return<kPair>(tmem_base, S::kColumns);
    }
}

// The parts of a split reduction, which stand `pitch` words apart row by row and `split_rows` rows apart, added and scaled: four columns a thread.
template <bool kLong>
__global__ void __launch_bounds__(256) lin_join_kernel(const __grid_constant__ LinGemmArgs a, const int32_t *__restrict__ part, size_t pitch)
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
            v[j] = __fmaf_rn(f * rs, in && a.col_scale ? __ldg(a.col_scale + col + j) : 1.0f, in && a.bias ? __ldg(a.bias + col + j) : 0.0f);
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

struct GemmPlan {
    bool pair;
    int tile_n, m_tiles, n_tiles, splits, k_stages, stages_per_split;
};

constexpr int kMostStages = 1023;   // of a part: 130,944 products of codes, at most 2^14 each, are an int32

int tile_m(const GemmPlan &p) { return p.pair ? 2 * kTileM : kTileM; }
size_t partial_pitch(int n) { return ((size_t)n + 3) & ~(size_t)3; }

// Tiles and splits that take the least time by a model of waves of blocks: cycles of a stage (the MMAs', or what its loads take), and some 6000 cycles in front
// of and behind a block's work.
GemmPlan plan_of(size_t m, size_t n, size_t k)
{
    const int k_stages = (int)((k + kStageK - 1) / kStageK), least = (k_stages + kMostStages - 1) / kMostStages;
    GemmPlan best = {};
    double best_time = 0.0;
    for (int w = 0; w < 4; ++w) {
        GemmPlan p;
        p.tile_n = 32 << w;
        p.pair = p.tile_n == 256;
        if (p.pair && (m <= kTileM || n <= 128)) continue;
        if (w > 0 && !p.pair && n <= (size_t)p.tile_n / 2) continue;
        p.m_tiles = (int)((m + tile_m(p) - 1) / tile_m(p));
        p.n_tiles = (int)((n + p.tile_n - 1) / p.tile_n);
        p.k_stages = k_stages;
        const size_t tiles = (size_t)p.m_tiles * p.n_tiles, room = kPartSms / (p.pair ? 2 : 1);
        static const double kStage[4] = {260.0, 290.0, 380.0, 560.0};
        for (int fill = 0; fill <= 2; ++fill) {
            size_t splits = fill == 0 ? 1 : fill * room / tiles;
            if (fill > 0 && splits <= 1) continue;
            if (splits < (size_t)least) splits = least;
            if (splits > (size_t)k_stages) splits = k_stages;
            p.stages_per_split = (int)((k_stages + splits - 1) / splits);
            p.splits = (k_stages + p.stages_per_split - 1) / p.stages_per_split;
            const double waves = (double)((tiles * p.splits + room - 1) / room);
            double time = 6000.0 + waves * ((double)p.stages_per_split * kStage[w] + 8.0 * p.tile_n);
            if (p.splits > 1) time += 7000.0 + (double)p.splits * m * n * 4.0 * 2.0 / 2500.0;
            if (best_time == 0.0 || time < best_time) {
                best = p;
                best_time = time;
            }
        }
    }
    return best;
}

template <int kMajor, int kN, bool kPair>
cudaError_t launch(const LinGemmArgs &a, const void *pa, size_t pitch_a, const void *pb, size_t pitch_b, size_t k, const void *out, cudaStream_t st)
{
    using S = GemmShape<kN, kPair>;
    CUtensorMap ma, mb, mo = {};
    const bool got =
        (kMajor == kBothMn ? tiled_map_of(&ma, pa, 1, a.m, k, pitch_a, 128, kStageK, 128) : tiled_map_of(&ma, pa, 1, k, a.m, pitch_a, kStageK, kTileM, 128)) &&
        (kMajor == kBothK ? tiled_map_of(&mb, pb, 1, k, a.n, pitch_b, kStageK, S::kOwnN, 128)
                          : tiled_map_of(&mb, pb, 1, a.n, k, pitch_b, S::kOwnN, kStageK, S::kOwnN));
    if (!got) return cudaErrorInvalidValue;
    if (a.tensor_store) {
        const int e = a.out_type == EOQ_F16 || a.out_type == EOQ_BF16 ? 2 : 4;
        if (!tiled_map_of(&mo, out, e, a.n, a.out_type == EOQ_I32 ? a.splits * a.split_rows : (size_t)a.m, a.out_pitch, 64 / e, 32, 64)) return cudaErrorInvalidValue;
    }
    static_assert(S::kBytes <= kMaxSmem && S::kStages >= 4, "shared memory of a block");
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)lin_gemm_kernel<kMajor, kN, kPair>, S::kBytes, allowed);
    if (e != cudaSuccess) return e;
    const size_t units = (size_t)a.m_tiles * a.n_tiles * a.splits, room = a.sm_count / S::kBlocks;
    const unsigned grid = (unsigned)(units < room ? units : room) * S::kBlocks;
    return launch_chained_clusters(S::kBlocks, lin_gemm_kernel<kMajor, kN, kPair>, dim3(grid), dim3(kThreads), S::kBytes, st, a, ma, mb, mo);
}

template <int kMajor>
cudaError_t of_width(const LinGemmArgs &a, int tile_n, const void *pa, size_t pitch_a, const void *pb, size_t pitch_b, size_t k, const void *out, cudaStream_t st)
{
    if (tile_n == 32) return launch<kMajor, 32, false>(a, pa, pitch_a, pb, pitch_b, k, out, st);
    if (tile_n == 64) return launch<kMajor, 64, false>(a, pa, pitch_a, pb, pitch_b, k, out, st);
    if (tile_n == 128) return launch<kMajor, 128, false>(a, pa, pitch_a, pb, pitch_b, k, out, st);
    return launch<kMajor, 256, true>(a, pa, pitch_a, pb, pitch_b, k, out, st);
}

}  // namespace

size_t lin_gemm_workspace_bytes(size_t m, size_t n, size_t k)
{
    const GemmPlan p = plan_of(m, n, k);
    return p.splits > 1 ? sizeof(int32_t) * (size_t)p.splits * p.m_tiles * tile_m(p) * partial_pitch((int)n) : 0;
}

cudaError_t launch_lin_gemm(LinGemmArgs a, int pass, const int8_t *pa, size_t pitch_a, const int8_t *pb, size_t pitch_b, size_t k, void *workspace, int *launches,
                            cudaStream_t st)
{
    const GemmPlan p = plan_of(a.m, a.n, k);
    a.m_tiles = p.m_tiles;
    a.n_tiles = p.n_tiles;
    a.splits = p.splits;
    a.k_stages = p.k_stages;
    a.stages_per_split = p.stages_per_split;
    a.split_rows = p.m_tiles * tile_m(p);
    LinGemmArgs g = a;
    // (a tensor copy writes whole pieces of 16 bytes at the end of a row, past the last column)
    g.tensor_store = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && a.out_pitch % 16 == 0 && (size_t)a.n * (a.out_type == EOQ_F32 ? 4 : 2) % 16 == 0;
    if (p.splits > 1) {
        g.out = workspace;
        g.out_type = EOQ_I32;
        g.out_pitch = partial_pitch(a.n) * 4;
        g.tensor_store = true;
        g.launch_early = true;
    }
    const cudaError_t err = pass == EOQ_PASS_FWD     ? of_width<kBothK>(g, p.tile_n, pa, pitch_a, pb, pitch_b, k, g.out, st)
                            : pass == EOQ_PASS_DGRAD ? of_width<kBMn>(g, p.tile_n, pa, pitch_a, pb, pitch_b, k, g.out, st)
                                                     : of_width<kBothMn>(g, p.tile_n, pa, pitch_a, pb, pitch_b, k, g.out, st);
    ++*launches;
    if (err != cudaSuccess || p.splits == 1) return err;
    ++*launches;
    const size_t pieces = (size_t)a.m * ((a.n + 3) / 4), blocks = (pieces + 255) / 256, cap = 8 * (size_t)a.sm_count;
    const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
    const int32_t *part = reinterpret_cast<const int32_t *>(workspace);
    if (p.k_stages > kMostStages) return launch_chained(lin_join_kernel<true>, grid, dim3(256), 0, st, a, part, partial_pitch(a.n));
    return launch_chained(lin_join_kernel<false>, grid, dim3(256), 0, st, a, part, partial_pitch(a.n));
}

}  // namespace eoq
