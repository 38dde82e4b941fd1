// Weight gradient of a linear layer (a 1x1 convolution) from floating-point errors and the 8-bit form of its input (eoq_ckpt_wgrad):
//   dw[o][i] = sum over rows r of  dy[r][o] * codes[r][i] * 2^(s[r][i / 32] - 127).
// Steps are powers of two and codes have seven bits, so code * step is a bf16 number exactly: the 8-bit form needs no rounding on its
// way into tcgen05.mma kind::f16.  Errors in fp16 and fp32 are cut into two and three bf16 parts whose sum they are, exactly
// (11 = 8 + 3 and 24 = 8 + 8 + 8 bits), and every part is an operand of its own: products are exact whatever the type, sums are fp32.
//
// The reduction runs over rows, the slow axis of both operands, so both are MN-major tiles [rows][64 columns], 128 bytes a row,
// swizzled.  Eight warps read dy and codes from global memory a stage ahead into registers, convert and write the tiles; one warp issues
// the MMAs; the eight store the accumulators.  Row ranges are split over blocks where there are few tiles; their sums stand side by
// side in the workspace and a second kernel adds them in a fixed order.  All waits are bounded.
#include "eoq_block8.cuh"
#include "eoq_epilogue.cuh"

namespace eoq {

namespace {

constexpr int kProducers = 256;             // threads of the eight warps
constexpr int kThreads = kProducers + 32;   // and the MMA warp, the last one
constexpr int kRows = 64;                   // rows of a stage
constexpr int kSub = kRows * 128;           // bytes of a tile of 64 columns
constexpr int kStagesMax = 4;

// bf16 parts that hold an error of the type
template <int kType> struct DyParts;
template <> struct DyParts<EOQ_BF16> { static constexpr int kParts = 1; };
template <> struct DyParts<EOQ_F16> { static constexpr int kParts = 2; };
template <> struct DyParts<EOQ_F32> { static constexpr int kParts = 3; };

// byte offset of eight columns (16 bytes) of a row within an operand tile
__device__ __forceinline__ uint32_t tile_at(int col8, int row)
{
    return (uint32_t)((col8 >> 3) * kSub + row * 128 + (((col8 & 7) ^ (row & 7)) << 4));
}
__device__ __forceinline__ void st_shared_128(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ void mma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t leader)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader));
}

// bf16 pair of two codes: 128 + (low seven bits) less 128 or, for a negative code, 256; both are bf16 numbers, and so is the result
__device__ __forceinline__ uint32_t two_codes(uint32_t halves, __nv_bfloat162 step)
{
    const uint32_t up = (halves & 0x007f007fu) | 0x43004300u, down = (halves & 0x00800080u) | 0x43004300u;
    const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&up), *reinterpret_cast<const __nv_bfloat162 *>(&down)), step);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// What a thread carries of a stage: kDy chunks of eight errors and kX chunks of 16 codes, rows apart.
template <int kType, int kN, bool kWide>
struct StageRegs {
    static constexpr int kE = Elem<kType>::kSize;
    static constexpr int kDy = kTileM / 8 * kRows / kProducers;     // 4
    static constexpr int kXLanes = kN / 16, kX = kXLanes * kRows / kProducers;
    uint4 dy[kDy][kE / 2];
    uint4 x[kX];
    uint32_t s[kX];

    __device__ __forceinline__ void load(const CkptWgradArgs &a, size_t row0, size_t row_end, int o0, int i0)
    {
        const int t = threadIdx.x;
        const int o = o0 + (t % (kTileM / 8)) * 8;
#pragma unroll
        for (int k = 0; k < kDy; ++k) {
            const size_t r = row0 + t / (kTileM / 8) + k * (kProducers / (kTileM / 8));
            const char *src = reinterpret_cast<const char *>(a.dy) + (r * a.dy_stride + o) * kE;
#pragma unroll
            for (int j = 0; j < kE / 2; ++j) dy[k][j] = make_uint4(0, 0, 0, 0);
            if (r < row_end && o < a.c_out) {
                if (kWide) {
#pragma unroll
                    for (int j = 0; j < kE / 2; ++j) dy[k][j] = __ldg(reinterpret_cast<const uint4 *>(src) + j);
                } else {
                    uint32_t w[4 * (kE / 2)];
#pragma unroll
                    for (int j = 0; j < 2 * kE; ++j) w[j] = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (o + j < a.c_out) {
                            if (kE == 2) w[j / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(src) + j) << (16 * (j & 1));
                            else w[j % (2 * kE)] = __ldg(reinterpret_cast<const uint32_t *>(src) + j);
                        }
#pragma unroll
                    for (int j = 0; j < kE / 2; ++j) dy[k][j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                }
            }
        }
        const int i = i0 + (t % kXLanes) * 16;
#pragma unroll
        for (int k = 0; k < kX; ++k) {
            const size_t r = row0 + t / kXLanes + k * (kProducers / kXLanes);
            x[k] = make_uint4(0, 0, 0, 0);
            s[k] = 1;
            if (r < row_end && i < a.c_in) {
                const int8_t *src = a.codes + r * a.c_in + i;
                if (kWide) x[k] = __ldg(reinterpret_cast<const uint4 *>(src));
                else {
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (i + j < a.c_in) w[j / 4] |= (uint32_t)(uint8_t)__ldg(src + j) << (8 * (j & 3));
                    x[k] = make_uint4(w[0], w[1], w[2], w[3]);
                }
                s[k] = __ldg(a.exps + r * a.blocks + i / kBlock8);
            }
        }
    }

    // converts and writes the stage's tiles: the parts of dy one after the other at `at`, then x
    __device__ __forceinline__ void store(uint32_t at) const
    {
        constexpr int kParts = DyParts<kType>::kParts;
        const int t = threadIdx.x;
#pragma unroll
        for (int k = 0; k < kDy; ++k) {
            const uint32_t dst = at + tile_at(t % (kTileM / 8), t / (kTileM / 8) + k * (kProducers / (kTileM / 8)));
            if (kType == EOQ_BF16) {
                st_shared_128(dst, dy[k][0]);
            } else {
                float v[8];
                if (kE == 2) {
                    Raw<16> r;
                    r.w = dy[k][0];
                    Elem<EOQ_F16>::to_f32(r, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        v[4 * j] = __uint_as_float(dy[k][j % (kE / 2)].x);
                        v[4 * j + 1] = __uint_as_float(dy[k][j % (kE / 2)].y);
                        v[4 * j + 2] = __uint_as_float(dy[k][j % (kE / 2)].z);
                        v[4 * j + 3] = __uint_as_float(dy[k][j % (kE / 2)].w);
                    }
                }
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __byte_perm(__float_as_uint(v[2 * j]), __float_as_uint(v[2 * j + 1]), 0x7632);
                    st_shared_128(dst + p * (kTileM / 64 * kSub), make_uint4(w[0], w[1], w[2], w[3]));
                    // what the upper halves leave: exact; nothing of an infinity
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float hi = __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u);
                        v[j] = fabsf(v[j]) == INFINITY ? 0.0f : v[j] - hi;
                    }
                }
            }
        }
        const uint32_t at_x = at + kParts * (kTileM / 64 * kSub);
#pragma unroll
        for (int k = 0; k < kX; ++k) {
            const int g = t % kXLanes, row = t / kXLanes + k * (kProducers / kXLanes);
            const uint32_t sw = s[k] << 7 | s[k] << 23;
            const __nv_bfloat162 step = *reinterpret_cast<const __nv_bfloat162 *>(&sw);
            const uint32_t c[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            uint4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                half[h] = make_uint4(two_codes(__byte_perm(c[2 * h], 0, 0x4140), step), two_codes(__byte_perm(c[2 * h], 0, 0x4342), step),
                                     two_codes(__byte_perm(c[2 * h + 1], 0, 0x4140), step), two_codes(__byte_perm(c[2 * h + 1], 0, 0x4342), step));
            // neighbouring tiles begin at the same bank: every other one takes its odd chunks first
            const int first = (g >> 2) & 1;
            st_shared_128(at_x + tile_at(2 * g + first, row), first ? half[1] : half[0]);
            st_shared_128(at_x + tile_at(2 * g + 1 - first, row), first ? half[0] : half[1]);
        }
    }
};

template <int kType, int kN> struct StageSize {
    static constexpr uint32_t kA = DyParts<kType>::kParts * (kTileM / 64) * kSub, kBytes = kA + kN / 64 * kSub;
    static constexpr int kFit = (int)((200u * 1024u) / kBytes), kStages = kFit < kStagesMax ? kFit : kStagesMax;
};

template <int kType, int kN, bool kWide>
__global__ void __launch_bounds__(kThreads, 1) ckpt_wgrad_kernel(const __grid_constant__ CkptWgradArgs a)
{
    using Size = StageSize<kType, kN>;
    constexpr int kStages = Size::kStages, kParts = DyParts<kType>::kParts;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStagesMax + 1];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t abort_s;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kStagesMax + s); };
    const uint32_t done_bar = bar0 + 8u * (2 * kStagesMax);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(full_bar(s), kProducers / 32);
            ptx::mbar_init(empty_bar(s), 1);
        }
        ptx::mbar_init(done_bar, 1);
        abort_s = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kProducers / 32) {
        ptx::tmem_alloc(ptx::smem_u32(&tmem_base_s), kN);
        ptx::tmem_relinquish();
    }
    const int tiles = a.m_tiles * a.n_tiles, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int o0 = tile / a.n_tiles * kTileM, i0 = tile % a.n_tiles * kN;
    const size_t row_begin = (size_t)split * a.rows_per_split, row_end = min(a.rows, row_begin + a.rows_per_split);
    const int stages = (int)((row_end - row_begin + kRows - 1) / kRows);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    ptx::grid_dep_wait();
    const uint32_t tmem_base = tmem_base_s;
    const RoleCtx ctx{&abort_s, a.dev};

    if (warp < kProducers / 32) {
        StageRegs<kType, kN, kWide> cur, next;
        cur.load(a, row_begin, row_end, o0, i0);
        int stage = 0;
        uint32_t phase = 0;
        for (int it = 0; it < stages; ++it) {
            if (it + 1 < stages) next.load(a, row_begin + (size_t)(it + 1) * kRows, row_end, o0, i0);
            if (!__all_sync(0xffffffffu, wait_bar(empty_bar(stage), phase ^ 1u, ctx))) break;
            cur.store(smem_base + stage * Size::kBytes);
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(full_bar(stage));
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
            cur = next;
        }
        // a row of the tile a lane; two warps share 32 rows, half of the columns each
        const int quad = warp & 3, o = o0 + quad * 32 + lane;
        const bool ok = __all_sync(0xffffffffu, wait_bar<64>(done_bar, 0, ctx));
        if (ok) {
            ptx::tc_fence_after();
            float *dst = a.out + (size_t)split * a.c_out * a.c_in + (size_t)o * a.c_in;
            constexpr int kHalf = kN / 2;
#pragma unroll 1
            for (int c0 = (warp >> 2) * kHalf; c0 < (warp >> 2) * kHalf + kHalf; c0 += 32) {
                uint32_t r[32];
                ptx::tmem_ld_32x32(tmem_base + ((uint32_t)(quad * 32) << 16) + c0, r);
                ptx::tmem_ld_wait();
                if (o < a.c_out) {
                    if (a.c_in % 4 == 0) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (i0 + c0 + j < a.c_in)
                                *reinterpret_cast<uint4 *>(dst + i0 + c0 + j) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (i0 + c0 + j < a.c_in) dst[i0 + c0 + j] = __uint_as_float(r[j]);
                    }
                }
            }
        }
    } else {
        const uint32_t leader = elect_one();
        // fp32 accumulator, bf16 operands, both MN-major
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(kTileM >> 4) << 24);
        const uint64_t proto = make_smem_desc(0, kSub, 1024, 2);
        const uint32_t hi = (uint32_t)(proto >> 32), lead = (uint32_t)proto;
        int stage = 0;
        uint32_t phase = 0, accumulate = 0;
        bool ok = true;
        for (int it = 0; it < stages; ++it) {
            if (!(ok = __all_sync(0xffffffffu, wait_bar(full_bar(stage), phase, ctx)))) break;
            ptx::tc_fence_after();
            const uint32_t a16 = ((smem_base + stage * Size::kBytes) >> 4) | lead, b16 = ((smem_base + stage * Size::kBytes + Size::kA) >> 4) | lead;
#pragma unroll
            for (int k = 0; k < kRows / 16; ++k)
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    mma_bf16(tmem_base, smem_desc_join(a16 + p * ((kTileM / 64 * kSub) >> 4) + k * 128, hi), smem_desc_join(b16 + k * 128, hi), idesc,
                             accumulate, leader);
                    accumulate = 1;
                }
            ptx::mma_commit(empty_bar(stage), leader);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        ptx::mma_commit(done_bar, leader);
        if (!ok)
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (ptx::mbar_try_wait(done_bar, 0)) break;
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == kProducers / 32) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, kN);
    }
}

// dw = the splits' sums, added in their order
template <int kV>
__global__ void __launch_bounds__(256) ckpt_wgrad_join_kernel(const float *__restrict__ part, size_t n, int splits, float *__restrict__ dw)
{
    ptx::grid_dep_wait_launch_small();
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * kV; i < n; i += (size_t)gridDim.x * 256 * kV) {
        float t[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) t[j] = 0.0f;
        for (int s = 0; s < splits; ++s) {
            float v[kV];
            Elem<EOQ_F32>::to_f32(load_raw<4 * kV>(part + (size_t)s * n + i), v);
#pragma unroll
            for (int j = 0; j < kV; ++j) t[j] += v[j];
        }
        store_raw(dw + i, Elem<EOQ_F32>::from_f32(t));
    }
}

struct WgradPlan8 {
    int n_tile, m_tiles, n_tiles, splits;
    size_t rows_per_split;
};

WgradPlan8 plan_of(size_t rows, int c_out, int c_in)
{
    WgradPlan8 p;
    p.n_tile = c_in <= 64 ? 64 : c_in <= 128 ? 128 : 256;
    p.m_tiles = (c_out + kTileM - 1) / kTileM;
    p.n_tiles = (c_in + p.n_tile - 1) / p.n_tile;
    const size_t tiles = (size_t)p.m_tiles * p.n_tiles, stages = (rows + kRows - 1) / kRows;
    size_t splits = tiles < (size_t)kPartSms ? kPartSms / tiles : 1;
    if (splits > stages) splits = stages;
    const size_t per = (stages + splits - 1) / splits;
    p.splits = (int)((stages + per - 1) / per);
    p.rows_per_split = per * kRows;
    return p;
}

template <int kType, int kN, bool kWide>
cudaError_t launch(const CkptWgradArgs &a, int grid, cudaStream_t st)
{
    using Size = StageSize<kType, kN>;
    constexpr int bytes = Size::kBytes * Size::kStages + 1024;
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)ckpt_wgrad_kernel<kType, kN, kWide>, bytes, allowed);
    if (e != cudaSuccess) return e;
    return launch_chained(ckpt_wgrad_kernel<kType, kN, kWide>, dim3(grid), dim3(kThreads), bytes, st, a);
}

template <int kType, bool kWide>
cudaError_t of_width(const CkptWgradArgs &a, int n_tile, int grid, cudaStream_t st)
{
    if (n_tile == 64) return launch<kType, 64, kWide>(a, grid, st);
    if (n_tile == 128) return launch<kType, 128, kWide>(a, grid, st);
    return launch<kType, 256, kWide>(a, grid, st);
}

template <int kType>
cudaError_t of_type(const CkptWgradArgs &a, int n_tile, int grid, cudaStream_t st)
{
    const bool wide = a.c_out % 8 == 0 && a.c_in % 16 == 0 && a.dy_stride % (16 / Elem<kType>::kSize) == 0 &&
                      reinterpret_cast<uintptr_t>(a.dy) % 16 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 16 == 0;
    return wide ? of_width<kType, true>(a, n_tile, grid, st) : of_width<kType, false>(a, n_tile, grid, st);
}

}  // namespace

size_t ckpt_wgrad_workspace_bytes(size_t rows, int c_out, int c_in)
{
    const WgradPlan8 p = plan_of(rows, c_out, c_in);
    return p.splits > 1 ? sizeof(float) * (size_t)p.splits * c_out * c_in : 0;
}

cudaError_t launch_ckpt_wgrad(CkptWgradArgs a, int dtype, float *dw, void *workspace, int *launches, cudaStream_t st)
{
    const WgradPlan8 p = plan_of(a.rows, a.c_out, a.c_in);
    a.blocks = (a.c_in + kBlock8 - 1) / kBlock8;
    a.m_tiles = p.m_tiles;
    a.n_tiles = p.n_tiles;
    a.rows_per_split = p.rows_per_split;
    a.out = p.splits > 1 ? reinterpret_cast<float *>(workspace) : dw;
    const int grid = p.m_tiles * p.n_tiles * p.splits;
    const cudaError_t e = dtype == EOQ_F32   ? of_type<EOQ_F32>(a, p.n_tile, grid, st)
                          : dtype == EOQ_F16 ? of_type<EOQ_F16>(a, p.n_tile, grid, st)
                                             : of_type<EOQ_BF16>(a, p.n_tile, grid, st);
    ++*launches;
    if (e != cudaSuccess || p.splits == 1) return e;
    ++*launches;
    const size_t n = (size_t)a.c_out * a.c_in, per = n % 4 == 0 ? 4 : 1, blocks = (n / per + 255) / 256, cap = 8 * kPartSms;
    const dim3 join((unsigned)(blocks < cap ? blocks : cap));
    if (per == 4) return launch_chained(ckpt_wgrad_join_kernel<4>, join, dim3(256), 0, st, (const float *)a.out, n, p.splits, dw);
    return launch_chained(ckpt_wgrad_join_kernel<1>, join, dim3(256), 0, st, (const float *)a.out, n, p.splits, dw);
}

}  // namespace eoq
