// Weight gradient of a linear layer (a 1x1 convolution) from floating-point errors and the 8-bit form of its input (eoq_ckpt_wgrad):
//   dw[o][i] = sum over rows r of  dy[r][o] * codes[r][i] * 2^(s[r][i / 32] - 127).
// Steps are powers of two and codes have seven bits, so code * step is a bf16 number exactly: the 8-bit form needs no rounding on its
// way into tcgen05.mma kind::f16.  Errors in fp16 and fp32 are cut into two and three bf16 parts whose sum they are, exactly
// (11 = 8 + 3 and 24 = 8 + 8 + 8 bits), and every part is an operand of its own: products are exact whatever the type, sums are fp32.
//
// The reduction runs over rows, the slow axis of both operands, so both are MN-major tiles [rows][64 columns], 128 bytes a row,
// swizzled.  Roles: sixteen warps bring dy and codes in (asynchronous copies, some stages ahead), convert and write the operand tiles; one
// warp issues the MMAs; four move the accumulator on.  Row ranges are split over blocks where there are few tiles; their sums stand side
// by side in the workspace and a second kernel adds them in a fixed order.  All waits are bounded.
//
// The tensor core adds to its fp32 accumulator without rounding to nearest: sums lose about 2^-27 of themselves with every step of 16
// rows, always towards zero (16,384 rows: 8e-6 of the result's norm).  So every kSteps steps the accumulator is added to a second one in
// tensor memory, in ordinary fp32 additions, and starts again: 2.4e-7 (1024 to 4096 channels; fp32 products of
// a library: 5.7e-7).
//
// A copied chunk is only ever read back by the thread that copied it.  Where rows are not 16-byte aligned, the aligned words around a
// chunk are copied and shifted into place; a word is only touched when it holds part of the row.
#include "eoq_block8.cuh"
#include "eoq_epilogue.cuh"
#include "eoq_pair.cuh"

namespace eoq {

namespace {

constexpr int kProducers = 512;                  // threads of the sixteen warps
constexpr int kMmaWarp = kProducers / 32;        // then the MMA warp, then four that move the accumulator on
constexpr int kThreads = kProducers + 32 + 128;
constexpr int kSteps = 64;                       // MMA steps before the accumulator moves on
constexpr int kMaxSmem = 226 * 1024;   // (of dynamic shared memory)

// bf16 parts that hold an error of the type
template <int kType> struct DyParts;
template <> struct DyParts<EOQ_BF16> { static constexpr int kParts = 1; };
template <> struct DyParts<EOQ_F16> { static constexpr int kParts = 2; };
template <> struct DyParts<EOQ_F32> { static constexpr int kParts = 3; };

// Shapes and shared memory of a kernel.
template <int kType, int kN, bool kWide>
struct Shape {
    static constexpr int kE = Elem<kType>::kSize, kParts = DyParts<kType>::kParts;
    static constexpr int kRows = kE == 2 && kN <= 128 ? 64 : 32;         // rows of a stage
    static constexpr int kSub = kRows * 128;                             // bytes of a tile of 64 columns
    static constexpr int kATile = kTileM / 64 * kSub, kA = kParts * kATile, kB = kN / 64 * kSub;
    // A thread's share of a stage: kDy times eight errors, and kCodes neighbouring codes of a row (of threads without any there may be some).
    static constexpr int kDyLanes = kTileM / 8, kDyPass = kProducers / kDyLanes, kDy = kRows / kDyPass;
    static constexpr int kCodes = kN * kRows / kProducers >= 32 ? 32 : 16, kXLanes = kN / kCodes;
    static_assert(kDyPass % 8 == 0 && kDy * kDyPass == kRows, "rows of a thread's chunks share their swizzle");
    static_assert(kXLanes * kRows <= kProducers, "one piece of codes a thread");
    // words of a chunk as copied: an unaligned one of n words touches n + 1
    static constexpr int kDyWords = kE == 4 ? 8 : kWide ? 4 : 5, kXWords = kCodes / 4 + (kWide ? 0 : 1);
    static constexpr int kRawBytes = kProducers * 4 * (kDy * kDyWords + kXWords);
    // Stages of operand tiles, of copies and of barriers, all of which divide four, so that a loop over four stages knows its slots.
    static constexpr int kRing = 4, kAhead = 3;
    static constexpr int size(int ops) { return ops * (kA + kB) + kRing * kRawBytes + 1024; }
    static constexpr int kOps = size(4) <= kMaxSmem ? 4 : 2;
    static constexpr int kBytes = size(kOps);
    static constexpr int kChunk = kSteps / (kRows / 16 * kParts);        // stages before the accumulator moves on
};

// byte offset of eight columns (16 bytes) of a row within an operand tile
template <int kSub>
__device__ __forceinline__ uint32_t tile_at(int col8, int row)
{
    return (uint32_t)((col8 >> 3) * kSub + row * 128 + (((col8 & 7) ^ (row & 7)) << 4));
}
// asynchronous copies that write zeros where `in` is false
__device__ __forceinline__ void copy_16(uint32_t to, const void *from, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_4(uint32_t to, const void *from, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_shared_128(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// kPair: over the operands of two blocks, issued by the first
template <bool kPair>
__device__ __forceinline__ void mma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t leader)
{
    if constexpr (kPair)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "setp.ne.b32 q, %5, 0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader));
    else
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

// What a thread of the sixteen warps does to a stage.
template <int kType, int kN, bool kWide>
struct Feeder {
    using S = Shape<kType, kN, kWide>;
    const void *safe;
    const char *dy, *x;                  // the thread's first chunks of the next stage to copy
    const uint8_t *exps;
    size_t dy_pass, dy_step, x_step, exps_step;   // to its next chunk, S::kDyPass rows on; to the next stage
    int dy_left, x_left;                 // rows from that chunk to the end of the range; 0 where the columns are past the end
    int dy_cols, x_cols;                 // bytes from the chunk to the end of its row
    uint32_t smem, raw;                  // operand tiles; the thread's first copied word: word j of its chunks at j * kProducers
    uint32_t dy_tile, x_tile;            // places of the first chunks in their tiles
    uint32_t dy_bytes, x_bytes;          // addresses of the chunks to convert next, of which two bits count

    __device__ __forceinline__ Feeder(const CkptWgradArgs &a, size_t begin, size_t end, int o0, int i0, uint32_t smem_base)
        : safe(a.safe), smem(smem_base), raw(smem_base + S::kOps * S::kA + S::kOps * S::kB + threadIdx.x * (kWide ? 16 : 4))
    {
        // Eight lanes that store together should meet eight different places of 16 bytes: of codes, the even (or a quarter of the) chunks
        // of a tile's row, in neighbouring rows, which the swizzle turns against one another.
        constexpr int kInTile = 64 / S::kCodes, kRowBits = 8 / kInTile;   // pieces of a row in a tile; rows of eight lanes
        const int t = threadIdx.x, o8 = t % S::kDyLanes, dy_row = t / S::kDyLanes;
        const int piece = t % kInTile + t / 8 % (S::kXLanes / kInTile) * kInTile, x_row = t / kInTile % kRowBits + t / (8 * (S::kXLanes / kInTile)) * kRowBits;
        const int o = o0 + o8 * 8, i = i0 + piece * S::kCodes, rows = (int)(end - begin);
        dy = reinterpret_cast<const char *>(a.dy) + ((begin + dy_row) * a.dy_stride + o) * S::kE;
        x = reinterpret_cast<const char *>(a.codes) + (begin + x_row) * a.c_in + i;
        exps = a.exps + (begin + x_row) * a.blocks + i / kBlock8;
        dy_pass = (size_t)S::kDyPass * a.dy_stride * S::kE;
        dy_step = (size_t)S::kRows * a.dy_stride * S::kE;
        x_step = (size_t)S::kRows * a.c_in;
        exps_step = (size_t)S::kRows * a.blocks;
        dy_left = o < a.c_out ? rows - dy_row : 0;
        x_left = i < a.c_in && x_row < S::kRows ? rows - x_row : 0;
        dy_cols = (a.c_out - o) * S::kE;
        x_cols = a.c_in - i;
        dy_tile = tile_at<S::kSub>(o8, dy_row);
        x_tile = x_row < S::kRows ? tile_at<S::kSub>(piece * (S::kCodes / 8), x_row) : ~0u;
        dy_bytes = (uint32_t)reinterpret_cast<uintptr_t>(dy);
        x_bytes = (uint32_t)reinterpret_cast<uintptr_t>(x);
    }

    // words that hold the bytes from p to p + valid; word j goes to at + j * kProducers * 4
    template <int kWords>
    __device__ __forceinline__ void copy_words(uint32_t at, const char *p, int valid, bool in) const
    {
        const uintptr_t first = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3;
        const int bytes = in ? valid + (int)(reinterpret_cast<uintptr_t>(p) & 3) : 0;
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            const bool has = 4 * j < bytes;
            copy_4(at + j * kProducers * 4, has ? reinterpret_cast<const void *>(first + 4 * j) : safe, has);
        }
    }
    // pieces of 16 bytes that hold the bytes from p to p + valid (a multiple of 16)
    template <int kWords>
    __device__ __forceinline__ void copy_wide(uint32_t at, const char *p, int valid, bool in) const
    {
#pragma unroll
        for (int j = 0; j < kWords / 4; ++j) {
            const bool has = in && (j == 0 || 16 * j < valid);
            copy_16(at + j * kProducers * 16, has ? p + 16 * j : safe, has);
        }
    }

    // starts the copies of the next stage, whose slot of the copies is `slot`; the byte of its codes is on its way
    __device__ __forceinline__ void start(int slot, uint32_t &s)
    {
        uint32_t at = raw + slot * S::kRawBytes;
        const char *p = dy;
#pragma unroll
        for (int k = 0; k < S::kDy; ++k, p += dy_pass) {
            const bool in = k * S::kDyPass < dy_left;
            if constexpr (kWide) copy_wide<S::kDyWords>(at, p, dy_cols, in);
            else copy_words<S::kDyWords>(at, p, dy_cols, in);
            at += S::kDyWords * kProducers * 4;
        }
        const bool in = x_left > 0;
        if constexpr (kWide) copy_wide<S::kXWords>(at, x, x_cols, in);
        else copy_words<S::kXWords>(at, x, x_cols, in);
        s = in ? __ldg(exps) : 1u;
        dy += dy_step;
        x += x_step;
        exps += exps_step;
        dy_left -= S::kRows;
        x_left -= S::kRows;
    }

    template <int kWords>
    __device__ __forceinline__ void copied(uint32_t at, uint32_t (&w)[kWords]) const
    {
        if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < kWords; j += 4) {
                const int4 v = ptx::ld_shared_128(at + j / 4 * kProducers * 16);
                w[j] = v.x;
                w[j + 1] = v.y;
                w[j + 2] = v.z;
                w[j + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kWords; ++j) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[j]) : "r"(at + j * kProducers * 4) : "memory");
        }
    }
    // aligned words to the ones that begin at an address of that remainder in the first
    template <int kWords>
    static __device__ __forceinline__ void shift(uint32_t (&w)[kWords], uint32_t bytes)
    {
#pragma unroll
        for (int j = 0; j + 1 < kWords; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], 8 * (bytes & 3u));
    }

    // converts the next stage, whose copies have arrived in `raw_slot`, into its operand tiles
    __device__ __forceinline__ void convert(int raw_slot, int slot, uint32_t s)
    {
        uint32_t at = raw + raw_slot * S::kRawBytes;
#pragma unroll
        for (int k = 0; k < S::kDy; ++k) {
            uint32_t w[S::kDyWords];
            copied(at, w);
            at += S::kDyWords * kProducers * 4;
            const uint32_t dst = smem + slot * S::kA + dy_tile + k * S::kDyPass * 128;
            if constexpr (S::kDyWords == 5) shift(w, dy_bytes + k * (uint32_t)dy_pass);
            if constexpr (kType == EOQ_BF16) {
                st_shared_128(dst, make_uint4(w[0], w[1], w[2], w[3]));
            } else {
                float v[8];
                if constexpr (S::kE == 2) {
                    Raw<16> r;
                    r.w = make_uint4(w[0], w[1], w[2], w[3]);
                    Elem<EOQ_F16>::to_f32(r, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
                }
#pragma unroll
                for (int p = 0; p < S::kParts; ++p) {
                    uint32_t h[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[j] = __byte_perm(__float_as_uint(v[2 * j]), __float_as_uint(v[2 * j + 1]), 0x7632);
                    st_shared_128(dst + p * S::kATile, make_uint4(h[0], h[1], h[2], h[3]));
                    // what the upper halves leave: exact; nothing of an infinity
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float hi = __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u);
                        v[j] = fabsf(v[j]) == INFINITY ? 0.0f : v[j] - hi;
                    }
                }
            }
        }
        dy_bytes += (uint32_t)dy_step;
        if (S::kXLanes * S::kRows == kProducers || x_tile != ~0u) {
            uint32_t w[S::kXWords];
            copied(at, w);
            if constexpr (!kWide) shift(w, x_bytes);
            const uint32_t sw = s << 7 | s << 23;
            const __nv_bfloat162 step = *reinterpret_cast<const __nv_bfloat162 *>(&sw);
            const uint32_t dst = smem + S::kOps * S::kA + slot % S::kOps * S::kB + x_tile;
#pragma unroll
            for (int j = 0; j < S::kCodes / 8; ++j) {
                const uint32_t c0 = w[2 * j], c1 = w[2 * j + 1];
                // (the pieces of a row begin at a multiple of their number: chunk j differs in bits of the swizzled place)
                st_shared_128(dst ^ (j << 4), make_uint4(two_codes(__byte_perm(c0, 0, 0x4140), step), two_codes(__byte_perm(c0, 0, 0x4342), step),
                                                         two_codes(__byte_perm(c1, 0, 0x4140), step), two_codes(__byte_perm(c1, 0, 0x4342), step)));
            }
        }
        x_bytes += (uint32_t)x_step;
    }
};

// fp32 accumulator, bf16 operands, both MN-major, m x n
__device__ __forceinline__ uint32_t wgrad_idesc(int m, int n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// The first eight warps, once everything is done: the tile to memory.  A row of the tile a lane; two warps share 32 rows, half of the
// columns each.
template <int kN>
__device__ __forceinline__ void store_tile(const CkptWgradArgs &a, int split, int o0, int i0, uint32_t tmem_base, uint32_t tmem_run, int chunks,
                                           uint32_t end_bar, const RoleCtx &ctx)
{
    const int warp = warp_index_uniform(), quad = warp & 3, o = o0 + quad * 32 + (threadIdx.x & 31);
    if (warp >= 8 || !__all_sync(0xffffffffu, wait_bar<64>(end_bar, 0, ctx))) return;
    ptx::tc_fence_after();
    float *dst = a.out + (size_t)split * a.pitch + (size_t)o * a.c_in;
    constexpr int kHalf = kN / 2;
#pragma unroll 1
    for (int c0 = (warp >> 2) * kHalf; c0 < (warp >> 2) * kHalf + kHalf; c0 += 32) {
        uint32_t r[32];
        ptx::tmem_ld_32x32(tmem_base + ((uint32_t)(quad * 32) << 16) + c0, r);
        ptx::tmem_ld_wait();
        if (chunks > 1) {
            uint32_t run[32];
            ptx::tmem_ld_32x32(tmem_run + ((uint32_t)(quad * 32) << 16) + c0, run);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(run[j]) + __uint_as_float(r[j]));
        }
        if (o < a.c_out) {
            if (a.c_in % 4 == 0) {
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                    if (i0 + c0 + j < a.c_in) *reinterpret_cast<uint4 *>(dst + i0 + c0 + j) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (i0 + c0 + j < a.c_in) dst[i0 + c0 + j] = __uint_as_float(r[j]);
            }
        }
    }
}

// The four warps that add the accumulator to the one of the chunks before.
template <int kN, bool kPair>
__device__ __forceinline__ void move_sums(uint32_t tmem_base, uint32_t tmem_run, int chunks, uint32_t sums_bar, uint32_t moved_bar, const RoleCtx &ctx)
{
    const uint32_t row = (uint32_t)((warp_index_uniform() & 3) * 32) << 16;
    for (int chunk = 0; chunk + 1 < chunks; ++chunk) {
        if (!__all_sync(0xffffffffu, wait_bar<64>(sums_bar, chunk & 1, ctx))) break;
        ptx::tc_fence_after();
#pragma unroll 1
        for (int c0 = 0; c0 < kN; c0 += 32) {
            uint32_t r[32];
            ptx::tmem_ld_32x32(tmem_base + row + c0, r);
            ptx::tmem_ld_wait();
            if (chunk) {
                uint32_t run[32];
                ptx::tmem_ld_32x32(tmem_run + row + c0, run);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(run[j]) + __uint_as_float(r[j]));
            }
            tmem_st_32x32(tmem_run + row + c0, r);
        }
        tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) arrive_first<kPair>(moved_bar);
    }
}

template <int kType, int kN, bool kWide>
__global__ void __launch_bounds__(kThreads, 1) ckpt_wgrad_kernel(const __grid_constant__ CkptWgradArgs a)
{
    using S = Shape<kType, kN, kWide>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kRing + 3];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t abort_s;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
    // of stage `it`: operands written; MMAs done.  Of the chunks of steps: sums complete; sums moved on.  All done.
    auto full_bar = [&](int it) { return bar0 + 8u * (it % S::kRing); };
    auto done_bar = [&](int it) { return bar0 + 8u * (S::kRing + it % S::kRing); };
    auto parity = [](int it) { return (uint32_t)(it / S::kRing) & 1u; };
    const uint32_t sums_bar = bar0 + 8u * (2 * S::kRing), moved_bar = sums_bar + 8, end_bar = sums_bar + 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kRing; ++s) {
            ptx::mbar_init(full_bar(s), kProducers / 32);
            ptx::mbar_init(done_bar(s), 1);
        }
        ptx::mbar_init(sums_bar, 1);
        ptx::mbar_init(moved_bar, 4);
        ptx::mbar_init(end_bar, 1);
        abort_s = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(ptx::smem_u32(&tmem_base_s), 2 * kN);
        ptx::tmem_relinquish();
    }
    const int tiles = a.m_tiles * a.n_tiles, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int o0 = tile / a.n_tiles * kTileM, i0 = tile % a.n_tiles * kN;
    const size_t row_begin = (size_t)split * a.rows_per_split, row_end = min(a.rows, row_begin + a.rows_per_split);
    const int stages = (int)((row_end - row_begin + S::kRows - 1) / S::kRows), chunks = (stages + S::kChunk - 1) / S::kChunk;
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    ptx::grid_dep_wait();
    if (a.joins) ptx::grid_dep_launch();   // (the joining kernel comes up beside this one)
    const uint32_t tmem_base = tmem_base_s, tmem_run = tmem_base + kN;
    const RoleCtx ctx{&abort_s, a.dev};

    if (warp < kMmaWarp) {
        Feeder<kType, kN, kWide> feed(a, row_begin, row_end, o0, i0, smem_base);
        uint32_t s[S::kRing] = {};
        auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
#pragma unroll
        for (int j = 0; j < S::kAhead; ++j) {
            if (j < stages) feed.start(j, s[j]);
            commit();
        }
        bool ok = true;
        for (int it0 = 0; it0 < stages && ok; it0 += S::kRing) {
#pragma unroll
            for (int j = 0; j < S::kRing; ++j) {
                const int it = it0 + j, ahead = (j + S::kAhead) % S::kRing;
                if (it >= stages || !ok) break;
                // stage it - kOps has left the tiles that stage `it` goes to
                if (it >= S::kOps) ok = __all_sync(0xffffffffu, wait_bar(done_bar(j + S::kRing - S::kOps), parity(it - S::kOps), ctx));
                if (!ok) break;
                if (it + S::kAhead < stages) feed.start(ahead, s[ahead]);
                commit();
                asm volatile("cp.async.wait_group %0;" ::"n"(S::kAhead) : "memory");
                feed.convert(j, j % S::kOps, s[j]);
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(full_bar(j));
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        store_tile<kN>(a, split, o0, i0, tmem_base, tmem_run, chunks, end_bar, ctx);
    } else if (warp == kMmaWarp) {
        const uint32_t leader = elect_one();
        const uint32_t idesc = wgrad_idesc(kTileM, kN);
        const uint64_t proto = make_smem_desc(0, S::kSub, 1024, 2);
        const uint32_t hi = (uint32_t)(proto >> 32), lead = (uint32_t)proto;
        bool ok = true;
        int chunk = 0, in_chunk = 0;
        for (int it = 0; it < stages; ++it) {
            if (in_chunk == S::kChunk) {   // hand the sums over and wait until they have been taken
                ptx::mma_commit(sums_bar, leader);
                if (!(ok = __all_sync(0xffffffffu, wait_bar(moved_bar, chunk & 1, ctx)))) break;
                ptx::tc_fence_after();
                ++chunk;
                in_chunk = 0;
            }
            if (!(ok = __all_sync(0xffffffffu, wait_bar(full_bar(it), parity(it), ctx)))) break;
            ptx::tc_fence_after();
            const uint32_t a16 = ((smem_base + (it % S::kOps) * S::kA) >> 4) | lead;
            const uint32_t b16 = ((smem_base + S::kOps * S::kA + (it % S::kOps) * S::kB) >> 4) | lead;
#pragma unroll
            for (int k = 0; k < S::kRows / 16; ++k)
#pragma unroll
                for (int p = 0; p < S::kParts; ++p)
                    mma_bf16<false>(tmem_base, smem_desc_join(a16 + p * (S::kATile >> 4) + k * 128, hi), smem_desc_join(b16 + k * 128, hi), idesc,
                             (k | p | in_chunk) != 0 ? 1u : 0u, leader);
            ptx::mma_commit(done_bar(it), leader);
            ++in_chunk;
        }
        ptx::mma_commit(end_bar, leader);
        if (!ok)
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (ptx::mbar_try_wait(end_bar, 0)) break;
    } else {
        move_sums<kN, false>(tmem_base, tmem_run, chunks, sums_bar, moved_bar, ctx);
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, 2 * kN);
    }
}

// ------------------------------------------------------------------ bf16 errors, 16-byte rows: tensor copies
// The same with both operands brought in by tensor copies (one thread's work), errors straight into their operand tiles and codes as
// they are, four to five stages ahead; the sixteen converting warps only convert.  With copies of their own between the conversions
// 1024 to 4096 channels, 16,384 rows took 250 us: 159 of it for the copies alone, which two stages in flight do not feed, 96 for the MMAs alone.
//
// kPair: two blocks, a cluster, work on a tile of 256 x 256 as one.  Each brings in its 128 columns of dy and of codes, converts its
// codes and holds its 128 rows of the accumulator; the MMAs are the first block's, over both blocks' operands.  What bounds the kernel is
// the conversion, and a pair converts half as much for the same MMAs.
template <int kN, bool kPair>
struct TmaShape {
    static constexpr int kOwn = kPair ? kN / 2 : kN;                      // columns of codes of a block
    static constexpr int kRows = 64, kSub = kRows * 128, kA = kTileM / 64 * kSub, kB = kOwn / 64 * kSub, kCodesBytes = kRows * kOwn;
    static constexpr int kOps = kOwn <= 128 ? 3 : 2;                      // stages of converted tiles
    static constexpr int kRing = (kMaxSmem - 1024 - kOps * kB) / (kA + kCodesBytes) < 8 ? (kMaxSmem - 1024 - kOps * kB) / (kA + kCodesBytes) : 8;
    static constexpr int kBytes = kRing * (kA + kCodesBytes) + kOps * kB + 1024;
    static constexpr int kChunk = kSteps / (kRows / 16);
    static constexpr int kPieces = kProducers / kRows, kCodes = kOwn / kPieces, kChunks8 = kCodes / 8;   // codes of a thread: a piece of a row
    static_assert(kPieces == 8 && kChunks8 >= 1 && kCodes <= kBlock8, "a row's pieces are those of eight lanes");
};
constexpr int kTmaThreads = kThreads + 32;   // one more warp, for the copies

template <int kN, bool kPair>
__global__ void __launch_bounds__(kTmaThreads, 1)
ckpt_wgrad_tma_kernel(const __grid_constant__ CkptWgradArgs a, const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x)
{
    using S = TmaShape<kN, kPair>;
    constexpr int kBlocks = kPair ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kRing + 2 * S::kOps + 3];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t abort_s;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
    const uint32_t b_base = smem_base + S::kRing * S::kA, code_base = b_base + S::kOps * S::kB;
    // by slot of the ring: copies landed; codes read and MMAs on the errors done.  By slot of converted tiles: written; MMAs done.
    auto in_bar = [&](int s) { return bar0 + 8u * s; };
    auto free_bar = [&](int s) { return bar0 + 8u * (S::kRing + s); };
    auto full_bar = [&](int s) { return bar0 + 8u * (2 * S::kRing + s); };
    auto done_bar = [&](int s) { return bar0 + 8u * (2 * S::kRing + S::kOps + s); };
    const uint32_t sums_bar = bar0 + 8u * (2 * S::kRing + 2 * S::kOps), moved_bar = sums_bar + 8, end_bar = sums_bar + 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kRing; ++s) {
            ptx::mbar_init(in_bar(s), 1);
            ptx::mbar_init(free_bar(s), kProducers / 32 + 1);
        }
        for (int s = 0; s < S::kOps; ++s) {
            ptx::mbar_init(full_bar(s), kBlocks * kProducers / 32);
            ptx::mbar_init(done_bar(s), 1);
        }
        ptx::mbar_init(sums_bar, 1);
        ptx::mbar_init(moved_bar, kBlocks * 4);
        ptx::mbar_init(end_bar, 1);
        abort_s = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&map_dy);
        ptx::prefetch_tensormap(&map_x);
    }
    if (warp == kMmaWarp) tmem_take<kPair>(ptx::smem_u32(&tmem_base_s), 2 * kN);
    const int rank = kPair ? blockIdx.x & 1 : 0, id = blockIdx.x / kBlocks;
    const int tiles = a.m_tiles * a.n_tiles, split = id / tiles, tile = id % tiles;
    const int o0 = (tile / a.n_tiles * kBlocks + rank) * kTileM, i0 = tile % a.n_tiles * kN, own_i0 = i0 + rank * S::kOwn;
    const size_t row_begin = (size_t)split * a.rows_per_split, row_end = min(a.rows, row_begin + a.rows_per_split);
    const int stages = (int)((row_end - row_begin + S::kRows - 1) / S::kRows), chunks = (stages + S::kChunk - 1) / S::kChunk;
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (the other block's barriers are ready)
    else __syncthreads();
    ptx::tc_fence_after();
    ptx::grid_dep_wait();
    if (a.joins) ptx::grid_dep_launch();   // (the joining kernel comes up beside this one)
    const uint32_t tmem_base = tmem_base_s, tmem_run = tmem_base + kN;
    const RoleCtx ctx{&abort_s, a.dev};

    if (warp < kMmaWarp) {
        const int piece = threadIdx.x % S::kPieces, row = threadIdx.x / S::kPieces, i = own_i0 + piece * S::kCodes;
        int left = i < a.c_in ? (int)(row_end - row_begin) - row : 0;
        const uint8_t *exps = a.exps + (row_begin + row) * a.blocks + i / kBlock8;
        const size_t step = (size_t)S::kRows * a.blocks;
        auto next_byte = [&] {
            const uint32_t s = left > 0 ? __ldg(exps) : 1u;
            exps += step;
            left -= S::kRows;
            return s;
        };
        uint32_t s0 = next_byte(), s1 = next_byte();
        // Each lane takes its chunks of eight codes in an order of its own, so that lanes that store (and load) together meet different banks.
        const int turn = piece * S::kChunks8 / 8 + (row & 1);
        uint32_t from[S::kChunks8], to[S::kChunks8];
#pragma unroll
        for (int j = 0; j < S::kChunks8; ++j) {
            const int c = (j + turn) % S::kChunks8;
            from[j] = (uint32_t)(row * S::kOwn + piece * S::kCodes + c * 8);
            to[j] = tile_at<S::kSub>(piece * S::kChunks8 + c, row);
        }
        int slot = 0, op = 0;
        uint32_t ring_phase = 0, op_phase = 0;
        for (int it = 0; it < stages; ++it) {
            const uint32_t s2 = next_byte();
            if (!__all_sync(0xffffffffu, wait_bar(in_bar(slot), ring_phase, ctx))) break;
            const uint32_t src = code_base + slot * S::kCodesBytes;
            uint4 v[S::kChunks8];
            const uint32_t sw = s0 << 7 | s0 << 23;
            const __nv_bfloat162 unit = *reinterpret_cast<const __nv_bfloat162 *>(&sw);
#pragma unroll
            for (int j = 0; j < S::kChunks8; ++j) {
                uint32_t c0, c1;
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c0), "=r"(c1) : "r"(src + from[j]) : "memory");
                v[j] = make_uint4(two_codes(__byte_perm(c0, 0, 0x4140), unit), two_codes(__byte_perm(c0, 0, 0x4342), unit),
                                  two_codes(__byte_perm(c1, 0, 0x4140), unit), two_codes(__byte_perm(c1, 0, 0x4342), unit));
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(free_bar(slot));
            if (!__all_sync(0xffffffffu, wait_bar(done_bar(op), op_phase ^ 1u, ctx))) break;
            const uint32_t dst = b_base + op * S::kB;
#pragma unroll
            for (int j = 0; j < S::kChunks8; ++j) st_shared_128(dst + to[j], v[j]);
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) arrive_first<kPair>(full_bar(op));
            s0 = s1;
            s1 = s2;
            if (++slot == S::kRing) { slot = 0; ring_phase ^= 1u; }
            if (++op == S::kOps) { op = 0; op_phase ^= 1u; }
        }
        store_tile<kN>(a, split, o0, i0, tmem_base, tmem_run, chunks, end_bar, ctx);
    } else if (warp == kMmaWarp && rank == 0) {
        const uint32_t leader = elect_one();
        const uint32_t idesc = wgrad_idesc(kBlocks * kTileM, kN);
        const uint64_t proto = make_smem_desc(0, S::kSub, 1024, 2);
        const uint32_t hi = (uint32_t)(proto >> 32), lead = (uint32_t)proto;
        bool ok = true;
        int chunk = 0, in_chunk = 0, slot = 0, op = 0;
        uint32_t ring_phase = 0, op_phase = 0;
        for (int it = 0; it < stages; ++it) {
            if (in_chunk == S::kChunk) {   // hand the sums over and wait until they have been taken
                commit_both<kPair>(sums_bar, leader);
                if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(moved_bar, chunk & 1, ctx)))) break;
                ptx::tc_fence_after();
                ++chunk;
                in_chunk = 0;
            }
            if (!(ok = __all_sync(0xffffffffu, wait_bar(in_bar(slot), ring_phase, ctx)))) break;
            if (!(ok = __all_sync(0xffffffffu, wait_both<kPair>(full_bar(op), op_phase, ctx)))) break;
            ptx::tc_fence_after();
            const uint32_t a16 = ((smem_base + slot * S::kA) >> 4) | lead, b16 = ((b_base + op * S::kB) >> 4) | lead;
#pragma unroll
            for (int k = 0; k < S::kRows / 16; ++k)
                mma_bf16<kPair>(tmem_base, smem_desc_join(a16 + k * 128, hi), smem_desc_join(b16 + k * 128, hi), idesc, (k | in_chunk) != 0 ? 1u : 0u, leader);
            commit_both<kPair>(done_bar(op), leader);
            commit_both<kPair>(free_bar(slot), leader);
            ++in_chunk;
            if (++slot == S::kRing) { slot = 0; ring_phase ^= 1u; }
            if (++op == S::kOps) { op = 0; op_phase ^= 1u; }
        }
        commit_both<kPair>(end_bar, leader);
        if (!ok)
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (ptx::mbar_try_wait(end_bar, 0)) break;
    } else if (warp == kMmaWarp) {
        // (the other block of a pair: its MMAs are issued by the first)
    } else if (warp < kMmaWarp + 5) {
        move_sums<kN, kPair>(tmem_base, tmem_run, chunks, sums_bar, moved_bar, ctx);
    } else {
        bool ok = true;
        int slot = 0, started = 0;
        uint32_t ring_phase = 0;
        for (int it = 0; it < stages; ++it) {
            if (!(ok = __all_sync(0xffffffffu, wait_bar<32>(free_bar(slot), ring_phase ^ 1u, ctx)))) break;
            if (lane == 0) {
                const int r = (int)row_begin + it * S::kRows;
                ptx::mbar_expect_tx(in_bar(slot), S::kA + S::kCodesBytes);
#pragma unroll
                for (int j = 0; j < kTileM / 64; ++j) ptx::tma_load_2d(smem_base + slot * S::kA + j * S::kSub, &map_dy, in_bar(slot), o0 + 64 * j, r);
                ptx::tma_load_2d(code_base + slot * S::kCodesBytes, &map_x, in_bar(slot), own_i0, r);
            }
            __syncwarp();
            ++started;
            if (++slot == S::kRing) { slot = 0; ring_phase ^= 1u; }
        }
        if (!ok && lane == 0)   // (copies still in flight land before the block ends)
            for (int it = started > S::kRing ? started - S::kRing : 0; it < started; ++it)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (ptx::mbar_try_wait(in_bar(it % S::kRing), (uint32_t)(it / S::kRing) & 1u)) break;
    }
    ptx::tc_fence_before();
    if (kPair) ptx::cluster_sync();   // (neither block ends while the other's MMAs or arrivals may reach it)
    else __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after();
        tmem_return<kPair>(tmem_base, 2 * kN);
    }
}


// dw = the splits' sums, which stand `pitch` floats apart: four neighbouring ones a thread, kShares warps of a block to the same ones, each
// with every kShares-th split in order, then the shares in order.  (One share leaves too few loads in flight where the matrix is small.)
template <int kShares>
__global__ void __launch_bounds__(256) ckpt_wgrad_join_kernel(const float *__restrict__ part, size_t n, size_t pitch, int splits, float *__restrict__ dw)
{
    __shared__ float4 share[kShares][256 / kShares];
    ptx::grid_dep_wait_launch_small();
    constexpr int kPieces = 256 / kShares;
    const int piece = threadIdx.x % kPieces, own = threadIdx.x / kPieces;
    for (size_t i0 = (size_t)blockIdx.x * kPieces * 4; i0 < n; i0 += (size_t)gridDim.x * kPieces * 4) {
        const size_t i = i0 + piece * 4;
        float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto add = [&](const float4 &v) {
            t.x += v.x;
            t.y += v.y;
            t.z += v.z;
            t.w += v.w;
        };
        if (i < n)
#pragma unroll 4
            for (int s = own; s < splits; s += kShares) add(__ldg(reinterpret_cast<const float4 *>(part + (size_t)s * pitch + i)));
        if (kShares > 1) {
            share[own][piece] = t;
            __syncthreads();
            t = share[0][piece];
            if (own == 0)
                for (int w = 1; w < kShares; ++w) add(share[w][piece]);
            __syncthreads();
        }
        if (own == 0 && i < n) {
            if (i + 4 <= n) {
                *reinterpret_cast<float4 *>(dw + i) = t;
            } else {
                const float v[3] = {t.x, t.y, t.z};
                for (int j = 0; j < (int)(n - i); ++j) dw[i + j] = v[j];
            }
        }
    }
}

constexpr int kPlanRows = 64;   // (whole stages of every kernel)

struct WgradPlan8 {
    bool pair;
    int n_tile, m_tiles, n_tiles, splits;
    size_t rows_per_split;
};

// Microseconds of a block for 64 rows, by the width of its tile (64, 128, 256), as measured with every SM at work: what the conversions
// take, not the MMAs (0.27 at 256).
double rows_time(int dtype, bool wide, int width)
{
    static const double kTimes[2][3][3] = {{{2.3, 2.45, 2.8}, {1.2, 1.45, 1.85}, {1.07, 1.13, 1.69}},    // fp32, fp16, bf16
                                           {{1.85, 1.85, 2.1}, {0.8, 0.86, 1.33}, {0.35, 0.43, 0.5}}};
    return kTimes[wide ? 1 : 0][dtype == EOQ_F32 ? 0 : dtype == EOQ_F16 ? 1 : 2][width];
}

// The tile and the number of splits that take the least time by that: waves of blocks, each with some 6 us in front of and behind its
// rows, and the joining kernel's launch and reading (512 to 2048 channels, 1,568 rows of bf16: 14 us without splits in tiles of 64,
// 17 us in four splits of tiles of two blocks).  wide: rows of both operands 16-byte aligned; bf16 then has a tile of 256 x 256 for two
// blocks, and none of 128 x 256.
WgradPlan8 plan_of(size_t rows, int c_out, int c_in, int dtype, bool wide)
{
    const bool tma = wide && dtype == EOQ_BF16;
    const size_t stages = (rows + kPlanRows - 1) / kPlanRows;
    WgradPlan8 best = {};
    double best_time = 0.0;
    for (int width = 0; width < 3; ++width) {
        WgradPlan8 p;
        p.n_tile = 64 << width;
        p.pair = tma && width == 2;
        if (p.pair && (c_out <= kTileM || c_in <= 128)) continue;
        if (width > 0 && c_in <= p.n_tile / 2) continue;
        const int m_tile = p.pair ? 2 * kTileM : kTileM;
        p.m_tiles = (c_out + m_tile - 1) / m_tile;
        p.n_tiles = (c_in + p.n_tile - 1) / p.n_tile;
        const size_t tiles = (size_t)p.m_tiles * p.n_tiles, room = kPartSms / (p.pair ? 2 : 1);
        for (size_t fill = 0; fill <= 2; ++fill) {
            size_t splits = fill == 0 ? 1 : fill * room / tiles;
            if (splits < 1 || (fill > 0 && splits == 1)) continue;
            if (splits > stages) splits = stages;
            const size_t per = (stages + splits - 1) / splits;
            splits = (stages + per - 1) / per;
            p.splits = (int)splits;
            p.rows_per_split = per * kPlanRows;
            const double waves = (double)((tiles * splits + room - 1) / room);
            const double time = waves * (6.0 + (double)per * rows_time(dtype, wide, width)) +
                                (splits > 1 ? 3.0 + (double)splits * c_out * c_in * 4.0 / 4e6 : 0.0);
            if (best_time == 0.0 || time < best_time) {
                best = p;
                best_time = time;
            }
        }
    }
    return best;
}

bool wide_rows(const void *dy, int dtype, int c_out, size_t dy_stride, const void *codes, int c_in)
{
    return c_out % 8 == 0 && c_in % 16 == 0 && dy_stride % (dtype == EOQ_F32 ? 4 : 8) == 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 &&
           reinterpret_cast<uintptr_t>(codes) % 16 == 0;
}

template <int kType, int kN, bool kWide>
cudaError_t launch(const CkptWgradArgs &a, int grid, cudaStream_t st)
{
    constexpr int bytes = Shape<kType, kN, kWide>::kBytes;
    static_assert(bytes <= kMaxSmem, "shared memory of a block");
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)ckpt_wgrad_kernel<kType, kN, kWide>, bytes, allowed);
    if (e != cudaSuccess) return e;
    return launch_chained(ckpt_wgrad_kernel<kType, kN, kWide>, dim3(grid), dim3(kThreads), bytes, st, a);
}

template <int kN, bool kPair>
cudaError_t launch_tma(const CkptWgradArgs &a, int grid, cudaStream_t st)
{
    using S = TmaShape<kN, kPair>;
    CUtensorMap map_dy, map_x;
    if (!tiled_map_2d(&map_dy, a.dy, true, a.c_out, a.rows, a.dy_stride * 2, 64, S::kRows, true) ||
        !tiled_map_2d(&map_x, a.codes, false, a.c_in, a.rows, a.c_in, S::kOwn, S::kRows, false))
        return cudaErrorInvalidValue;
    static_assert(S::kBytes <= kMaxSmem, "shared memory of a block");
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)ckpt_wgrad_tma_kernel<kN, kPair>, S::kBytes, allowed);
    if (e != cudaSuccess) return e;
    return launch_chained_clusters(kPair ? 2 : 1, ckpt_wgrad_tma_kernel<kN, kPair>, dim3(grid), dim3(kTmaThreads), S::kBytes, st, a, map_dy, map_x);
}

template <int kType, bool kWide>
cudaError_t of_width(const CkptWgradArgs &a, int n_tile, int grid, cudaStream_t st)
{
    if (n_tile == 64) return launch<kType, 64, kWide>(a, grid, st);
    if (n_tile == 128) return launch<kType, 128, kWide>(a, grid, st);
    return launch<kType, 256, kWide>(a, grid, st);
}

template <int kType>
cudaError_t of_type(const CkptWgradArgs &a, int n_tile, bool wide, bool pair, int grid, cudaStream_t st)
{
    if (!wide) return of_width<kType, false>(a, n_tile, grid, st);
    if constexpr (kType == EOQ_BF16) {
        if (pair) return launch_tma<256, true>(a, 2 * grid, st);
        return n_tile == 64 ? launch_tma<64, false>(a, grid, st) : launch_tma<128, false>(a, grid, st);
    } else {
        return of_width<kType, true>(a, n_tile, grid, st);
    }
}

}  // namespace

// floats of a split's sums: whole pieces of 16 bytes
static size_t split_pitch(int c_out, int c_in) { return ((size_t)c_out * c_in + 3) & ~(size_t)3; }

// for either alignment of the call's tensors
size_t ckpt_wgrad_workspace_bytes(size_t rows, int c_out, int c_in, int dtype)
{
    const WgradPlan8 w = plan_of(rows, c_out, c_in, dtype, true), n = plan_of(rows, c_out, c_in, dtype, false);
    const int splits = w.splits > n.splits ? w.splits : n.splits;
    return splits > 1 ? sizeof(float) * (size_t)splits * split_pitch(c_out, c_in) : 0;
}

cudaError_t launch_ckpt_wgrad(CkptWgradArgs a, int dtype, float *dw, void *workspace, int *launches, cudaStream_t st)
{
    const bool wide = wide_rows(a.dy, dtype, a.c_out, a.dy_stride, a.codes, a.c_in);
    const WgradPlan8 p = plan_of(a.rows, a.c_out, a.c_in, dtype, wide);
    a.blocks = (a.c_in + kBlock8 - 1) / kBlock8;
    a.m_tiles = p.m_tiles;
    a.n_tiles = p.n_tiles;
    a.rows_per_split = p.rows_per_split;
    a.safe = reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(a.exps) & ~(uintptr_t)15);   // (never read: copies of nothing)
    a.joins = p.splits > 1;
    a.pitch = split_pitch(a.c_out, a.c_in);
    a.out = p.splits > 1 ? reinterpret_cast<float *>(workspace) : dw;
    const int grid = p.m_tiles * p.n_tiles * p.splits;
    const cudaError_t e = dtype == EOQ_F32   ? of_type<EOQ_F32>(a, p.n_tile, wide, p.pair, grid, st)
                          : dtype == EOQ_F16 ? of_type<EOQ_F16>(a, p.n_tile, wide, p.pair, grid, st)
                                             : of_type<EOQ_BF16>(a, p.n_tile, wide, p.pair, grid, st);
    ++*launches;
    if (e != cudaSuccess || p.splits == 1) return e;
    ++*launches;
    const size_t n = (size_t)a.c_out * a.c_in, pieces = (n + 3) / 4, cap = 8 * kPartSms;
    const bool small = pieces < (size_t)kPartSms * 256;
    const size_t blocks = small ? (pieces + 31) / 32 : (pieces + 255) / 256;
    const dim3 join((unsigned)(blocks < cap ? blocks : cap));
    if (small) return launch_chained(ckpt_wgrad_join_kernel<8>, join, dim3(256), 0, st, (const float *)a.out, n, a.pitch, p.splits, dw);
    return launch_chained(ckpt_wgrad_join_kernel<1>, join, dim3(256), 0, st, (const float *)a.out, n, a.pitch, p.splits, dw);
}

}  // namespace eoq
