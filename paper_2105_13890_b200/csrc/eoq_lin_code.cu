// Codes of floating-point rows and columns with a scale each (eoq_lin_quantize, and the first steps of eoq_lin_fwd and eoq_lin_bwd):
//   scale = max(largest magnitude, 2^-119) / 127,  code = R(value * fl(127 / max(..))).
//
// Bound: memory.  A row belongs to up to 256 neighbouring threads, which keep it in registers as it came between the look for its maximum and its coding; only
// rows longer than they hold are read a second time.  The errors of a layer are coded by rows and by columns, and columns need all rows before the first code, so
// there are two looks at the tensor: the first leaves the maxima of parts of rows and columns (and the parts' sums of columns), the second writes both codes.
// Neither look has a thread wait for another row's: coding the rows in the first one, with a barrier of 256 threads for each row, took 155 us for
// 16,384 x 4096 of bf16 where the floor of reading is 21.
#include <type_traits>

#include "eoq_lin.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256;
// blocks of the rows' kernel on an SM, by the vectors that a thread holds
template <int kHeld> constexpr int kRowBlocks = kHeld <= 1 ? 6 : kHeld <= 4 ? 4 : 2;
// Strips, and elements of a tensor, whose maxima the second look puts together by itself; others take a kernel between the two.
constexpr int kFoldStrips = 32;
constexpr size_t kFoldSize = 1 << 20;

// the largest of `lanes` neighbouring threads' values, a power of two; of more than a warp by way of `cells`, one for each of the block's warps
__device__ __forceinline__ uint32_t lanes_top(uint32_t top, int lanes, uint32_t *cells)
{
    if (lanes >= 32) {
        top = __reduce_max_sync(0xffffffffu, top);
        if (lanes > 32) {
            if (threadIdx.x % 32 == 0) cells[threadIdx.x / 32] = top;
            __syncthreads();
            const int warps = lanes / 32, first = threadIdx.x / lanes * warps;
            top = cells[first];
            for (int w = 1; w < warps; ++w) top = max(top, cells[first + w]);
        }
        return top;
    }
    for (int d = lanes / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    return top;
}

// Rows: kHold groups of a row at a time, the next row's on their way meanwhile.
template <int kType, int kU, int kHold>
__global__ void __launch_bounds__(kThreads, kRowBlocks<kHold>) lin_rows_kernel(const __grid_constant__ LinCodeArgs a, const int lanes)
{
    using S = Span<kType, kU>;
    constexpr int kN = S::kN;
    __shared__ uint32_t cells[2][kThreads / 32];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slots = kThreads / lanes, groups = (a.cols + lanes * kN - 1) / (lanes * kN);
    const size_t at_once = slots, stride = a.stride * S::kE;
    auto scaled = [&](const Raw<16> &r, const S &at, float (&v)[kN]) {
        Elem<kType>::to_f32(r, v);
        if (a.factors) {
            float f[kN];
            at.get_exact(a.factors, f);
#pragma unroll
            for (int i = 0; i < kN; ++i) v[i] *= f[i];
        }
    };
    auto more = [&](uint32_t top, const Raw<16> &r, const S &at) {
        if (!a.factors) return raw_top<kType>(r, top);
        float v[kN];
        scaled(r, at, v);
#pragma unroll
        for (int i = 0; i < kN; ++i) top = max(top, abs_bits(v[i]));
        return top;
    };
    Raw<16> next[kHold];
    auto fetch = [&](size_t row) {
#pragma unroll
        for (int h = 0; h < kHold; ++h) next[h] = S(h, lane, lanes, a.cols).get(reinterpret_cast<const char *>(a.src) + row * stride, row < a.rows);
    };
    const size_t step = gridDim.x * at_once;
    size_t row = blockIdx.x * at_once + threadIdx.x / lanes;
    int turn = 0;
    fetch(row);
    for (size_t first = blockIdx.x * at_once; first < a.rows; first += step, row += step, turn ^= 1) {   // (the same rounds for every thread)
        Raw<16> held[kHold];
#pragma unroll
        for (int h = 0; h < kHold; ++h) held[h] = next[h];
        if (first + step < a.rows) fetch(row + step);
        const bool mine = row < a.rows;
        const char *src = reinterpret_cast<const char *>(a.src) + row * stride;
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < kHold; ++h) top = more(top, held[h], S(h, lane, lanes, a.cols));
        if (mine)
            for (int g = kHold; g < groups; ++g) {
                const S at(g, lane, lanes, a.cols);
                top = more(top, at.get(src, true), at);
            }
        const float t = __uint_as_float(lanes_top(top, lanes, cells[turn]));
        if (!mine) continue;
        const bool fine = finite_top(t);
        const float per = fine ? row_per_of(t) : 0.0f;
        if (lane == 0) {
            a.scales[row] = row_scale_of(t);
            if (!fine) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
        }
        auto put = [&](const Raw<16> &r, const S &at) {
            float v[kN];
            uint32_t q[kN];
            scaled(r, at, v);
#pragma unroll
            for (int i = 0; i < kN; ++i) q[i] = row_code(v[i], per);
            if (!fine) {
#pragma unroll
                for (int i = 0; i < kN; ++i) q[i] = 0;
            }
            at.put_codes(a.codes + row * a.pitch, q);
        };
#pragma unroll
        for (int h = 0; h < kHold; ++h) put(held[h], S(h, lane, lanes, a.cols));
        for (int g = kHold; g < groups; ++g) {
            const S at(g, lane, lanes, a.cols);
            put(at.get(src, true), at);
        }
    }
}

// ------------------------------------------------------------------ the errors of a layer

constexpr int kAhead = 4;   // rows of a thread in flight

// the largest magnitude of three, NaN if one is; two products or sums of neighbouring values in one instruction, each rounded as it is alone
__device__ __forceinline__ float max3_abs(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float2 mul_2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 c, a, b;\n\t"
        "mov.b64 {%0, %1}, c;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 add_2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 c, a, b;\n\t"
        "mov.b64 {%0, %1}, c;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// The values of the block's threads that have the same lane, put together in those of slot 0, by way of kCells arrays of a value a thread.
template <int kN, int kCells, bool kMax>
__device__ __forceinline__ void meet_threads(float *cells, float (&mine)[kN], int lane, int slot, int slots, int lanes)
{
    constexpr int kAtOnce = kCells < kN ? kCells : kN;
#pragma unroll
    for (int i0 = 0; i0 < kN; i0 += kAtOnce) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) cells[i * kThreads + threadIdx.x] = mine[i0 + i];
        __syncthreads();
        if (slot == 0)
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                for (int s = 1; s < slots; ++s) {
                    const float v = cells[i * kThreads + s * lanes + lane];
                    mine[i0 + i] = kMax ? max_abs(mine[i0 + i], v) : mine[i0 + i] + v;
                }
    }
}

// Block (x, y): strip x of the rows, kVec groups of the columns from y * kVec on, `lanes` (at most 32) threads a row.  kRows: the rows' maxima too.
// Vectors come in by asynchronous copies, each read back by the thread that copied it, some rows ahead.  What bounds it is issue: two vectors of a row a thread share the
// row's own work (its factor, its maximum, what is ahead).  16,384 x 4096 of bf16: 36 us; 43 with one.  (That form's 16-bit variants spill 48 bytes at the 80 registers that three
// blocks an SM leave.)
template <int kType, int kU, int kVec, bool kRows>
__global__ void __launch_bounds__(kThreads, 3) lin_look_kernel(const __grid_constant__ LinErrorArgs a, const int lanes)
{
    using S = Span<kType, kU>;
    constexpr int kN = S::kN, kRing = kU == 16 ? (kVec == 2 ? 3 : 4) : 1, kPair = 2;   // stages of two rows
    __shared__ __align__(16) uint4 ring[kRing * kPair * kVec][kThreads];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes, slots = kThreads / lanes;
    const size_t begin = (size_t)blockIdx.x * a.strip, end = min(a.rows, begin + a.strip);
    const size_t step = slots * a.stride * S::kE;
    const char *src = reinterpret_cast<const char *>(a.src) + (begin + slot) * a.stride * S::kE;
    const int stages = (int)((end - begin + kPair * slots - 1) / (kPair * slots));   // (the same for every lane)
    int left = (int)(end - begin) - slot;                                           // rows from `src` on
    S at[kVec];
    int bytes[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
        at[j] = S(blockIdx.y * kVec + j, lane, lanes, a.cols);
        bytes[j] = min(16, max(0, (a.cols - at[j].first) * S::kE));   // (of a vector; zeros behind them)
    }
    Raw<16> now[kPair][kVec];
    // the next stage's copies or, without a ring, loads
    auto fetch = [&](int slot_) {
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            const bool mine = u * slots < left;
            const char *row = mine ? src + u * step : reinterpret_cast<const char *>(a.src);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                if constexpr (kU == 16) {
                    const int n = mine ? bytes[j] : 0;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(&ring[(slot_ * kPair + u) * kVec + j][threadIdx.x])),
                                 "l"(row + (n ? (size_t)at[j].first * S::kE : 0)), "r"(n)
                                 : "memory");
                } else {
                    now[u][j] = at[j].get(row, mine);
                }
            }
        }
        src += kPair * step;
        left -= kPair * slots;
        if constexpr (kU == 16) asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const float *factor = a.row_factors + begin + slot;
    int f_left = left;
    auto fetch_factors = [&](float (&to)[kPair]) {
#pragma unroll
        for (int u = 0; u < kPair; ++u) to[u] = a.row_factors && u * slots < f_left ? __ldg(factor + u * slots) : 0.0f;
        factor += kPair * slots;
        f_left -= kPair * slots;
    };
    float f[kPair] = {}, next_f[kPair] = {}, w[kVec][kN], top[kVec][kN] = {};
    float2 sum[kVec][kN / 2] = {};
    if constexpr (kU == 16)
        for (int j = 0; j < kRing - 1; ++j) fetch(j);   // (nothing but empty groups past the last one)
    fetch_factors(next_f);
    if (kRows)
#pragma unroll
        for (int j = 0; j < kVec; ++j) at[j].get_exact(a.factors, w[j]);
    float *row_top = kRows ? a.row_tops + blockIdx.y * a.rows + begin + slot : nullptr;
    int row_left = left + (kU == 16 ? (kRing - 1) * kPair * slots : 0), here = 0, ahead = kRing - 1;
    for (int it = 0; it < stages; ++it) {
#pragma unroll
        for (int u = 0; u < kPair; ++u) f[u] = next_f[u];
        fetch_factors(next_f);
        if constexpr (kU == 16) {
            fetch(ahead);
            asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
#pragma unroll
            for (int u = 0; u < kPair; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) now[u][j].w = ring[(here * kPair + u) * kVec + j][threadIdx.x];
            here = here + 1 == kRing ? 0 : here + 1;
            ahead = ahead + 1 == kRing ? 0 : ahead + 1;
        } else {
            fetch(0);
        }
        float m[kPair] = {};
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            float v[kPair][kN];
            Elem<kType>::to_f32(now[0][j], v[0]);
            Elem<kType>::to_f32(now[1][j], v[1]);
#pragma unroll
            for (int i = 0; i < kN; i += 2) {
                const float2 a0 = make_float2(v[0][i], v[0][i + 1]), a1 = make_float2(v[1][i], v[1][i + 1]);
                const float2 p0 = mul_2(a0, make_float2(f[0], f[0])), p1 = mul_2(a1, make_float2(f[1], f[1]));
                top[j][i] = max3_abs(top[j][i], p0.x, p1.x);
                top[j][i + 1] = max3_abs(top[j][i + 1], p0.y, p1.y);
                sum[j][i / 2] = add_2(add_2(sum[j][i / 2], a0), a1);
                if (kRows) {
                    const float2 ww = make_float2(w[j][i], w[j][i + 1]), r0 = mul_2(a0, ww), r1 = mul_2(a1, ww);
                    m[0] = max3_abs(m[0], r0.x, r0.y);
                    m[1] = max3_abs(m[1], r1.x, r1.y);
                }
            }
        }
        if (kRows) {
#pragma unroll
            for (int u = 0; u < kPair; ++u) {
                const uint32_t t = lanes_top(__float_as_uint(m[u]), lanes, nullptr);
                if (lane == 0 && u * slots < row_left) row_top[u * slots] = __uint_as_float(t);
            }
            row_top += kPair * slots;
            row_left -= kPair * slots;
        }
    }
    if constexpr (kU == 16) asm volatile("cp.async.wait_all;" ::: "memory");
    float *cells = reinterpret_cast<float *>(&ring[0][0]);
    constexpr int kCells = kRing * kPair * kVec * 4;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
        if (a.strip_tops) {
            meet_threads<kN, kCells, true>(cells, top[j], lane, slot, slots, lanes);
            if (slot == 0) at[j].put_padded(a.strip_tops + blockIdx.x * a.col_pitch, top[j]);
        }
        if (a.strip_sums) {
            float sums[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) sums[i] = i & 1 ? sum[j][i / 2].y : sum[j][i / 2].x;
            meet_threads<kN, kCells, false>(cells, sums, lane, slot, slots, lanes);
            if (slot == 0) at[j].put_padded(a.strip_sums + blockIdx.x * a.col_pitch, sums);
        }
    }
}

// Scale and factor of a row or column from its maximum.  One without codes (it holds a NaN or an infinity) has the factor 0: its codes do not matter, its scale
// is NaN.
__device__ __forceinline__ float finish_top(float top, float *scale, DeviceState *dev)
{
    *scale = row_scale_of(top);
    if (finite_top(top)) return row_per_of(top);
    atomicOr(&dev->status, EOQ_DEV_NONFINITE);
    return 0.0f;
}

// What the parts left, put together: by the first blocks 32 columns each, a share of the strips a warp, by the others a row a thread.  Sums of up to kFoldStrips strips are
// added one by one, as the second look adds them: the same bits whatever else a call is asked for.
constexpr int kJoinThreads = 512;
__global__ void __launch_bounds__(kJoinThreads) lin_join_looks_kernel(const __grid_constant__ LinErrorArgs a)
{
    constexpr int kWarps = kJoinThreads / 32;
    static_assert(kFoldStrips == 2 * kWarps, "two strips a warp");
    __shared__ float tops_s[kWarps][32], sums_s[kFoldStrips][32];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, across = (a.cols + 31) / 32;
    if ((int)blockIdx.x >= across) {
        const size_t row = (size_t)(blockIdx.x - across) * kJoinThreads + threadIdx.x;
        if (row >= a.rows) return;
        float top = 0.0f;
#pragma unroll 8
        for (int c = 0; c < a.chunks; ++c) top = fmaxf(top, __ldg(a.row_tops + c * a.rows + row));   // (NaN is kept below)
        bool bad = false;
        for (int c = 0; c < a.chunks; ++c) bad = bad || !finite_top(__ldg(a.row_tops + c * a.rows + row));
        a.row_per[row] = finish_top(bad ? __uint_as_float(0x7fc00000u) : top, a.scales + row, a.dev);
        return;
    }
    const int col = blockIdx.x * 32 + lane;
    const bool apart = a.strips <= kFoldStrips;
    float top = 0.0f, sum = 0.0f, second = 0.0f;
    if (col < a.cols) {
#pragma unroll 4
        for (int s = warp; s < a.strips; s += kWarps) {
            if (a.strip_tops) top = max_abs(top, __ldg(a.strip_tops + (size_t)s * a.col_pitch + col));
            if (a.strip_sums) {
                const float v = __ldg(a.strip_sums + (size_t)s * a.col_pitch + col);
                if (apart && s >= kWarps) second += v;
                else sum += v;
            }
        }
    }
    tops_s[warp][lane] = top;
    sums_s[warp][lane] = sum;
    sums_s[warp + kWarps][lane] = second;
    __syncthreads();
    if (warp == 0 && col < a.cols) {
        float whole = 0.0f;
        for (int w = 1; w < kWarps; ++w) top = max_abs(top, tops_s[w][lane]);
#pragma unroll
        for (int s = 0; s < kFoldStrips; ++s) whole += sums_s[s][lane];
        if (a.strip_tops) a.col_per[col] = finish_top(top, a.col_scales + col, a.dev);
        if (a.strip_sums) a.sums[col] = whole;
    }
}

// The second look.  Block (x, y): `range` rows from x * range on, group y of the columns.  kFold: what the parts left is put together here, column by
// column and row by row, by every thread that needs it.
template <int kType, int kU, bool kRows, bool kFold>
__global__ void __launch_bounds__(kThreads, 3) lin_codes_kernel(const __grid_constant__ LinErrorArgs a, const int lanes, const size_t range)
{
    using S = Span<kType, kU>;
    constexpr int kN = S::kN;
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes, slots = kThreads / lanes;
    const S at(blockIdx.y, lane, lanes, a.cols);
    const size_t begin = (size_t)blockIdx.x * range, end = min(a.rows, begin + range);
    if (!at.any()) return;
    const char *src = reinterpret_cast<const char *>(a.src) + (begin + slot) * a.stride * S::kE;
    const size_t step = slots * a.stride * S::kE;
    float w[kN], per[kN];
    if (kRows) at.get_exact(a.factors, w);
    if (kFold) {
        float top[kN] = {};
#pragma unroll 4
        for (int s = 0; s < a.strips; ++s) {
            float t[kN];
            at.get_padded(a.strip_tops + s * a.col_pitch, t);
#pragma unroll
            for (int i = 0; i < kN; ++i) top[i] = max_abs(top[i], t[i]);
        }
        const bool writes = blockIdx.x == 0 && slot == 0;
        if (writes && a.strip_sums) {
            float sum[kN] = {};
#pragma unroll 4
            for (int s = 0; s < a.strips; ++s) {
                float t[kN];
                at.get_padded(a.strip_sums + s * a.col_pitch, t);
#pragma unroll
                for (int i = 0; i < kN; ++i) sum[i] += t[i];
            }
            at.put_exact(a.sums, sum);
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (writes && at.column(i) < a.cols) finish_top(top[i], a.col_scales + at.column(i), a.dev);
            per[i] = finite_top(top[i]) ? row_per_of(top[i]) : 0.0f;
        }
    } else {
        at.get_padded(a.col_per, per);
    }
    for (size_t row0 = begin + slot; row0 < end; row0 += kAhead * slots, src += kAhead * step) {
        Raw<16> raw[kAhead];
        float f[kAhead], row_per[kAhead] = {};
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const size_t row = row0 + u * slots;
            const bool mine = row < end;
            raw[u] = at.get(src + u * step, mine);
            f[u] = mine ? __ldg(a.row_factors + row) : 0.0f;
            if (kRows && !kFold) row_per[u] = mine ? __ldg(a.row_per + row) : 0.0f;
            if (kRows && kFold && mine)
                for (int c = 0; c < a.chunks; ++c) row_per[u] = max_abs(row_per[u], __ldg(a.row_tops + c * a.rows + row));
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const size_t row = row0 + u * slots;
            if (row >= end) break;
            float v[kN];
            uint32_t q[kN];
            Elem<kType>::to_f32(raw[u], v);
#pragma unroll
            for (int i = 0; i < kN; ++i) q[i] = row_code(v[i] * f[u], per[i]);
            at.put_codes(a.col_codes + row * a.pitch, q);
            if (kRows) {
                if (kFold) {
                    const float t = row_per[u];
                    row_per[u] = finite_top(t) ? row_per_of(t) : 0.0f;
                    if (blockIdx.y == 0 && lane == 0) finish_top(t, a.scales + row, a.dev);
                }
#pragma unroll
                for (int i = 0; i < kN; ++i) q[i] = row_code(v[i] * w[i], row_per[u]);
                at.put_codes(a.codes + row * a.pitch, q);
            }
        }
    }
}

// the power of two of lanes that hold `vectors`, `hold` each
int lanes_of(int vectors, int hold)
{
    int lanes = 1;
    while (lanes < kThreads && lanes * hold < vectors) lanes *= 2;
    return lanes;
}

template <int kType, int kU, int kHold>
cudaError_t launch_rows(const LinCodeArgs &a, int vectors, cudaStream_t st)
{
    const int lanes = lanes_of(vectors, kHold);
    const size_t at_once = kThreads / lanes, rounds = (a.rows + at_once - 1) / at_once, room = (size_t)kRowBlocks<kHold> * kPartSms;
    return launch_chained(lin_rows_kernel<kType, kU, kHold>, dim3((unsigned)(rounds < room ? rounds : room)), dim3(kThreads), 0, st, a, lanes);
}

// As few threads a row as hold it in 64 bytes each (128 of the longest rows), since a row's own work is every thread's: 8,192 x 4096 of bf16 take 19.7 us, 24 with 32
// bytes a thread, 21 with 128.  Rows that leave SMs without a block are spread over more threads.
template <int kType, int kU>
cudaError_t rows_of(const LinCodeArgs &a, cudaStream_t st)
{
    const int vectors = (a.cols + Span<kType, kU>::kN - 1) / Span<kType, kU>::kN;
    const bool few = a.rows * vectors < (size_t)kPartSms * kThreads * 4;
    if (vectors > 4 * kThreads) return launch_rows<kType, kU, 8>(a, vectors, st);
    if (vectors <= 32 || (few && vectors <= kThreads)) return launch_rows<kType, kU, 1>(a, vectors, st);
    if (vectors <= 64) return launch_rows<kType, kU, 2>(a, vectors, st);
    return launch_rows<kType, kU, 4>(a, vectors, st);
}

// Two groups of columns a block of the first look: of tensors that keep every SM busy for some rounds all the same.
bool lin_two_groups(size_t rows, int cols, int dtype) { return cols > (dtype == EOQ_F32 ? 128 : 256) && rows * cols >= (size_t)1 << 22; }

template <int kType, int kU, bool kRows>
cudaError_t looks_of(LinErrorArgs a, int *launches, cudaStream_t st)
{
    const int vectors = (a.cols + Span<kType, kU>::kN - 1) / Span<kType, kU>::kN;
    const int lanes = vectors < 32 ? lanes_of(vectors, 1) : 32, across = (vectors + lanes - 1) / lanes, slots = kThreads / lanes;
    ++*launches;
    cudaError_t e;
    if (kU == 16 && lin_two_groups(a.rows, a.cols, kType)) {
        a.chunks = (across + 1) / 2;
        e = launch_chained(lin_look_kernel<kType, kU, kU == 16 ? 2 : 1, kRows>, dim3((unsigned)a.strips, a.chunks), dim3(kThreads), 0, st, a, lanes);
    } else {
        a.chunks = across;
        e = launch_chained(lin_look_kernel<kType, kU, 1, kRows>, dim3((unsigned)a.strips, a.chunks), dim3(kThreads), 0, st, a, lanes);
    }
    if (e != cudaSuccess) return e;
    const bool fold = a.strip_tops && a.strips <= kFoldStrips && a.rows * a.cols <= kFoldSize;
    if (!fold) {
        const size_t rows = kRows ? (a.rows + kJoinThreads - 1) / kJoinThreads : 0;
        ++*launches;
        e = launch_chained(lin_join_looks_kernel, dim3((unsigned)((a.cols + 31) / 32 + rows)), dim3(kJoinThreads), 0, st, a);
        if (e != cudaSuccess || !a.strip_tops) return e;
    }
    // eight rounds of four rows a thread, or as many as leave every SM four blocks
    size_t range = (size_t)slots * kAhead * 8;
    while (range > (size_t)slots && (a.rows + range - 1) / range * across < 4 * kPartSms) range /= 2;
    const dim3 grid((unsigned)((a.rows + range - 1) / range), across);
    ++*launches;
    if (fold) return launch_chained(lin_codes_kernel<kType, kU, kRows, true>, grid, dim3(kThreads), 0, st, a, lanes, range);
    return launch_chained(lin_codes_kernel<kType, kU, kRows, false>, grid, dim3(kThreads), 0, st, a, lanes, range);
}

template <int kType, int kU>
cudaError_t errors_of(LinErrorArgs a, int *launches, cudaStream_t st)
{
    const LinStrips s = lin_strips(a.rows, a.cols, kType);
    a.strip = s.rows;
    a.strips = (int)((a.rows + s.rows - 1) / s.rows);
    a.col_pitch = s.col_pitch;
    if (a.codes && a.strip_tops) return looks_of<kType, kU, true>(a, launches, st);
    if (a.codes) {
        LinCodeArgs r = {};
        r.src = a.src;
        r.rows = a.rows;
        r.stride = a.stride;
        r.cols = a.cols;
        r.factors = a.factors;
        r.codes = a.codes;
        r.pitch = a.pitch;
        r.scales = a.scales;
        r.dev = a.dev;
        ++*launches;
        const cudaError_t e = rows_of<kType, kU>(r, st);
        if (e != cudaSuccess) return e;
    }
    return a.strip_tops || a.strip_sums ? looks_of<kType, kU, false>(a, launches, st) : cudaSuccess;
}

template <int kType, typename F>
cudaError_t with_width(const void *src, size_t stride, F &&f)
{
    const int u = row_alignment(src, stride, Elem<kType>::kSize);
    if (u == 16) return f(std::integral_constant<int, kType>(), std::integral_constant<int, 16>());
    if (u == 8) return f(std::integral_constant<int, kType>(), std::integral_constant<int, 8>());
    if (u == 4 || kType == EOQ_F32) return f(std::integral_constant<int, kType>(), std::integral_constant<int, 4>());
    return f(std::integral_constant<int, kType>(), std::integral_constant<int, kType == EOQ_F32 ? 4 : 2>());
}
template <typename F>
cudaError_t with_type(const void *src, size_t stride, int dtype, F &&f)
{
    if (dtype == EOQ_F32) return with_width<EOQ_F32>(src, stride, f);
    if (dtype == EOQ_F16) return with_width<EOQ_F16>(src, stride, f);
    return with_width<EOQ_BF16>(src, stride, f);
}

}  // namespace

// Strips of rows: as many as let every block run at once, three on an SM, of at least eight rows; at most 512, so that what they leave stays small beside the tensor.
LinStrips lin_strips(size_t rows, int cols, int dtype)
{
    const int wide = dtype == EOQ_F32 ? 128 : 256;   // columns of a block
    const size_t chunks = (cols + wide - 1) / wide, blocks = lin_two_groups(rows, cols, dtype) ? (chunks + 1) / 2 : chunks;
    size_t strips = 3 * kPartSms / blocks;
    if (strips < 1) strips = 1;
    if (strips > 512) strips = 512;
    LinStrips s;
    s.rows = (rows + strips - 1) / strips;
    if (s.rows < 8) s.rows = 8;
    s.col_pitch = ((size_t)cols + 7) & ~(size_t)7;
    s.floats = (rows + s.rows - 1) / s.rows * s.col_pitch;
    s.row_floats = rows * chunks;
    return s;
}

cudaError_t launch_lin_rows(const LinCodeArgs &a, int dtype, int *launches, cudaStream_t st)
{
    ++*launches;
    return with_type(a.src, a.stride, dtype, [&](auto type, auto v) { return rows_of<decltype(type)::value, decltype(v)::value>(a, st); });
}
cudaError_t launch_lin_errors(const LinErrorArgs &a, int dtype, int *launches, cudaStream_t st)
{
    return with_type(a.src, a.stride, dtype, [&](auto type, auto v) { return errors_of<decltype(type)::value, decltype(v)::value>(a, launches, st); });
}

}  // namespace eoq
