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
constexpr int kFoldStrips = 32;   // strips whose maxima the second look finds by itself; more take a kernel between the two

// magnitudes as unsigned bits: their order, with infinity and then NaN above all numbers
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// the largest magnitude among the elements of a vector, as an fp32's bits
template <int kType, int kBytes>
__device__ __forceinline__ uint32_t raw_top(const Raw<kBytes> &r, uint32_t top)
{
    if constexpr (kType == EOQ_F32) {
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) top = max(top, raw_word(r, i) & 0x7fffffffu);
        return top;
    } else {
        // the halves of a word side by side
        uint32_t m = 0;
        if constexpr (kBytes == 2) {
            m = raw_word(r, 0) & 0x7fffu;
        } else {
#pragma unroll
            for (int i = 0; i < kBytes / 4; ++i) m = __vmaxs2(m, raw_word(r, i) & 0x7fff7fffu);
            m = max(m & 0xffffu, m >> 16);
        }
        if constexpr (kType == EOQ_BF16) return max(top, m << 16);
        else return max(top, abs_bits(__half2float(__ushort_as_half((unsigned short)m))));
    }
}

// a vector of a row from `col` on, zeros behind the row's end
template <int kType, int kV>
__device__ __forceinline__ Raw<kV * Elem<kType>::kSize> get_raw(const char *row, int col, int cols, bool mine)
{
    constexpr int kE = Elem<kType>::kSize;
    if (mine && col + kV <= cols) return load_raw<kV * kE>(row + (size_t)col * kE);
    Raw<kV * kE> r = zero_raw<kV * kE>();
    if constexpr (kV > 1) {
        if (mine && col < cols) {
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                if (col + i >= cols) break;
                const uint32_t w = raw_word(load_raw<kE>(row + (size_t)(col + i) * kE), 0);
                if constexpr (kE == 4) set_word(r, i, w);
                else set_word(r, i / 2, i & 1 ? raw_word(r, i / 2) | w << 16 : w);
            }
        }
    }
    return r;
}

// factors of kV columns; ones (of nothing) behind the end
template <int kV>
__device__ __forceinline__ void get_factors(const float *factors, int col, int cols, float (&f)[kV])
{
#pragma unroll
    for (int i = 0; i < kV; ++i) f[i] = col + i < cols ? __ldg(factors + col + i) : 1.0f;
}

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

template <int kV>
__device__ __forceinline__ void put_codes(int8_t *row, int col, const float (&v)[kV], float per, bool fine)
{
    uint32_t q[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) q[i] = row_code(v[i], per);
    Raw<kV> r = pack_codes(q);
    store_raw(row + col, fine ? r : zero_raw<kV>());   // (a row of codes is whole pieces of 16 bytes)
}

// Rows: kHold vectors of kV elements a lane of each of kRows rows at a time.
template <int kType, int kV, int kHold, int kRows>
__global__ void __launch_bounds__(kThreads) lin_rows_kernel(const __grid_constant__ LinCodeArgs a, const int lanes)
{
    constexpr int kE = Elem<kType>::kSize;
    __shared__ uint32_t cells[kThreads / 32];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slots = kThreads / lanes;
    const size_t row0 = (size_t)blockIdx.x * kRows * slots + threadIdx.x / lanes;
    const char *src = reinterpret_cast<const char *>(a.src) + row0 * a.stride * kE;
    const size_t step = slots * a.stride * kE;
    auto scaled = [&](const Raw<kV * kE> &r, int col, float (&v)[kV]) {
        Elem<kType>::to_f32(r, v);
        if (a.factors) {
            float f[kV];
            get_factors(a.factors, col, a.cols, f);
#pragma unroll
            for (int i = 0; i < kV; ++i) v[i] *= f[i];
        }
    };
    auto more = [&](uint32_t top, const Raw<kV * kE> &r, int col) {
        if (!a.factors) return raw_top<kType, kV * kE>(r, top);
        float v[kV];
        scaled(r, col, v);
#pragma unroll
        for (int i = 0; i < kV; ++i) top = max(top, abs_bits(v[i]));
        return top;
    };
    Raw<kV * kE> held[kRows][kHold];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int h = 0; h < kHold; ++h) held[u][h] = get_raw<kType, kV>(src + u * step, (h * lanes + lane) * kV, a.cols, row0 + u * slots < a.rows);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const size_t row = row0 + u * slots;
        const bool mine = row < a.rows;
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < kHold; ++h) top = more(top, held[u][h], (h * lanes + lane) * kV);
        if (mine)
            for (int col = (kHold * lanes + lane) * kV; col < a.cols; col += lanes * kV) top = more(top, get_raw<kType, kV>(src + u * step, col, a.cols, true), col);
        const float t = __uint_as_float(lanes_top(top, lanes, cells));
        if (kRows > 1 && lanes > 32) __syncthreads();   // (the cells are read)
        if (!mine) continue;
        const bool fine = finite_top(t);
        const float per = row_per_of(t);
        if (lane == 0) {
            a.scales[row] = row_scale_of(t);
            if (!fine) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
        }
        int8_t *dst = a.codes + row * a.pitch;
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            const int col = (h * lanes + lane) * kV;
            if (col >= a.cols) break;
            float v[kV];
            scaled(held[u][h], col, v);
            put_codes(dst, col, v, per, fine);
        }
        for (int col = (kHold * lanes + lane) * kV; col < a.cols; col += lanes * kV) {
            float v[kV];
            scaled(get_raw<kType, kV>(src + u * step, col, a.cols, true), col, v);
            put_codes(dst, col, v, per, fine);
        }
    }
}

// ------------------------------------------------------------------ the errors of a layer

// kV floats from an address that is a multiple of their size
template <int kV>
__device__ __forceinline__ void get_floats(const float *p, float (&v)[kV])
{
    if constexpr (kV % 4 == 0) {
#pragma unroll
        for (int i = 0; i < kV; i += 4) {
            const float4 w = __ldg(reinterpret_cast<const float4 *>(p + i));
            v[i] = w.x;
            v[i + 1] = w.y;
            v[i + 2] = w.z;
            v[i + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) v[i] = __ldg(p + i);
    }
}
template <int kV>
__device__ __forceinline__ void put_floats(float *p, const float (&v)[kV])
{
    if constexpr (kV % 4 == 0) {
#pragma unroll
        for (int i = 0; i < kV; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) p[i] = v[i];
    }
}

constexpr int kAhead = 4;   // rows of a thread in flight

// Block (x, y): strip x of the rows, `lanes` (at most 32) vectors of columns.  kRows: the rows' maxima too.
template <int kType, int kV, bool kRows>
__global__ void __launch_bounds__(kThreads) lin_look_kernel(const __grid_constant__ LinErrorArgs a, const int lanes)
{
    constexpr int kE = Elem<kType>::kSize;
    __shared__ float tops_s[kThreads][kV], sums_s[kThreads][kV];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes, slots = kThreads / lanes, col = (blockIdx.y * lanes + lane) * kV;
    const size_t begin = (size_t)blockIdx.x * a.strip, end = min(a.rows, begin + a.strip);
    const char *src = reinterpret_cast<const char *>(a.src) + (begin + slot) * a.stride * kE;
    const size_t step = slots * a.stride * kE;
    float w[kV], top[kV] = {}, sum[kV] = {};
    if (kRows) get_factors(a.factors, col, a.cols, w);
    Raw<kV * kE> next[kAhead];
    float next_f[kAhead];
    auto fetch = [&](size_t row) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool mine = row + u * slots < end;
            next[u] = get_raw<kType, kV>(src + u * step, col, a.cols, mine);
            next_f[u] = mine && a.row_factors ? __ldg(a.row_factors + row + u * slots) : 0.0f;
        }
        src += kAhead * step;
    };
    fetch(begin + slot);
    for (size_t row0 = begin; row0 < end; row0 += kAhead * slots) {   // (the same rounds for every lane)
        Raw<kV * kE> held[kAhead];
        float f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            held[u] = next[u];
            f[u] = next_f[u];
        }
        fetch(row0 + slot + kAhead * slots);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float v[kV], m = 0.0f;
            Elem<kType>::to_f32(held[u], v);
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                if (kRows) m = max_abs(m, v[i] * w[i]);
                top[i] = max_abs(top[i], v[i] * f[u]);
                sum[i] += v[i];
            }
            if (kRows) {
                const uint32_t t = lanes_top(__float_as_uint(m), lanes, nullptr);
                const size_t row = row0 + slot + u * slots;
                if (lane == 0 && row < end) a.row_tops[blockIdx.y * a.rows + row] = __uint_as_float(t);
            }
        }
    }
    put_floats(tops_s[threadIdx.x], top);
    put_floats(sums_s[threadIdx.x], sum);
    __syncthreads();
    if (slot == 0 && col < a.cols) {
        for (int s = 1; s < slots; ++s) {
            const int at = s * lanes + lane;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                top[i] = max_abs(top[i], tops_s[at][i]);
                sum[i] += sums_s[at][i];
            }
        }
        const size_t at = (size_t)blockIdx.x * a.col_pitch + col;
        if (a.strip_tops) put_floats(a.strip_tops + at, top);
        if (a.strip_sums) put_floats(a.strip_sums + at, sum);
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

// What the parts left, put together: by the first blocks 32 columns each, a share of the strips a warp, by the others a row a thread.
constexpr int kJoinThreads = 512;
__global__ void __launch_bounds__(kJoinThreads) lin_join_looks_kernel(const __grid_constant__ LinErrorArgs a)
{
    constexpr int kWarps = kJoinThreads / 32;
    __shared__ float tops_s[kWarps][32], sums_s[kWarps][32];
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
    float top = 0.0f, sum = 0.0f;
    if (col < a.cols) {
#pragma unroll 4
        for (int s = warp; s < a.strips; s += kWarps) {
            if (a.strip_tops) top = max_abs(top, __ldg(a.strip_tops + (size_t)s * a.col_pitch + col));
            if (a.strip_sums) sum += __ldg(a.strip_sums + (size_t)s * a.col_pitch + col);
        }
    }
    tops_s[warp][lane] = top;
    sums_s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < a.cols) {
        for (int w = 1; w < kWarps; ++w) {
            top = max_abs(top, tops_s[w][lane]);
            sum += sums_s[w][lane];
        }
        if (a.strip_tops) a.col_per[col] = finish_top(top, a.col_scales + col, a.dev);
        if (a.strip_sums) a.sums[col] = sum;
    }
}

// The second look.  Block (x, y): `range` rows from x * range on, `lanes` vectors of columns.  kFold: what the parts left is put together here, column by
// column and row by row, by every thread that needs it.
template <int kType, int kV, bool kRows, bool kFold>
__global__ void __launch_bounds__(kThreads) lin_codes_kernel(const __grid_constant__ LinErrorArgs a, const int lanes, const size_t range)
{
    constexpr int kE = Elem<kType>::kSize;
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes, slots = kThreads / lanes, col = (blockIdx.y * lanes + lane) * kV;
    const size_t begin = (size_t)blockIdx.x * range, end = min(a.rows, begin + range);
    if (col >= a.cols) return;
    const char *src = reinterpret_cast<const char *>(a.src) + (begin + slot) * a.stride * kE;
    const size_t step = slots * a.stride * kE;
    Raw<kV * kE> next[kAhead];
    float next_f[kAhead], next_per[kAhead];
    auto fetch = [&](size_t row0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const size_t row = row0 + u * slots;
            const bool mine = row < end;
            next[u] = get_raw<kType, kV>(src + u * step, col, a.cols, mine);
            next_f[u] = mine ? __ldg(a.row_factors + row) : 0.0f;
            if (kRows && !kFold) next_per[u] = mine ? __ldg(a.row_per + row) : 0.0f;
            if (kRows && kFold) {
                next_per[u] = 0.0f;
                if (mine)
                    for (int c = 0; c < a.chunks; ++c) next_per[u] = max_abs(next_per[u], __ldg(a.row_tops + c * a.rows + row));
            }
        }
        src += kAhead * step;
    };
    fetch(begin + slot);
    float w[kV], per[kV];
    if (kRows) get_factors(a.factors, col, a.cols, w);
    if (kFold) {
        float top[kV] = {}, sum[kV] = {};
#pragma unroll 4
        for (int s = 0; s < a.strips; ++s) {
            float t[kV];
            get_floats(a.strip_tops + (size_t)s * a.col_pitch + col, t);
#pragma unroll
            for (int i = 0; i < kV; ++i) top[i] = max_abs(top[i], t[i]);
        }
        const bool writes = blockIdx.x == 0 && slot == 0;
        if (writes && a.strip_sums) {
#pragma unroll 4
            for (int s = 0; s < a.strips; ++s) {
                float t[kV];
                get_floats(a.strip_sums + (size_t)s * a.col_pitch + col, t);
#pragma unroll
                for (int i = 0; i < kV; ++i) sum[i] += t[i];
            }
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (col + i < a.cols) a.sums[col + i] = sum[i];
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            if (writes && col + i < a.cols) finish_top(top[i], a.col_scales + col + i, a.dev);
            per[i] = finite_top(top[i]) ? row_per_of(top[i]) : 0.0f;
        }
    } else {
        get_floats(a.col_per + col, per);
    }
    for (size_t row0 = begin + slot; row0 < end; row0 += kAhead * slots) {
        Raw<kV * kE> held[kAhead];
        float f[kAhead], row_per[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            held[u] = next[u];
            f[u] = next_f[u];
            row_per[u] = next_per[u];
        }
        fetch(row0 + kAhead * slots);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const size_t row = row0 + u * slots;
            if (row >= end) break;
            float v[kV];
            Elem<kType>::to_f32(held[u], v);
            uint32_t q[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) q[i] = row_code(v[i] * f[u], per[i]);
            store_raw(a.col_codes + row * a.pitch + col, pack_codes(q));
            if (kRows) {
                if (kFold) {
                    const float t = row_per[u];
                    row_per[u] = finite_top(t) ? row_per_of(t) : 0.0f;
                    if (blockIdx.y == 0 && lane == 0) finish_top(t, a.scales + row, a.dev);
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) q[i] = row_code(v[i] * w[i], row_per[u]);
                store_raw(a.codes + row * a.pitch + col, pack_codes(q));
            }
        }
    }
}

// elements of the widest vectors that every row begins and ends pieces of
int vector_of(const void *src, size_t stride, int e)
{
    const size_t at = reinterpret_cast<uintptr_t>(src) | stride * e;
    return at % 16 == 0 ? 16 / e : e == 2 && at % 4 == 0 ? 2 : 1;
}

// the power of two of lanes that hold `vectors`, `hold` each
int lanes_of(int vectors, int hold)
{
    int lanes = 1;
    while (lanes < kThreads && lanes * hold < vectors) lanes *= 2;
    return lanes;
}

template <int kType, int kV, int kHold, int kRows>
cudaError_t launch_rows(const LinCodeArgs &a, int vectors, cudaStream_t st)
{
    const int lanes = lanes_of(vectors, kHold);
    const size_t at_once = (size_t)kThreads / lanes * kRows;
    return launch_chained(lin_rows_kernel<kType, kV, kHold, kRows>, dim3((unsigned)((a.rows + at_once - 1) / at_once)), dim3(kThreads), 0, st, a, lanes);
}

// 64 bytes a thread in flight (128 for the longest rows), of one row or of four; rows that leave SMs without a block are spread over more threads.
template <int kType, int kV>
cudaError_t rows_of(const LinCodeArgs &a, cudaStream_t st)
{
    const int vectors = (a.cols + kV - 1) / kV;
    const bool few = a.rows * vectors < (size_t)kPartSms * kThreads * 4;
    if (vectors > 4 * kThreads) return launch_rows<kType, kV, 8, 1>(a, vectors, st);
    if (few && vectors <= kThreads) return launch_rows<kType, kV, 1, 1>(a, vectors, st);
    if (vectors <= 32) return launch_rows<kType, kV, 1, 4>(a, vectors, st);
    if (vectors <= 64) return launch_rows<kType, kV, 2, 2>(a, vectors, st);
    return launch_rows<kType, kV, 4, 1>(a, vectors, st);
}

template <int kType, int kV, bool kRows>
cudaError_t looks_of(LinErrorArgs a, int vectors, int *launches, cudaStream_t st)
{
    const int lanes = vectors < 32 ? lanes_of(vectors, 1) : 32, across = (vectors + lanes - 1) / lanes, slots = kThreads / lanes;
    a.chunks = across;
    ++*launches;
    cudaError_t e = launch_chained(lin_look_kernel<kType, kV, kRows>, dim3((unsigned)a.strips, across), dim3(kThreads), 0, st, a, lanes);
    if (e != cudaSuccess) return e;
    const bool fold = a.strip_tops && a.strips <= kFoldStrips && across <= kFoldStrips;
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
    if (fold) return launch_chained(lin_codes_kernel<kType, kV, kRows, true>, grid, dim3(kThreads), 0, st, a, lanes, range);
    return launch_chained(lin_codes_kernel<kType, kV, kRows, false>, grid, dim3(kThreads), 0, st, a, lanes, range);
}

template <int kType, int kV>
cudaError_t errors_of(LinErrorArgs a, int *launches, cudaStream_t st)
{
    const int vectors = (a.cols + kV - 1) / kV;
    const LinStrips s = lin_strips(a.rows, a.cols);
    a.strip = s.rows;
    a.strips = (int)((a.rows + s.rows - 1) / s.rows);
    a.col_pitch = s.col_pitch;
    if (a.codes && a.strip_tops) return looks_of<kType, kV, true>(a, vectors, launches, st);
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
        const cudaError_t e = rows_of<kType, kV>(r, st);
        if (e != cudaSuccess) return e;
    }
    return a.strip_tops || a.strip_sums ? looks_of<kType, kV, false>(a, vectors, launches, st) : cudaSuccess;
}

template <int kType, typename F>
cudaError_t with_vectors(const void *src, size_t stride, F &&f)
{
    constexpr int kWide = 16 / Elem<kType>::kSize;
    const int v = vector_of(src, stride, Elem<kType>::kSize);
    if (v == kWide) return f(std::integral_constant<int, kType>(), std::integral_constant<int, kWide>());
    if constexpr (kWide == 8)
        if (v == 2) return f(std::integral_constant<int, kType>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, kType>(), std::integral_constant<int, 1>());
}
template <typename F>
cudaError_t with_type(const void *src, size_t stride, int dtype, F &&f)
{
    if (dtype == EOQ_F32) return with_vectors<EOQ_F32>(src, stride, f);
    if (dtype == EOQ_F16) return with_vectors<EOQ_F16>(src, stride, f);
    return with_vectors<EOQ_BF16>(src, stride, f);
}

}  // namespace

// Strips of rows: some eight blocks of 256 columns for each SM, of at least eight rows; at most 512, so that what they leave stays small beside the tensor.
LinStrips lin_strips(size_t rows, int cols)
{
    size_t strips = (8 * kPartSms + (cols + 255) / 256 - 1) / ((cols + 255) / 256);
    if (strips > 512) strips = 512;
    LinStrips s;
    s.rows = (rows + strips - 1) / strips;
    if (s.rows < 8) s.rows = 8;
    s.col_pitch = ((size_t)cols + 7) & ~(size_t)7;
    s.floats = (rows + s.rows - 1) / s.rows * s.col_pitch;
    s.row_floats = rows * ((cols + 31) / 32);   // (of the narrowest vectors: chunks of 32 columns)
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
