// Codes of floating-point rows and columns with a scale each (eoq_lin_quantize, and the first steps of eoq_lin_fwd and eoq_lin_bwd):
//   scale = max(largest magnitude, 2^-119) / 127,  code = R(value * fl(127 / max(..))).
//
// Bound: memory.  A row belongs to 32 to 256 neighbouring threads, which keep it in registers between the look for its maximum and its coding; only
// rows longer than they hold are read a second time.  Columns need all rows before the first code: two looks at the tensor.
#include "eoq_lin.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256;

// kHold vectors of kV elements a lane; `lanes` of a row (32, 64, 128 or 256)
template <int kType, int kV>
__global__ void __launch_bounds__(kThreads) lin_rows_kernel(const __grid_constant__ LinCodeArgs a, const int lanes)
{
    constexpr int kE = Elem<kType>::kSize, kHold = kV == 1 ? 16 : 64 / (kV * kE);
    __shared__ float top_s[kThreads / 32];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes, slots = kThreads / lanes;
    const size_t row = (size_t)blockIdx.x * slots + slot;
    const bool mine = row < a.rows;
    const char *src = reinterpret_cast<const char *>(a.src) + row * a.stride * kE;
    // a vector of the row, times the columns' factors; zeros behind the end
    auto get = [&](int col, float (&v)[kV]) {
        if (mine && col + kV <= a.cols) {
            Elem<kType>::to_f32(load_raw<kV * kE>(src + (size_t)col * kE), v);
        } else {
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                float one[1] = {0.0f};
                if (mine && col + i < a.cols) Elem<kType>::to_f32(load_raw<kE>(src + (size_t)(col + i) * kE), one);
                v[i] = one[0];
            }
        }
        if (a.factors)
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (col + i < a.cols) v[i] *= __ldg(a.factors + col + i);
    };
    float held[kHold][kV], top = 0.0f;
#pragma unroll
    for (int h = 0; h < kHold; ++h) {
        get((h * lanes + lane) * kV, held[h]);
#pragma unroll
        for (int i = 0; i < kV; ++i) top = max_abs(top, held[h][i]);
    }
    for (int col = (kHold * lanes + lane) * kV; col < a.cols; col += lanes * kV) {
        float v[kV];
        get(col, v);
#pragma unroll
        for (int i = 0; i < kV; ++i) top = max_abs(top, v[i]);
    }
    top = lanes_max_abs<32>(top);
    if (lanes > 32) {
        if (threadIdx.x % 32 == 0) top_s[threadIdx.x / 32] = top;
        __syncthreads();
        const int first = slot * (lanes / 32);
        top = top_s[first];
        for (int w = 1; w < lanes / 32; ++w) top = max_abs(top, top_s[first + w]);
    }
    if (!mine) return;
    const bool fine = finite_top(top);
    const float per = row_per_of(top);
    if (lane == 0) {
        a.scales[row] = row_scale_of(top);
        if (!fine) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
    }
    int8_t *dst = a.codes + row * a.pitch;
    auto put = [&](int col, const float (&v)[kV]) {
        if (col >= a.cols) return;
        uint32_t q[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) q[i] = fine ? row_code(v[i], per) : 0u;
        store_raw(dst + col, pack_codes(q));   // (a row of codes is whole pieces of 16 bytes)
    };
#pragma unroll
    for (int h = 0; h < kHold; ++h) put((h * lanes + lane) * kV, held[h]);
    for (int col = (kHold * lanes + lane) * kV; col < a.cols; col += lanes * kV) {
        float v[kV];
        get(col, v);
        put(col, v);
    }
}

// Largest magnitudes of the columns, values times the rows' factors, and the columns' sums (without factors) by strips of rows.  32 x kV columns and a strip
// a block, eight rows at a time.
template <int kType, int kV>
__global__ void __launch_bounds__(kThreads) lin_column_tops_kernel(const __grid_constant__ LinCodeArgs a)
{
    constexpr int kE = Elem<kType>::kSize;
    __shared__ float top_s[8][32 * kV], sum_s[8][32 * kV];
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % 32, slot = threadIdx.x / 32, col = (blockIdx.x * 32 + lane) * kV;
    const size_t begin = (size_t)blockIdx.y * a.strip, end = min(a.rows, begin + a.strip);
    float top[kV] = {}, sum[kV] = {};
#pragma unroll 4
    for (size_t row = begin + slot; row < end; row += 8) {
        const char *src = reinterpret_cast<const char *>(a.src) + (row * a.stride + col) * kE;
        const float f = a.factors ? __ldg(a.factors + row) : 1.0f;
        if (col + kV <= a.cols) {
            float v[kV];
            Elem<kType>::to_f32(load_raw<kV * kE>(src), v);
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                top[i] = max_abs(top[i], v[i] * f);
                sum[i] += v[i];
            }
        } else {
            for (int i = 0; i < kV; ++i)
                if (col + i < a.cols) {
                    float one[1];
                    Elem<kType>::to_f32(load_raw<kE>(src + i * kE), one);
                    top[i] = max_abs(top[i], one[0] * f);
                    sum[i] += one[0];
                }
        }
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        top_s[slot][lane * kV + i] = top[i];
        sum_s[slot][lane * kV + i] = sum[i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * kV; c += kThreads) {
        const int at = blockIdx.x * 32 * kV + c;
        if (at >= a.cols) continue;
        float m = top_s[0][c], s = sum_s[0][c];
        for (int w = 1; w < 8; ++w) {
            m = max_abs(m, top_s[w][c]);
            s += sum_s[w][c];
        }
        if (a.tops) atomicMax(a.tops + at, __float_as_uint(m));   // (of magnitudes, the order of the bits; NaN above all)
        if (a.sums) a.strip_sums[(size_t)blockIdx.y * a.cols + at] = s;
    }
}

// Codes of the columns, and the strips' sums added.
template <int kType, int kV>
__global__ void __launch_bounds__(kThreads) lin_columns_kernel(const __grid_constant__ LinCodeArgs a)
{
    constexpr int kE = Elem<kType>::kSize;
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x % 32, slot = threadIdx.x / 32, col = (blockIdx.x * 32 + lane) * kV;
    const size_t begin = (size_t)blockIdx.y * a.strip, end = min(a.rows, begin + a.strip);
    if (a.sums && blockIdx.y == 0)
        for (int c = threadIdx.x; c < 32 * kV; c += kThreads) {
            const int at = blockIdx.x * 32 * kV + c;
            if (at >= a.cols) continue;
            float s = 0.0f;
            for (int y = 0; y < a.strips; ++y) s += __ldg(a.strip_sums + (size_t)y * a.cols + at);
            a.sums[at] = s;
        }
    if (!a.tops || col >= a.cols) return;
    float per[kV];
    bool fine[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const float top = col + i < a.cols ? __uint_as_float(a.tops[col + i]) : 0.0f;
        fine[i] = finite_top(top);
        per[i] = row_per_of(top);
        if (blockIdx.y == 0 && slot == 0 && col + i < a.cols) {
            a.scales[col + i] = row_scale_of(top);
            if (!fine[i]) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
        }
    }
#pragma unroll 4
    for (size_t row = begin + slot; row < end; row += 8) {
        const char *src = reinterpret_cast<const char *>(a.src) + (row * a.stride + col) * kE;
        const float f = __ldg(a.factors + row);
        float v[kV];
        if (col + kV <= a.cols) {
            Elem<kType>::to_f32(load_raw<kV * kE>(src), v);
        } else {
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                float one[1] = {0.0f};
                if (col + i < a.cols) Elem<kType>::to_f32(load_raw<kE>(src + i * kE), one);
                v[i] = one[0];
            }
        }
        uint32_t q[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) q[i] = fine[i] ? row_code(v[i] * f, per[i]) : 0u;
        store_raw(a.codes + row * a.pitch + col, pack_codes(q));
    }
}

// elements of the widest vectors that every row begins and ends pieces of
int vector_of(const void *src, size_t stride, int e)
{
    const size_t at = reinterpret_cast<uintptr_t>(src) | stride * e;
    return at % 16 == 0 ? 16 / e : e == 2 && at % 4 == 0 ? 2 : 1;
}

template <int kType, int kV>
cudaError_t rows_of(const LinCodeArgs &a, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kHold = kV == 1 ? 16 : 64 / (kV * kE);
    int lanes = 32;
    while (lanes < kThreads && lanes * kV * kHold < a.cols) lanes *= 2;
    const size_t slots = kThreads / lanes;
    return launch_chained(lin_rows_kernel<kType, kV>, dim3((unsigned)((a.rows + slots - 1) / slots)), dim3(kThreads), 0, st, a, lanes);
}

template <int kType, int kV>
cudaError_t columns_of(LinCodeArgs a, int *launches, cudaStream_t st)
{
    const unsigned across = (a.cols + 32 * kV - 1) / (32 * kV);
    if (a.tops) {
        const cudaError_t e = cudaMemsetAsync(a.tops, 0, (size_t)a.cols * 4, st);
        if (e != cudaSuccess) return e;
    }
    a.strip = lin_strip_rows(a.rows);
    a.strips = (int)((a.rows + a.strip - 1) / a.strip);
    ++*launches;
    cudaError_t e = launch_chained(lin_column_tops_kernel<kType, kV>, dim3(across, a.strips), dim3(kThreads), 0, st, a);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_chained(lin_columns_kernel<kType, kV>, dim3(across, a.tops ? a.strips : 1), dim3(kThreads), 0, st, a);
}

template <int kType>
cudaError_t of_type(const LinCodeArgs &a, bool columns, int *launches, cudaStream_t st)
{
    const int v = vector_of(a.src, a.stride, Elem<kType>::kSize);
    if (!columns) ++*launches;
    if (v == 16 / Elem<kType>::kSize) return columns ? columns_of<kType, 16 / Elem<kType>::kSize>(a, launches, st) : rows_of<kType, 16 / Elem<kType>::kSize>(a, st);
    if constexpr (Elem<kType>::kSize == 2)
        if (v == 2) return columns ? columns_of<kType, 2>(a, launches, st) : rows_of<kType, 2>(a, st);
    return columns ? columns_of<kType, 1>(a, launches, st) : rows_of<kType, 1>(a, st);
}

cudaError_t dispatch(const LinCodeArgs &a, int dtype, bool columns, int *launches, cudaStream_t st)
{
    if (dtype == EOQ_F32) return of_type<EOQ_F32>(a, columns, launches, st);
    if (dtype == EOQ_F16) return of_type<EOQ_F16>(a, columns, launches, st);
    return of_type<EOQ_BF16>(a, columns, launches, st);
}

}  // namespace

// rows of a strip: at least 64, and at most 512 strips
size_t lin_strip_rows(size_t rows)
{
    const size_t least = (rows + 511) / 512;
    return least < 64 ? 64 : (least + 7) / 8 * 8;
}

cudaError_t launch_lin_rows(const LinCodeArgs &a, int dtype, int *launches, cudaStream_t st) { return dispatch(a, dtype, false, launches, st); }
cudaError_t launch_lin_columns(const LinCodeArgs &a, int dtype, int *launches, cudaStream_t st) { return dispatch(a, dtype, true, launches, st); }

}  // namespace eoq
