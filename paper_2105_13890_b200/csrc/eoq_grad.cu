// Norm of the gradients of a step, of many tensors together, and their clipping (eoq_grad_norm, eoq_grad_clip):
//   norm = sqrt(sum of squares over all elements),  g <- g * min(1, max_norm / norm).
//
// Bound: memory, or the launches where the gradients are few.  The tensors are cut into pieces of kPiece elements, dealt out to blocks in turn; a block's squares
// are added in 64 bits (no overflow, no digits lost over long sums) in an order that depends on the sizes and alignments alone, the blocks' sums by the block that comes last.
#include "eoq_block8.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256;

// the tensor that holds piece `p`
__device__ __forceinline__ int tensor_of(const GradBatch &b, unsigned p)
{
    int lo = 0, hi = b.num - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (b.first[mid] <= p) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename F>
__device__ __forceinline__ void with_type(int dtype, F &&f)
{
    if (dtype == EOQ_F32) f(Elem<EOQ_F32>());
    else if (dtype == EOQ_F16) f(Elem<EOQ_F16>());
    else f(Elem<EOQ_BF16>());
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double sum_s[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sum_s[threadIdx.x / 32] = v;
    __syncthreads();
    v = sum_s[0];
    for (int w = 1; w < kThreads / 32; ++w) v += sum_s[w];
    return v;
}

// Of elements [0, n) at p: the first ones up to a 16-byte boundary and the last ones behind one go one at a time, the others 16 bytes at a time.
template <typename E>
__device__ __forceinline__ int head_of(const void *p, int n)
{
    return min(n, (int)((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16) / E::kSize);
}

__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const __grid_constant__ GradBatch b)
{
    ptx::grid_dep_wait_launch_small();
    double sum = 0.0;
    for (unsigned p = blockIdx.x; p < b.pieces; p += gridDim.x) {
        const int t = tensor_of(b, p);
        const size_t at = (size_t)(p - b.first[t]) * kGradPiece;
        const int n = (int)min((unsigned long long)kGradPiece, (unsigned long long)(b.size[t] - at));
        with_type(b.dtype[t], [&](auto type) {
            using E = decltype(type);
            constexpr int kV = 16 / E::kSize;
            const char *src = reinterpret_cast<const char *>(b.in[t]) + at * E::kSize;
            const int head = head_of<E>(src, n), body = (n - head) / kV;
            auto one = [&](int i) {
                float v[1];
                E::to_f32(load_raw<E::kSize>(src + (size_t)i * E::kSize), v);
                sum += (double)v[0] * v[0];
            };
            if ((int)threadIdx.x < head) one(threadIdx.x);
            if ((int)threadIdx.x < n - head - body * kV) one(head + body * kV + threadIdx.x);
#pragma unroll 4
            for (int i = threadIdx.x; i < body; i += kThreads) {
                float v[kV];
                E::to_f32(load_raw<16>(src + ((size_t)head + (size_t)i * kV) * E::kSize), v);
#pragma unroll
                for (int j = 0; j < kV; ++j) sum += (double)v[j] * v[j];
            }
        });
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) b.sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double whole_sum(const double *sums, int blocks)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < blocks; i += kThreads) s += sums[i];
    return block_sum(s);
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double *sums, int blocks, float *norm, DeviceState *dev)
{
    ptx::grid_dep_wait_launch_small();
    const double s = whole_sum(sums, blocks);
    if (threadIdx.x == 0) {
        const float n = (float)sqrt(s);
        *norm = n;
        if (!(n <= 3.402823466e38f)) atomicOr(&dev->status, EOQ_DEV_NONFINITE);
    }
}

__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const __grid_constant__ GradBatch b, const double *sums, int blocks, float max_norm, float *norm, DeviceState *dev)
{
    ptx::grid_dep_wait_launch_small();
    const double whole = sqrt(whole_sum(sums, blocks));
    const bool fine = whole <= 3.402823466e38;
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm) {
        *norm = (float)whole;
        if (!fine) atomicOr(&dev->status, EOQ_DEV_NONFINITE);
    }
    const float scale = fine && whole > max_norm ? (float)(max_norm / whole) : 1.0f;
    for (unsigned p = blockIdx.x; p < b.pieces; p += gridDim.x) {
        const int t = tensor_of(b, p);
        if (b.in[t] == b.out[t] && scale == 1.0f) continue;
        const size_t at = (size_t)(p - b.first[t]) * kGradPiece;
        const int n = (int)min((unsigned long long)kGradPiece, (unsigned long long)(b.size[t] - at));
        with_type(b.dtype[t], [&](auto type) {
            using E = decltype(type);
            constexpr int kV = 16 / E::kSize;
            const char *src = reinterpret_cast<const char *>(b.in[t]) + at * E::kSize;
            char *dst = reinterpret_cast<char *>(b.out[t]) + at * E::kSize;
            const bool together = reinterpret_cast<uintptr_t>(src) % 16 == reinterpret_cast<uintptr_t>(dst) % 16;
            const int head = together ? head_of<E>(src, n) : n, body = (n - head) / kV;
            auto one = [&](int i) {
                float v[1];
                E::to_f32(*reinterpret_cast<const Raw<E::kSize> *>(src + (size_t)i * E::kSize), v);
                v[0] *= scale;
                store_raw(dst + (size_t)i * E::kSize, E::from_f32(v));
            };
            for (int i = threadIdx.x; i < head; i += kThreads) one(i);
            for (int i = head + body * kV + threadIdx.x; i < n; i += kThreads) one(i);
#pragma unroll 4
            for (int i = threadIdx.x; i < body; i += kThreads) {
                const size_t o = ((size_t)head + (size_t)i * kV) * E::kSize;
                float v[kV];
                E::to_f32(*reinterpret_cast<const Raw<16> *>(src + o), v);
#pragma unroll
                for (int j = 0; j < kV; ++j) v[j] *= scale;
                store_raw(dst + o, E::from_f32(v));
            }
        });
    }
}

}  // namespace

constexpr unsigned kMostBlocks = 4u * kPartSms;   // of a launch: the order of the sums depends on the sizes alone

static size_t batches_of(int num) { return ((size_t)num + kGradTensors - 1) / kGradTensors; }
size_t grad_workspace_bytes(int num) { return sizeof(double) * kMostBlocks * batches_of(num); }

cudaError_t launch_grad(const GradList &l, bool clip, float max_norm, float *norm, void *workspace, DeviceState *dev, int *launches, cudaStream_t st)
{
    double *sums = reinterpret_cast<double *>(workspace);
    int blocks = 0;
    // tensors [first, first + kGradTensors) as a launch takes them; those without elements are left out
    auto batch = [&](int first, GradBatch &b) {
        b.num = 0;
        b.pieces = 0;
        for (int i = first; i < l.num && i < first + kGradTensors; ++i) {
            if (l.size[i] == 0) continue;
            b.in[b.num] = l.in[i];
            b.out[b.num] = l.out ? l.out[i] : const_cast<void *>(l.in[i]);
            b.size[b.num] = l.size[i];
            b.dtype[b.num] = (uint8_t)l.dtype[i];
            b.first[b.num] = b.pieces;
            b.pieces += (unsigned)((l.size[i] + kGradPiece - 1) / kGradPiece);
            ++b.num;
        }
        return b.pieces < kMostBlocks ? b.pieces : kMostBlocks;
    };
    GradBatch b;
    for (int first = 0; first < l.num; first += kGradTensors) {
        const unsigned grid = batch(first, b);
        if (grid == 0) continue;
        b.sums = sums + blocks;
        ++*launches;
        const cudaError_t e = launch_chained(grad_squares_kernel, dim3(grid), dim3(kThreads), 0, st, b);
        if (e != cudaSuccess) return e;
        blocks += (int)grid;
    }
    if (!clip) {
        ++*launches;
        return launch_chained(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, (const double *)sums, blocks, norm, dev);
    }
    for (int first = 0, done = 0; first < l.num || !done; first += kGradTensors, ++done) {
        const unsigned grid = batch(first, b);
        if (grid == 0 && done) continue;
        ++*launches;
        const cudaError_t e = launch_chained(grad_scale_kernel, dim3(grid ? grid : 1), dim3(kThreads), 0, st, b, (const double *)sums, blocks, max_norm,
                                             done ? (float *)nullptr : norm, dev);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace eoq
