// Norm of the gradients of a step, of many tensors together, and their clipping (eoq_grad_norm, eoq_grad_clip):
//   norm = sqrt(sum of squares over all elements),  g <- g * min(1, max_norm / norm).
//
// Bound: memory, or the launches where the gradients are few.  The tensors are cut into pieces, dealt out to blocks in turn; the squares of 16 bytes are added in
// 32 bits and these sums in 64, in an order that depends on the sizes and alignments alone, the blocks' sums by the block that comes last.  (Every square in 64 bits:
// the conversions hold the kernel at 1.5 T elements a second, 133 us for 200 M of two types.)  A thread has 64 bytes on their way while it uses as many: with load
// and store in turn, that many took 240 us to scale instead of 159.
#include "eoq_block8.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256, kFlight = 4;        // vectors of a thread in flight
constexpr unsigned kAddBlocks = 4 * kPartSms, kScaleBlocks = 4 * kPartSms;   // of a launch, all at once on the part; the order of the sums depends on the sizes alone
constexpr int kFewTensors = 128, kMostTensors = 960, kRanges = 512;   // (some 32 KB of parameters at most)

// What a launch has to know of a tensor, side by side: parameters come from far away the first time, a line at a time.
struct alignas(32) GradTensor {
    const void *in;
    void *out;
    unsigned long long size;
    unsigned first;                    // pieces of the tensors before
    int dtype;
};
template <int kTensors>
struct GradBatch {                     // a launch's tensors
    GradTensor tensor[kTensors];
    uint16_t start[kRanges];           // tensor of the first piece of every range of 2^shift pieces
    unsigned pieces;
    int num, shift;
};

// What the launches of a call share.
struct GradSums {
    double *sums;                      // a block's sum of squares each, of all launches
    int before;                        // blocks of the launches before this one
    bool last;                         // this one is the last of a norm without clipping, which adds them
    float *norm;
    DeviceState *dev;
};

// Elements of a piece: what the threads of a block have in flight.  Pieces begin at multiples of 128 bytes: a tensor's first one has `skew` elements less.
__host__ __device__ inline unsigned piece_of(int dtype) { return kFlight * kThreads * (dtype == EOQ_F32 ? 4 : 8); }
__host__ __device__ inline unsigned skew_of(const void *p, int dtype) { return (unsigned)(reinterpret_cast<uintptr_t>(p) % 128) / (dtype == EOQ_F32 ? 4 : 2); }

// The tensor of a piece.  It is looked up in a table of the pieces' ranges and then among the few that share one: parameters are read one at a time, and a search by
// halves waits for ten such reads one after the other.
template <int kTensors>
__device__ __forceinline__ int tensor_of(const GradBatch<kTensors> &b, unsigned p)
{
    int t = b.start[p >> b.shift];
    while (t + 1 < b.num && b.tensor[t + 1].first <= p) ++t;
    return t;
}

template <typename F>
__device__ __forceinline__ void with_type(int dtype, F &&f)
{
    if (dtype == EOQ_F32) f(Elem<EOQ_F32>());
    else if (dtype == EOQ_F16) f(Elem<EOQ_F16>());
    else f(Elem<EOQ_BF16>());
}

// sum over the block, in every thread
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double sum_s[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sum_s[threadIdx.x / 32] = v;
    __syncthreads();
    v = sum_s[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v += sum_s[w];
    return v;
}

// The squares of 16 bytes in fp32: off by 5 * 2^-24 of their sum at most, as long as that is a good one.
template <typename E>
__device__ __forceinline__ float squares(const Raw<16> &r)
{
    constexpr int kV = 16 / E::kSize;
    float v[kV];
    E::to_f32(r, v);
    float even = v[0] * v[0], odd = v[1] * v[1];
#pragma unroll
    for (int j = 2; j < kV; j += 2) {
        even = __fmaf_rn(v[j], v[j], even);
        odd = __fmaf_rn(v[j + 1], v[j + 1], odd);
    }
    return even + odd;
}
// Neither so small that squares may have been lost among the smallest numbers (2^-123 of 2^-76 together, above that) nor too large for fp32, infinite or NaN; those
// are added in 64 bits.
__device__ __forceinline__ bool good_sum(float s) { return s >= 0x1p-76f && s <= 0x1p126f; }
template <typename E>
__device__ __noinline__ double wide_squares(Raw<16> r)
{
    constexpr int kV = 16 / E::kSize;
    float v[kV];
    E::to_f32(r, v);
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kV; ++j) sum += (double)v[j] * v[j];
    return sum;
}

// A piece on its way: its tensor, its place there, this thread's vectors if they are all the tensor's.
struct Flight {
    int t;
    unsigned k;
    bool whole;
    Raw<16> r[kFlight];
};
// The block's pieces, every gridDim.x-th one, the next one's vectors on their way while use() has one's: two flights in turn, since a copy of what is on its way would
// wait for it.
template <typename F, typename G>
__device__ __forceinline__ void two_ahead(unsigned pieces, F &&fetch, G &&use)
{
    Flight f, g;
    unsigned p = blockIdx.x;
    if (p < pieces) fetch(p, f);
    while (p < pieces) {
        const unsigned q = p + gridDim.x;
        if (q < pieces) fetch(q, g);
        use(f);
        if (q >= pieces) break;
        p = q + gridDim.x;
        if (p < pieces) fetch(p, f);
        use(g);
    }
}

// This thread's vectors of piece `k` of tensor `t`, if they are all the tensor's.
template <int kTensors>
__device__ __forceinline__ bool fetch_piece(const GradBatch<kTensors> &b, int t, unsigned k, Raw<16> (&r)[kFlight])
{
    const int shift = b.tensor[t].dtype == EOQ_F32 ? 2 : 1;
    const char *p = reinterpret_cast<const char *>(b.tensor[t].in);
    constexpr long long kBytes = kFlight * kThreads * 16;
    const long long begin = (long long)k * kBytes - (long long)(reinterpret_cast<uintptr_t>(p) % 128);   // (of the piece, in bytes)
    if (begin < 0 || begin + kBytes > (long long)b.tensor[t].size << shift) return false;
#pragma unroll
    for (int u = 0; u < kFlight; ++u) r[u] = *reinterpret_cast<const Raw<16> *>(p + begin + (u * kThreads + threadIdx.x) * 16);
    return true;
}
// Of a piece that is not: f(vector, bytes from `p` to it) for those whose elements are, g(element) for the elements of the others.
template <typename E, typename F, typename G>
__device__ __forceinline__ void piece_ends(const char *p, unsigned long long n, unsigned skew, unsigned k, F &&f, G &&g)
{
    constexpr int kV = 16 / E::kSize;
    const long long begin = (long long)k * kFlight * kThreads * kV - skew;   // (of the piece, in elements)
#pragma unroll 1
    for (int u = 0; u < kFlight; ++u) {
        const long long e = begin + (long long)(u * kThreads + threadIdx.x) * kV;
        if (e >= 0 && e + kV <= (long long)n) f(*reinterpret_cast<const Raw<16> *>(p + e * E::kSize), e * E::kSize);
        else
            for (long long i = e < 0 ? 0 : e; i < e + kV && i < (long long)n; ++i) g(i);
    }
}

// root of the sum of the blocks' sums, in every thread
__device__ __forceinline__ double whole_norm(const double *sums, int blocks)
{
    double v[4] = {};
    for (int i = threadIdx.x; i < blocks; i += 4 * kThreads)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kThreads < blocks) v[u] += __ldcg(sums + i + u * kThreads);
    return sqrt(block_sum((v[0] + v[1]) + (v[2] + v[3])));
}
// whether an fp32 number holds the norm, which is rounded to it
__device__ __forceinline__ bool holds(double whole) { return __double2float_rn(whole) <= 3.4028234663852886e38f; }
__device__ __forceinline__ void write_norm(double whole, float *norm, DeviceState *dev)
{
    if (threadIdx.x != 0) return;
    *norm = __double2float_rn(whole);
    if (!holds(whole)) atomicOr(&dev->status, EOQ_DEV_NONFINITE);
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads, 4) grad_squares_kernel(const __grid_constant__ GradBatch<kTensors> b, const GradSums s)
{
    __shared__ bool last_s;
    ptx::grid_dep_wait_launch_small();
    double sum = 0.0;
    two_ahead(b.pieces, [&](unsigned p, Flight &f) {
        f.t = tensor_of(b, p);
        f.k = p - b.tensor[f.t].first;
        f.whole = fetch_piece(b, f.t, f.k, f.r);
    }, [&](const Flight &f) {
        const int t = f.t;
        const unsigned k = f.k;
        const bool whole = f.whole;
        const Raw<16> (&r)[kFlight] = f.r;
        with_type(b.tensor[t].dtype, [&](auto type) {
            using E = decltype(type);
            if (whole) {
                float q[kFlight];
                bool good = true;
#pragma unroll
                for (int u = 0; u < kFlight; ++u) good = good_sum(q[u] = squares<E>(r[u])) && good;
                if (good) {
                    sum += ((double)q[0] + (double)q[1]) + ((double)q[2] + (double)q[3]);
                } else {
#pragma unroll
                    for (int u = 0; u < kFlight; ++u)
                        if ((r[u].w.x | r[u].w.y | r[u].w.z | r[u].w.w) != 0) sum += wide_squares<E>(r[u]);
                }
            } else {
                const char *src = reinterpret_cast<const char *>(b.tensor[t].in);
                piece_ends<E>(
                    src, b.tensor[t].size, skew_of(src, b.tensor[t].dtype), k,
                    [&](const Raw<16> &v, long long) {
                        const float q = squares<E>(v);
                        if (good_sum(q)) sum += (double)q;
                        else if ((v.w.x | v.w.y | v.w.z | v.w.w) != 0) sum += wide_squares<E>(v);
                    },
                    [&](long long i) {
                        float v[1];
                        E::to_f32(load_raw<E::kSize>(src + i * E::kSize), v);
                        sum += (double)v[0] * v[0];
                    });
            }
        });
    });
    const double own = block_sum(sum);
    if (threadIdx.x == 0) {
        s.sums[s.before + blockIdx.x] = own;
        __threadfence();
        last_s = s.last && atomicInc(&s.dev->ticket, gridDim.x - 1) == gridDim.x - 1;   // (back to zero by itself)
    }
    __syncthreads();
    if (!last_s) return;
    __threadfence();
    write_norm(whole_norm(s.sums, s.before + gridDim.x), s.norm, s.dev);
}

// A block's pieces last to first: what the norm read last is still in the L2.
template <int kTensors>
__global__ void __launch_bounds__(kThreads, 4) grad_scale_kernel(const __grid_constant__ GradBatch<kTensors> b, const GradSums s, float max_norm)
{
    ptx::grid_dep_wait_launch_small();
    const double whole = whole_norm(s.sums, s.before);
    if (blockIdx.x == 0 && s.last) write_norm(whole, s.norm, s.dev);
    const float scale = holds(whole) && whole > max_norm ? (float)(max_norm / whole) : 1.0f;
    two_ahead(b.pieces, [&](unsigned back, Flight &f) {
        const unsigned p = b.pieces - 1 - back;
        f.t = tensor_of(b, p);
        f.k = p - b.tensor[f.t].first;
        f.whole = (b.tensor[f.t].in != b.tensor[f.t].out || scale != 1.0f) && fetch_piece(b, f.t, f.k, f.r);
    }, [&](const Flight &f) {
        const int t = f.t;
        const unsigned k = f.k;
        const bool all = f.whole;
        const Raw<16> (&r)[kFlight] = f.r;
        if (b.tensor[t].in == b.tensor[t].out && scale == 1.0f) return;
        with_type(b.tensor[t].dtype, [&](auto type) {
            using E = decltype(type);
            constexpr int kV = 16 / E::kSize;
            const char *src = reinterpret_cast<const char *>(b.tensor[t].in);
            char *dst = reinterpret_cast<char *>(b.tensor[t].out);
            const unsigned skew = skew_of(src, b.tensor[t].dtype);
            const bool together = (reinterpret_cast<uintptr_t>(src) - reinterpret_cast<uintptr_t>(dst)) % 16 == 0;
            auto put = [&](const Raw<16> &in, long long at) {
                float v[kV];
                E::to_f32(in, v);
#pragma unroll
                for (int j = 0; j < kV; ++j) v[j] *= scale;
                if (together) {
                    store_raw(dst + at, E::from_f32(v));
                } else {
#pragma unroll
                    for (int j = 0; j < kV; ++j) {
                        const float one[1] = {v[j]};
                        store_raw(dst + at + j * E::kSize, E::from_f32(one));
                    }
                }
            };
            if (all) {
                const long long begin = (long long)k * kFlight * kThreads * 16 - (long long)(skew * E::kSize);
#pragma unroll
                for (int u = 0; u < kFlight; ++u) put(r[u], begin + (u * kThreads + threadIdx.x) * 16);
            } else {
                piece_ends<E>(src, b.tensor[t].size, skew, k, put, [&](long long i) {
                    float v[1];
                    E::to_f32(*reinterpret_cast<const Raw<E::kSize> *>(src + i * E::kSize), v);
                    v[0] *= scale;
                    store_raw(dst + i * E::kSize, E::from_f32(v));
                });
            }
        });
    });
}

// tensors [first, first + kTensors) as a launch takes them, those without elements left out; the blocks it takes
template <int kTensors>
unsigned batch_of(const GradList &l, int first, unsigned most, GradBatch<kTensors> &b)
{
    b.num = 0;
    b.pieces = 0;
    for (int i = first; i < l.num && i < first + kTensors; ++i) {
        if (l.size[i] == 0) continue;
        b.tensor[b.num].in = l.in[i];
        b.tensor[b.num].out = l.out ? l.out[i] : const_cast<void *>(l.in[i]);
        b.tensor[b.num].size = l.size[i];
        b.tensor[b.num].dtype = l.dtype[i];
        b.tensor[b.num].first = b.pieces;
        b.pieces += (unsigned)((l.size[i] + skew_of(l.in[i], l.dtype[i]) + piece_of(l.dtype[i]) - 1) / piece_of(l.dtype[i]));
        ++b.num;
    }
    b.shift = 0;
    while (b.pieces >> b.shift >= kRanges) ++b.shift;
    for (unsigned r = 0, t = 0; r << b.shift < b.pieces; ++r) {
        while ((int)t + 1 < b.num && b.tensor[t + 1].first <= r << b.shift) ++t;
        b.start[r] = (uint16_t)t;
    }
    return b.pieces == 0 ? 1 : b.pieces < most ? b.pieces : most;   // (a launch without elements has a block that adds nothing)
}

template <int kTensors>
cudaError_t launch(const GradList &l, bool clip, float max_norm, float *norm, double *sums, DeviceState *dev, int *launches, cudaStream_t st)
{
    GradBatch<kTensors> b;
    GradSums s = {sums, 0, false, norm, dev};
    for (int first = 0; first < l.num; first += kTensors) {
        const unsigned grid = batch_of(l, first, kAddBlocks, b);
        s.last = !clip && l.num - first <= kTensors;
        ++*launches;
        const cudaError_t e = launch_chained(grad_squares_kernel<kTensors>, dim3(grid), dim3(kThreads), 0, st, b, s);
        if (e != cudaSuccess) return e;
        s.before += (int)grid;
    }
    if (!clip) return cudaSuccess;
    for (int first = (l.num - 1) / kTensors * kTensors; first >= 0; first -= kTensors) {
        const unsigned grid = batch_of(l, first, kScaleBlocks, b);
        s.last = first == 0;   // (of several launches the last one writes the norm)
        if (b.pieces == 0 && !s.last) continue;
        ++*launches;
        const cudaError_t e = launch_chained(grad_scale_kernel<kTensors>, dim3(grid), dim3(kThreads), 0, st, b, s, max_norm);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

size_t grad_workspace_bytes(int num) { return sizeof(double) * kAddBlocks * (((size_t)num + kMostTensors - 1) / kMostTensors); }

// (a launch's parameters are copied with it: short lists take the small form)
cudaError_t launch_grad(const GradList &l, bool clip, float max_norm, float *norm, void *workspace, DeviceState *dev, int *launches, cudaStream_t st)
{
    double *sums = reinterpret_cast<double *>(workspace);
    if (l.num <= kFewTensors) return launch<kFewTensors>(l, clip, max_norm, norm, sums, dev, launches, st);
    return launch<kMostTensors>(l, clip, max_norm, norm, sums, dev, launches, st);
}

}  // namespace eoq
