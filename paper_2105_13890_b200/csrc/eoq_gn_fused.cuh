// Group normalisation that reads every element once: what its forward and backward kernels share.
//
// A sample's chunk of whole groups stays on the chip between the sums and their use, dealt out by pixels to the blocks of a cluster.
// A thread copies its vectors to shared memory (asynchronously where they have 4 bytes or more) and only ever reads back what it
// copied itself, so the data needs no barrier; sums meet in shared memory, and over the cluster through distributed shared memory.
#pragma once
#include "eoq_gn.cuh"

namespace eoq {

constexpr int kGnThreads = 256, kGnWarps = kGnThreads / 32;

template <int kBytes>
__device__ __forceinline__ void copy_in(uint32_t smem, const void *src)
{
    static_assert(kBytes >= 4, "asynchronous copies have 4, 8 or 16 bytes");
    if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ float2 ld_cluster_f2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// A thread's vectors of a tensor: element i at base[i * kGnThreads + thread].
template <int kBytes>
struct OwnVectors {
    using Word = decltype(Raw<kBytes>::w);
    Word *base;
    __device__ __forceinline__ explicit OwnVectors(void *smem) : base(reinterpret_cast<Word *>(smem) + threadIdx.x) {}
    __device__ __forceinline__ Raw<kBytes> get(int i) const
    {
        Raw<kBytes> r;
        r.w = base[i * kGnThreads];
        return r;
    }
    // vectors first, first + step, ... of `count`; `at(i)` is their address
    template <typename At>
    __device__ __forceinline__ void fetch(int count, At at) const
    {
        if constexpr (kBytes >= 4) {
            for (int i = 0; i < count; ++i) copy_in<kBytes>(ptx::smem_u32(base + i * kGnThreads), at(i));
        } else {
            constexpr int kBatch = 8;
            for (int i0 = 0; i0 < count; i0 += kBatch) {
                Raw<kBytes> r[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (i0 + j < count) r[j] = load_raw<kBytes>(at(i0 + j));
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (i0 + j < count) base[(i0 + j) * kGnThreads] = r[j].w;
            }
        }
    }
};

// How a call is dealt out.
struct FusedPlan {
    int cv, slots, chunks, ranks, vecs;
    size_t smem;
};

// v: channels of a vector; bytes: what a thread keeps of one; unit: channels that must stay together (a multiple of v); fixed(cv):
// further bytes of shared memory.  Blocks want to share an SM, so that one loads while another stores: the first limit that some
// cluster meets is taken, small blocks before large ones, clusters of up to 8 before 16.
template <typename Fixed>
bool fused_plan(FusedPlan &p, int n, int hw, int c, int v, int unit, int bytes, int x_bytes, Fixed fixed)
{
    const int total = c / v, unit_v = unit / v;
    if (unit_v > kGnThreads) return false;
    const int units = total / unit_v;
    // 64 bytes of a pixel's channels at least, and no more idle threads than small images force
    int m = (64 + x_bytes * unit_v - 1) / (x_bytes * unit_v);
    while (m < units && (long long)m * unit_v * hw < kGnThreads) ++m;
    if (m > units) m = units;
    while (m > 1 && m * unit_v > kGnThreads) --m;
    const int chunks = (units + m - 1) / m;
    m = (units + chunks - 1) / chunks;
    p.cv = m * unit_v;
    p.chunks = (units + m - 1) / m;
    p.slots = kGnThreads / p.cv;
    const size_t rest = fixed(p.cv);
    auto fits = [&](int ranks, size_t limit) {
        const int per = (hw + ranks - 1) / ranks;
        p.ranks = ranks;
        p.vecs = (per + p.slots - 1) / p.slots;
        p.smem = (size_t)p.vecs * kGnThreads * bytes + rest;
        return p.smem <= limit;
    };
    const size_t kQuarter = 54 * 1024, kHalf = 110 * 1024, kWhole = 220 * 1024;
    const struct {
        size_t limit;
        int most;
    } tries[] = {{kQuarter, 8}, {kHalf, 8}, {kQuarter, 16}, {kHalf, 16}, {kWhole, 16}};
    for (const auto &t : tries)
        for (int ranks = 1; ranks <= t.most; ranks *= 2)
            if (fits(ranks, t.limit)) {
                // few blocks: spread them over more SMs as long as every thread has two vectors
                while (ranks < 8 && p.vecs > 2 && (long long)n * p.chunks * ranks < 2 * kPartSms) fits(ranks *= 2, t.limit);
                return true;
            }
    return false;
}

inline int gcd_of(int a, int b) { return b ? gcd_of(b, a % b) : a; }

// Allows a kernel its shared memory and clusters of 16, once per device.
inline cudaError_t allow_fused(const void *kernel, std::atomic<unsigned long long> &done)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = device < 64 ? 1ull << device : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

}  // namespace eoq
