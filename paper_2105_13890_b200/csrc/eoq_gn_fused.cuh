// Group normalisation in one launch: what its forward and backward kernels share.
//
// A sample's chunk of whole groups belongs to a cluster, dealt out by pixels to its blocks.  The blocks read their pixels once for the
// sums, which meet in shared memory and, over the cluster, in distributed shared memory, and look at them once more for the results.
// Between the two looks the vectors stay in shared memory where that leaves room for four blocks on an SM, forward also where it leaves
// room for two; larger samples are read again, from the L2 cache as far as what the resident clusters work on has room there.  (256
// channels 56 x 56, 32 fp16 samples: 25 us kept, 30 read again; 64 channels 112 x 112, 64 bf16 samples: kept in 104 KB by two blocks an
// SM 72 us forward and 209 backward, read again 83 and 110.  Samples that do not fit go to eight blocks whether or not the SMs need as many.)
#pragma once
#include "eoq_gn.cuh"

namespace eoq {

constexpr int kGnThreads = 256, kGnWarps = kGnThreads / 32;
constexpr int kGnBatch = 4;   // vectors of a thread at a time

// to the same place in shared memory of block `rank` of the cluster
__device__ __forceinline__ void st_cluster_f2(const float2 *at, int rank, float2 v)
{
    const uint32_t to = ptx::cluster_addr(ptx::smem_u32(at), (uint32_t)rank);
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
}
template <int kBytes>
__device__ __forceinline__ void copy_in(uint32_t smem, const void *src)
{
    static_assert(kBytes >= 4, "asynchronous copies have 4, 8 or 16 bytes");
    if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A thread's vectors of a tensor, `step` bytes apart from `at` on; kept: vector i at base[i * kGnThreads] of shared memory, where the
// thread only ever reads back what it copied itself, so that no barrier is needed.
template <int kBytes, bool kKeep>
struct Vectors {
    using Word = decltype(Raw<kBytes>::w);
    const char *at;
    size_t step;
    Word *base;
    __device__ __forceinline__ Vectors(const void *from, size_t step_, void *smem)
        : at(reinterpret_cast<const char *>(from)), step(step_), base(reinterpret_cast<Word *>(smem) + threadIdx.x)
    {
    }
    __device__ __forceinline__ void fetch(int count) const
    {
        if constexpr (kKeep) {
            const char *p = at;
            if constexpr (kBytes >= 4) {
                uint32_t to = ptx::smem_u32(base);
#pragma unroll 4
                for (int i = 0; i < count; ++i, p += step, to += kGnThreads * kBytes) copy_in<kBytes>(to, p);
            } else {
                constexpr int kMany = 8;
                for (int i0 = 0; i0 < count; i0 += kMany, p += kMany * step) {
                    Raw<kBytes> r[kMany];
#pragma unroll
                    for (int j = 0; j < kMany; ++j)
                        if (i0 + j < count) r[j] = load_raw<kBytes>(p + j * step);
#pragma unroll
                    for (int j = 0; j < kMany; ++j)
                        if (i0 + j < count) base[(i0 + j) * kGnThreads] = r[j].w;
                }
            }
        }
    }
    // vectors i, i + 1, ... of which `p` (vectors_at(0), moved on by next) is the first's address
    __device__ __forceinline__ const char *first() const { return at; }
    template <int kCount>
    __device__ __forceinline__ void get(Raw<kBytes> (&r)[kCount], int i, const char *&p) const
    {
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            if constexpr (kKeep) r[u].w = base[(i + u) * kGnThreads];
            else r[u] = load_raw<kBytes>(p + u * step);
        }
        if constexpr (!kKeep) p += kCount * step;
    }
};

// How a call is dealt out.
struct FusedPlan {
    int cv, slots, chunks, ranks, vecs;
    bool keep;
    size_t smem;
};

// v: channels of a vector, x_bytes long; unit: channels that must stay together (a multiple of v); kept: bytes of a vector in shared
// memory, as long as a block needs no more than `limit`; fixed(cv): further bytes of it.
template <typename Fixed>
bool fused_plan(FusedPlan &p, int n, int hw, int c, int v, int unit, int x_bytes, int kept, size_t limit, Fixed fixed)
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
    p.ranks = 1;
    // (more blocks to a sample while the vectors do not fit, and while there are few and every thread has more than two)
    auto vecs = [&] { return p.vecs = ((hw + p.ranks - 1) / p.ranks + p.slots - 1) / p.slots; };
    auto size = [&] { return (size_t)vecs() * kGnThreads * kept + fixed(p.cv); };
    while (p.ranks < 8 && (size() > limit || (vecs() > 2 && (long long)n * p.chunks * p.ranks < 2 * kPartSms))) p.ranks *= 2;
    p.keep = size() <= limit;
    p.smem = p.keep ? size() : fixed(p.cv);
    if (p.smem > 200 * 1024) return false;
    // (divisions by multiplication: dividend times divisor below 2^32)
    return (size_t)n * p.chunks * p.ranks < (1ull << 32) / (p.chunks > 8 ? p.chunks : 8) && (size_t)p.slots * hw < (1ull << 32);
}

inline void use_plan(GnArgs &a, const FusedPlan &p, int kw)
{
    a.cv = p.cv;
    a.slots = p.slots;
    a.chunks = p.chunks;
    a.ranks = p.ranks;
    a.vecs = p.vecs;
    a.per = (a.hw + p.ranks - 1) / p.ranks;
    a.run = run_of(p.vecs);
    a.by_slots = FastDiv(p.slots);
    a.by_chunks = FastDiv(p.chunks);
    a.by_ranks = FastDiv(p.ranks);
    a.by_cv = FastDiv(p.cv);
    a.by_cpg = FastDiv(a.cpg);
    a.by_part = FastDiv(a.cpg / kw);
}

inline int gcd_of(int a, int b) { return b ? gcd_of(b, a % b) : a; }

}  // namespace eoq
