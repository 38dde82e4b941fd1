// Group normalisation backward, every element read once (eoq_gn_bwd): see eoq_gn_fused.cuh for how the data stays on the chip, and
// eoq_gn.cu for the formulas.  The first look at the kept vectors sums dz and dz u per channel, which is all that S1, S2, dgamma and
// dbeta need; the second writes dx.  When all samples of a chunk fit a cluster it also adds dgamma and dbeta over them, and the call is
// one launch; otherwise a small kernel behind adds the samples in their order.
#include "eoq_gn_fused.cuh"

namespace eoq {

namespace {

// shared memory behind the vectors: cells of the threads, rows of sums by warp, sums of the block, of the sample, (S1, S2), gamma
template <int kV>
struct BwdLayout {
    __host__ __device__ static size_t bytes(int cv)
    {
        const int slots = kGnThreads / cv, width = cv * kV;
        return sizeof(float2) * ((size_t)kGnThreads * kV + (size_t)(slots < kGnWarps ? slots : kGnWarps) * width + (size_t)width * 7 / 2);
    }
};

template <int kType, int kV, bool kUni, bool kCodes>
__global__ void __launch_bounds__(kGnThreads, 2) gn_fused_bwd_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    using Input = GnInput<kType, kV, kCodes, kUni>;
    constexpr int kE = Elem<kType>::kSize, kDyE = Elem<Types::kY>::kSize, kG = kUni ? 1 : kV;
    extern __shared__ __align__(16) uint8_t smem[];
    const size_t all = (size_t)a.vecs * kGnThreads;
    const OwnVectors<Input::kDyB> own_dy(smem);
    const OwnVectors<Input::kXB> own_x(smem + all * Input::kDyB);
    uint8_t *own_s = smem + all * (Input::kDyB + Input::kXB) + threadIdx.x;
    const int width = a.cv * kV, rows = min(a.slots, kGnWarps);
    float2 *cell = reinterpret_cast<float2 *>(smem + all * (Input::kDyB + Input::kXB + (kCodes ? 1 : 0)));
    float2 *by_warp = cell + kGnThreads * kV, *mine = by_warp + rows * width, *total = mine + width, *means = total + width;
    float *gamma_s = reinterpret_cast<float *>(means + width);

    const int rank = blockIdx.x % a.cluster, id = blockIdx.x / a.cluster, chunk = id % a.chunks, samples = a.cluster / a.ranks;
    const int smp = id / a.chunks * samples + rank / a.ranks, part = rank % a.ranks;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch0 = chunk * width, ch = ch0 + cv * kV;
    const int per = (a.hw + a.ranks - 1) / a.ranks, p_begin = min(part * per, a.hw), pixels = min(a.hw, p_begin + per) - p_begin;
    const int channels = min(width, a.c - ch0), groups = channels / a.cpg;
    const bool active = slot < a.slots && ch < a.c;
    const int vecs = active && slot < pixels ? (pixels - slot + a.slots - 1) / a.slots : 0;
    const size_t pix0 = (size_t)smp * a.hw + p_begin + slot;

    ptx::grid_dep_wait_launch_small();
    own_dy.fetch(vecs, [&](int i) { return reinterpret_cast<const char *>(a.dy) + ((pix0 + (size_t)i * a.slots) * a.dy_stride + ch) * kDyE; });
    if constexpr (kCodes) {
        own_x.fetch(vecs, [&](int i) { return a.codes + (pix0 + (size_t)i * a.slots) * a.c + ch; });
        OwnVectors<1> bytes(own_s - threadIdx.x);
        bytes.fetch(vecs, [&](int i) { return a.exps + (pix0 + (size_t)i * a.slots) * a.blocks + ch / kBlock8; });
    } else {
        own_x.fetch(vecs, [&](int i) { return reinterpret_cast<const char *>(a.x) + ((pix0 + (size_t)i * a.slots) * a.x_stride + ch) * kE; });
    }
    float gamma[kV], beta[kV], mean[kG], rstd[kG];
#pragma unroll
    for (int j = 0; j < kV; ++j) {
        gamma[j] = active && a.gamma ? __ldg(a.gamma + ch + j) : 1.0f;
        beta[j] = active && a.beta ? __ldg(a.beta + ch + j) : 0.0f;
        if (j < kG) {
            const float2 st = active ? a.stats[(size_t)smp * a.groups + (ch + j) / a.cpg] : make_float2(0.0f, 0.0f);
            mean[j] = st.x;
            rstd[j] = st.y;
        }
    }
    for (int k = threadIdx.x; k < channels; k += kGnThreads) gamma_s[k] = a.gamma ? __ldg(a.gamma + ch0 + k) : 1.0f;
    const float dy_scale = error_scale<kType>(a);
    copy_wait();

    {
        float s0[kV], s1[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) s0[j] = s1[j] = 0.0f;
#pragma unroll 2
        for (int i = 0; i < vecs; ++i) {
            float u[kV], dz[kV];
            gn_terms<kType, kV, kCodes, kUni>(own_x.get(i), kCodes ? own_s[i * kGnThreads] : 0, own_dy.get(i), a.x_scale, dy_scale, a.act, mean, rstd,
                                              gamma, beta, u, dz);
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                s0[j] += dz[j];
                s1[j] = __fmaf_rn(dz[j], u[j], s1[j]);
            }
        }
        if (slot < a.slots)
#pragma unroll
            for (int j = 0; j < kV; ++j) cell[(slot * a.cv + cv) * kV + j] = make_float2(s0[j], s1[j]);
    }
    __syncthreads();
    // channels by lanes, slots by warps; then the warps' rows
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    if (warp < rows)
        for (int k = lane; k < channels; k += 32) {
            float2 t = make_float2(0.0f, 0.0f);
            for (int j = warp; j < a.slots; j += rows) {
                const float2 e = cell[j * width + k];
                t.x += e.x;
                t.y += e.y;
            }
            by_warp[warp * width + k] = t;
        }
    __syncthreads();
    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        float2 t = make_float2(0.0f, 0.0f);
        for (int j = 0; j < rows; ++j) {
            t.x += by_warp[j * width + k].x;
            t.y += by_warp[j * width + k].y;
        }
        mine[k] = t;
    }
    if (a.cluster > 1) ptx::cluster_sync();
    else __syncthreads();

    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        const uint32_t at = ptx::smem_u32(mine + k);
        auto add = [&](float2 &t, int r) {
            const float2 e = a.cluster > 1 ? ld_cluster_f2(ptx::cluster_addr(at, (uint32_t)r)) : mine[k];
            t.x += e.x;
            t.y += e.y;
        };
        float2 t = make_float2(0.0f, 0.0f);
        for (int r = 0; r < a.ranks; ++r) add(t, rank - part + r);
        total[k] = t;
        if (samples == a.n) {   // the cluster has every sample
            if (rank == 0) {
                for (int r = a.ranks; r < a.cluster; ++r) add(t, r);
                if (a.dbeta) a.dbeta[ch0 + k] = t.x;
                if (a.dgamma) a.dgamma[ch0 + k] = t.y;
            }
        } else if (part == 0) {
            a.part[(size_t)smp * a.c + ch0 + k] = t;
        }
    }
    __syncthreads();
    if (a.cluster > 1) ptx::cluster_arrive();   // (this block has read what it needs of the others)
    const float inv = (float)(1.0 / ((double)a.hw * a.cpg));
    for (int g = warp; g < groups; g += kGnWarps) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int i = lane; i < a.cpg; i += 32) {
            const float2 e = total[g * a.cpg + i];
            s0 = __fmaf_rn(gamma_s[g * a.cpg + i], e.x, s0);
            s1 = __fmaf_rn(gamma_s[g * a.cpg + i], e.y, s1);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            s0 += __shfl_xor_sync(0xffffffffu, s0, d);
            s1 += __shfl_xor_sync(0xffffffffu, s1, d);
        }
        if (lane == 0) means[g] = make_float2(s0 * inv, s1 * inv);
    }
    __syncthreads();
    float k0[kG], k1[kG];
#pragma unroll
    for (int j = 0; j < kG; ++j) {
        const float2 m = active ? means[(cv * kV + j) / a.cpg] : make_float2(0.0f, 0.0f);
        k0[j] = -rstd[j] * m.x;
        k1[j] = -rstd[j] * m.y;
    }
#pragma unroll 2
    for (int i = 0; i < vecs; ++i) {
        float u[kV], dz[kV];
        gn_terms<kType, kV, kCodes, kUni>(own_x.get(i), kCodes ? own_s[i * kGnThreads] : 0, own_dy.get(i), a.x_scale, dy_scale, a.act, mean, rstd, gamma,
                                          beta, u, dz);
#pragma unroll
        for (int j = 0; j < kV; ++j)
            dz[j] = __fmaf_rn(dz[j] * gamma[j], rstd[kUni ? 0 : j], __fmaf_rn(u[j], k1[kUni ? 0 : j], k0[kUni ? 0 : j]));
        store_raw(reinterpret_cast<char *>(a.dx) + ((pix0 + (size_t)i * a.slots) * a.dx_stride + ch) * Elem<Types::kDx>::kSize,
                  Elem<Types::kDx>::from_f32(dz));
    }
    if (a.cluster > 1) ptx::cluster_wait();
}

template <int kType, int kV, bool kUni, bool kCodes>
cudaError_t launch(GnArgs a, const FusedPlan &p, int *launches, cudaStream_t st)
{
    static std::atomic<unsigned long long> allowed;
    const auto kernel = gn_fused_bwd_kernel<kType, kV, kUni, kCodes>;
    cudaError_t e = allow_fused((const void *)kernel, allowed);
    if (e != cudaSuccess) return e;
    a.cv = p.cv;
    a.slots = p.slots;
    a.chunks = p.chunks;
    a.ranks = p.ranks;
    a.vecs = p.vecs;
    const bool together = a.n == 1 || (long long)a.n * p.ranks <= 8;   // all samples of a chunk in one cluster
    a.cluster = together ? a.n * p.ranks : p.ranks;
    e = launch_chained_clusters(a.cluster, kernel, dim3((unsigned)((size_t)a.n * p.chunks * p.ranks)), dim3(kGnThreads), p.smem, st, a);
    ++*launches;
    if (e != cudaSuccess || together || (!a.dgamma && !a.dbeta)) return e;
    ++*launches;
    return launch_gn_channel_sums(a, st);
}

template <int kType, int kV, bool kCodes>
bool of_width(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kDyB = kV * Elem<GnTypes<kType>::kY>::kSize, kXB = kCodes ? kV : kV * kE;
    const int unit = a.cpg / gcd_of(a.cpg, kV) * kV;
    FusedPlan p;
    if (!fused_plan(p, a.n, a.hw, a.c, kV, unit, kDyB + kXB + (kCodes ? 1 : 0), kV * kE, [&](int cv) { return BwdLayout<kV>::bytes(cv); }) ||
        (size_t)a.n * p.chunks * p.ranks > 0x7fffffffull)
        return false;
    if (kV == 1 || a.cpg % kV == 0) *result = launch<kType, kV, true, kCodes>(a, p, launches, st);
    else if constexpr (kV > 1) *result = launch<kType, kV, false, kCodes>(a, p, launches, st);
    return true;
}

template <int kType, bool kCodes>
bool of_source(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kY = Elem<GnTypes<kType>::kY>::kSize, kDx = Elem<GnTypes<kType>::kDx>::kSize;
    auto of = [&](int v) {
        return a.c % v == 0 && a.dy_stride % v == 0 && a.dx_stride % v == 0 && (kCodes || (a.x_stride % v == 0 && aligned_at(a.x, v * kE))) &&
               aligned_at(a.codes, v) && aligned_at(a.dy, v * kY) && aligned_at(a.dx, v * kDx);
    };
    if (of(GnTypes<kType>::kWide)) return of_width<kType, GnTypes<kType>::kWide, kCodes>(a, result, launches, st);
    if (of(2)) return of_width<kType, 2, kCodes>(a, result, launches, st);
    return of_width<kType, 1, kCodes>(a, result, launches, st);
}

template <int kType>
bool of_type(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    return a.codes ? of_source<kType, true>(a, result, launches, st) : of_source<kType, false>(a, result, launches, st);
}

}  // namespace

bool gn_fused_bwd(GnArgs a, int dtype, cudaError_t *result, int *launches, cudaStream_t st)
{
    switch (dtype) {
        case EOQ_F32: return of_type<EOQ_F32>(a, result, launches, st);
        case EOQ_F16: return of_type<EOQ_F16>(a, result, launches, st);
        case EOQ_BF16: return of_type<EOQ_BF16>(a, result, launches, st);
        default: return of_type<EOQ_I32>(a, result, launches, st);
    }
}

}  // namespace eoq
