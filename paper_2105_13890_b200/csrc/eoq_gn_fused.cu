// Group normalisation forward, every element read once (eoq_gn_fwd): see eoq_gn_fused.cuh for how the data stays on the chip.
// Mean and squares about it come from two looks at the kept vectors, joined as (count, mean, squares), so a mean far from zero costs
// no digits and a group of equal values has exactly that value as its mean.
#include "eoq_gn_fused.cuh"

namespace eoq {

namespace {

// shared memory behind the vectors: cells of the threads, (mean, squares) of the block's groups, (mean, rstd), gamma, beta
template <int kV, bool kUni>
struct FwdLayout {
    static constexpr int kCells = kGnThreads * (kUni ? 1 : kV);
    // (a group has at least one channel)
    __host__ __device__ static size_t bytes(int cv) { return sizeof(float2) * (kCells + 3 * (size_t)cv * kV); }
};

template <int kType, int kV, bool kUni, bool kSave>
__global__ void __launch_bounds__(kGnThreads, 4) gn_fused_fwd_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    constexpr int kE = Elem<kType>::kSize, kB = kV * kE, kLanes = kBlock8 / kV, kG = kUni ? 1 : kV;
    extern __shared__ __align__(16) uint8_t smem[];
    const OwnVectors<kB> own(smem);
    const int width = a.cv * kV;   // channels of a chunk
    float2 *cell = reinterpret_cast<float2 *>(smem + (size_t)a.vecs * kGnThreads * kB);
    float2 *mine = cell + FwdLayout<kV, kUni>::kCells, *final = mine + width;
    float *gamma = reinterpret_cast<float *>(final + width), *beta = gamma + width;

    const int rank = blockIdx.x % a.ranks, id = blockIdx.x / a.ranks, chunk = id % a.chunks, smp = id / a.chunks;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch0 = chunk * width, ch = ch0 + cv * kV;
    const int per = (a.hw + a.ranks - 1) / a.ranks, p_begin = min(rank * per, a.hw), pixels = min(a.hw, p_begin + per) - p_begin;
    const int channels = min(width, a.c - ch0), groups = channels / a.cpg;
    const int vecs = slot < a.slots && ch < a.c && slot < pixels ? (pixels - slot + a.slots - 1) / a.slots : 0;   // of this thread
    const size_t pix0 = (size_t)smp * a.hw + p_begin + slot;

    ptx::grid_dep_wait_launch_small();
    own.fetch(vecs, [&](int i) { return reinterpret_cast<const char *>(a.x) + ((pix0 + (size_t)i * a.slots) * a.x_stride + ch) * kE; });
    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        gamma[k] = a.gamma ? __ldg(a.gamma + ch0 + k) : 1.0f;
        beta[k] = a.beta ? __ldg(a.beta + ch0 + k) : 0.0f;
    }
    copy_wait();

    // ---- the thread's vectors: mean about the first value, squares about the mean
    {
        float first[kG], s[kG], q[kG];
#pragma unroll
        for (int j = 0; j < kG; ++j) first[j] = s[j] = q[j] = 0.0f;
        if (vecs > 0) {
            float v[kV];
            x_values<kType, kV>(own.get(0), a.x_scale, v);
#pragma unroll
            for (int j = 0; j < kG; ++j) first[j] = v[j];
#pragma unroll 4
            for (int i = 0; i < vecs; ++i) {
                x_values<kType, kV>(own.get(i), a.x_scale, v);
#pragma unroll
                for (int j = 0; j < kV; ++j) s[kUni ? 0 : j] += v[j] - first[kUni ? 0 : j];
            }
            const float per_value = 1.0f / (float)(kUni ? vecs * kV : vecs);
#pragma unroll
            for (int j = 0; j < kG; ++j) s[j] = __fmaf_rn(s[j], per_value, first[j]);
#pragma unroll 4
            for (int i = 0; i < vecs; ++i) {
                x_values<kType, kV>(own.get(i), a.x_scale, v);
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    const float d = v[j] - s[kUni ? 0 : j];
                    q[kUni ? 0 : j] = __fmaf_rn(d, d, q[kUni ? 0 : j]);
                }
            }
        }
        if (slot < a.slots)
#pragma unroll
            for (int j = 0; j < kG; ++j) cell[(slot * a.cv + cv) * kG + j] = make_float2(s[j], q[j]);
    }
    __syncthreads();

    // ---- a warp per group joins the block's cells
    const int per_group = kUni ? a.cpg / kV : a.cpg, row = a.cv * kG, used = min(a.slots, pixels);   // (cells of a group in a slot, of a slot)
    const int full = pixels / a.slots, more = pixels % a.slots;
    const int lane = threadIdx.x & 31;
    for (int g = threadIdx.x / 32; g < groups; g += kGnWarps) {
        const float2 *src = cell + g * per_group;
        const float first = src[0].x;
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < used * per_group; i += 32) {
            const int j = i / per_group;
            s = __fmaf_rn(src[j * row + i - j * per_group].x - first, (float)(full + (j < more)), s);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s = pixels ? first + s / ((float)pixels * (float)per_group) : 0.0f;
        constexpr float kValues = kUni ? (float)kV : 1.0f;   // values a pixel adds to a cell
        for (int i = lane; i < used * per_group; i += 32) {
            const int j = i / per_group;
            const float2 e = src[j * row + i - j * per_group];
            q += __fmaf_rn((e.x - s) * (e.x - s), kValues * (float)(full + (j < more)), e.y);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
        if (lane == 0) mine[g] = make_float2(s, q);
    }
    if (a.ranks > 1) ptx::cluster_sync();
    else __syncthreads();

    // ---- the blocks of the sample; every one joins them for itself
    for (int g = threadIdx.x; g < groups; g += kGnThreads) {
        const uint32_t at = ptx::smem_u32(mine + g);
        auto part = [&](int r) { return a.ranks > 1 ? ld_cluster_f2(ptx::cluster_addr(at, (uint32_t)r)) : mine[g]; };
        auto count = [&](int r) { return (float)(min(a.hw, (r + 1) * per) - min(a.hw, r * per)); };
        const float first = part(0).x;
        float s = 0.0f, q = 0.0f;
        for (int r = 1; r < a.ranks; ++r) s = __fmaf_rn(count(r) > 0.0f ? part(r).x - first : 0.0f, count(r), s);
        s = first + s / (float)a.hw;
        for (int r = 0; r < a.ranks; ++r) {
            const float2 e = part(r);
            if (count(r) > 0.0f) q += __fmaf_rn((e.x - s) * (e.x - s), count(r) * (float)a.cpg, e.y);
        }
        const float rstd = (float)(1.0 / sqrt((double)q / ((double)a.hw * a.cpg) + (double)a.eps));
        final[g] = make_float2(s, rstd);
        if (rank == 0 && a.stats) a.stats[(size_t)smp * a.groups + ch0 / a.cpg + g] = make_float2(s, rstd);
    }
    __syncthreads();
    if (a.ranks > 1) ptx::cluster_arrive();   // (this block has read what it needs of the others)

    // ---- y, and the 8-bit form
    float mul[kV], add[kV], mean[kG];
#pragma unroll
    for (int j = 0; j < kV; ++j) {
        const bool in = ch + j < a.c && slot < a.slots;
        const float2 st = in ? final[(cv * kV + j) / a.cpg] : make_float2(0.0f, 0.0f);
        if (j < kG) mean[j] = st.x;
        mul[j] = in ? st.y * gamma[cv * kV + j] : 0.0f;
        add[j] = in ? beta[cv * kV + j] : 0.0f;
    }
    unsigned bad = 0;
    const int rounds = kSave ? a.vecs : vecs;   // (lanes that share a block of the 8-bit form stay together)
#pragma unroll 2
    for (int i = 0; i < rounds; ++i) {
        const bool in = !kSave || i < vecs;
        const size_t pix = pix0 + (size_t)i * a.slots;
        float v[kV];
        x_values<kType, kV>(in ? own.get(i) : zero_raw<kB>(), a.x_scale, v);
        if constexpr (kSave) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < kV; ++j) m = max_abs(m, v[j]);
            m = lanes_max_abs<kLanes>(m);
            const int s = block_exp(m);
            uint32_t w[(kV + 3) / 4];
            block_codes(v, s, w);
            if (in) {
                Raw<kV> out;
#pragma unroll
                for (int j = 0; j < (kV + 3) / 4; ++j) set_word(out, j, w[j]);
                store_raw(a.codes_out + pix * a.c + ch, out);
                if (ch % kBlock8 == 0) a.exps_out[pix * a.blocks + ch / kBlock8] = (uint8_t)s;
                bad |= s == 255;
            }
        }
        if (in) {
#pragma unroll
            for (int j = 0; j < kV; ++j) v[j] = __fmaf_rn(v[j] - mean[kUni ? 0 : j], mul[j], add[j]);
            activate(v, a.act);
            store_raw(reinterpret_cast<char *>(a.y) + (pix * a.y_stride + ch) * Elem<Types::kY>::kSize, Elem<Types::kY>::from_f32(v));
        }
    }
    if (kSave && bad) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
    if (a.ranks > 1) ptx::cluster_wait();
}

template <int kType, int kV, bool kUni, bool kSave>
cudaError_t launch(GnArgs a, const FusedPlan &p, cudaStream_t st)
{
    static std::atomic<unsigned long long> allowed;
    const auto kernel = gn_fused_fwd_kernel<kType, kV, kUni, kSave>;
    const cudaError_t e = allow_fused((const void *)kernel, allowed);
    if (e != cudaSuccess) return e;
    a.cv = p.cv;
    a.slots = p.slots;
    a.chunks = p.chunks;
    a.ranks = p.ranks;
    a.vecs = p.vecs;
    return launch_chained_clusters(p.ranks, kernel, dim3((unsigned)((size_t)a.n * p.chunks * p.ranks)), dim3(kGnThreads), p.smem, st, a);
}

template <int kType, int kV>
bool of_width(const GnArgs &a, cudaError_t *result, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize;
    const bool uni = a.cpg % kV == 0, save = a.codes_out != nullptr && a.c % kBlock8 == 0;
    int unit = a.cpg / gcd_of(a.cpg, kV) * kV;
    if (save) unit = unit / gcd_of(unit, kBlock8) * kBlock8;
    FusedPlan p;
    if (!fused_plan(p, a.n, a.hw, a.c, kV, unit, kV * kE, kV * kE,
                    [&](int cv) { return uni ? FwdLayout<kV, true>::bytes(cv) : FwdLayout<kV, false>::bytes(cv); }) ||
        (size_t)a.n * p.chunks * p.ranks > 0x7fffffffull)
        return false;
    if (kV == 1 || uni) *result = save ? launch<kType, kV, true, true>(a, p, st) : launch<kType, kV, true, false>(a, p, st);
    else if constexpr (kV > 1) *result = save ? launch<kType, kV, false, true>(a, p, st) : launch<kType, kV, false, false>(a, p, st);
    return true;
}

template <int kType>
bool of_type(const GnArgs &a, cudaError_t *result, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kY = Elem<GnTypes<kType>::kY>::kSize;
    auto of = [&](int v) {
        return a.c % v == 0 && a.x_stride % v == 0 && a.y_stride % v == 0 && aligned_at(a.x, v * kE) && aligned_at(a.y, v * kY) && aligned_at(a.codes_out, v);
    };
    if (of(GnTypes<kType>::kWide)) return of_width<kType, GnTypes<kType>::kWide>(a, result, st);
    if (of(2)) return of_width<kType, 2>(a, result, st);
    return of_width<kType, 1>(a, result, st);
}

}  // namespace

bool gn_fused_fwd(GnArgs a, int dtype, cudaError_t *result, int *launches, cudaStream_t st)
{
    bool done;
    switch (dtype) {
        case EOQ_F32: done = of_type<EOQ_F32>(a, result, st); break;
        case EOQ_F16: done = of_type<EOQ_F16>(a, result, st); break;
        case EOQ_BF16: done = of_type<EOQ_BF16>(a, result, st); break;
        default: done = of_type<EOQ_I32>(a, result, st); break;
    }
    if (!done) return false;
    ++*launches;
    if (*result == cudaSuccess && a.codes_out && a.c % kBlock8) {   // a row of blocks that ends inside one
        ++*launches;
        *result = launch_ckpt_save(a.x, dtype, a.x_exp, (size_t)a.n * a.hw, a.c, a.x_stride, a.codes_out, a.exps_out, a.dev, a.sm_count, st);
    }
    return true;
}

}  // namespace eoq
