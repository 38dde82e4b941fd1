// Group normalisation forward in one launch (eoq_gn_fwd): see eoq_gn_fused.cuh for how a sample is dealt out.
// Batches of a thread's vectors give their mean and the squares about it; (count, mean, squares) are joined pairwise, so a mean far from
// zero costs no digits, and a group of equal values has exactly that value as its mean.
//
// Where samples are kept, a block reads, joins, then writes, so that reads and writes overlap only between blocks: 256 channels 56 x 56, 32 fp16 samples,
// ReLU: 25 us, 4.1 TB/s in 1,024 blocks for 592 places.  Small calls take the launch and a cluster barrier (512 channels 7 x 7, one
// sample: 3.7 us).  With SiLU and the 8-bit form (64 channels 112 x 112, 64 bf16 samples: 72 us, 3.6 TB/s) issue slots are busy for 44% of the cycles.
// The form that reads again and writes the 8-bit form holds three unrolled batches in 64 registers and spills 300 to 570 bytes a thread of 16-bit
// types (16 samples 150 x 150 x 64: 49 us, of which memory needs 18).
#include <type_traits>

#include "eoq_gn_fused.cuh"

namespace eoq {

namespace {

// shared memory: cells of the threads, (mean, squares) of every block of the cluster, (mean, rstd), gamma, beta
template <int kV, int kW>
struct FwdLayout {
    static constexpr int kCells = kGnThreads * (kV / kW);
    __host__ __device__ static size_t bytes(int cv, int groups) { return sizeof(float2) * (kCells + (8 + 1) * (size_t)groups + (size_t)cv * kV); }
};

// kW: so many neighbouring channels of a vector are always of one group (the common divisor of both widths)
template <int kType, int kV, int kW, bool kSave, bool kKeep>
__global__ void __launch_bounds__(kGnThreads, 4) gn_fused_fwd_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    constexpr int kE = Elem<kType>::kSize, kB = kV * kE, kLanes = kBlock8 / kV, kG = kV / kW;
    extern __shared__ __align__(16) uint8_t smem[];
    const int width = a.cv * kV, most = a.by_cpg(width);   // channels and groups of a chunk (the last one may have fewer)
    float2 *cell = reinterpret_cast<float2 *>(smem + (kKeep ? (size_t)a.vecs * kGnThreads * kB : 0));
    float2 *parts = cell + FwdLayout<kV, kW>::kCells, *final = parts + 8 * most;   // parts [rank][group]
    float *gamma = reinterpret_cast<float *>(final + most), *beta = gamma + width;

    const int id = a.by_ranks(blockIdx.x), rank = blockIdx.x - id * a.ranks, smp = a.by_chunks(id), chunk = id - smp * a.chunks;
    const int slot = a.by_cv(threadIdx.x), cv = threadIdx.x - slot * a.cv, ch0 = chunk * width, ch = ch0 + cv * kV;
    const int per = a.per, p_begin = min(rank * per, a.hw), pixels = min(a.hw, p_begin + per) - p_begin;
    const int channels = min(width, a.c - ch0), groups = a.by_cpg(channels);
    const int full = a.by_slots(pixels), more = pixels - full * a.slots;   // slot j has `full` pixels, the first `more` one more
    const bool active = slot < a.slots && ch < a.c;
    const int vecs = active ? full + (slot < more) : 0;                  // of this thread
    const size_t pix0 = (size_t)smp * a.hw + p_begin + slot;
    const Vectors<kB, kKeep> x(reinterpret_cast<const char *>(a.x) + (pix0 * a.x_stride + ch) * kE, a.slots * a.x_stride * kE, smem);

    if (a.ranks > 1) ptx::cluster_arrive();   // (waited for below: the others have started when their memory is written)
    ptx::grid_dep_wait_launch_small();
    x.fetch(vecs);
    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        gamma[k] = a.gamma ? __ldg(a.gamma + ch0 + k) : 1.0f;
        beta[k] = a.beta ? __ldg(a.beta + ch0 + k) : 0.0f;
    }

    if (kKeep) copy_wait();

    // ---- the thread's vectors
    {
        constexpr int kA = kW == 1 ? kPairs<kV> : kG;   // accumulators: a channel to a lane of a pair, or a group to a pair
        Pair mean[kA], sq[kA];   // of a run of vectors; mean: with its sign turned
        auto acc = [](int i) { return kW == 1 ? i : 2 * i / kW; };   // of pair i of a vector
        // i0: vectors of the run in front of the batch; inv: 1 / values of the batch
        auto batch = [&](const char *&at, int i, int i0, auto count, float inv) {
            constexpr int kCount = decltype(count)::value;
            Raw<kB> raw[kCount];
            float v[kCount][kV];
            Pair s[kA], q[kA], first[kA];
            x.get(raw, i, at);
#pragma unroll
            for (int u = 0; u < kCount; ++u) Elem<kType>::to_f32(raw[u], v[u]);   // (integer sums as they are)
            // (about the first value, so that equal values have themselves as their mean; sums of a few 16-bit values are exact anyway)
            constexpr bool kShift = kE > 2;
#pragma unroll
            for (int j = 0; j < kA; ++j) {
                s[j] = q[j] = both(0.0f);
                first[j] = kW == 1 ? pair_of(v[0], j) * both(-1.0f) : both(-v[0][j * kW]);
            }
#pragma unroll
            for (int u = 0; u < kCount; ++u)
#pragma unroll
                for (int j = 0; j < kPairs<kV>; ++j) s[acc(j)] = s[acc(j)] + (kShift ? pair_of(v[u], j) + first[acc(j)] : pair_of(v[u], j));
#pragma unroll
            for (int j = 0; j < kA; ++j) {   // s: minus the mean
                if (kW > 1) s[j] = both(s[j].x + s[j].y);
                s[j] = kShift ? fma2(s[j], both(-inv), first[j]) : s[j] * both(-inv);
            }
#pragma unroll
            for (int u = 0; u < kCount; ++u)
#pragma unroll
                for (int j = 0; j < kPairs<kV>; ++j) {
                    const Pair d = pair_of(v[u], j) + s[acc(j)];
                    q[acc(j)] = fma2(d, d, q[acc(j)]);
                }
            const float share = __fdividef((float)kCount, (float)(i0 + kCount)), between = (float)(i0 * kW) * share;
            // (each lane of a pair holds half of a group's squares: half of what the means' distance adds goes to each)
#pragma unroll
            for (int j = 0; j < kA; ++j) {
                const Pair d = fma2(mean[j], both(-1.0f), s[j]);
                mean[j] = i0 ? fma2(d, both(share), mean[j]) : s[j];
                sq[j] = sq[j] + fma2(d * d, both(kW > 1 ? 0.5f * between : between), q[j]);
            }
        };
        const char *at = x.first();
        int done = 0;   // vectors in the cells (kept ones are few: a single run)
        do {
            const int end = kKeep ? vecs : min(vecs, done + a.run);
#pragma unroll
            for (int j = 0; j < kA; ++j) mean[j] = sq[j] = both(0.0f);
            int i = done;
            for (; i + kGnBatch <= end; i += kGnBatch) batch(at, i, i - done, std::integral_constant<int, kGnBatch>(), 1.0f / (kGnBatch * kW));
            if (i + 2 <= end) {
                batch(at, i, i - done, std::integral_constant<int, 2>(), 0.5f / kW);
                i += 2;
            }
            if (i < end) batch(at, i, i - done, std::integral_constant<int, 1>(), 1.0f / kW);
            if (slot < a.slots) {
                const float share = kKeep || done == 0 ? 1.0f : __fdividef((float)(end - done), (float)end), between = (float)(done * kW) * share;
#pragma unroll
                for (int j = 0; j < kG; ++j) {
                    const Pair m = mean[kW == 1 ? j / 2 : j], e = sq[kW == 1 ? j / 2 : j];
                    float2 c = kW == 1 ? (j % 2 ? make_float2(-m.y, e.y) : make_float2(-m.x, e.x)) : make_float2(-m.x, e.x + e.y);
                    float2 &at_cell = cell[(slot * a.cv + cv) * kG + j];
                    if (!kKeep && done > 0) {
                        const float2 was = at_cell;
                        const float d = c.x - was.x;
                        c = make_float2(__fmaf_rn(d, share, was.x), was.y + __fmaf_rn(d * d, between, c.y));
                    }
                    at_cell = c;
                }
            }
            done = end;
        } while (!kKeep && done < vecs);
    }
    if (!kKeep) copy_wait();
    __syncthreads();
    if (a.ranks > 1) ptx::cluster_wait();

    // ---- a warp per group joins the block's cells and hands the result to every block of the sample
    const int per_group = a.cpg / kW, row = a.cv * kG, used = min(a.slots, pixels);   // (cells of a group in a slot, of a slot)
    const int lane = threadIdx.x & 31;
    for (int g = threadIdx.x / 32; g < groups; g += kGnWarps) {
        const float2 *cells = cell + g * per_group;
        const float first = cells[0].x;
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < used * per_group; i += 32) {
            const int j = a.by_part(i);
            s = __fmaf_rn(cells[j * row + i - j * per_group].x - first, (float)(full + (j < more)), s);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s = pixels ? first + s / ((float)pixels * (float)per_group) : 0.0f;
        for (int i = lane; i < used * per_group; i += 32) {
            const int j = a.by_part(i);
            const float2 e = cells[j * row + i - j * per_group];
            q += __fmaf_rn((e.x - s) * (e.x - s), (float)((full + (j < more)) * kW), e.y);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
        if (a.ranks == 1) {
            if (lane == 0) parts[g] = make_float2(s, q);
        } else if (lane < a.ranks) {
            st_cluster_f2(parts + rank * most + g, lane, make_float2(s, q));
        }
    }
    if (a.ranks > 1) ptx::cluster_sync();
    else __syncthreads();

    // ---- the blocks of the sample; every one joins them for itself
    for (int g = threadIdx.x; g < groups; g += kGnThreads) {
        auto count = [&](int r) { return (float)(min(a.hw, (r + 1) * per) - min(a.hw, r * per)); };
        const float first = parts[g].x;
        float s = 0.0f, q = 0.0f;
        for (int r = 1; r < a.ranks; ++r) s = __fmaf_rn(count(r) > 0.0f ? parts[r * most + g].x - first : 0.0f, count(r), s);
        s = first + s / (float)a.hw;
        for (int r = 0; r < a.ranks; ++r) {
            const float2 e = parts[r * most + g];
            if (count(r) > 0.0f) q += __fmaf_rn((e.x - s) * (e.x - s), count(r) * (float)a.cpg, e.y);
        }
        const float var = q / ((float)a.hw * (float)a.cpg);
        float rstd = __frsqrt_rn(var + a.eps);
        if constexpr (kType == EOQ_I32) {   // (squares of sums at exponent 60 are no fp32 numbers: what the exponent adds comes in 64 bits)
            s *= a.x_scale;
            rstd = (float)(1.0 / sqrt((double)var * a.x_scale * a.x_scale + (double)a.eps));
        }
        final[g] = make_float2(s, rstd);
        if (rank == 0 && a.stats) a.stats[(size_t)smp * a.groups + a.by_cpg(ch0) + g] = make_float2(s, rstd);
    }
    __syncthreads();

    // ---- y, and the 8-bit form
    float mul[kV], add[kV], mean[kG];
    const float scale = act_scale(a.act);
    int g = a.by_cpg(cv * kV), in_g = cv * kV - g * a.cpg;   // group of the next kW channels, and where in it
#pragma unroll
    for (int k = 0; k < kG; ++k) {
        const float2 st = active ? final[g] : make_float2(0.0f, 0.0f);
        mean[k] = -st.x;
#pragma unroll
        for (int j = k * kW; j < (k + 1) * kW; ++j) {
            mul[j] = active ? st.y * gamma[cv * kV + j] * scale : 0.0f;
            add[j] = active ? beta[cv * kV + j] * scale : 0.0f;
        }
        in_g += kW;
        if (in_g == a.cpg) {
            in_g = 0;
            ++g;
        }
    }
    constexpr int kYE = Elem<Types::kY>::kSize;
    char *y = reinterpret_cast<char *>(a.y) + (pix0 * a.y_stride + ch) * kYE;
    int8_t *codes = kSave ? a.codes_out + pix0 * a.c + ch : nullptr;
    uint8_t *exps = kSave ? a.exps_out + pix0 * a.blocks + ch / kBlock8 : nullptr;
    const size_t y_step = a.slots * a.y_stride * kYE, codes_step = (size_t)a.slots * a.c, exps_step = (size_t)a.slots * a.blocks;
    unsigned bad = 0;
    auto emit = [&](auto kind, const Raw<kB> &raw, bool in) {
        float v[kV];
        x_values<kType, kV>(raw, a.x_scale, v);
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
                store_raw(codes, out);
                if (ch % kBlock8 == 0) *exps = (uint8_t)s;
                bad |= s == 255;
            }
            codes += codes_step;
            exps += exps_step;
        }
        if (in) {
#pragma unroll
            for (int j = 0; j < kPairs<kV>; ++j) {
                const Pair m = {mean[2 * j / kW], mean[kV == 1 ? 0 : (2 * j + 1) / kW]};
                set_pair(v, j, fma2(pair_of(v, j) + m, pair_of(mul, j), pair_of(add, j)));
            }
            activate<decltype(kind)::value>(v);
            store_raw(y, Elem<Types::kY>::from_f32(v));
        }
        y += y_step;
    };
    // Lanes that share a block of the 8-bit form stay together: full batches are those of the whole warp.
    const int least = kSave ? (int)__reduce_min_sync(0xffffffffu, (unsigned)vecs) : vecs;
    const int rounds = kSave ? (int)__reduce_max_sync(0xffffffffu, (unsigned)vecs) : vecs;
    with_act(a.act, [&](auto kind) {
        const char *at = x.first();
        int i = 0;
        for (; i + kGnBatch <= least; i += kGnBatch) {
            Raw<kB> raw[kGnBatch];
            x.get(raw, i, at);
#pragma unroll
            for (int u = 0; u < kGnBatch; ++u) emit(kind, raw[u], true);
        }
        for (; i < rounds; ++i) {
            Raw<kB> raw[1] = {zero_raw<kB>()};
            if (i < vecs) x.get(raw, i, at);
            emit(kind, raw[0], i < vecs);
        }
    });
    if (kSave && bad) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
}

template <int kType, int kV, int kW, bool kSave, bool kKeep>
cudaError_t launch(GnArgs a, const FusedPlan &p, cudaStream_t st)
{
    const auto kernel = gn_fused_fwd_kernel<kType, kV, kW, kSave, kKeep>;
    use_plan(a, p, kW);
    static std::atomic<unsigned long long> allowed;
    const cudaError_t e = allow_smem((const void *)kernel, 200 * 1024, allowed);
    if (e != cudaSuccess) return e;
    return launch_chained_clusters(p.ranks, kernel, dim3((unsigned)((size_t)a.n * p.chunks * p.ranks)), dim3(kGnThreads), p.smem, st, a);
}

// whether a plan is taken that leaves SMs without a block, or vectors unkept
constexpr int kAlways = 0, kAllSms = 1, kKept = 2;

template <int kType, int kV, int kW>
bool of_part(const GnArgs &a, cudaError_t *result, cudaStream_t st, int only)
{
    constexpr int kB = kV * Elem<kType>::kSize;
    const bool save = a.codes_out != nullptr && a.c % kBlock8 == 0;
    int unit = a.cpg / kW * kV;
    if (save) unit = unit / gcd_of(unit, kBlock8) * kBlock8;
    constexpr size_t kFour = 56 * 1024, kTwo = 112 * 1024;   // blocks to an SM
    FusedPlan p;
    auto fixed = [&](int cv) { return FwdLayout<kV, kW>::bytes(cv, cv * kV / a.cpg); };
    if (!fused_plan(p, a.n, a.hw, a.c, kV, unit, kB, kB, kFour, fixed)) return false;
    if (!p.keep && !fused_plan(p, a.n, a.hw, a.c, kV, unit, kB, kB, kTwo, fixed)) return false;
    if ((only == kAllSms && (size_t)a.n * p.chunks * p.ranks < kPartSms) || (only == kKept && !p.keep)) return false;
    if (p.keep) *result = save ? launch<kType, kV, kW, true, true>(a, p, st) : launch<kType, kV, kW, false, true>(a, p, st);
    else *result = save ? launch<kType, kV, kW, true, false>(a, p, st) : launch<kType, kV, kW, false, false>(a, p, st);
    return true;
}

template <int kType, int kV>
bool of_width(const GnArgs &a, cudaError_t *result, cudaStream_t st, int only = kAlways)
{
    const int w = gcd_of(a.cpg, kV);
    if constexpr (kV == 8)
        if (w == 8) return of_part<kType, kV, 8>(a, result, st, only);
    if constexpr (kV >= 4)
        if (w == 4) return of_part<kType, kV, 4>(a, result, st, only);
    if constexpr (kV >= 2)
        if (w == 2) return of_part<kType, kV, 2>(a, result, st, only);
    return of_part<kType, kV, 1>(a, result, st, only);
}

template <int kType>
bool of_type(const GnArgs &a, cudaError_t *result, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kY = Elem<GnTypes<kType>::kY>::kSize;
    auto of = [&](int v) {
        return a.c % v == 0 && a.x_stride % v == 0 && a.y_stride % v == 0 && aligned_at(a.x, v * kE) && aligned_at(a.y, v * kY) && aligned_at(a.codes_out, v);
    };
    constexpr int kWide = GnTypes<kType>::kWide;
    if (of(kWide)) {
        // Narrower vectors where groups then fall into more chunks and the call has no block for every SM otherwise (13 samples 45 x 45, 120 fp16
        // channels in groups of 15: 8.5 us, 11.3 with 16-byte vectors).
        // Whole blocks of the 8-bit form may make a group too wide for narrower vectors alone: few blocks then, which are worth it where they
        // keep their vectors (1,056 fp16 channels in 32 groups, one sample 7 x 7: 10.4 us, 13.6 in three launches; 112 x 112, read again: 1048 and 308).
        if (a.cpg % kWide != 0)
            return of_width<kType, kWide>(a, result, st, kAllSms) || of_width<kType, kWide / 2>(a, result, st) || of_width<kType, kWide>(a, result, st, kKept);
        return of_width<kType, kWide>(a, result, st);
    }
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
