// Group normalisation backward in one launch, or two (eoq_gn_bwd): see eoq_gn_fused.cuh for how a sample is dealt out, and eoq_gn.cu for
// the formulas.  The first look at a block's pixels sums dz and dz u per channel, which is all that S1, S2, dgamma and dbeta need; the
// second writes dx.  When all samples of a chunk fit a cluster it also adds dgamma and dbeta over them, and the call is one launch;
// otherwise a small kernel behind adds the samples in their order.
//
// 64 channels 112 x 112, 64 bf16 samples from the 8-bit form, SiLU: 109 us, 2.4 TB/s of what has to move (3.0 TB/s with what is read a second time).
// No unit is full: 38 instructions per element keep issue 58% and the exponentials' unit 48% busy, 27 of 64 warps are there, and
// their longest wait is for loads (3.3 per issue; next 1.7 for dependent arithmetic).  Registers allow four blocks on an SM; fp32 vectors read again
// spill at that bound (116 bytes a thread stored, 48 from the 8-bit form; the 16-bit types 8 to 16).
#include <type_traits>

#include "eoq_gn_fused.cuh"

namespace eoq {

namespace {

// shared memory: cells of the threads, rows of sums by warp, sums of every block of the cluster, of the sample, (S1, S2); gamma, gamma times rstd,
// that and beta times act_scale()
template <int kV>
struct BwdLayout {
    __host__ __device__ static size_t bytes(int cv)
    {
        const int slots = kGnThreads / cv, width = cv * kV;
        return sizeof(float2) * ((size_t)kGnThreads * kV + (size_t)(slots < kGnWarps ? slots : kGnWarps) * width + (8 + 4) * (size_t)width);
    }
};

// kW: so many neighbouring channels of a vector are always of one group (the common divisor of both widths)
template <int kType, int kV, int kW, bool kCodes, bool kKeep>
__global__ void __launch_bounds__(kGnThreads, kW == kV ? 4 : 3) gn_fused_bwd_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    using Input = GnInput<kType, kV, kCodes>;
    constexpr int kE = Elem<kType>::kSize, kDyE = Elem<Types::kY>::kSize, kG = kV / kW;
    extern __shared__ __align__(16) uint8_t smem[];
    const int width = a.cv * kV, rows = min(a.slots, kGnWarps);
    const size_t all = kKeep ? (size_t)a.vecs * kGnThreads : 0;
    float2 *cell = reinterpret_cast<float2 *>(smem + all * (Input::kDyB + Input::kXB));
    float2 *by_warp = cell + kGnThreads * kV, *parts = by_warp + rows * width, *total = parts + 8 * width, *means = total + width;   // parts [rank][channel]
    float *gamma_s = reinterpret_cast<float *>(means + width), *gamma_r = gamma_s + width, *mul_z = gamma_r + width, *beta_z = mul_z + width;

    const int id = a.by_cluster(blockIdx.x), rank = blockIdx.x - id * a.cluster, set = a.by_chunks(id), chunk = id - set * a.chunks;
    const int samples = a.by_ranks(a.cluster), own = a.by_ranks(rank), smp = set * samples + own, part = rank - own * a.ranks;
    const int slot = a.by_cv(threadIdx.x), cv = threadIdx.x - slot * a.cv, ch0 = chunk * width, ch = ch0 + cv * kV;
    const int per = a.per, p_begin = min(part * per, a.hw), pixels = min(a.hw, p_begin + per) - p_begin;
    const int channels = min(width, a.c - ch0), groups = a.by_cpg(channels);
    const bool active = slot < a.slots && ch < a.c;
    const int vecs = active && slot < pixels ? 1 + a.by_slots(pixels - 1 - slot) : 0;
    const size_t pix0 = (size_t)smp * a.hw + p_begin + slot;

    const Vectors<Input::kDyB, kKeep> dys(reinterpret_cast<const char *>(a.dy) + (pix0 * a.dy_stride + ch) * kDyE, a.slots * a.dy_stride * kDyE, smem);
    const Vectors<Input::kXB, kKeep> xs(kCodes ? reinterpret_cast<const char *>(a.codes + pix0 * a.c + ch)
                                               : reinterpret_cast<const char *>(a.x) + (pix0 * a.x_stride + ch) * kE,
                                        kCodes ? (size_t)a.slots * a.c : a.slots * a.x_stride * kE, smem + all * Input::kDyB);
    const Vectors<1, false> bytes(kCodes ? a.exps + pix0 * a.blocks + ch / kBlock8 : nullptr, (size_t)a.slots * a.blocks, smem);

    if (a.cluster > 1) ptx::cluster_arrive();   // (waited for below: the others have started when their memory is written)
    ptx::grid_dep_wait_launch_small();
    dys.fetch(vecs);
    xs.fetch(vecs);
    if (kKeep && kCodes) {   // (into the L1 cache, where both looks find them)
        const char *p = bytes.first();
#pragma unroll 4
        for (int i = 0; i < vecs; ++i, p += bytes.step) ptx::prefetch_l1(p);
    }
    float less[kG], rstd[kG];
    const int g0 = a.by_cpg(cv * kV), in_g0 = cv * kV - g0 * a.cpg;   // group of the first channel within the chunk, and where in it
    const float2 *stats = a.stats + (size_t)smp * a.groups + a.by_cpg(ch0);
    int g = g0, in_g = in_g0;
#pragma unroll
    for (int k = 0; k < kG; ++k) {
        const float2 st = active ? __ldg(stats + g) : make_float2(0.0f, 0.0f);
        less[k] = -st.x;
        rstd[k] = st.y;
        in_g += kW;
        if (in_g == a.cpg) {
            in_g = 0;
            ++g;
        }
    }
    for (int k = threadIdx.x; k < width; k += kGnThreads) {
        const bool in = k < channels;
        const float gamma = in && a.gamma ? __ldg(a.gamma + ch0 + k) : 1.0f, r = in ? __ldg(stats + a.by_cpg(k)).y : 0.0f;
        gamma_s[k] = gamma;
        gamma_r[k] = gamma * r;
        mul_z[k] = gamma * r * act_scale(a.act);   // (as the forward pass has it)
        beta_z[k] = (in && a.beta ? __ldg(a.beta + ch0 + k) : 0.0f) * act_scale(a.act);
    }
    const float dy_scale = kType == EOQ_I32 ? error_scale(a) : 1.0f;

    if (kKeep) copy_wait();

    __syncthreads();   // (gamma and beta)

    // Both looks: a few vectors at a time.  use(u, dz, gamma rstd) gets what a vector holds; first to last, after(i) follows the batch in front of vector i.
    const float *const mul_at = mul_z + cv * kV, *const beta_at = beta_z + cv * kV, *const gamma_r_at = gamma_r + cv * kV;
    // back: from the last vector to the first, so that what is read again was read a short while ago (64 channels 112 x 112, 64 bf16
    // samples: 109 us instead of 120).
    auto look = [&](auto kind, auto back, auto use, auto after) {
        constexpr bool kBack = decltype(back)::value;
        const char *dy_at = dys.first(), *x_at = xs.first(), *s_at = bytes.first();
        if (kBack) {
            dy_at += vecs * dys.step;
            x_at += vecs * xs.step;
            s_at += vecs * bytes.step;
        }
        auto batch = [&](int i, auto count) {
            constexpr int kCount = decltype(count)::value;
            if (kBack) {
                dy_at -= kCount * dys.step;
                x_at -= kCount * xs.step;
                s_at -= kCount * bytes.step;
            }
            Raw<Input::kXB> x[kCount];
            Raw<Input::kDyB> dy[kCount];
            Raw<1> s[kCount] = {};
            dys.get(dy, i, dy_at);
            xs.get(x, i, x_at);
            if (kCodes) bytes.get(s, i, s_at);
            if (kBack) {   // (get has moved them on)
                if (!kKeep) {
                    dy_at -= kCount * dys.step;
                    x_at -= kCount * xs.step;
                }
                s_at -= kCount * bytes.step;
            }
            float mul[kV], beta[kV], by[kV];
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                mul[j] = mul_at[j];
                beta[j] = beta_at[j];
                by[j] = gamma_r_at[j];
            }
#pragma unroll
            for (int j = 0; j < kCount; ++j) {
                float u[kV], dz[kV];
                gn_terms<decltype(kind)::value, kType, kV, kCodes, kW>(x[j], s[j].w, dy[j], a.x_scale, a.act, less, rstd, mul, beta, u, dz);
                if constexpr (kBack) use(i + j, u, dz, by);
                else use(0, u, dz, by);
            }
        };
        if constexpr (kBack) {
            int i = vecs;
#pragma unroll 1
            for (; i % kGnBatch; --i) batch(i - 1, std::integral_constant<int, 1>());
#pragma unroll 1
            for (; i > 0; i -= kGnBatch) batch(i - kGnBatch, std::integral_constant<int, kGnBatch>());
        } else {
            int i = 0;
#pragma unroll 1
            for (; i + kGnBatch <= vecs; i += kGnBatch) {
                batch(i, std::integral_constant<int, kGnBatch>());
                after(i + kGnBatch);
            }
#pragma unroll 1
            for (; i < vecs; ++i) batch(i, std::integral_constant<int, 1>());
        }
    };

    // Vectors read again from the cache are worked on one by one, with what registers the loads of a batch leave (64 channels 112 x 112, 64 bf16
    // samples, first to last: 117 us; a batch at a time 138, with three blocks on an SM 153); kept ones a batch at a time (256 channels 56 x 56, 32 bf16
    // samples: 68 us instead of 70).
    auto by_act = [&](auto f) {
        if constexpr (kKeep) with_act(a.act, f);
        else f(std::integral_constant<int, kAnyAct>());
    };

    {
        float s0[kV], s1[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) s0[j] = s1[j] = 0.0f;
        float2 *const own = cell + (slot * a.cv + cv) * kV;
        auto to_cell = [&](bool first) {
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                const float2 was = first ? make_float2(0.0f, 0.0f) : own[j];
                own[j] = make_float2(was.x + s0[j], was.y + s1[j]);
                s0[j] = s1[j] = 0.0f;
            }
        };
        by_act([&](auto kind) {
            look(kind, std::false_type(), [&](int, const float (&u)[kV], const float (&dz)[kV], const float (&)[kV]) {
#pragma unroll
                for (int j = 0; j < kPairs<kV>; ++j) {
                    set_pair(s0, j, pair_of(s0, j) + pair_of(dz, j));
                    set_pair(s1, j, fma2(pair_of(dz, j), pair_of(u, j), pair_of(s1, j)));
                }
            }, [&](int i) {
                if (!kKeep && (i & (a.run - 1)) == 0) to_cell(i == a.run);   // (kept vectors are few)
            });
        });
        if (slot < a.slots) to_cell(kKeep || vecs < a.run);
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
    if (a.cluster > 1) ptx::cluster_wait();
    // who needs a block's sums: the blocks of its sample, and the first block where that adds the samples up
    const bool whole = samples == a.n;
    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        float2 t = make_float2(0.0f, 0.0f);
        for (int j = 0; j < rows; ++j) {
            t.x += by_warp[j * width + k].x;
            t.y += by_warp[j * width + k].y;
        }
        if (a.cluster == 1) {
            parts[k] = t;
        } else {
            for (int r = rank - part; r < rank - part + a.ranks; ++r) st_cluster_f2(parts + rank * width + k, r, t);
            if (whole && rank >= a.ranks) st_cluster_f2(parts + rank * width + k, 0, t);
        }
    }
    if (a.cluster > 1) ptx::cluster_sync();
    else __syncthreads();

    for (int k = threadIdx.x; k < channels; k += kGnThreads) {
        float2 t = make_float2(0.0f, 0.0f);
        auto add = [&](int r) {
            const float2 e = parts[r * width + k];
            t.x += e.x;
            t.y += e.y;
        };
        for (int r = 0; r < a.ranks; ++r) add(rank - part + r);
        total[k] = t;
        if (whole) {
            if (rank == 0) {
                for (int r = a.ranks; r < a.cluster; ++r) add(r);
                if (a.dbeta) a.dbeta[ch0 + k] = t.x * dy_scale;
                if (a.dgamma) a.dgamma[ch0 + k] = t.y * dy_scale;
            }
        } else if (part == 0) {
            a.part[(size_t)smp * a.c + ch0 + k] = t;
        }
    }
    __syncthreads();
    const float inv = 1.0f / ((float)a.hw * (float)a.cpg);
    for (int k = warp; k < groups; k += kGnWarps) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int i = lane; i < a.cpg; i += 32) {
            const float2 e = total[k * a.cpg + i];
            s0 = __fmaf_rn(gamma_s[k * a.cpg + i], e.x, s0);
            s1 = __fmaf_rn(gamma_s[k * a.cpg + i], e.y, s1);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            s0 += __shfl_xor_sync(0xffffffffu, s0, d);
            s1 += __shfl_xor_sync(0xffffffffu, s1, d);
        }
        if (lane == 0) means[k] = make_float2(s0 * inv, s1 * inv);
    }
    __syncthreads();
    float k0[kG], k1[kG];
    g = g0;
    in_g = in_g0;
#pragma unroll
    for (int k = 0; k < kG; ++k) {
        const float2 m = active ? means[g] : make_float2(0.0f, 0.0f);
        k0[k] = -rstd[k] * m.x;
        k1[k] = -rstd[k] * m.y;
        in_g += kW;
        if (in_g == a.cpg) {
            in_g = 0;
            ++g;
        }
    }
    constexpr int kDxE = Elem<Types::kDx>::kSize;
    char *dx = reinterpret_cast<char *>(a.dx) + (pix0 * a.dx_stride + ch) * kDxE;
    const size_t dx_step = a.slots * a.dx_stride * kDxE;
    by_act([&](auto kind) {
        look(kind, std::bool_constant<!kKeep>(), [&](int i, const float (&u)[kV], float (&dz)[kV], const float (&by)[kV]) {
#pragma unroll
            for (int j = 0; j < kPairs<kV>; ++j) {
                const int l = 2 * j / kW, h = kV == 1 ? 0 : (2 * j + 1) / kW;
                set_pair(dz, j, fma2(pair_of(dz, j), pair_of(by, j), fma2(pair_of(u, j), Pair{k1[l], k1[h]}, Pair{k0[l], k0[h]})));
                if (kType == EOQ_I32) set_pair(dz, j, pair_of(dz, j) * both(dy_scale));
            }
            if constexpr (kKeep) {
                store_raw(dx, Elem<Types::kDx>::from_f32(dz));
                dx += dx_step;
            } else {
                store_raw(dx + i * dx_step, Elem<Types::kDx>::from_f32(dz));
            }
        }, [](int) {});
    });
}

template <int kType, int kV, int kW, bool kCodes, bool kKeep>
cudaError_t launch(GnArgs a, const FusedPlan &p, int *launches, cudaStream_t st)
{
    const auto kernel = gn_fused_bwd_kernel<kType, kV, kW, kCodes, kKeep>;
    use_plan(a, p, kW);
    const bool together = a.n == 1 || (long long)a.n * p.ranks <= 8;   // all samples of a chunk in one cluster
    a.cluster = together ? a.n * p.ranks : p.ranks;
    a.by_cluster = FastDiv(a.cluster);
    static std::atomic<unsigned long long> allowed;
    cudaError_t e = allow_smem((const void *)kernel, 200 * 1024, allowed);
    if (e != cudaSuccess) return e;
    e = launch_chained_clusters(a.cluster, kernel, dim3((unsigned)((size_t)a.n * p.chunks * p.ranks)), dim3(kGnThreads), p.smem, st, a);
    ++*launches;
    if (e != cudaSuccess || together || (!a.dgamma && !a.dbeta)) return e;
    ++*launches;
    return launch_gn_channel_sums(a, st);
}

template <int kType, int kV, int kW, bool kCodes>
bool of_part(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    constexpr int kB = kV * Elem<kType>::kSize, kKept = kV * Elem<GnTypes<kType>::kY>::kSize + (kCodes ? kV : kB);
    constexpr size_t kLimit = 56 * 1024;   // four blocks to an SM
    FusedPlan p;
    if (!fused_plan(p, a.n, a.hw, a.c, kV, a.cpg / kW * kV, kB, kKept, kLimit, [](int cv) { return BwdLayout<kV>::bytes(cv); })) return false;
    *result = p.keep ? launch<kType, kV, kW, kCodes, true>(a, p, launches, st) : launch<kType, kV, kW, kCodes, false>(a, p, launches, st);
    return true;
}

template <int kType, int kV, bool kCodes>
bool of_width(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    const int w = gcd_of(a.cpg, kV);
    if constexpr (kV >= 4)
        if (w == 4) return of_part<kType, kV, 4, kCodes>(a, result, launches, st);
    if constexpr (kV >= 2)
        if (w == 2) return of_part<kType, kV, 2, kCodes>(a, result, launches, st);
    return of_part<kType, kV, 1, kCodes>(a, result, launches, st);
}

template <int kType, bool kCodes>
bool of_source(const GnArgs &a, cudaError_t *result, int *launches, cudaStream_t st)
{
    constexpr int kE = Elem<kType>::kSize, kY = Elem<GnTypes<kType>::kY>::kSize, kDx = Elem<GnTypes<kType>::kDx>::kSize;
    auto of = [&](int v) {
        return a.c % v == 0 && a.dy_stride % v == 0 && a.dx_stride % v == 0 && (kCodes || (a.x_stride % v == 0 && aligned_at(a.x, v * kE))) &&
               aligned_at(a.codes, v) && aligned_at(a.dy, v * kY) && aligned_at(a.dx, v * kDx);
    };
    // (eight 16-bit channels a thread take more registers than four blocks on an SM leave: 145 us instead of 117 for 64 channels 112 x 112,
    // 64 bf16 samples)
    if (of(4)) return of_width<kType, 4, kCodes>(a, result, launches, st);
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
