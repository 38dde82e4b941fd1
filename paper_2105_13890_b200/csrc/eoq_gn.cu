// Group normalisation with an activation on channels-last tensors, forward and backward (eoq_gn_fwd, eoq_gn_bwd).  Beside
// eoq_bn.cu, the comparison case of arXiv 2105.13890, Sec. 5.3, it is the normalisation that does not look over the batch, which
// is what the paper's small-batch training needs:
//   u = (x - mean) rstd over the pixels and channels of a (sample, group),  z = gamma u + beta,  y = act(z);
//   dz = dy act'(z),  dbeta = sum dz,  dgamma = sum dz u,  dx = rstd (gamma dz - S1 - u S2),
//   S1 and S2 the means of gamma dz and gamma dz u over the (sample, group).
//
// The kernels here serve what the one-launch forms (eoq_gn_fused.cu, eoq_gn_fused_bwd.cu) leave: groups wider than a thread block, or than
// its shared memory.  A pass that reduces, a small one that joins, a pass that writes.  For calls that both forms take they are the slower ones
// where there are samples for every SM (256 channels 56 x 56, 32 fp16 samples, forward: 43 us against 25; 64 channels 112 x 112, 64 bf16 samples,
// both passes: 303 against 181), since everything is read from memory twice and a call is three launches.  They would be the faster ones for a few
// large images, whose pixels they deal to all SMs instead of eight for each chunk of channels (one 512 x 512 of 64 channels in 16 groups, bf16: 62 and 68
// us against 373 and 488; in one group 480 and 215 against 502 and 974): such calls take the one-launch form all the same.  A thread owns kV
// neighbouring channels (16 bytes of x, or one element where widths or addresses rule that out) and walks pixels of one sample, so
// that what depends on the channel stays in registers.  Sums never leave the thread as raw squares: a batch of pixels gives its mean
// and its squares about that mean, and (count, mean, squares) are joined pairwise, so a mean far from zero costs no digits.
#include "eoq_gn.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

template <int kType, int kV>
__global__ void __launch_bounds__(kThreads) gn_stats_kernel(const __grid_constant__ GnArgs a)
{
    extern __shared__ float2 cell[];   // [slots][channels of the chunk]: mean, squares
    ptx::grid_dep_wait();
    const int smp = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch = (blockIdx.y * a.cv + cv) * kV;
    const int p_begin = split * a.per_split, p_end = min(a.hw, p_begin + a.per_split);
    constexpr int kB = kV * Elem<kType>::kSize;
    if (slot < a.slots && ch < a.c) {
        const char *src = reinterpret_cast<const char *>(a.x) + ((size_t)smp * a.hw * a.x_stride + ch) * Elem<kType>::kSize;
        int in_cell = 0, p0 = p_begin + slot;   // pixels that the cell holds
        do {
            float mean[kV], sq[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) mean[i] = sq[i] = 0.0f;
            int count = 0;
            for (; p0 < p_end && count < a.run; p0 += kUnroll * a.slots) {
                Raw<kB> raw[kUnroll];
                float v[kUnroll][kV];
                int m = 0;
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const int p = p0 + u * a.slots;
                    raw[u] = p < p_end ? load_raw<kB>(src + (size_t)p * a.x_stride * Elem<kType>::kSize) : zero_raw<kB>();
                    m += p < p_end;
                }
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) Elem<kType>::to_f32(raw[u], v[u]);   // (integer sums as they are)
                const float inv_m = 1.0f / (float)m, share = (float)m / (float)(count + m), both = (float)count * share;
                count += m;
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    // about the first pixel: equal values have exactly themselves as their mean
                    const float k = v[0][i];
                    float s = 0.0f, q = 0.0f;
#pragma unroll
                    for (int u = 1; u < kUnroll; ++u) s += u < m ? v[u][i] - k : 0.0f;   // (the valid pixels come first)
                    s = __fmaf_rn(s, inv_m, k);
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u) {
                        const float d = u < m ? v[u][i] - s : 0.0f;
                        q = __fmaf_rn(d, d, q);
                    }
                    const float d = s - mean[i];
                    mean[i] = __fmaf_rn(d, share, mean[i]);
                    sq[i] += __fmaf_rn(d * d, both, q);
                }
            }
            const float share = in_cell ? (float)count / (float)(in_cell + count) : 1.0f, both = (float)in_cell * share;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                float2 &at = cell[(slot * a.cv + cv) * kV + i];
                const float2 was = in_cell ? at : make_float2(0.0f, 0.0f);
                const float d = mean[i] - was.x;
                at = in_cell ? make_float2(__fmaf_rn(d, share, was.x), was.y + __fmaf_rn(d * d, both, sq[i])) : make_float2(mean[i], sq[i]);
            }
            in_cell += count;
        } while (p0 < p_end);
    }
    __syncthreads();
    // a thread per channel joins the slots: the mean of the means by their counts, then the squares about it
    const int width = a.cv * kV, total = p_end - p_begin;
    for (int k = threadIdx.x; k < width; k += kThreads) {
        const int c = blockIdx.y * width + k;
        if (c >= a.c) break;
        float s = 0.0f, q = 0.0f;
        const int full = total / a.slots, more = total % a.slots;   // slot j has `full` pixels, the first `more` one more
        const float first = cell[k].x;
        for (int j = 1; j < a.slots; ++j) s = __fmaf_rn(full + (j < more) ? cell[j * width + k].x - first : 0.0f, (float)(full + (j < more)), s);
        s = first + s / (float)total;
        for (int j = 0; j < a.slots; ++j) {
            const float2 e = cell[j * width + k];
            const int cnt = full + (j < more);
            if (cnt) q += __fmaf_rn((e.x - s) * (e.x - s), (float)cnt, e.y);
        }
        a.part[((size_t)smp * a.splits + split) * a.c + c] = make_float2(s, q);
    }
}

// a warp per (sample, group): mean and 1 / sqrt(variance + eps), in 64 bits.  The partial results of integer sums are those of the sums as they are:
// with their exponent the squares may be beyond fp32.
__global__ void __launch_bounds__(kThreads) gn_join_kernel(const __grid_constant__ GnArgs a)
{
    ptx::grid_dep_wait_launch_small();
    const int lane = threadIdx.x & 31;
    const size_t id = (size_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (id >= (size_t)a.n * a.groups) return;
    const int smp = (int)(id / a.groups), g = (int)(id % a.groups), cells = a.splits * a.cpg;
    const float2 *part = a.part + (size_t)smp * a.splits * a.c + (size_t)g * a.cpg;
    auto count_of = [&](int split) { return (double)(min(a.hw, (split + 1) * a.per_split) - split * a.per_split); };
    double s = 0.0;
    for (int i = lane; i < cells; i += 32) s += count_of(i / a.cpg) * part[(size_t)(i / a.cpg) * a.c + i % a.cpg].x;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    const double total = (double)a.hw * a.cpg, mean = s / total;
    double q = 0.0;
    for (int i = lane; i < cells; i += 32) {
        const float2 e = part[(size_t)(i / a.cpg) * a.c + i % a.cpg];
        q += e.y + count_of(i / a.cpg) * (e.x - mean) * (e.x - mean);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
    const double scale = a.x_scale;   // (of integer sums)
    if (lane == 0) a.stats[id] = make_float2((float)(mean * scale), (float)(1.0 / sqrt(q / total * scale * scale + (double)a.eps)));
}

template <int kType, int kV, bool kSave>
__global__ void __launch_bounds__(kThreads) gn_apply_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    constexpr int kB = kV * Elem<kType>::kSize, kLanes = kBlock8 / kV;
    ptx::grid_dep_wait_launch_small();
    const int smp = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch = (blockIdx.y * a.cv + cv) * kV;
    const int p_begin = split * a.per_split, p_end = min(a.hw, p_begin + a.per_split);
    const bool mine = slot < a.slots && ch < a.c;
    float mul[kV], add[kV], mean[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) mul[i] = add[i] = mean[i] = 0.0f;
    if (mine)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float2 st = a.stats[(size_t)smp * a.groups + (ch + i) / a.cpg];
            mean[i] = st.x;
            mul[i] = (a.gamma ? st.y * a.gamma[ch + i] : st.y) * act_scale(a.act);
            add[i] = a.beta ? a.beta[ch + i] * act_scale(a.act) : 0.0f;
        }
    const size_t pix0 = (size_t)smp * a.hw;
    unsigned bad = 0;
    with_act(a.act, [&](auto kind) {
        for (int p0 = p_begin; p0 < p_end; p0 += kUnroll * a.slots) {
            Raw<kB> raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + slot + u * a.slots;
                raw[u] = mine && p < p_end ? load_raw<kB>(reinterpret_cast<const char *>(a.x) + ((pix0 + p) * a.x_stride + ch) * Elem<kType>::kSize)
                                           : zero_raw<kB>();
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + slot + u * a.slots;
                const bool in = mine && p < p_end;
                float v[kV];
                x_values<kType, kV>(raw[u], a.x_scale, v);
                if constexpr (kSave) {
                    float m = 0.0f;
#pragma unroll
                    for (int i = 0; i < kV; ++i) m = max_abs(m, v[i]);
                    m = lanes_max_abs<kLanes>(m);
                    const int s = block_exp(m);
                    uint32_t w[(kV + 3) / 4];
                    block_codes(v, s, w);
                    if (in) {
                        Raw<kV> out;
#pragma unroll
                        for (int i = 0; i < (kV + 3) / 4; ++i) set_word(out, i, w[i]);
                        store_raw(a.codes_out + (pix0 + p) * a.c + ch, out);
                        if (ch % kBlock8 == 0) a.exps_out[(pix0 + p) * a.blocks + ch / kBlock8] = (uint8_t)s;
                        bad |= s == 255;
                    }
                }
                if (in) {
#pragma unroll
                    for (int i = 0; i < kV; ++i) v[i] = __fmaf_rn(v[i] - mean[i], mul[i], add[i]);
                    activate<decltype(kind)::value>(v);
                    store_raw(reinterpret_cast<char *>(a.y) + ((pix0 + p) * a.y_stride + ch) * Elem<Types::kY>::kSize,
                              Elem<Types::kY>::from_f32(v));
                }
            }
        }
    });
    if (kSave && bad) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
}

template <int kType, int kV, bool kCodes>
__global__ void __launch_bounds__(kThreads) gn_bwd_sums_kernel(const __grid_constant__ GnArgs a)
{
    extern __shared__ float2 cell[];   // [slots][channels of the chunk]: sum dz, sum dz u
    ptx::grid_dep_wait();
    const int smp = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch = (blockIdx.y * a.cv + cv) * kV;
    const int p_begin = split * a.per_split, p_end = min(a.hw, p_begin + a.per_split);
    if (slot < a.slots && ch < a.c) {
        float rstd[kV], less[kV], mul[kV], beta[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float2 st = a.stats[(size_t)smp * a.groups + (ch + i) / a.cpg];
            rstd[i] = st.y;
            less[i] = -st.x;
            mul[i] = (a.gamma ? st.y * a.gamma[ch + i] : st.y) * act_scale(a.act);
            beta[i] = a.beta ? a.beta[ch + i] * act_scale(a.act) : 0.0f;
        }
        const size_t pix0 = (size_t)smp * a.hw;
        with_act(a.act, [&](auto kind) {
            int p0 = p_begin + slot;
            bool first = true;
            do {
                float s0[kV], s1[kV];
#pragma unroll
                for (int i = 0; i < kV; ++i) s0[i] = s1[i] = 0.0f;
                for (int count = 0; p0 < p_end && count < a.run; count += kUnroll, p0 += kUnroll * a.slots) {
                    GnInput<kType, kV, kCodes> in[kUnroll];
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u) in[u].load(a, pix0 + p0 + u * a.slots, ch, p0 + u * a.slots < p_end);
#pragma unroll
                    for (int k = 0; k < kUnroll; ++k) {
                        if (p0 + k * a.slots >= p_end) break;
                        float u[kV], dz[kV];
                        in[k].template values<decltype(kind)::value>(a, rstd, less, mul, beta, u, dz);
#pragma unroll
                        for (int i = 0; i < kV; ++i) {
                            s0[i] += dz[i];
                            s1[i] = __fmaf_rn(dz[i], u[i], s1[i]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    float2 &at = cell[(slot * a.cv + cv) * kV + i];
                    const float2 was = first ? make_float2(0.0f, 0.0f) : at;
                    at = make_float2(was.x + s0[i], was.y + s1[i]);
                }
                first = false;
            } while (p0 < p_end);
        });
    }
    __syncthreads();
    const int width = a.cv * kV;
    for (int k = threadIdx.x; k < width; k += kThreads) {
        const int c = blockIdx.y * width + k;
        if (c >= a.c) break;
        float2 t = make_float2(0.0f, 0.0f);
        for (int j = 0; j < a.slots; ++j) {
            const float2 e = cell[j * width + k];
            t.x += e.x;
            t.y += e.y;
        }
        a.part[((size_t)smp * a.splits + split) * a.c + c] = t;
    }
}

// Blocks in front: a warp per (sample, group) forms S1 and S2.  Blocks behind: kJoin channels each, dgamma and dbeta over samples and
// splits, 32 threads a channel in a fixed order.  Both in 64 bits where there are many, since nothing bounds the numbers of samples and splits.
constexpr int kJoin = 8;
__global__ void __launch_bounds__(kThreads) gn_bwd_join_kernel(const __grid_constant__ GnArgs a, int group_blocks)
{
    ptx::grid_dep_wait_launch_small();
    if ((int)blockIdx.x < group_blocks) {
        const int lane = threadIdx.x & 31;
        const size_t id = (size_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
        if (id >= (size_t)a.n * a.groups) return;
        const int smp = (int)(id / a.groups), g = (int)(id % a.groups), cells = a.splits * a.cpg;
        const float2 *part = a.part + (size_t)smp * a.splits * a.c + (size_t)g * a.cpg;
        double s0 = 0.0, s1 = 0.0;
        for (int i = lane; i < cells; i += 32) {
            const float2 e = part[(size_t)(i / a.cpg) * a.c + i % a.cpg];
            const double gamma = a.gamma ? a.gamma[g * a.cpg + i % a.cpg] : 1.0f;
            s0 += gamma * e.x;
            s1 += gamma * e.y;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            s0 += __shfl_xor_sync(0xffffffffu, s0, d);
            s1 += __shfl_xor_sync(0xffffffffu, s1, d);
        }
        const double total = (double)a.hw * a.cpg;
        if (lane == 0) a.means[id] = make_float2((float)(s0 / total), (float)(s1 / total));
        return;
    }
    __shared__ float2 red[kThreads / 32][kJoin];
    const int k = threadIdx.x % kJoin, j = threadIdx.x / kJoin, c = ((int)blockIdx.x - group_blocks) * kJoin + k;
    constexpr int kRows = kThreads / kJoin, kRun = 32;
    const size_t rows = (size_t)a.n * a.splits;
    auto sum = [&](size_t from, size_t to) {
        float2 t = make_float2(0.0f, 0.0f);
#pragma unroll 4
        for (size_t r = from; r < to; r += kRows) {
            const float2 e = a.part[r * a.c + c];
            t.x += e.x;
            t.y += e.y;
        }
        return t;
    };
    float2 t = make_float2(0.0f, 0.0f);
    if (c < a.c && rows <= kRun * kRows) {
        t = sum(j, rows);
    } else if (c < a.c) {
        double2 far = make_double2(0.0, 0.0);
        for (size_t r0 = j; r0 < rows; r0 += kRun * kRows) {
            t = sum(r0, min(rows, r0 + kRun * kRows));
            far.x += t.x;
            far.y += t.y;
        }
        t = make_float2((float)far.x, (float)far.y);
    }
#pragma unroll
    for (int d = kJoin; d < 32; d *= 2) {
        t.x += __shfl_xor_sync(0xffffffffu, t.x, d);
        t.y += __shfl_xor_sync(0xffffffffu, t.y, d);
    }
    if (threadIdx.x % 32 < kJoin) red[threadIdx.x / 32][k] = t;
    __syncthreads();
    if (threadIdx.x < kJoin && c < a.c) {
#pragma unroll
        for (int i = 1; i < kThreads / 32; ++i) {
            t.x += red[i][k].x;
            t.y += red[i][k].y;
        }
        const float scale = error_scale(a);
        if (a.dbeta) a.dbeta[c] = t.x * scale;
        if (a.dgamma) a.dgamma[c] = t.y * scale;
    }
}

template <int kType, int kV, bool kCodes>
__global__ void __launch_bounds__(kThreads) gn_bwd_apply_kernel(const __grid_constant__ GnArgs a)
{
    using Types = GnTypes<kType>;
    ptx::grid_dep_wait_launch_small();
    const int smp = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int cv = threadIdx.x % a.cv, slot = threadIdx.x / a.cv, ch = (blockIdx.y * a.cv + cv) * kV;
    if (slot >= a.slots || ch >= a.c) return;
    const int p_begin = split * a.per_split, p_end = min(a.hw, p_begin + a.per_split);
    float rstd[kV], less[kV], mul[kV], beta[kV], by[kV], k0[kV], k1[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const size_t g = (size_t)smp * a.groups + (ch + i) / a.cpg;
        const float2 st = a.stats[g], m = a.means[g];
        rstd[i] = st.y;
        less[i] = -st.x;
        by[i] = a.gamma ? st.y * a.gamma[ch + i] : st.y;
        mul[i] = by[i] * act_scale(a.act);
        beta[i] = a.beta ? a.beta[ch + i] * act_scale(a.act) : 0.0f;
        k0[i] = -st.y * m.x;
        k1[i] = -st.y * m.y;
    }
    const float dy_scale = kType == EOQ_I32 ? error_scale(a) : 1.0f;
    const size_t pix0 = (size_t)smp * a.hw;
    with_act(a.act, [&](auto kind) {
        for (int p0 = p_begin + slot; p0 < p_end; p0 += kUnroll * a.slots) {
            GnInput<kType, kV, kCodes> in[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) in[u].load(a, pix0 + p0 + u * a.slots, ch, p0 + u * a.slots < p_end);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int p = p0 + k * a.slots;
                if (p >= p_end) break;
                float u[kV], dz[kV];
                in[k].template values<decltype(kind)::value>(a, rstd, less, mul, beta, u, dz);
#pragma unroll
                for (int i = 0; i < kV; ++i) dz[i] = __fmaf_rn(dz[i], by[i], __fmaf_rn(u[i], k1[i], k0[i])) * dy_scale;
                store_raw(reinterpret_cast<char *>(a.dx) + ((pix0 + p) * a.dx_stride + ch) * Elem<Types::kDx>::kSize,
                          Elem<Types::kDx>::from_f32(dz));
            }
        }
    });
}

// How the channels and pixels of a call are dealt out to thread blocks.
struct GnPlan {
    int cv, slots, chunks, splits, per_split;
};

// `blocks`: how many thread blocks are wanted in all.  Splits are whole rounds of the block's pixels.
GnPlan gn_plan(int n, int hw, int c, int v, int blocks)
{
    GnPlan p;
    const int per_pixel = (c + v - 1) / v, lanes = kBlock8 / v;
    p.chunks = (per_pixel + kThreads - 1) / kThreads;
    p.cv = (per_pixel + p.chunks - 1) / p.chunks;
    if (c % kBlock8 == 0) p.cv = (p.cv + lanes - 1) / lanes * lanes;   // blocks of the 8-bit form stay within a warp
    p.slots = kThreads / p.cv;
    const int rounds = (hw + p.slots * kUnroll - 1) / (p.slots * kUnroll);
    long long splits = (blocks + (long long)n * p.chunks - 1) / ((long long)n * p.chunks);
    if (splits > rounds) splits = rounds;
    if (splits < 1) splits = 1;
    p.per_split = (int)((rounds + splits - 1) / splits) * p.slots * kUnroll;
    p.splits = (hw + p.per_split - 1) / p.per_split;
    return p;
}

constexpr int kStatBlocks = 4 * kPartSms, kApplyBlocks = 8 * kPartSms;

int wide_of(int dtype) { return dtype == EOQ_F32 || dtype == EOQ_I32 ? 4 : 8; }

void use_plan(GnArgs &a, const GnPlan &p)
{
    a.cv = p.cv;
    a.slots = p.slots;
    a.splits = p.splits;
    a.per_split = p.per_split;
    a.run = run_of(p.per_split / p.slots);
}

size_t parts_bytes(int n, int hw, int c, int dtype)
{
    // either width may be taken, by the addresses of the call
    const GnPlan w = gn_plan(n, hw, c, wide_of(dtype), kStatBlocks), s = gn_plan(n, hw, c, 1, kStatBlocks);
    const size_t splits = (size_t)(w.splits > s.splits ? w.splits : s.splits);
    return (sizeof(float2) * (size_t)n * splits * c + 255) & ~(size_t)255;
}

template <int kType, int kV>
cudaError_t run_fwd(GnArgs a, int *launches, cudaStream_t st)
{
    GnPlan p = gn_plan(a.n, a.hw, a.c, kV, kStatBlocks);
    use_plan(a, p);
    cudaError_t e = launch_chained(gn_stats_kernel<kType, kV>, dim3(a.n * p.splits, p.chunks), dim3(kThreads),
                                   sizeof(float2) * p.slots * p.cv * kV, st, a);
    if (e != cudaSuccess) return e;
    const size_t warps = (size_t)a.n * a.groups;
    e = launch_chained(gn_join_kernel, dim3((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32))), dim3(kThreads), 0, st, a);
    if (e != cudaSuccess) return e;
    p = gn_plan(a.n, a.hw, a.c, kV, kApplyBlocks);
    use_plan(a, p);
    *launches += 3;
    const dim3 grid(a.n * p.splits, p.chunks);
    if (!a.codes_out) return launch_chained(gn_apply_kernel<kType, kV, false>, grid, dim3(kThreads), 0, st, a);
    if (a.c % kBlock8 == 0) return launch_chained(gn_apply_kernel<kType, kV, true>, grid, dim3(kThreads), 0, st, a);
    // a row of blocks that ends inside one
    e = launch_chained(gn_apply_kernel<kType, kV, false>, grid, dim3(kThreads), 0, st, a);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_ckpt_save(a.x, kType, a.x_exp, (size_t)a.n * a.hw, a.c, a.x_stride, a.codes_out, a.exps_out, a.dev, a.sm_count, st);
}

template <int kType, int kV, bool kCodes>
cudaError_t run_bwd(GnArgs a, int *launches, cudaStream_t st)
{
    GnPlan p = gn_plan(a.n, a.hw, a.c, kV, kStatBlocks);
    use_plan(a, p);
    cudaError_t e = launch_chained(gn_bwd_sums_kernel<kType, kV, kCodes>, dim3(a.n * p.splits, p.chunks), dim3(kThreads),
                                   sizeof(float2) * p.slots * p.cv * kV, st, a);
    if (e != cudaSuccess) return e;
    const size_t warps = (size_t)a.n * a.groups;
    const int group_blocks = (int)((warps + kThreads / 32 - 1) / (kThreads / 32)), channel_blocks = (a.c + kJoin - 1) / kJoin;
    e = launch_chained(gn_bwd_join_kernel, dim3(group_blocks + channel_blocks), dim3(kThreads), 0, st, a, group_blocks);
    if (e != cudaSuccess) return e;
    p = gn_plan(a.n, a.hw, a.c, kV, kApplyBlocks);
    use_plan(a, p);
    *launches += 3;
    return launch_chained(gn_bwd_apply_kernel<kType, kV, kCodes>, dim3(a.n * p.splits, p.chunks), dim3(kThreads), 0, st, a);
}

template <int kType>
cudaError_t fwd_of_type(const GnArgs &a, int *launches, cudaStream_t st)
{
    constexpr int kV = GnTypes<kType>::kWide, kY = Elem<GnTypes<kType>::kY>::kSize;
    const bool wide = a.c % kV == 0 && a.x_stride % kV == 0 && a.y_stride % kV == 0 && aligned_at(a.x, 16) && aligned_at(a.y, kV * kY) &&
                      aligned_at(a.codes_out, kV);
    return wide ? run_fwd<kType, kV>(a, launches, st) : run_fwd<kType, 1>(a, launches, st);
}

template <int kType>
cudaError_t bwd_of_type(const GnArgs &a, int *launches, cudaStream_t st)
{
    constexpr int kV = GnTypes<kType>::kWide, kY = Elem<GnTypes<kType>::kY>::kSize;
    const bool wide = a.c % kV == 0 && a.dy_stride % kV == 0 && a.dx_stride % kV == 0 && (!a.x || a.x_stride % kV == 0) && aligned_at(a.x, 16) &&
                      aligned_at(a.codes, kV) && aligned_at(a.dy, kV * kY) && aligned_at(a.dx, 16);
    if (a.codes) return wide ? run_bwd<kType, kV, true>(a, launches, st) : run_bwd<kType, 1, true>(a, launches, st);
    return wide ? run_bwd<kType, kV, false>(a, launches, st) : run_bwd<kType, 1, false>(a, launches, st);
}

}  // namespace

cudaError_t launch_gn_channel_sums(GnArgs a, cudaStream_t st)
{
    a.splits = 1;
    return launch_chained(gn_bwd_join_kernel, dim3((a.c + kJoin - 1) / kJoin), dim3(kThreads), 0, st, a, 0);
}

// [partial sums][means of the backward pass, or the statistics of a call that keeps none]
size_t gn_workspace_bytes(const eoq_gn_desc_t &d)
{
    return parts_bytes(d.n, d.hw, d.c, d.dtype) + sizeof(float2) * (size_t)d.n * d.groups;
}

static void place(GnArgs &a, int dtype, void *workspace)
{
    a.part = reinterpret_cast<float2 *>(workspace);
    a.means = reinterpret_cast<float2 *>(reinterpret_cast<char *>(workspace) + parts_bytes(a.n, a.hw, a.c, dtype));
}

cudaError_t launch_gn_fwd(GnArgs a, int dtype, void *workspace, int *launches, cudaStream_t st)
{
    place(a, dtype, workspace);
    cudaError_t e;
    if (gn_fused_fwd(a, dtype, &e, launches, st)) return e;
    if (!a.stats) a.stats = a.means;
    switch (dtype) {
        case EOQ_F32: return fwd_of_type<EOQ_F32>(a, launches, st);
        case EOQ_F16: return fwd_of_type<EOQ_F16>(a, launches, st);
        case EOQ_BF16: return fwd_of_type<EOQ_BF16>(a, launches, st);
        default: return fwd_of_type<EOQ_I32>(a, launches, st);
    }
}

cudaError_t launch_gn_bwd(GnArgs a, int dtype, void *workspace, int *launches, cudaStream_t st)
{
    place(a, dtype, workspace);
    cudaError_t e;
    if (gn_fused_bwd(a, dtype, &e, launches, st)) return e;
    switch (dtype) {
        case EOQ_F32: return bwd_of_type<EOQ_F32>(a, launches, st);
        case EOQ_F16: return bwd_of_type<EOQ_F16>(a, launches, st);
        case EOQ_BF16: return bwd_of_type<EOQ_BF16>(a, launches, st);
        default: return bwd_of_type<EOQ_I32>(a, launches, st);
    }
}

}  // namespace eoq
