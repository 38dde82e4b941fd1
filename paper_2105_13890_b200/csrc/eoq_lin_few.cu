// Forward pass of an integer linear layer for a few tokens (up to eight), the form of serving single ones (eoq_lin_fwd):
//   y[t][o] = x_scale[t] w_scale[o] sum over i of x_code[t][i] w_code[o][i]  (+ bias[o]).
//
// Bound: reading the weights, or latency where they are few; a tile of 128 tokens would leave the tensor core's tiles empty and its sums to a second kernel (one token,
// 4096 to 4096: 11.1 us).  Weights go from memory straight into the registers of mma.sync (16 channels by 8 tokens by 32): which bytes of the reduction a thread holds does not matter as long
// as it holds the same ones of weights and tokens, so a thread takes 16 neighbouring bytes of a row and the four threads of a row 64.  A block has 16 channels at a
// time (or more, where the reduction is short), its warps a share of the reduction each; the shares meet in shared memory, exactly.  Every block codes the tokens for
// itself while its first weights are on their way, so that the call is one launch; that is what limits their number.
#include <type_traits>

#include "eoq_lin.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kSteps = 4;           // of 64 bytes of the reduction in flight
constexpr int kTokens = 8, kMostCodes = 16384;   // tokens of a call; codes of all of them
constexpr int kMostShared = kMostCodes + kTokens * 96;

struct FewArgs {
    LinFewArgs l;
    int k_warps;                    // warps that share a reduction (a power of two); the block's others have other channels
    int pitch_s;                    // bytes from token to token in shared memory
};

__device__ __forceinline__ void mma_16x8x32(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// kType: of x, y.  kCode: x is coded here.
template <int kType, bool kCode, int kU>
__global__ void __launch_bounds__(kThreads, 2) lin_few_kernel(const __grid_constant__ FewArgs f)
{
    using E = Elem<kType>;
    const LinFewArgs &a = f.l;
    extern __shared__ __align__(16) uint8_t codes_s[];
    __shared__ int sums_s[kWarps][16][kTokens + 1];
    __shared__ float scales_s[kTokens];
    __shared__ uint32_t tops_s[kWarps];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();   // (a chain of small calls: the next one's launch is most of its time)

    const int warp = warp_index_uniform(), lane = threadIdx.x % 32, g = lane / 4, q = lane % 4;
    const int k_warp = warp % f.k_warps, group = warp / f.k_warps, groups = kWarps / f.k_warps;
    const int steps = ((int)a.pitch + 63) / 64;
    auto channel0 = [&](int unit) { return (unit * groups + group) * 16; };
    // kSteps steps of the warp's, from its j-th on: rows g and g + 8 of the 16 channels
    uint4 w[kSteps][2];
    auto fetch = [&](int unit, int j) {
        const int o = channel0(unit);
        // (rows behind the last one: the last one again; nothing is written for them)
        const int8_t *r0 = a.w_codes + (size_t)min(o + g, a.c_out - 1) * a.pitch, *r1 = a.w_codes + (size_t)min(o + g + 8, a.c_out - 1) * a.pitch;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int k = ((j + s) * f.k_warps + k_warp) * 64 + q * 16;
            const bool in = k < (int)a.pitch;
            w[s][0] = in ? __ldg(reinterpret_cast<const uint4 *>(r0 + k)) : make_uint4(0, 0, 0, 0);
            w[s][1] = in ? __ldg(reinterpret_cast<const uint4 *>(r1 + k)) : make_uint4(0, 0, 0, 0);
        }
    };
    const int units = (a.c_out + 16 * groups - 1) / (16 * groups), mine = (steps - k_warp + f.k_warps - 1) / f.k_warps;
    fetch(blockIdx.x, 0);

    if constexpr (kCode) {
        // a token has a share of the warps
        using S = Span<kType, kU>;
        int tokens = 1;
        while (tokens < a.rows) tokens *= 2;
        const int lanes = kThreads / tokens, token = threadIdx.x / lanes, at_lane = threadIdx.x % lanes, span_groups = (a.c_in + lanes * S::kN - 1) / (lanes * S::kN);
        const char *src = reinterpret_cast<const char *>(a.x) + (size_t)token * a.x_stride * S::kE;
        constexpr int kHold = 2;   // vectors that stay between the look and the coding; of a longer row the others come from the L1 again
        Raw<16> held[kHold];
#pragma unroll
        for (int i = 0; i < kHold; ++i) held[i] = S(i, at_lane, lanes, a.c_in).get(src, token < a.rows);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kHold; ++i) top = raw_top<kType>(held[i], top);
#pragma unroll 4
        for (int i = kHold; i < span_groups; ++i) top = raw_top<kType>(S(i, at_lane, lanes, a.c_in).get(src, token < a.rows), top);
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) tops_s[warp] = top;
        // what lies between the last code and the next piece of 64 bytes
        for (int t = 0; t < a.rows; ++t)
            for (int k = a.c_in + threadIdx.x; k < steps * 64; k += kThreads) codes_s[t * f.pitch_s + k] = 0;
        __syncthreads();
        for (int i = 0; i < lanes / 32; ++i) top = max(top, tops_s[token * (lanes / 32) + i]);
        const float t = __uint_as_float(top);
        const bool fine = finite_top(t);
        const float per = row_per_of(t);
        if (token < a.rows) {
            if (at_lane == 0) {
                scales_s[token] = row_scale_of(t);
                if (!fine && blockIdx.x == 0) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
            }
            auto put = [&](const Raw<16> &r, const S &at) {
                float v[S::kN];
                uint32_t c[S::kN];
                E::to_f32(r, v);
#pragma unroll
                for (int j = 0; j < S::kN; ++j) c[j] = fine ? row_code(v[j], per) : 0u;
                at.put_codes(reinterpret_cast<int8_t *>(codes_s) + token * f.pitch_s, c);
            };
#pragma unroll
            for (int i = 0; i < kHold; ++i) put(held[i], S(i, at_lane, lanes, a.c_in));
#pragma unroll 4
            for (int i = kHold; i < span_groups; ++i) put(S(i, at_lane, lanes, a.c_in).get(src, true), S(i, at_lane, lanes, a.c_in));
        }
    } else {
        for (int t = 0; t < a.rows; ++t)
            for (int k = threadIdx.x * 16; k < steps * 64; k += kThreads * 16) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (k < (int)a.pitch) v = __ldg(reinterpret_cast<const uint4 *>(a.x_codes + (size_t)t * a.pitch + k));
                if (k + 16 > a.c_in) {   // (bytes behind the last code count as nothing)
                    uint32_t *const p[4] = {&v.x, &v.y, &v.z, &v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int left = a.c_in - k - 4 * i;
                        *p[i] = left >= 4 ? *p[i] : left <= 0 ? 0u : *p[i] & ((1u << (8 * left)) - 1u);
                    }
                }
                *reinterpret_cast<uint4 *>(codes_s + t * f.pitch_s + k) = v;
            }
        if ((int)threadIdx.x < a.rows) scales_s[threadIdx.x] = __ldg(a.x_scales + threadIdx.x);
    }
    __syncthreads();

    for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int d[4] = {};
        // 16 neighbouring threads: the channels of a group and token.  The first ones' scales and biases are on their way beside the products.
        auto out_channel = [&](int i) { return (unit * groups + i / 16 / a.rows) * 16 + i % 16; };
        const int o_first = min(out_channel(threadIdx.x), a.c_out - 1);
        const float scale_first = __ldg(a.w_scales + o_first), bias_first = a.bias ? __ldg(a.bias + o_first) : 0.0f;
        for (int j = 0; j < mine;) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (j + s >= mine) break;
                const int k = ((j + s) * f.k_warps + k_warp) * 64 + q * 16;
                int4 x = make_int4(0, 0, 0, 0);
                if (g < a.rows) x = *reinterpret_cast<const int4 *>(codes_s + g * f.pitch_s + k);
                mma_16x8x32(d, w[s][0].x, w[s][1].x, w[s][0].y, w[s][1].y, x.x, x.y);
                mma_16x8x32(d, w[s][0].z, w[s][1].z, w[s][0].w, w[s][1].w, x.z, x.w);
            }
            j += kSteps;
            if (j < mine) fetch(unit, j);
        }
        if (unit + (int)gridDim.x < units) fetch(unit + gridDim.x, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) sums_s[warp][g + (i / 2) * 8][q * 2 + i % 2] = d[i];
        __syncthreads();
        for (int i = threadIdx.x; i < groups * 16 * a.rows; i += kThreads) {
            const int c = i % 16, t = i / 16 % a.rows, gr = i / 16 / a.rows, o = out_channel(i);
            int sum = 0;
            for (int s = 0; s < f.k_warps; ++s) sum += sums_s[gr * f.k_warps + s][c][t];
            if (o < a.c_out) {
                const bool first = i == (int)threadIdx.x;
                const float scale = first ? scale_first : __ldg(a.w_scales + o), bias = first ? bias_first : a.bias ? __ldg(a.bias + o) : 0.0f;
                const float v[1] = {scaled_sum(__int2float_rn(sum), scales_s[t], scale, bias)};
                store_raw(reinterpret_cast<char *>(a.y) + ((size_t)t * a.y_stride + o) * E::kSize, E::from_f32(v));
            }
        }
        __syncthreads();
    }
}

template <int kType, bool kCode, int kU>
cudaError_t launch(const FewArgs &f, int sm_count, cudaStream_t st)
{
    const int per_block = 16 * (kWarps / f.k_warps), units = (f.l.c_out + per_block - 1) / per_block, room = 2 * sm_count;
    return launch_chained(lin_few_kernel<kType, kCode, kU>, dim3(units < room ? units : room), dim3(kThreads), (size_t)f.l.rows * f.pitch_s, st, f);
}

template <int kType>
cudaError_t of_type(const FewArgs &f, int sm_count, cudaStream_t st)
{
    const LinFewArgs &a = f.l;
    if (!a.x) return launch<kType, false, 16>(f, sm_count, st);
    const int u = row_alignment(a.x, a.x_stride, Elem<kType>::kSize);
    if (u == 16) return launch<kType, true, 16>(f, sm_count, st);
    if (u >= 4) return launch<kType, true, 4>(f, sm_count, st);
    return launch<kType, true, kType == EOQ_F32 ? 4 : 2>(f, sm_count, st);
}

// the token's codes, then room that has the tokens begin 16 bytes off one another in the banks
int shared_pitch(int pitch) { return (pitch + 63) / 64 * 64 + 16; }

}  // namespace

// Up to eight tokens of 16,384 values together.  Eight of 2048 values to 1000 channels take 5.1 us here and 6.8 through the tiles of the large form, four of 4096 to 4096 8.9 and
// 11.6; eight of 4096 to 16,384 take 24 and 18, because every block codes 32,768 values in front of its products.
bool lin_few_fits(size_t rows, int c_in)
{
    static_assert(kMostShared <= 48 * 1024, "no opt-in");
    return rows <= kTokens && rows * c_in <= kMostCodes;
}

cudaError_t launch_lin_few(const LinFewArgs &a, int dtype, int sm_count, cudaStream_t st)
{
    FewArgs f;
    f.l = a;
    f.pitch_s = shared_pitch((int)a.pitch);
    const int steps = ((int)a.pitch + 63) / 64;
    f.k_warps = 1;
    while (f.k_warps < kWarps && f.k_warps * 2 <= steps) f.k_warps *= 2;
    if (dtype == EOQ_F32) return of_type<EOQ_F32>(f, sm_count, st);
    if (dtype == EOQ_F16) return of_type<EOQ_F16>(f, sm_count, st);
    return of_type<EOQ_BF16>(f, sm_count, st);
}

}  // namespace eoq
