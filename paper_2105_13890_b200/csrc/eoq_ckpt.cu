// A tensor in 8 bits and back (eoq_ckpt_save, eoq_ckpt_load): the scale quantizer of arXiv 2105.13890, Sec. 3.2.2, with a step per
// block of 32 neighbouring columns instead of one for the tensor, chosen so that nothing clips.  See eoq_block8.cuh for the form.
//
// Both directions are bound by memory (a bf16 element: 2 bytes in, 1 + 1/32 out; 200,704 rows of 128 bf16 there and back: 29 us, 5.3 TB/s).  A block belongs to 32 / kV neighbouring lanes,
// each with kV elements (16 bytes of the wider side); rows are dealt out to thread groups of fixed width, so that no element needs a
// division.  Columns, strides or addresses that rule 16-byte loads out take kV = 1, a lane per element and a warp per block.
#include "eoq_block8.cuh"

namespace eoq {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

struct CkptArgs {
    const void *src;          // save: values; load: codes
    void *dst;                // save: codes; load: values
    uint8_t *exps;
    size_t rows, stride;      // stride of the values, in elements
    int cols, blocks;         // blocks of a row
    int lanes;                // lanes of a row in this launch's chunk
    int slots;                // rows that a thread block works on at a time
    float scale;              // of int32 values: 2^exponent
    DeviceState *dev;
};

template <int kType, int kV, bool kSave>
__global__ void __launch_bounds__(kThreads) ckpt_kernel(const __grid_constant__ CkptArgs a)
{
    constexpr int kLanes = kBlock8 / kV;
    ptx::grid_dep_wait_launch_small();
    const int lane_in_row = blockIdx.y * a.lanes + threadIdx.x % a.lanes, slot = threadIdx.x / a.lanes;
    const int col = lane_in_row * kV;
    const bool mine = slot < a.slots && col < a.cols;
    const int block = lane_in_row / kLanes;
    const size_t step = (size_t)gridDim.x * a.slots;
    constexpr int kE = Elem<kType>::kSize;
    unsigned bad = 0;
    for (size_t r0 = (size_t)blockIdx.x * a.slots; r0 < a.rows; r0 += kUnroll * step) {   // (the same rounds for every lane of a warp)
        if (kSave) {
            Raw<kV * kE> raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const size_t r = r0 + slot + u * step;
                raw[u] = mine && r < a.rows ? load_raw<kV * kE>(reinterpret_cast<const char *>(a.src) + (r * a.stride + col) * kE) : zero_raw<kV * kE>();
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const size_t r = r0 + slot + u * step;
                float v[kV], m = 0.0f;
                Elem<kType>::to_f32(raw[u], v);
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    if (kType == EOQ_I32) v[i] *= a.scale;
                    m = max_abs(m, v[i]);
                }
                m = lanes_max_abs<kLanes>(m);
                const int s = block_exp(m);
                uint32_t w[(kV + 3) / 4];
                block_codes(v, s, w);
                if (mine && r < a.rows) {
                    Raw<kV> out;
#pragma unroll
                    for (int i = 0; i < (kV + 3) / 4; ++i) set_word(out, i, w[i]);
                    store_raw(reinterpret_cast<int8_t *>(a.dst) + r * a.cols + col, out);
                    if (lane_in_row % kLanes == 0) a.exps[r * a.blocks + block] = (uint8_t)s;
                    bad |= s == 255;
                }
            }
        } else {
            Raw<kV> raw[kUnroll];
            int s[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const size_t r = r0 + slot + u * step;
                const bool in = mine && r < a.rows;
                raw[u] = in ? load_raw<kV>(reinterpret_cast<const int8_t *>(a.src) + r * a.cols + col) : zero_raw<kV>();
                s[u] = in ? __ldg(a.exps + r * a.blocks + block) : 1;
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const size_t r = r0 + slot + u * step;
                if (!mine || r >= a.rows) continue;
                float v[kV];
                block_values(raw[u], s[u], v);
                if (kType == EOQ_F16) {
                    // a code may stand for a value just above the largest fp16 number: it reads back as that number
                    if (s[u] != 255)
#pragma unroll
                        for (int i = 0; i < kV; ++i) v[i] = fminf(fmaxf(v[i], -65504.0f), 65504.0f);
                }
                if constexpr (kType != EOQ_I32)
                    store_raw(reinterpret_cast<char *>(a.dst) + (r * a.stride + col) * kE, Elem<kType>::from_f32(v));
            }
        }
    }
    if (kSave && bad) atomicOr(&a.dev->status, EOQ_DEV_NONFINITE);
}

template <int kType, int kV, bool kSave>
cudaError_t launch(CkptArgs a, int sm_count, cudaStream_t st)
{
    constexpr int kLanes = kBlock8 / kV;
    // A whole number of blocks and of warps' worth of rows: lanes of a block never straddle a warp.
    const int row_lanes = a.blocks * kLanes;
    const int chunks = (row_lanes + kThreads - 1) / kThreads;
    a.lanes = ((a.blocks + chunks - 1) / chunks) * kLanes;
    a.slots = kThreads / a.lanes;
    const size_t rounds = (a.rows + (size_t)a.slots * kUnroll - 1) / ((size_t)a.slots * kUnroll);
    const size_t cap = ((size_t)sm_count * 8 + chunks - 1) / chunks;
    const dim3 grid((unsigned)(rounds < cap ? rounds : cap), (unsigned)chunks);
    return launch_chained(ckpt_kernel<kType, kV, kSave>, grid, dim3(kThreads), 0, st, a);
}

template <bool kSave>
cudaError_t dispatch(CkptArgs a, int dtype, const void *values, const void *codes, int sm_count, cudaStream_t st)
{
    const int per16 = dtype == EOQ_F32 || dtype == EOQ_I32 ? 4 : 8;
    a.blocks = (a.cols + kBlock8 - 1) / kBlock8;
    const bool wide = a.cols % per16 == 0 && a.stride % per16 == 0 && reinterpret_cast<uintptr_t>(values) % 16 == 0 &&
                      reinterpret_cast<uintptr_t>(codes) % per16 == 0;
    if (a.stride == (size_t)a.cols && a.cols % kBlock8 == 0) {   // one row of blocks after the other: no row ends inside a block
        a.rows *= a.blocks;
        a.cols = kBlock8;
        a.stride = kBlock8;
        a.blocks = 1;
    }
    switch (dtype) {
        case EOQ_F32: return wide ? launch<EOQ_F32, 4, kSave>(a, sm_count, st) : launch<EOQ_F32, 1, kSave>(a, sm_count, st);
        case EOQ_F16: return wide ? launch<EOQ_F16, 8, kSave>(a, sm_count, st) : launch<EOQ_F16, 1, kSave>(a, sm_count, st);
        case EOQ_BF16: return wide ? launch<EOQ_BF16, 8, kSave>(a, sm_count, st) : launch<EOQ_BF16, 1, kSave>(a, sm_count, st);
        default: break;
    }
    if constexpr (kSave)
        if (dtype == EOQ_I32) return wide ? launch<EOQ_I32, 4, kSave>(a, sm_count, st) : launch<EOQ_I32, 1, kSave>(a, sm_count, st);
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_ckpt_save(const void *src, int dtype, int src_exp, size_t rows, int cols, size_t stride, int8_t *codes, uint8_t *exps,
                             DeviceState *dev, int sm_count, cudaStream_t st)
{
    CkptArgs a{src, codes, exps, rows, stride, cols, 0, 0, 0, ldexpf(1.0f, src_exp), dev};
    return dispatch<true>(a, dtype, src, codes, sm_count, st);
}

cudaError_t launch_ckpt_load(const int8_t *codes, const uint8_t *exps, size_t rows, int cols, void *dst, int dtype, size_t stride,
                             DeviceState *dev, int sm_count, cudaStream_t st)
{
    CkptArgs a{codes, dst, const_cast<uint8_t *>(exps), rows, stride, cols, 0, 0, 0, 1.0f, dev};
    return dispatch<false>(a, dtype, dst, codes, sm_count, st);
}

}  // namespace eoq
