// Products of narrow layers: at most 128 columns (four blocks) and 128 outputs, any
// number of rows.  Bound by memory, so the weights stay in registers and the rows
// go through once; with values as inputs they are quantised on the way, and the codes
// that the backward reads are stored beside the outputs.
#include <algorithm>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct NarrowArgs {
    const void *x;        // values, or null: a's codes are there
    int64_t x_stride;
    int cols;
    Mx4View a, w;
    const float *bias;
    bool relu;
    void *out;
    int64_t out_stride;
    int32_t out_dtype;
    int64_t units;
};

// The lane's outputs of one row: NT tiles of four.  kPair: pairs of tiles hold
// eight outputs in a row (the weights' rows are laid out for that).
template <typename V, int NT, bool PAIR>
__device__ __forceinline__ void put_row(const NarrowArgs &b, int64_t row, const v4f32 *acc,
                                        const float *bias) {
    const int q = (threadIdx.x & 63) / 16, outs = (int)b.w.rows;
    typename V::T *to = (typename V::T *)b.out + row * b.out_stride;
    constexpr int kRun = PAIR ? 8 : 4;
#pragma unroll
    for (int r = 0; r < NT * 4 / kRun; ++r) {
        float y[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            y[k] = acc[(r * kRun + k) / 4][k % 4] + bias[r * kRun + k];
            if (b.relu && y[k] < 0.0f) y[k] = 0.0f;
        }
        const int n = r * 4 * kRun + q * kRun;
        if (n >= outs) continue;
        if constexpr (PAIR)
            store8<V>(to + n, y, outs - n);
        else
            store4<V>(to + n, y, outs - n);
    }
}

// A wave takes four units (a block of a row group each) at a time: 16 KB-th of
// 64 / KB rows.  The matrix instruction multiplies 16 rows of four blocks; where rows
// have fewer, the blocks of other rows are blanked: one instruction a row group.
// V: type of the values, or int: codes.
template <typename V, int KB, int NT>
__global__ __launch_bounds__(kThreads) void narrow(NarrowArgs b) {
    constexpr bool kValues = !std::is_same<V, int>::value;
    constexpr int kSubs = 4 / KB;   // row groups at a time
    __shared__ Words4 codes[kWaves][64];
    __shared__ uint8_t scales[kWaves][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool pair = NT > 1 && b.out_dtype != OCTNCA_F32;

    // weights: row r of tile t is output n, so that a lane's four of each tile (or
    // eight of two) are outputs in a row
    Mx4Operand w[NT];
    float bias[4 * NT];
    const int outs = (int)b.w.rows;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = lane % 16;
        const int n = pair ? t / 2 * 32 + r / 4 * 8 + t % 2 * 4 + r % 4 : t * 16 + r;
        const int block = lane / 16 % KB;
        const bool in = n < outs && block < b.w.blocks;
        const int at = in ? (n / kMxGroup * b.w.blocks + block) * kMxGroup + n % kMxGroup : 0;
        w[t].codes = ((const Words4 *)b.w.codes)[at] & (in ? ~0u : 0u);
        w[t].scale = in ? b.w.scales[at] : 127;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int q = lane / 16;
            const int m = pair ? t / 2 * 32 + q * 8 + t % 2 * 4 + k : t * 16 + q * 4 + k;
            bias[t * 4 + k] = b.bias && m < outs ? b.bias[m] : 0.0f;
        }
    }
    // Rows have KB blocks, or three (KB 4): a wave's units are then those of its row
    // group, the fourth blank.
    const int per = KB == 4 ? b.a.blocks : 4;
    const int64_t turns = (b.units + per - 1) / per;
    for (int64_t turn = (int64_t)blockIdx.x * kWaves + wave; turn < turns;
         turn += (int64_t)gridDim.x * kWaves) {
        const int64_t u = turn * per;
        const int64_t unit = std::min<int64_t>(u + lane / 16, b.units - 1);
        const bool there = lane / 16 < per && u + lane / 16 < b.units;
        Mx4Operand a;
        if constexpr (kValues) {
            const Place p = place_of(u, b.a.blocks);
            Eight<V> raw[kPasses];
            const auto x = (const typename V::T *)b.x;
            if (b.cols < 8)
                load_units<V, true>(x, b.x_stride, b.cols, b.a.rows, p, raw);
            else
                load_units<V, false>(x, b.x_stride, b.cols, b.a.rows, p, raw);
            uint32_t c[kPasses], s[kPasses];
            quantise_units(raw, c, s);
#pragma unroll
            for (int k = 0; k < kPasses; ++k)
                ((uint32_t *)codes[wave])[lane % 16 / 4 * 64 + (4 * k + lane / 16) * 4 + lane % 4] = c[k];
            scales[wave][lane % 16 / 4 * 16 + lane % 4 * 4 + lane / 16] = (uint8_t)quad_pick(s);
            lds_fence();
            a.codes = codes[wave][lane];
            a.scale = scales[wave][lane];
            lds_fence();
            const int64_t row = (KB == 4 ? turn : turn * kSubs + lane / 16 / KB) * kMxGroup + lane % 16;
            if (there && row < b.a.rows) {
                ((Words4 *)b.a.codes)[u * kMxGroup + lane] = a.codes;
                b.a.scales[u * kMxGroup + lane] = (uint8_t)a.scale;
            }
        } else {
            const int64_t at = unit * kMxGroup + lane % 16;
            a.codes = ((const Words4 *)b.a.codes)[at];
            a.scale = b.a.scales[at];
        }
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            const bool mine = there && (KB == 4 || lane / 16 / KB == sub);
            const Mx4Operand only{a.codes & (mine ? ~0u : 0u), mine ? a.scale : 127u};
            v4f32 acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mx4_mfma(w[t], only, v4f32{});
            const int64_t row = (turn * kSubs + sub) * kMxGroup + lane % 16;
            if (row >= b.a.rows) continue;
            if (b.out_dtype == OCTNCA_F32)
                put_row<Values<OCTNCA_F32>, NT, false>(b, row, acc, bias);
            else if (b.out_dtype == OCTNCA_F16)
                put_row<Values<OCTNCA_F16>, NT, (NT > 1)>(b, row, acc, bias);
            else
                put_row<Values<OCTNCA_BF16>, NT, (NT > 1)>(b, row, acc, bias);
        }
    }
}

template <typename V, int KB, int NT>
hipError_t run(const NarrowArgs &b, hipStream_t stream) {
    const int64_t per = KB == 4 ? b.a.blocks : 4;
    const int64_t turns = (b.units + per - 1) / per;
    const int64_t grid = std::min<int64_t>((turns + kWaves - 1) / kWaves, 4 * device_cus());
    narrow<V, KB, NT><<<(unsigned)grid, kThreads, 0, stream>>>(b);
    return hipGetLastError();
}

template <typename V, int KB> hipError_t run(const NarrowArgs &b, hipStream_t stream) {
    return b.w.rows <= 16   ? run<V, KB, 1>(b, stream)
           : b.w.rows <= 32 ? run<V, KB, 2>(b, stream)
           : b.w.rows <= 64 ? run<V, KB, 4>(b, stream)
                            : run<V, KB, 8>(b, stream);
}

template <typename V> hipError_t run(const NarrowArgs &b, hipStream_t stream) {
    return b.a.blocks == 1   ? run<V, 1>(b, stream)
           : b.a.blocks == 2 ? run<V, 2>(b, stream)
                             : run<V, 4>(b, stream);
}

}  // namespace

bool mx4_narrow_serves(int64_t cols, int64_t outs) { return cols <= 128 && outs <= 128; }

hipError_t launch_mx4_narrow(const octnca_rows *x, const octnca_mx4 &a, const octnca_mx4 &w,
                             const float *bias, bool relu, const octnca_rows &out,
                             hipStream_t stream) {
    const Mx4View view = mx4_view(a);
    const NarrowArgs b{x ? x->data : nullptr, x ? x->stride : 0, (int)a.cols, view, mx4_view(w),
                       bias, relu, out.data, out.stride, out.dtype,
                       (a.rows + kMxGroup - 1) / kMxGroup * view.blocks};
    if (x == nullptr) return run<int>(b, stream);
    return with_type(x->dtype, [&](auto type) { return run<decltype(type)>(b, stream); });
}

}  // namespace octnca
