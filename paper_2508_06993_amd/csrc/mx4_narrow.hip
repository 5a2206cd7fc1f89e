// Products of narrow layers: at most 128 columns (four blocks) and 128 outputs, any
// number of rows.  Bound by memory, so the weights stay in registers and the rows
// go through once; with values as inputs they are quantised on the way, and the codes
// that the backward reads are stored beside the outputs.
#include <algorithm>
#include <type_traits>

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
    bool dense;           // out's rows follow each other
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

// The outputs of a row group whose rows follow each other: through the wave's part of
// LDS, so that a store has 1 KB in a row.  (Of 64 fp16 outputs a lane has two times
// 16 bytes of a row, and a store of one of them 64 bytes of each of sixteen rows.)
template <typename V, int NT>
__device__ __forceinline__ void put_group(const NarrowArgs &b, int64_t group, const v4f32 *acc,
                                          const float *bias, char *stage) {
    using T = typename V::T;
    const int lane = threadIdx.x & 63, outs = (int)b.w.rows;
    T *to = (T *)stage + lane % 16 * outs + lane / 16 * 4;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[k] = acc[t][k] + bias[t * 4 + k];
            if (b.relu && y[k] < 0.0f) y[k] = 0.0f;
        }
        const int n = t * 16 + lane / 16 * 4;
        if (outs % 4 == 0) {
            if (n < outs) V::put4(to + t * 16, y);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n + k < outs) to[t * 16 + k] = (T)y[k];
        }
    }
    lds_fence();
    const int64_t rows = std::min<int64_t>(b.a.rows - group * kMxGroup, kMxGroup);
    const int values = (int)rows * outs;
    using At = std::conditional_t<V::kBytes == 4, Words4At4, Words4At2>;
    constexpr int kEach = 16 / V::kBytes;
    T *out = (T *)b.out + group * kMxGroup * outs;
    for (int at = lane * kEach; at < values; at += 64 * kEach) {
        if (at + kEach <= values) {
            *(At *)(out + at) = *(const Words4 *)((const T *)stage + at);
        } else {
            for (int k = at; k < values; ++k) out[k] = ((const T *)stage)[k];
        }
    }
    lds_fence();
}

// A wave takes four units (a block of a row group each) at a time: 64 / KB rows, the
// next ones being loaded meanwhile.  The matrix instruction multiplies 16 rows of four
// blocks; where rows have fewer, the blocks of other rows are blanked: one instruction
// a row group.  V: type of the values, or int: codes.
template <typename V, int KB, int NT>
__global__ __launch_bounds__(kThreads) void narrow(NarrowArgs b) {
    constexpr bool kValues = !std::is_same<V, int>::value;
    constexpr int kSubs = 4 / KB;   // row groups at a time
    __shared__ Words4 codes[kWaves][64];
    __shared__ uint8_t scales[kWaves][64];
    __shared__ __align__(16) char stage[kWaves][kMxGroup * 16 * NT * 4];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool pair = NT > 1 && b.out_dtype != OCTNCA_F32 && !b.dense;

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
    const int64_t all = (int64_t)gridDim.x * kWaves;
    Eight<std::conditional_t<kValues, V, Values<OCTNCA_F32>>> raw[kPasses];
    Mx4Operand next;
    // what a turn reads (past the end: what the last one does, used by no one)
    const auto load = [&](int64_t turn) {
        const int64_t u = std::min(turn, turns - 1) * per;
        if constexpr (kValues) {
            const Place p = place_of(u, b.a.blocks);
            const auto x = (const typename V::T *)b.x;
            if (b.cols < 8)
                load_units<V, true>(x, b.x_stride, b.cols, b.a.rows, p, raw);
            else
                load_units<V, false>(x, b.x_stride, b.cols, b.a.rows, p, raw);
        } else {
            const int64_t at = std::min<int64_t>(u + lane / 16, b.units - 1) * kMxGroup + lane % 16;
            next.codes = ((const Words4 *)b.a.codes)[at];
            next.scale = b.a.scales[at];
        }
    };
    int64_t turn = (int64_t)blockIdx.x * kWaves + wave;
    if (turn < turns) load(turn);
    for (; turn < turns; turn += all) {
        const int64_t u = turn * per;
        const bool there = lane / 16 < per && u + lane / 16 < b.units;
        Mx4Operand a;
        if constexpr (kValues) {
            uint32_t c[kPasses], s[kPasses];
            quantise_units(raw, c, s);
#pragma unroll
            for (int k = 0; k < kPasses; ++k)
                ((uint32_t *)codes[wave])[lane % 16 / 4 * 64 + (4 * k + lane / 16) * 4 + lane % 4] = c[k];
            scales[wave][lane % 16 / 4 * 16 + lane % 4 * 4 + lane / 16] = (uint8_t)quad_pick(s);
            load(turn + all);
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
            a = next;
            load(turn + all);
        }
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            const bool mine = there && (KB == 4 || lane / 16 / KB == sub);
            const Mx4Operand only{a.codes & (mine ? ~0u : 0u), mine ? a.scale : 127u};
            v4f32 acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mx4_mfma(w[t], only, v4f32{});
            const int64_t group = turn * kSubs + sub, row = group * kMxGroup + lane % 16;
            if (b.dense) {
                if (group * kMxGroup >= b.a.rows) continue;
                if (b.out_dtype == OCTNCA_F32)
                    put_group<Values<OCTNCA_F32>, NT>(b, group, acc, bias, stage[wave]);
                else if (b.out_dtype == OCTNCA_F16)
                    put_group<Values<OCTNCA_F16>, NT>(b, group, acc, bias, stage[wave]);
                else
                    put_group<Values<OCTNCA_BF16>, NT>(b, group, acc, bias, stage[wave]);
                continue;
            }
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
    // as many workgroups as are resident; us with 2, 3, 4 and 8 a compute unit: 1M x 32
    // fp32 values -> 64 fp16 63, 63, 70, 70, 1M x 64 codes -> 19 fp32 38, 29, 27, 29
    const int64_t grid = std::min<int64_t>((turns + kWaves - 1) / kWaves,
                                           (std::is_same<V, int>::value ? 4 : 3) * device_cus());
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
                       out.stride == w.rows || a.rows == 1,
                       (a.rows + kMxGroup - 1) / kMxGroup * view.blocks};
    if (x == nullptr) return run<int>(b, stream);
    return with_type(x->dtype, [&](auto type) { return run<decltype(type)>(b, stream); });
}

}  // namespace octnca
