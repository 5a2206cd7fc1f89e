// Matrices in microscaled 4 bits: quantisation and product (formulas and layout
// in octree_nca.h).
#include <algorithm>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 23;

// x of lane K of each four lanes; of the lane's partner in them.
template <int K> __device__ __forceinline__ uint32_t quad_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, K * 0x55, 15, 15, true);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 15, 15, true));
    return std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 15, 15, true));
}

// A unit is a block of a row group, 256 bytes of codes; a wave takes kUnits in a row.
// Four lanes have a block of a row, eight columns each; sixteen the same row of all
// units (with four blocks of a row 256 bytes of fp16 in a row), and a pass of the wave
// four rows of each unit.
constexpr int kUnits = 4, kPasses = 4;
struct Place {
    int64_t unit, row;   // row: of pass 0; of pass k 4 k more
    int col;
};
__device__ __forceinline__ Place place_of(int64_t first, int blocks) {
    const int lane = threadIdx.x & 63, unit = lane % 16 / 4;
    int64_t group = first / blocks;
    int block = (int)(first - group * blocks) + unit;
    if (blocks >= kUnits) {
        if (block >= blocks) block -= blocks, ++group;
    } else {
        group += block / blocks;
        block %= blocks;
    }
    return Place{first + unit, group * kMxGroup + lane / 16, block * kMxBlock + lane % 4 * 8};
}

// NARROW: rows of fewer than eight columns.
template <typename V, bool NARROW>
__global__ __launch_bounds__(kThreads) void quantise(const typename V::T *__restrict__ x,
                                                     int64_t stride, int cols, Mx4View m,
                                                     int64_t units) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t u = ((int64_t)blockIdx.x * (kThreads / 64) + wave) * kUnits; u < units;
         u += (int64_t)gridDim.x * (kThreads / 64) * kUnits) {
        const Place p = place_of(u, m.blocks);
        Eight<V> raw[kPasses];
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const typename V::T *row = x + std::min(p.row + 4 * k, m.rows - 1) * stride;
            if (NARROW) {
                raw[k].down = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    raw[k].v[e] = p.col + e < cols ? row[p.col + e] : (typename V::T)0.0f;
            } else {
                raw[k].load(row, p.col, cols);
            }
        }
        uint32_t scale[kPasses];
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            float v[8];
            raw[k].values(v);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = std::max(top, __float_as_uint(v[e]) & 0x7fffffffu);
            scale[k] = mx4_scale(quad_max(top));
            const uint32_t c = mx4_codes(v, mx4_inverse(scale[k]));
            if (p.row + 4 * k < m.rows)
                ((uint32_t *)m.codes)[p.unit * 64 + (4 * k + lane / 16) * 4 + lane % 4] = c;
        }
        // lane q of a block's four stores the scale of pass q's row
        const int q = lane % 4;
        const uint32_t s = q < 2 ? q == 0 ? scale[0] : scale[1] : q == 2 ? scale[2] : scale[3];
        if (p.row + 4 * q < m.rows)
            m.scales[p.unit * kMxGroup + 4 * q + lane / 16] = (uint8_t)s;
    }
}

template <typename V, bool STREAM>
__global__ __launch_bounds__(kThreads) void dequantise(Mx4View m, typename V::T *__restrict__ x,
                                                       int64_t stride, int cols, int64_t units) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t u = ((int64_t)blockIdx.x * (kThreads / 64) + wave) * kUnits; u < units;
         u += (int64_t)gridDim.x * (kThreads / 64) * kUnits) {
        const Place p = place_of(u, m.blocks);
        const int64_t unit = std::min(p.unit, units - 1);
        uint32_t c[kPasses];
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int64_t at = unit * 64 + (4 * k + lane / 16) * 4;
            if (V::kBytes == 4) {   // fours 4 q and 16 + 4 q: 64 bytes in a row a store
                const uint16_t *from = (const uint16_t *)((const uint32_t *)m.codes + at);
                c[k] = from[lane % 4] | (uint32_t)from[4 + lane % 4] << 16;
            } else {
                c[k] = ((const uint32_t *)m.codes)[at + lane % 4];
            }
        }
        // lane q of a block's four has the scale of pass q's row
        const uint32_t s = m.scales[unit * kMxGroup + lane % 4 * 4 + lane / 16];
        const uint32_t scale[kPasses] = {quad_lane<0>(s), quad_lane<1>(s), quad_lane<2>(s),
                                         quad_lane<3>(s)};
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            float v[8];
            mx4_values(c[k], v);
            const float factor = mx4_scale_value(scale[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            if (p.row + 4 * k >= m.rows) continue;
            typename V::T *row = x + (p.row + 4 * k) * stride;
            if (V::kBytes == 4) {
                const int col = p.col - lane % 4 * 4;
                if (col < cols) store4<V>(row + col, v, cols - col);
                if (col + 16 < cols) store4<V>(row + col + 16, v + 4, cols - col - 16);
            } else if (p.col < cols) {
                store8<V, STREAM>(row + p.col, v, cols - p.col);
            }
        }
    }
}

struct ProductArgs {
    Mx4View a, w;
    const float *bias;   // or null
    bool relu;
    void *out;
    int64_t stride;
    bool vec;            // four outputs of a row from a multiple of four on can be stored at once
};

// Outputs n .. n + 3 of a row.
template <typename V>
__device__ __forceinline__ void store4(const ProductArgs &p, int64_t row, int n, v4f32 acc) {
    const int outs = (int)p.w.rows;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = acc[i] + (p.bias && n + i < outs ? p.bias[n + i] : 0.0f);
        if (p.relu && y[i] < 0.0f) y[i] = 0.0f;
    }
    typename V::T *to = (typename V::T *)p.out + row * p.stride + n;
    if (p.vec && n + 4 <= outs) {
        V::put4(to, y);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < outs) V::put(to + i, y[i]);
    }
}

// A wave takes a row group and kTiles groups of outputs, straight from memory.
constexpr int kTiles = 4;
template <typename V>
__global__ __launch_bounds__(kThreads) void product(ProductArgs p) {
    const int lane = threadIdx.x & 63;
    const int64_t group = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    const int64_t groups = (p.a.rows + kMxGroup - 1) / kMxGroup;
    const int w_groups = (int)((p.w.rows + kMxGroup - 1) / kMxGroup);
    const int tile = blockIdx.y * kTiles;
    if (group >= groups) return;
    v4f32 acc[kTiles] = {};
    for (int k = 0; k < p.a.blocks; k += 4) {
        const Mx4Operand b = mx4_operand(p.a, group, k);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            acc[t] = mx4_mfma(mx4_operand(p.w, std::min(tile + t, w_groups - 1), k), b, acc[t]);
    }
    const int64_t row = group * kMxGroup + lane % kMxGroup;
    if (row >= p.a.rows) return;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        if (tile + t < w_groups)
            store4<V>(p, row, (tile + t) * kMxGroup + lane / kMxGroup * 4, acc[t]);
}

// Whether a matrix is so large (half the last-level cache) that its values are written
// past it.  us through it and past it: 1.2M x 128 fp16 72 and 58, 65536 x 4096 bf16
// 121 and 111.  Not where a store has less than 128 bytes in a row or lines stay half
// written: 600 thousand x 100 fp32 71 and 107, 30000 x 4100 fp16 74 and 89.
bool streams(const octnca_rows &x, int64_t rows, int64_t cols) {
    return rows * cols * (x.dtype == OCTNCA_F32 ? 4 : 2) >= int64_t(1) << 27;
}

bool rows_aligned(const octnca_rows &x, int to) {
    return (uintptr_t)x.data % to == 0 && x.stride * (x.dtype == OCTNCA_F32 ? 4 : 2) % to == 0;
}

}  // namespace

hipError_t launch_mx4_quantise(const octnca_rows &x, const octnca_mx4 &m, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const int64_t grid = (units + kUnits * 4 - 1) / (kUnits * 4);
        const auto from = (const typename V::T *)x.data;
        const unsigned n = (unsigned)std::min(grid, kMaxGrid);
        const auto run = [&](auto kernel) {
            kernel<<<n, kThreads, 0, stream>>>(from, x.stride, (int)m.cols, v, units);
        };
        if (m.cols < 8)
            run(quantise<V, true>);
        else
            run(quantise<V, false>);
        return hipGetLastError();
    });
}

hipError_t launch_mx4_dequantise(const octnca_mx4 &m, const octnca_rows &x, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const int64_t grid = (units + kUnits * 4 - 1) / (kUnits * 4);
        const auto run = [&](auto kernel) {
            kernel<<<(unsigned)std::min(grid, kMaxGrid), kThreads, 0, stream>>>(
                v, (typename V::T *)x.data, x.stride, (int)m.cols, units);
        };
        const bool whole = x.stride == m.cols && m.cols * V::kBytes % 16 == 0 && rows_aligned(x, 16);
        if (V::kBytes == 2 && whole && streams(x, m.rows, m.cols))
            run(dequantise<V, true>);
        else
            run(dequantise<V, false>);
        return hipGetLastError();
    });
}

hipError_t launch_mx4_product(const octnca_mx4 &a, const octnca_mx4 &w, const float *bias,
                              bool relu, const octnca_rows &out, hipStream_t stream) {
    return with_type(out.dtype, [&](auto type) {
        using V = decltype(type);
        const ProductArgs p{mx4_view(a), mx4_view(w), bias, relu, out.data, out.stride,
                            rows_aligned(out, 4 * V::kBytes)};
        const int64_t groups = (a.rows + kMxGroup - 1) / kMxGroup;
        const int64_t tiles = (w.rows + kMxGroup * kTiles - 1) / (kMxGroup * kTiles);
        product<V><<<dim3((unsigned)((groups + 3) / 4), (unsigned)tiles), kThreads, 0, stream>>>(p);
        return hipGetLastError();
    });
}

hipError_t launch_mx4_linear(const octnca_rows &x, const octnca_mx4 &kept, const octnca_mx4 &w,
                             const float *bias, bool relu, const octnca_rows &out,
                             hipStream_t stream) {
    const hipError_t e = launch_mx4_quantise(x, kept, stream);
    return e == hipSuccess ? launch_mx4_product(kept, w, bias, relu, out, stream) : e;
}

}  // namespace octnca
