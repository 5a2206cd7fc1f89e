// Matrices in microscaled 4 bits: quantisation and product (formulas and layout
// in octree_nca.h).
#include <algorithm>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 23;

// Eight columns of a row from column `col` on, zeros past the last.  VEC: rows
// start at multiples of 16 bytes.
template <typename V, bool VEC>
__device__ __forceinline__ void load_row8(const typename V::T *row, int col, int cols, float *x) {
    if (VEC && col + 8 <= cols) {
        V::get8(row + col, x);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = col + k < cols ? V::get(row + col + k) : 0.0f;
}

// A wave takes a block of a row group: four lanes a row, eight values each.
template <typename V, bool VEC>
__global__ __launch_bounds__(kThreads) void quantise(const typename V::T *__restrict__ x,
                                                     int64_t stride, int cols, Mx4View m,
                                                     int64_t units) {
    const int lane = threadIdx.x & 63;
    for (int64_t u = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); u < units;
         u += (int64_t)gridDim.x * (kThreads / 64)) {
        const int64_t group = u / m.blocks;
        const int block = (int)(u - group * m.blocks);
        const int64_t row = group * kMxGroup + lane / 4;
        const bool in = row < m.rows;
        float v[8];
        load_row8<V, VEC>(x + (in ? row : m.rows - 1) * stride, block * kMxBlock + lane % 4 * 8,
                          cols, v);
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = std::max(top, __float_as_uint(v[k]) & 0x7fffffffu);
        top = std::max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = std::max(top, (uint32_t)__shfl_xor((int)top, 2));
        const uint32_t scale = mx4_scale(top);
        const uint32_t c = mx4_codes(v, mx4_inverse(scale));
        if (in) {
            ((uint32_t *)m.codes)[u * 64 + lane] = c;
            if (lane % 4 == 0) m.scales[u * kMxGroup + lane / 4] = (uint8_t)scale;
        }
    }
}

template <typename V, bool VEC>
__global__ __launch_bounds__(kThreads) void dequantise(Mx4View m, typename V::T *__restrict__ x,
                                                       int64_t stride, int cols, int64_t units) {
    const int lane = threadIdx.x & 63;
    for (int64_t u = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); u < units;
         u += (int64_t)gridDim.x * (kThreads / 64)) {
        const int64_t group = u / m.blocks;
        const int col = (int)(u - group * m.blocks) * kMxBlock + lane % 4 * 8;
        const int64_t row = group * kMxGroup + lane / 4;
        if (row >= m.rows) continue;
        float v[8];
        mx4_values(((const uint32_t *)m.codes)[u * 64 + lane], v);
        const float scale = mx4_scale_value(m.scales[u * kMxGroup + lane / 4]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
        typename V::T *to = x + row * stride + col;
        if (VEC && col + 8 <= cols) {
            V::put8(to, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (col + k < cols) V::put(to + k, v[k]);
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

bool rows_aligned(const octnca_rows &x, int to) {
    return (uintptr_t)x.data % to == 0 && x.stride * (x.dtype == OCTNCA_F32 ? 4 : 2) % to == 0;
}

}  // namespace

hipError_t launch_mx4_quantise(const octnca_rows &x, const octnca_mx4 &m, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const unsigned grid = (unsigned)std::min((units + 3) / 4, kMaxGrid);
        const auto from = (const typename V::T *)x.data;
        if (rows_aligned(x, 16))
            quantise<V, true><<<grid, kThreads, 0, stream>>>(from, x.stride, (int)m.cols, v, units);
        else
            quantise<V, false><<<grid, kThreads, 0, stream>>>(from, x.stride, (int)m.cols, v, units);
        return hipGetLastError();
    });
}

hipError_t launch_mx4_dequantise(const octnca_mx4 &m, const octnca_rows &x, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const unsigned grid = (unsigned)std::min((units + 3) / 4, kMaxGrid);
        const auto to = (typename V::T *)x.data;
        if (rows_aligned(x, 16))
            dequantise<V, true><<<grid, kThreads, 0, stream>>>(v, to, x.stride, (int)m.cols, units);
        else
            dequantise<V, false><<<grid, kThreads, 0, stream>>>(v, to, x.stride, (int)m.cols, units);
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
