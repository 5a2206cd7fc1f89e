// Gradients of the 4-bit product (formulas in octree_nca.h).
//
// Both are products of the gradient G with a matrix in 4 bits whose values are
// exact in bf16 (a code has two significant bits, a scale is a power of two).  G is
// split into bf16 parts that add up to it: bf16 one, fp16 two, fp32 three.  So every
// product is exact and only the fp32 sums round.
#include <algorithm>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;      // rows and columns of a workgroup's tile of the result
constexpr int kStep = 32;      // of the summed index
constexpr int kPitch = 40;     // of a tile's rows in LDS, bf16 values

typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));

template <typename V> constexpr int kParts = 3;
template <> constexpr int kParts<Values<OCTNCA_F16>> = 2;
template <> constexpr int kParts<Values<OCTNCA_BF16>> = 1;

// part[p] of x, each cut off to bf16's 8 bits (no part overflows, and their signs
// agree): their sum is x, but for bits below bf16's smallest value.  What is not
// finite is its own first part.
template <int PARTS> __device__ __forceinline__ void split(float x, uint16_t *part) {
    const uint32_t u = __float_as_uint(x);
    const bool odd = (u & 0x7f800000u) == 0x7f800000u;
    uint32_t hi = u & 0xffff0000u;
    if (x != x) hi |= 0x00400000u;
    part[0] = (uint16_t)(hi >> 16);
#pragma unroll
    for (int p = 1; p < PARTS; ++p) {
        x = odd ? 0.0f : x - __uint_as_float(hi);
        hi = __float_as_uint(x) & 0xffff0000u;
        part[p] = (uint16_t)(hi >> 16);
    }
}

struct BackwardArgs {
    const void *grad;     // G
    int64_t stride;
    int64_t rows;
    int outs, cols;
    Mx4View q;            // the weights (grad_in) or the inputs (grad_weight)
    void *out;            // grad_in
    int64_t out_stride;
    float *sums;          // grad_weight: [splits][outs][cols], then bias [splits][outs]
    float *bias;          // or null
    int64_t per_split;    // rows of a split (a multiple of kStep)
};

// out[i][j] = sum over c of P[i][c] Q[c][j], Q the values of a matrix in 4 bits.
// WEIGHT: i an output, c a row of G, j a column of the inputs (P = G^T); else i a
// row of G, c an output, j a column of the weights.
template <typename V, bool WEIGHT>
__global__ __launch_bounds__(kThreads) void backward(BackwardArgs b) {
    constexpr int kP = kParts<V>;
    __shared__ __align__(16) uint16_t ps[kP][kTile][kPitch];
    __shared__ __align__(16) uint16_t qs[kTile][kPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i0 = WEIGHT ? (int64_t)blockIdx.y * kTile : (int64_t)blockIdx.x * kTile;
    const int j0 = WEIGHT ? blockIdx.x * kTile : blockIdx.y * kTile;
    const int64_t i_end = WEIGHT ? b.outs : b.rows;
    const int64_t c_begin = WEIGHT ? (int64_t)blockIdx.z * b.per_split : 0;
    const int64_t c_end = WEIGHT ? std::min(b.rows, c_begin + b.per_split) : b.outs;
    const bool sum_bias = WEIGHT && b.bias != nullptr && j0 == 0;
    const auto grad = (const typename V::T *)b.grad;
    v4f32 acc[2][2] = {};
    float bias = 0.0f;
    for (int64_t c0 = c_begin; c0 < c_end; c0 += kStep) {
        if (WEIGHT) {
            // a thread takes a column of G, eight rows of it
            const int64_t i = i0 + lane;
            uint16_t part[8][kP];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t c = c0 + wave * 8 + k;
                const float x = i < i_end && c < c_end ? V::get(grad + c * b.stride + i) : 0.0f;
                bias += x;
                split<kP>(x, part[k]);
            }
#pragma unroll
            for (int p = 0; p < kP; ++p)
#pragma unroll
                for (int k = 0; k < 8; ++k) ps[p][lane][wave * 8 + k] = part[k][p];
        } else {
            const int64_t i = i0 + threadIdx.x / 4;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t c = c0 + threadIdx.x % 4 * 8 + k;
                const float x = i < i_end && c < c_end ? V::get(grad + i * b.stride + c) : 0.0f;
                uint16_t part[kP];
                split<kP>(x, part);
#pragma unroll
                for (int p = 0; p < kP; ++p)
                    ps[p][threadIdx.x / 4][threadIdx.x % 4 * 8 + k] = part[p];
            }
        }
        {
            // a thread takes eight columns of a row of Q
            const int64_t c = c0 + threadIdx.x / 8;
            const int j = j0 + threadIdx.x % 8 * 8, block = j / kMxBlock;
            float v[8] = {};
            if (c < c_end && block < b.q.blocks) {
                const int64_t at = (c / kMxGroup * b.q.blocks + block) * kMxGroup + c % kMxGroup;
                mx4_values(((const uint32_t *)b.q.codes)[at * 4 + j % kMxBlock / 8], v);
                const float scale = mx4_scale_value(b.q.scales[at]);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= scale;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                qs[threadIdx.x % 8 * 8 + k][threadIdx.x / 8] =
                    (uint16_t)(__float_as_uint(v[k]) >> 16);
        }
        __syncthreads();
        v8bf16 q[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
            q[t] = *(const v8bf16 *)&qs[wave / 2 * 32 + t * 16 + lane % 16][lane / 16 * 8];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = kP - 1; p >= 0; --p) {
                const v8bf16 g =
                    *(const v8bf16 *)&ps[p][wave % 2 * 32 + s * 16 + lane % 16][lane / 16 * 8];
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    acc[s][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t], g, acc[s][t], 0, 0, 0);
            }
        __syncthreads();
    }
    // a lane has four columns j of row i
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t i = i0 + wave % 2 * 32 + s * 16 + lane % 16;
            const int j = j0 + wave / 2 * 32 + t * 16 + lane / 16 * 4;
            if (i >= i_end) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (j + k >= b.cols) continue;
                if (WEIGHT)
                    b.sums[((int64_t)blockIdx.z * b.outs + i) * b.cols + j + k] = acc[s][t][k];
                else
                    V::put((typename V::T *)b.out + i * b.out_stride + j + k, acc[s][t][k]);
            }
        }
    if (sum_bias) {
        float *sums = (float *)ps;   // every wave has passed the last barrier
        sums[threadIdx.x] = bias;
        __syncthreads();
        if (wave == 0 && i0 + lane < i_end)
            b.bias[(int64_t)blockIdx.z * b.outs + i0 + lane] =
                (sums[lane] + sums[lane + 64]) + (sums[lane + 128] + sums[lane + 192]);
    }
}

// to[e] = sum over the splits, in order
__global__ __launch_bounds__(kThreads) void join(const float *__restrict__ sums, float *to,
                                                 int64_t n, int splits) {
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < n;
         e += (int64_t)gridDim.x * kThreads) {
        double x = 0.0;
        for (int s = 0; s < splits; ++s) x += sums[s * n + e];
        to[e] = (float)x;
    }
}

// Splits of the rows for grad_weight.
int splits_of(int64_t rows, int64_t cols, int64_t outs) {
    const int64_t tiles = ((cols + kTile - 1) / kTile) * ((outs + kTile - 1) / kTile);
    const int64_t most = (rows + 255) / 256;
    return (int)std::max<int64_t>(1, std::min((512 + tiles - 1) / tiles, most));
}

size_t sums_bytes(int64_t splits, int64_t cols, int64_t outs) {
    return (size_t)splits * (size_t)outs * (size_t)(cols + 1) * 4;
}

}  // namespace

size_t mx4_backward_bytes(int64_t rows, int64_t cols, int64_t outs) {
    return std::max<size_t>(16, sums_bytes(splits_of(rows, cols, outs), cols, outs));
}

hipError_t launch_mx4_backward(const octnca_rows &grad_out, const octnca_mx4 &a,
                               const octnca_mx4 &w, const octnca_rows *grad_in, float *grad_weight,
                               float *grad_bias, void *workspace, hipStream_t stream) {
    return with_type(grad_out.dtype, [&](auto type) {
        using V = decltype(type);
        const int64_t rows = a.rows, cols = a.cols, outs = w.rows;
        BackwardArgs b{};
        b.grad = grad_out.data;
        b.stride = grad_out.stride;
        b.rows = rows;
        b.outs = (int)outs;
        b.cols = (int)cols;
        const auto tiles = [](int64_t n) { return (unsigned)((n + kTile - 1) / kTile); };
        if (grad_in && rows) {
            b.q = mx4_view(w);
            b.out = grad_in->data;
            b.out_stride = grad_in->stride;
            backward<V, false><<<dim3(tiles(rows), tiles(cols)), kThreads, 0, stream>>>(b);
        }
        if (grad_weight || grad_bias) {
            const int splits = splits_of(rows, cols, outs);
            b.q = mx4_view(a);
            b.sums = (float *)workspace;
            b.bias = grad_bias ? b.sums + (int64_t)splits * outs * cols : nullptr;
            b.per_split = ((rows + splits - 1) / splits + kStep - 1) / kStep * kStep;
            backward<V, true><<<dim3(grad_weight ? tiles(cols) : 1, tiles(outs), splits), kThreads,
                                0, stream>>>(b);
            const auto blocks = [](int64_t n) {
                return (unsigned)std::min<int64_t>((n + kThreads - 1) / kThreads, 4096);
            };
            if (grad_weight)
                join<<<blocks(outs * cols), kThreads, 0, stream>>>(b.sums, grad_weight, outs * cols,
                                                                   splits);
            if (grad_bias)
                join<<<blocks(outs), kThreads, 0, stream>>>(b.bias, grad_bias, outs, splits);
        }
        return hipGetLastError();
    });
}

}  // namespace octnca
