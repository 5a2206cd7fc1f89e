// Gradients of the 4-bit product (formulas in octree_nca.h).
//
// Both are products of the gradient G with a matrix in 4 bits whose values are
// exact in bf16 (a code has two significant bits, a scale is a power of two).  G is
// split into bf16 parts that add up to it: bf16 one, fp16 two, fp32 three.  So every
// product is exact and only the fp32 sums round; the split costs two or three times
// the matrix instructions.
//
// Wide layers are bound by the matrix cores and by what feeds them: 8192 x 4096 <- 4096
// in bf16 takes 289 us for grad_in and 333 for grad_weight under the profiler, 561 in
// all without (980 TFLOP/s; a library's bf16 product of 8192^3 reaches 1340).
// Both operands need the summed index along the rows of LDS tiles, so they are
// written row by row and read transposed.  What took it from 6069 us: transposed reads
// and tiles of 256 x 256 (802), no use of a loaded value before the products that
// cover its way (724), 32 x 32 instructions and the work for LDS between them (592),
// codes to bf16 with their scale in one instruction (551 to 561).
// Narrow layers are bound by memory: one pass over G gives all three.  320 x 320
// cells, 32 <- 64 in fp32 (41 MB): 16.6 us and 3.9 for joining the splits; as two
// passes on tiles it was 46, 27 and 6.
#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kStep = 32;      // of the summed index: the matrix instruction's
constexpr int kPad = 16;       // values after a row of a tile in LDS: four rows of 32 bytes are
                               // read at once, from different banks

typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));

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
    bool whole;           // G's rows have 8 n values
    Mx4View q;            // the weights (grad_in) or the inputs (grad_weight)
    void *out;            // grad_in, or grad_weight's sums [splits][outs][cols] or null
    int64_t out_stride;
    float *bias;          // sums [splits][outs], or null
    int64_t per_split;    // rows of a split (a multiple of kStep)
    int i_tiles, j_tiles; // of the result
};

// A tile of bf16 values in LDS, the summed index along the rows: the operand of 16
// columns from `col` on.  Lane l gets column l % 16, eight rows from 8 (l / 16) on:
// each read hands four rows of sixteen columns out to sixteen lanes, transposed.
template <int PITCH>
__device__ __forceinline__ v8bf16 read_columns(const uint16_t *tile, int col) {
    typedef __attribute__((address_space(3))) v4i16 *Lds;
    const int lane = threadIdx.x & 63;
    const uint16_t *at = tile + (lane / 16 * 8 + lane % 16 / 4) * PITCH + col + lane % 4 * 4;
    const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
    const v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * PITCH));
    return __builtin_bit_cast(v8bf16, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The same for 32 columns and 16 rows from `row` on (an operand of the 32 x 32
// instruction): lane l gets column l % 32, rows 8 (l / 32) .. + 7.  SWAP: the second
// and third four of each sixteen columns change places.
template <int PITCH, bool SWAP>
__device__ __forceinline__ v8bf16 read_columns32(const uint16_t *tile, int row, int col) {
    typedef __attribute__((address_space(3))) v4i16 *Lds;
    const int lane = threadIdx.x & 63;
    const int four = SWAP ? (lane & 1) * 2 + (lane >> 1 & 1) : lane & 3;
    const uint16_t *at = tile + (row + lane / 32 * 8 + lane % 16 / 4) * PITCH + col +
                         lane % 32 / 16 * 16 + four * 4;
    const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
    const v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * PITCH));
    return __builtin_bit_cast(v8bf16, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Eight values of G as loaded, ahead of their use.  WHOLE: rows of a multiple of eight
// columns, so that all eight lie in a row or none.
template <typename V, bool WHOLE> struct Raw8 {
    using T = typename V::T;
    using At = std::conditional_t<V::kBytes == 4, Words4At4, Words4At2>;
    Words4 w[V::kBytes / 2];
    bool in;     // whether they count; applied with their use, no wait before
    int down;    // so many of them come before the first
    // Columns col .. col + 7 of a row of `end` (zeros past it, and everywhere where
    // `row_in` is false; the row can be read all the same).  No branches but for rows of
    // fewer than eight: what lies outside is read from the row's other columns.
    __device__ __forceinline__ void load(const T *row, int64_t col, int64_t end, bool row_in) {
        in = row_in && col < end;
        if (!WHOLE && end < 8) {
            T x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[k] = col + k < end ? row[col + k] : (T)0.0f;
            __builtin_memcpy(w, x, sizeof(w));
            down = 0;
            return;
        }
        const int64_t at = col + 8 <= end ? col : WHOLE ? 0 : end - 8;
        down = !WHOLE && col < end ? (int)(col - at) : 0;
        const At *from = (const At *)(row + at);
#pragma unroll
        for (int k = 0; k < V::kBytes / 2; ++k) w[k] = from[k];
    }
    // Moves the values down to their places.
    __device__ __forceinline__ void settle() {
        if (WHOLE || !__any(down)) return;
        T v[8];
        __builtin_memcpy(v, w, sizeof(w));
#pragma unroll
        for (int step = 4; step; step /= 2)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const T here = v[k], after = k + step < 8 ? v[k + step < 8 ? k + step : k] : (T)0.0f;
                v[k] = down & step ? after : here;
            }
        __builtin_memcpy(w, v, sizeof(w));
    }
    __device__ __forceinline__ void values(float *x) const {
        T v[8];
        __builtin_memcpy(v, w, sizeof(w));
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = in ? (float)v[k] : 0.0f;
    }
    // part p of the eight, packed
    template <int P> __device__ __forceinline__ void parts(Words4 *out) const {
        if (P == 1) {   // bf16 as it is
            out[0] = w[0] & (in ? ~0u : 0u);
            return;
        }
        float x[8];
        values(x);
        uint16_t part[8][P];
#pragma unroll
        for (int k = 0; k < 8; ++k) split<P>(x[k], part[k]);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                out[p][k] = part[2 * k][p] | (uint32_t)part[2 * k + 1][p] << 16;
    }
};

// Eight codes as bf16 values (exact: a code has two significant bits).
__device__ __forceinline__ Words4 code_values(uint32_t codes, uint32_t scale) {
    const float s = mx4_scale_value(scale);
    Words4 out;
    out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return out;
}

// out[i][j] = sum over c of P[i][c] Q[c][j], Q the values of a matrix in 4 bits.
// WEIGHT: i an output, c a row of G, j a column of the inputs (P = G^T); else i a
// row of G, c an output, j a column of the weights.  A workgroup takes 64 I rows and
// 64 I columns, four waves with a quarter each, U steps at a time.  The next ones are
// loaded during the first half of the products and go to LDS, as bf16 values, during
// the second.
template <typename V, bool WEIGHT, int I, int U, bool WHOLE>
__global__ __launch_bounds__(kThreads) void backward(BackwardArgs b) {
    constexpr int kP = kParts<V>;
    constexpr int kSide = 64 * I;
    constexpr int kPitchP = WEIGHT ? kSide + kPad : kStep + 8;
    constexpr int kRowsP = WEIGHT ? kStep : kSide;
    constexpr int kPitchQ = kSide + kPad;
    constexpr int kLoads = kSide / 64;   // of a thread and side
    // a lane's results of four columns, or of eight for 16-bit types
    using O = std::conditional_t<WEIGHT, Values<OCTNCA_F32>, V>;
    constexpr int kRun = 16 / O::kBytes;
    __shared__ __align__(16) uint16_t ps[2][U][kP][kRowsP * kPitchP];
    __shared__ __align__(16) uint16_t qs[2][U][kStep * kPitchQ];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups next to each other share columns (grad_in), or rows
    const int64_t i0 = (int64_t)(WEIGHT ? blockIdx.x / b.j_tiles : blockIdx.x % b.i_tiles) * kSide;
    const int j0 = (int)(WEIGHT ? blockIdx.x % b.j_tiles : blockIdx.x / b.i_tiles) * kSide;
    const int64_t i_end = WEIGHT ? b.outs : b.rows;
    const int64_t c_begin = WEIGHT ? (int64_t)blockIdx.y * b.per_split : 0;
    const int64_t c_end = WEIGHT ? std::min(b.rows, c_begin + b.per_split) : b.outs;
    const bool sum_bias = WEIGHT && b.bias != nullptr && j0 == 0;
    const auto grad = (const typename V::T *)b.grad;

    Raw8<V, WHOLE> p[U][kLoads];
    uint32_t codes[U][kLoads], scales[U][kLoads];
    bool codes_in[U][kLoads];
    // where a thread's part k of P lies: row and first column of the tile
    const auto p_row = [&](int k) {
        return WEIGHT ? (threadIdx.x + k * kThreads) / (kSide / 8) : threadIdx.x / 4 + k * 64;
    };
    const auto p_col = [&](int k) {
        return WEIGHT ? (threadIdx.x + k * kThreads) % (kSide / 8) * 8 : threadIdx.x % 4 * 8;
    };
    // Piece x of what is loaded: a part of P, or a block of a row group of Q
    constexpr int kPieces = 2 * U * kLoads;
    const auto load = [&](int64_t from, int x) {
        const int u = x / (2 * kLoads), k = x % kLoads;
        const int64_t c0 = from + u * kStep;
        if (x % (2 * kLoads) < kLoads) {
            const int64_t row = (WEIGHT ? c0 : i0) + p_row(k), rows = WEIGHT ? c_end : i_end;
            p[u][k].load(grad + std::min(row, rows - 1) * b.stride,
                                       (WEIGHT ? i0 : c0) + p_col(k), WEIGHT ? i_end : c_end,
                                       row < rows);
        } else {
            const int unit = k * 4 + wave, block = j0 / kMxBlock + unit / 2;
            const int64_t c = c0 + unit % 2 * kMxGroup + lane / 4;
            codes_in[u][k] = c < c_end && block < b.q.blocks;
            const int64_t row = std::min(c, c_end - 1);
            const int64_t at = (row / kMxGroup * b.q.blocks + std::min(block, b.q.blocks - 1)) *
                                   kMxGroup + row % kMxGroup;
            codes[u][k] = ((const uint32_t *)b.q.codes)[at * 4 + lane % 4];
            scales[u][k] = b.q.scales[at];
        }
    };
    float bias[8] = {};
    const auto store = [&](int buffer, int x) {
        const int u = x / (2 * kLoads), k = x % kLoads;
        if (x % (2 * kLoads) < kLoads) {
            Words4 part[kP];
            p[u][k].settle();
            p[u][k].template parts<kP>(part);
#pragma unroll
            for (int q = 0; q < kP; ++q)
                *(Words4 *)&ps[buffer][u][q][p_row(k) * kPitchP + p_col(k)] = part[q];
            if (sum_bias) {   // a thread's parts are of the same eight columns
                float y[8];
                p[u][k].values(y);
#pragma unroll
                for (int e = 0; e < 8; ++e) bias[e] += y[e];
            }
        } else {
            const int unit = k * 4 + wave;
            *(Words4 *)&qs[buffer][u][(unit % 2 * kMxGroup + lane / 4) * kPitchQ +
                                      unit / 2 * kMxBlock + lane % 4 * 8] =
                code_values(codes_in[u][k] ? codes[u][k] : 0, codes_in[u][k] ? scales[u][k] : 127);
        }
    };

    const int wi = wave % 2 * (32 * I), wj = wave / 2 * (32 * I);
    // A turn: part turn % kP of 32 rows, 16 of the summed index; a pass: I * kP turns.
    constexpr int kTurns = 2 * U * I * kP;
    const auto operand = [&](int buffer, int turn) {
        const int pass = turn / (I * kP), row = wi + turn / kP % I * 32;
        const uint16_t *tile = ps[buffer][pass / 2][turn % kP];
        return WEIGHT ? read_columns32<kPitchP, false>(tile, pass % 2 * 16, row)
                      : *(const v8bf16 *)&tile[(row + lane % 32) * kPitchP + pass % 2 * 16 +
                                               lane / 32 * 8];
    };
    const auto column_operand = [&](int buffer, int pass, int t) {
        return read_columns32<kPitchQ, kRun == 8>(qs[buffer][pass / 2], pass % 2 * 16, wj + t * 32);
    };
    v16f32 acc[I][I] = {};
    if (c_begin < c_end) {
#pragma unroll
        for (int x = 0; x < kPieces; ++x) load(c_begin, x);
#pragma unroll
        for (int x = 0; x < kPieces; ++x) store(0, x);
    }
    int buffer = 0;
    for (int64_t c0 = c_begin; c0 < c_end; c0 += U * kStep, buffer ^= 1) {
        __syncthreads();
        v8bf16 q[2][I], g = operand(buffer, 0);
#pragma unroll
        for (int t = 0; t < I; ++t) q[0][t] = column_operand(buffer, 0, t);
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            const int pass = turn / (I * kP);
            const v8bf16 after = turn + 1 < kTurns ? operand(buffer, turn + 1) : g;
            if (pass + 1 < 2 * U && turn % kP == 0)
                q[(pass + 1) % 2][turn / kP % I] =
                    column_operand(buffer, pass + 1, turn / kP % I);
            __builtin_amdgcn_sched_barrier(0);   // on their way during these
#pragma unroll
            for (int t = 0; t < I; ++t)
                acc[turn / kP % I][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    q[pass % 2][t], g, acc[turn / kP % I][t], 0, 0, 0);
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {   // past the end: zeros, used by no one
                if (x * (kTurns / 2) / kPieces == turn) load(c0 + U * kStep, x);
                if (kTurns / 2 + x * (kTurns / 2) / kPieces == turn) store(buffer ^ 1, x);
            }
            g = after;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // kRun columns of row lane % 32 of each tile in a row, the next ones 2 kRun on
    auto out = (typename O::T *)b.out;
    if (WEIGHT && out) out += (int64_t)blockIdx.y * b.outs * b.cols;
#pragma unroll
    for (int s = 0; s < I; ++s) {
        const int64_t i = i0 + wi + s * 32 + lane % 32;
        if (i >= i_end || (WEIGHT && out == nullptr)) continue;
#pragma unroll
        for (int t = 0; t < I; ++t)
#pragma unroll
            for (int r = 0; r < 16 / kRun; ++r) {
                float y[kRun];
#pragma unroll
                for (int k = 0; k < kRun; ++k) y[k] = acc[s][t][r * kRun + k];
                const int j = j0 + wj + t * 32 + r * 2 * kRun + lane / 32 * kRun;
                if (j >= b.cols) continue;
                if constexpr (kRun == 8)
                    store8<O>(out + i * b.out_stride + j, y, b.cols - j);
                else
                    store4<O>(out + i * b.out_stride + j, y, b.cols - j);
            }
    }
    if (sum_bias) {
        // kSide / 8 threads hold the columns, the others more rows of them
        constexpr int kSets = kThreads / (kSide / 8);
        __shared__ float sums[kSets][kSide];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sums[threadIdx.x / (kSide / 8)][threadIdx.x % (kSide / 8) * 8 + e] = bias[e];
        __syncthreads();
        for (int i = threadIdx.x; i < kSide; i += kThreads) {
            float x = 0.0f;
            for (int k = 0; k < kSets; ++k) x += sums[k][i];
            if (i0 + i < i_end) b.bias[(int64_t)blockIdx.y * b.outs + i0 + i] = x;
        }
    }
}

// Narrow layers: at most 32 NT outputs and 16 KT columns, any number of rows.  One
// pass over G gives all three gradients.  A wave takes 32 rows at a time: G goes from
// memory straight into the operands of grad_in, whose other operand (the weights)
// stays in registers, and through the wave's part of LDS, transposed, into those of
// grad_weight, whose sums stay in registers over all of the wave's rows.
struct NarrowArgs {
    const void *grad;
    int64_t stride;
    int rows, outs, cols;
    Mx4View a, w;
    void *in;             // grad_in or null
    int64_t in_stride;
    bool in_vec;
    float *sums;          // [splits][outs][cols] or null
    float *bias;          // [splits][outs] or null
};

template <typename V, int NT, int KT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void narrow(NarrowArgs b) {
    constexpr int kP = kParts<V>, kWaves = kThreads / 64;
    constexpr int kN = 32 * NT, kK = 16 * KT, kB = KT / 2;   // kB: blocks of a row
    constexpr int kPitchG = kN + kPad, kPitchA = kK + kPad;
    constexpr int kWaveBytes = 2 * kStep * (kP * kPitchG + kPitchA);
    constexpr int kSumBytes = 4 * kN * (kK + 1);
    constexpr int kW = 2 * kN * kPitchA;
    constexpr int kLds = std::max(kWaves * std::max(kWaveBytes, kSumBytes), kW);
    __shared__ __align__(16) char lds[kLds];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // the weights as operands
    v8bf16 w[NT][KT];
    {
        uint16_t *t = (uint16_t *)lds;
        for (int u = wave; u < 2 * NT * kB; u += kWaves) {   // a block of a row group each
            const int group = u / kB, block = u % kB, n = group * kMxGroup + lane / 4;
            uint32_t codes = 0, scale = 127;
            if (n < b.outs && block < b.w.blocks) {
                const int at = (group * b.w.blocks + block) * kMxGroup + lane / 4;
                codes = ((const uint32_t *)b.w.codes)[at * 4 + lane % 4];
                scale = b.w.scales[at];
            }
            *(Words4 *)&t[n * kPitchA + block * kMxBlock + lane % 4 * 8] = code_values(codes, scale);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < KT; ++k) w[n][k] = read_columns<kPitchA>(t + n * 32 * kPitchA, k * 16);
        __syncthreads();
    }
    uint16_t *gs = (uint16_t *)(lds + wave * kWaveBytes);   // [kP][kStep][kPitchG]
    uint16_t *as = gs + kP * kStep * kPitchG;               // [kStep][kPitchA]

    Raw8<V, WHOLE> raw[2][NT];
    uint32_t codes[2][kB], scales[2][kB];
    bool codes_in[2][kB];
    const auto load = [&](int step) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int row = step * kStep + g * kMxGroup + lane % kMxGroup;
            const auto from = (const typename V::T *)b.grad + (int64_t)std::min(row, b.rows - 1) * b.stride;
#pragma unroll
            for (int n = 0; n < NT; ++n)
                raw[g][n].load(from, n * 32 + lane / 16 * 8, b.outs, row < b.rows);
            const int arow = step * kStep + g * kMxGroup + lane / 4;
#pragma unroll
            for (int k = 0; k < kB; ++k) {
                const int r = std::min(arow, b.rows - 1);
                const int64_t at = ((int64_t)(r / kMxGroup) * b.a.blocks + std::min(k, b.a.blocks - 1)) *
                                       kMxGroup + r % kMxGroup;
                codes[g][k] = ((const uint32_t *)b.a.codes)[at * 4 + lane % 4];
                scales[g][k] = b.a.scales[at];
                codes_in[g][k] = arow < b.rows && k < b.a.blocks;
            }
        }
    };
    const __bf16 one = (__bf16)1.0f;
    const v8bf16 ones = {one, one, one, one, one, one, one, one};
    v4f32 acc[2 * NT][KT] = {}, acc_bias[2 * NT] = {};
    const int steps = (b.rows + kStep - 1) / kStep, all = gridDim.x * kWaves;
    int step = blockIdx.x * kWaves + wave;
    if (step < steps) load(step);
    for (; step < steps; step += all) {
        // this step's operands, in registers and LDS
        Words4 part[2][NT][kP];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                raw[g][n].settle();
                raw[g][n].template parts<kP>(part[g][n]);
#pragma unroll
                for (int p = 0; p < kP; ++p)
                    *(Words4 *)&gs[(p * kStep + g * kMxGroup + lane % 16) * kPitchG + n * 32 +
                                   lane / 16 * 8] = part[g][n][p];
            }
#pragma unroll
            for (int k = 0; k < kB; ++k)
                *(Words4 *)&as[(g * kMxGroup + lane / 4) * kPitchA + k * kMxBlock + lane % 4 * 8] =
                    code_values(codes_in[g][k] ? codes[g][k] : 0, codes_in[g][k] ? scales[g][k] : 127);
        }
        load(step + all);   // past the end: zeros, used by no one
        if (b.in) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int row = step * kStep + g * kMxGroup + lane % kMxGroup;
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    v4f32 sum = {};
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = kP - 1; p >= 0; --p)
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                w[n][k], __builtin_bit_cast(v8bf16, part[g][n][p]), sum, 0, 0, 0);
                    const int j = k * 16 + lane / 16 * 4;
                    auto to = (typename V::T *)b.in + row * b.in_stride + j;
                    const float y[4] = {sum[0], sum[1], sum[2], sum[3]};
                    if (b.in_vec) {
                        if (row < b.rows && j < b.cols) V::put4(to, y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (row < b.rows && j + e < b.cols) V::put(to + e, y[e]);
                    }
                }
            }
        }
        lds_fence();
        if (b.sums || b.bias) {
            v8bf16 q[KT];
#pragma unroll
            for (int k = 0; k < KT; ++k) q[k] = read_columns<kPitchA>(as, k * 16);
#pragma unroll
            for (int n = 0; n < 2 * NT; ++n)
#pragma unroll
                for (int p = kP - 1; p >= 0; --p) {
                    const v8bf16 g = read_columns<kPitchG>(gs + p * kStep * kPitchG, n * 16);
#pragma unroll
                    for (int k = 0; k < KT; ++k)
                        acc[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[k], g, acc[n][k], 0, 0, 0);
                    acc_bias[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, g, acc_bias[n], 0, 0, 0);
                }
        }
        lds_fence();
    }
    if (!b.sums && !b.bias) return;
    // the waves' sums, [wave][kN][kK], then their biases [wave][kN]
    __syncthreads();
    float *sums = (float *)lds, *bias = sums + kWaves * kN * kK;
#pragma unroll
    for (int n = 0; n < 2 * NT; ++n) {
#pragma unroll
        for (int k = 0; k < KT; ++k)
            *(v4f32 *)&sums[(wave * kN + n * 16 + lane % 16) * kK + k * 16 + lane / 16 * 4] = acc[n][k];
        if (lane < 16) bias[wave * kN + n * 16 + lane] = acc_bias[n][0];
    }
    __syncthreads();
    if (b.sums)
        for (int e = threadIdx.x; e < kN * kK; e += kThreads) {
            float x = sums[e];
            for (int v = 1; v < kWaves; ++v) x += sums[v * kN * kK + e];
            const int n = e / kK, k = e % kK;
            if (n < b.outs && k < b.cols)
                b.sums[((int64_t)blockIdx.x * b.outs + n) * b.cols + k] = x;
        }
    if (b.bias)
        for (int n = threadIdx.x; n < b.outs; n += kThreads) {
            float x = bias[n];
            for (int v = 1; v < kWaves; ++v) x += bias[v * kN + n];
            b.bias[(int64_t)blockIdx.x * b.outs + n] = x;
        }
}

// to[e] = sum of from[s][e] over the splits s, of two lists.  Many splits: a wave takes
// every kJoin-th split of 64 elements, and the waves' sums are added in order.  us of all
// gradients with this and with a thread for an element: 512 splits (102400 cells 32 <- 64
// fp32) 20 and 140, 29 (13001 x 1030 <- 133 bf16) 53 and 55, 8 (8192 x 1024 <- 1024) 90 and
// 69.  With 8 waves for 16 the first takes 21.
constexpr int kJoin = 16;
struct JoinArgs {
    const float *from[2];
    float *to[2];
    int64_t n[2], blocks;   // blocks: of the first list
    int splits;
};
__global__ __launch_bounds__(64 * kJoin) void join(JoinArgs a) {
    __shared__ double sums[kJoin][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = blockIdx.x >= a.blocks;
    const int64_t n = a.n[which];
    const int64_t e = ((int64_t)blockIdx.x - (which ? a.blocks : 0)) * 64 + lane;
    const float *from = a.from[which];
    double x = 0.0;
    if (e < n)
#pragma unroll 8
        for (int s = wave; s < a.splits; s += kJoin) x += from[s * n + e];
    sums[wave][lane] = x;
    __syncthreads();
    if (wave == 0 && e < n) {
        for (int k = 1; k < kJoin; ++k) x += sums[k][lane];
        a.to[which][e] = (float)x;
    }
}

// Few splits: a thread takes an element.
__global__ __launch_bounds__(kThreads) void join_few(JoinArgs a) {
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < a.n[0] + a.n[1];
         e += (int64_t)gridDim.x * kThreads) {
        const int which = e >= a.n[0];
        const int64_t at = which ? e - a.n[0] : e;
        double x = 0.0;
        for (int s = 0; s < a.splits; ++s) x += a.from[which][s * a.n[which] + at];
        a.to[which][at] = (float)x;
    }
}

constexpr int kLarge = 4, kSmall = 2, kTiny = 1;   // I of the tile sizes

// Sizes of the narrow kernel for a layer; nt 0: it is too wide.
struct Narrow {
    int nt, kt;
};
Narrow narrow_of(int64_t cols, int64_t outs) {
    const int nt = outs <= 32 ? 1 : outs <= 64 ? 2 : 4;
    const int kt = cols <= 32 ? 2 : cols <= 64 ? 4 : 8;
    if (outs > 128 || cols > 128 || nt * kt > 16) return Narrow{0, 0};
    return Narrow{nt, kt};
}

// Splits of the rows for grad_weight: as many as fill the card.  us of all gradients with
// 256, 512 and 1024 workgroups: narrow 1M x 128 <- 32 fp16 130, 130, 142, 1M cells 32 <- 64 fp32
// 107, 88, 92, 102400 cells 19.1, 20.1, 24.7; small tiles, bf16, 8192 x 1024 <- 1024 77, 70,
// 84, 100000 x 300 <- 40 54, 49, 53.
int splits_of(int64_t rows, int64_t cols, int64_t outs) {
    const int64_t most = std::max<int64_t>(1, (rows + 127) / 128);
    if (narrow_of(cols, outs).nt) return (int)std::min<int64_t>(512, most);
    const bool large = mx4_large_tiles(outs, cols);
    const int64_t side = 64 * (large ? kLarge : kSmall);
    const int64_t tiles = ((cols + side - 1) / side) * ((outs + side - 1) / side);
    // two workgroups of small tiles a compute unit; one split where the tiles alone fill
    // the card
    const int64_t want = tiles >= 192 ? 1 : ((large ? 256 : 512) + tiles - 1) / tiles;
    return (int)std::min(want, (most + 1) / 2);
}

size_t sums_bytes(int64_t splits, int64_t cols, int64_t outs) {
    return (size_t)splits * (size_t)outs * (size_t)(cols + 1) * 4;
}

template <typename V, bool WEIGHT, int I>
void run_tiles(BackwardArgs b, int splits, bool products, hipStream_t stream) {
    // two steps at a time where LDS has room for them
    constexpr int U = kParts<V> == 1 ? 2 : 1;
    const auto tiles = [](int64_t n) { return (unsigned)((n + 64 * I - 1) / (64 * I)); };
    b.i_tiles = (int)tiles(WEIGHT ? b.outs : b.rows);
    b.j_tiles = products ? (int)tiles(b.cols) : 1;
    const dim3 grid((unsigned)(b.i_tiles * b.j_tiles), (unsigned)splits);
    if (b.whole)
        backward<V, WEIGHT, I, U, true><<<grid, kThreads, 0, stream>>>(b);
    else
        backward<V, WEIGHT, I, U, false><<<grid, kThreads, 0, stream>>>(b);
}

template <typename V, bool WEIGHT>
void run(const BackwardArgs &b, int splits, bool products, hipStream_t stream) {
    if (mx4_large_tiles(WEIGHT ? b.outs : b.rows, b.cols))
        return run_tiles<V, WEIGHT, kLarge>(b, splits, products, stream);
    // More workgroups of a quarter of the tile, for up to 128 tiles.  us of grad_in with them
    // and with tiles of 128 x 128, bf16: 40 tiles (1000 x 517 <- 1003) 12.5 and 20.4, 64 (1000
    // x 1024 <- 1024) 10.3 and 16.6, 128 (2048 x 1024 <- 1024) 13.9 and 16.6, 192 (2048 x 1500
    // <- 1000) 18.6 and 17.7; fp32, of the last two, 33 and 41, 43.5 and 42.9.
    if constexpr (!WEIGHT)
        if (((b.rows + 127) / 128) * ((b.cols + 127) / 128) <= 128)
            return run_tiles<V, WEIGHT, kTiny>(b, splits, products, stream);
    run_tiles<V, WEIGHT, kSmall>(b, splits, products, stream);
}

template <typename V, int NT, int KT>
void run_narrow(const NarrowArgs &b, bool whole, int splits, hipStream_t stream) {
    if (whole)
        narrow<V, NT, KT, true><<<splits, kThreads, 0, stream>>>(b);
    else
        narrow<V, NT, KT, false><<<splits, kThreads, 0, stream>>>(b);
}

template <typename V>
void run_narrow(const NarrowArgs &b, Narrow size, bool whole, int splits, hipStream_t stream) {
    switch (size.nt * 10 + size.kt) {
        case 12: return run_narrow<V, 1, 2>(b, whole, splits, stream);
        case 14: return run_narrow<V, 1, 4>(b, whole, splits, stream);
        case 18: return run_narrow<V, 1, 8>(b, whole, splits, stream);
        case 22: return run_narrow<V, 2, 2>(b, whole, splits, stream);
        case 24: return run_narrow<V, 2, 4>(b, whole, splits, stream);
        case 28: return run_narrow<V, 2, 8>(b, whole, splits, stream);
        case 42: return run_narrow<V, 4, 2>(b, whole, splits, stream);
        default: return run_narrow<V, 4, 4>(b, whole, splits, stream);
    }
}

}  // namespace

size_t mx4_backward_bytes(int64_t rows, int64_t cols, int64_t outs) {
    // One split's sums are the gradients themselves.  Fewer rows never have more splits,
    // so they need no more.
    const int splits = splits_of(rows, cols, outs);
    return splits == 1 ? 16 : std::max<size_t>(16, sums_bytes(splits, cols, outs));
}

hipError_t launch_mx4_backward(const octnca_rows &grad_out, const octnca_mx4 &a,
                               const octnca_mx4 &w, const octnca_rows *grad_in, float *grad_weight,
                               float *grad_bias, void *workspace, hipStream_t stream) {
    return with_type(grad_out.dtype, [&](auto type) {
        using V = decltype(type);
        const int64_t rows = a.rows, cols = a.cols, outs = w.rows;
        const auto aligned = [](const octnca_rows &x, int64_t to) {
            return (uintptr_t)x.data % to == 0 && x.stride * V::kBytes % to == 0;
        };
        const bool whole = outs % 8 == 0;
        const int splits = splits_of(rows, cols, outs);
        const Narrow size = narrow_of(cols, outs);
        float *sums = (float *)workspace;
        float *bias_sums = sums + (int64_t)splits * outs * cols;
        if (splits == 1) sums = grad_weight, bias_sums = grad_bias;
        if (size.nt) {
            NarrowArgs b{grad_out.data, grad_out.stride, (int)rows, (int)outs, (int)cols,
                         mx4_view(a), mx4_view(w), nullptr, 0, false, grad_weight ? sums : nullptr,
                         grad_bias ? bias_sums : nullptr};
            if (grad_in && rows) {
                b.in = grad_in->data;
                b.in_stride = grad_in->stride;
                b.in_vec = aligned(*grad_in, 4 * V::kBytes) && cols % 4 == 0;
            }
            if (b.in || b.sums || b.bias) run_narrow<V>(b, size, whole, splits, stream);
        } else {
            BackwardArgs b{};
            b.grad = grad_out.data;
            b.stride = grad_out.stride;
            b.rows = rows;
            b.outs = (int)outs;
            b.cols = (int)cols;
            b.whole = whole;
            if (grad_in && rows) {
                b.q = mx4_view(w);
                b.out = grad_in->data;
                b.out_stride = grad_in->stride;
                run<V, false>(b, 1, true, stream);
            }
            if (grad_weight || grad_bias) {
                b.q = mx4_view(a);
                b.out = grad_weight ? sums : nullptr;
                b.out_stride = cols;
                b.bias = grad_bias ? bias_sums : nullptr;
                b.per_split = ((rows + splits - 1) / splits + kStep - 1) / kStep * kStep;
                run<V, true>(b, splits, grad_weight != nullptr, stream);
            }
        }
        if (splits > 1 && (grad_weight || grad_bias)) {
            const int64_t n0 = grad_weight ? outs * cols : 0, n1 = grad_bias ? outs : 0;
            JoinArgs j{{sums, bias_sums}, {grad_weight, grad_bias}, {n0, n1}, (n0 + 63) / 64,
                       splits};
            if (splits > kJoin)
                join<<<(unsigned)(j.blocks + (n1 + 63) / 64), 64 * kJoin, 0, stream>>>(j);
            else
                join_few<<<(unsigned)std::min<int64_t>((n0 + n1 + kThreads - 1) / kThreads, 1 << 14),
                           kThreads, 0, stream>>>(j);
        }
        return hipGetLastError();
    });
}

}  // namespace octnca
