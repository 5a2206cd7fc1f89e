// Device-side building blocks of matrices in microscaled 4 bits (octnca_mx4).
// Internal header (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "values.h"

namespace octnca {

constexpr int kMxBlock = 32;      // columns that share a scale
constexpr int kMxGroup = 16;      // rows whose blocks lie together: 256 bytes of codes a block
constexpr uint32_t kMxNan = 255;  // scale byte of a block of NaN

typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef int v8i32 __attribute__((ext_vector_type(8)));

// Scale byte of a block from the largest magnitude's bits.  a = m 2^e with
// 1 <= m < 2: a <= 6 * 2^k = 1.5 * 2^(k + 2) from k = e - 2 on if m <= 1.5, else
// from e - 1; the addition carries into the exponent in the second case.  What is
// not finite has bits of at least 0x7f800000, above those of all numbers.
__device__ __forceinline__ uint32_t mx4_scale(uint32_t top) {
    const int byte = (int)((top + 0x3fffffu) >> 23) - 2;
    return top >= 0x7f800000u ? kMxNan : (uint32_t)(byte > 0 ? byte : 0);
}

// Power of two that takes a block's values to its codes' (0 for a block of NaN).
__device__ __forceinline__ float mx4_inverse(uint32_t scale) {
    return __uint_as_float(scale == kMxNan ? 0u : (254u - scale) << 23);
}

// Value of a scale byte: 2^-127 is a subnormal number.
__device__ __forceinline__ float mx4_scale_value(uint32_t scale) {
    return __uint_as_float(scale == 0 ? 0x00400000u : scale == kMxNan ? 0x7fc00000u : scale << 23);
}

// Codes of eight values times `inverse` (exact: a power of two), the first
// lowest.  A block of NaN has codes 0.
__device__ __forceinline__ uint32_t mx4_codes(const float *x, float inverse) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * inverse, x[1] * inverse, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * inverse, x[3] * inverse, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * inverse, x[5] * inverse, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * inverse, x[7] * inverse, 1.0f, 3);
    return inverse == 0.0f ? 0 : c;
}

// The values of eight codes (without their scale).
__device__ __forceinline__ void mx4_values(uint32_t c, float *x) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const auto v = k == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0)
                       : k == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1)
                       : k == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
        x[2 * k] = v[0];
        x[2 * k + 1] = v[1];
    }
}

// A matrix as the kernels see it.
struct Mx4View {
    uint8_t *codes, *scales;
    int64_t rows;
    int blocks;   // of a row
};
inline Mx4View mx4_view(const octnca_mx4 &m) {
    return Mx4View{(uint8_t *)m.codes, (uint8_t *)m.scales, m.rows,
                   (int)((m.cols + kMxBlock - 1) / kMxBlock)};
}

// A lane's part of an operand: a block of a row.  For the instruction of 16 rows and
// four blocks (128 columns) row lane % 16 of a group, block lane / 16 of the four,
// which lie in memory as one KB.
struct Mx4Operand {
    Words4 codes;
    uint32_t scale;
};

// acc[i] of lane l += sum over 128 columns of a's row 4 (l / 16) + i times b's row
// l % 16.
__device__ __forceinline__ v4f32 mx4_mfma(const Mx4Operand &a, const Mx4Operand &b, v4f32 acc) {
    const v8i32 x = {(int)a.codes[0], (int)a.codes[1], (int)a.codes[2], (int)a.codes[3], 0, 0, 0, 0};
    const v8i32 y = {(int)b.codes[0], (int)b.codes[1], (int)b.codes[2], (int)b.codes[3], 0, 0, 0, 0};
    // 4, 4: both operands e2m1; byte 0 of each lane's scale
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, a.scale, 0, b.scale);
}

// The same with 32 rows each and two blocks (64 columns): lane l of an operand has row
// l % 32, block l / 32; acc[i] of lane l is that of a's row 8 (i / 4) + 4 (l / 32) + i % 4
// and b's row l % 32.  About 1.5 times the rate of the other: with nothing but these
// instructions in a kernel 9.0 PFLOP/s and 5.4 of the other (one wave a SIMD; 7.0 and
// 5.2 with random codes).
typedef float v16f32 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ v16f32 mx4_mfma32(const Mx4Operand &a, const Mx4Operand &b, v16f32 acc) {
    const v8i32 x = {(int)a.codes[0], (int)a.codes[1], (int)a.codes[2], (int)a.codes[3], 0, 0, 0, 0};
    const v8i32 y = {(int)b.codes[0], (int)b.codes[1], (int)b.codes[2], (int)b.codes[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, 4, 4, 0, a.scale, 0, b.scale);
}

// x of lane K of each four lanes; the largest of the four.
template <int K> __device__ __forceinline__ uint32_t quad_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, K * 0x55, 15, 15, true);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 15, 15, true);
    x = x > y ? x : y;
    const uint32_t z = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 15, 15, true);
    return x > z ? x : z;
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

// The values of a wave's units.  NARROW: rows of fewer than eight columns.
template <typename V, bool NARROW>
__device__ __forceinline__ void load_units(const typename V::T *__restrict__ x, int64_t stride,
                                           int cols, int64_t rows, const Place &p,
                                           Eight<V> *raw) {
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
        const int64_t r = p.row + 4 * k;
        const typename V::T *row = x + (r < rows ? r : rows - 1) * stride;
        if (NARROW) {
            raw[k].down = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                raw[k].v[e] = p.col + e < cols ? row[p.col + e] : (typename V::T)0.0f;
        } else {
            raw[k].load(row, p.col, cols);
        }
    }
}

// Codes of a lane's eight values and the scale byte of their block, whose other
// values four lanes in a row have.
template <typename V>
__device__ __forceinline__ void quantise_eight(const Eight<V> &raw, uint32_t &codes,
                                               uint32_t &scale) {
    float v[8];
    raw.values(v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t mag = __float_as_uint(v[e]) & 0x7fffffffu;
        top = top > mag ? top : mag;
    }
    scale = mx4_scale(quad_max(top));
    codes = mx4_codes(v, mx4_inverse(scale));
}
template <typename V>
__device__ __forceinline__ void quantise_units(const Eight<V> *raw, uint32_t *codes,
                                               uint32_t *scale) {
#pragma unroll
    for (int k = 0; k < kPasses; ++k) quantise_eight(raw[k], codes[k], scale[k]);
}

// Entry q of four for lane q of each four lanes (selects of values: an index would
// put the array into memory).
__device__ __forceinline__ uint32_t quad_pick(const uint32_t *x) {
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    const uint32_t even = threadIdx.x & 2 ? x2 : x0, odd = threadIdx.x & 2 ? x3 : x1;
    return threadIdx.x & 1 ? odd : even;
}

// Orders a wave's own LDS accesses (a wave runs them in order; the compiler must
// too).
__device__ __forceinline__ void lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace octnca
