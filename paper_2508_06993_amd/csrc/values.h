// Rows of fp32, fp16 and bf16 values: one or eight consecutive ones as fp32.
// Internal header (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "octree_nca.h"

namespace octnca {

typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
// 16 bytes at any 2-byte (4-byte) address: one load or store, as global memory takes
// any alignment here.
typedef Words4 Words4At2 __attribute__((aligned(2)));
typedef Words4 Words4At4 __attribute__((aligned(4)));

// Values of type DT (octnca_dtype).  Rounding is to nearest, ties to even.
template <int DT> struct Values;

template <> struct Values<OCTNCA_F32> {
    using T = float;
    static constexpr int kBytes = 4;
    static __device__ __forceinline__ float get(const T *p) { return *p; }
    static __device__ __forceinline__ void put(T *p, float x) { *p = x; }
    // p 16-byte aligned
    static __device__ __forceinline__ void get8(const T *p, float *x) {
        const Words4 a = ((const Words4 *)p)[0], b = ((const Words4 *)p)[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = __uint_as_float(a[k]);
            x[k + 4] = __uint_as_float(b[k]);
        }
    }
    static __device__ __forceinline__ void put8(T *p, const float *x) {
        Words4 a, b;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = __float_as_uint(x[k]);
            b[k] = __float_as_uint(x[k + 4]);
        }
        ((Words4 *)p)[0] = a;
        ((Words4 *)p)[1] = b;
    }
    static __device__ __forceinline__ void put4(T *p, const float *x) {
        Words4 a;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(x[k]);
        *(Words4 *)p = a;
    }
};

// fp16 and bf16: a native 16-bit type each
template <typename H> struct Values16 {
    using T = H;
    static constexpr int kBytes = 2;
    typedef H H4 __attribute__((ext_vector_type(4)));
    typedef H H8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ float get(const T *p) { return (float)*p; }
    static __device__ __forceinline__ void put(T *p, float x) { *p = (T)x; }
    static __device__ __forceinline__ void get8(const T *p, float *x) {
        const H8 a = *(const H8 *)p;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (float)a[k];
    }
    static __device__ __forceinline__ void put8(T *p, const float *x) {
        H8 a;
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = (H)x[k];
        *(H8 *)p = a;
    }
    // p 8-byte aligned
    static __device__ __forceinline__ void put4(T *p, const float *x) {
        H4 a;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = (H)x[k];
        *(H4 *)p = a;
    }
};
template <> struct Values<OCTNCA_F16> : Values16<_Float16> {};
template <> struct Values<OCTNCA_BF16> : Values16<__bf16> {};

// Calls f with the type as a constant.
template <typename F> auto with_type(int32_t dtype, F f) {
    if (dtype == OCTNCA_F32) return f(Values<OCTNCA_F32>());
    if (dtype == OCTNCA_F16) return f(Values<OCTNCA_F16>());
    return f(Values<OCTNCA_BF16>());
}

}  // namespace octnca
