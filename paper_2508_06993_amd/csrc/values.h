// Rows of fp32, fp16 and bf16 values: one, four or eight consecutive ones as fp32.
// Internal header (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
    template <bool STREAM = false>
    static __device__ __forceinline__ void put8(T *p, const float *x) {
        Words4 a, b;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = __float_as_uint(x[k]);
            b[k] = __float_as_uint(x[k + 4]);
        }
        ((Words4At4 *)p)[0] = a;
        ((Words4At4 *)p)[1] = b;
    }
    // p 16-byte aligned
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
    template <bool STREAM = false>
    static __device__ __forceinline__ void put8(T *p, const float *x) {
        H8 a;
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = (H)x[k];
        const Words4 w = __builtin_bit_cast(Words4, a);
        if (STREAM)
            __builtin_nontemporal_store(w, (Words4At2 *)p);
        else
            *(Words4At2 *)p = w;
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

// Eight values from column `col` of a row of `cols` >= 8 on, as loaded: where the row
// ends before the eighth they are its last eight, and `down` of them come before
// `col`.
template <typename V> struct Eight {
    typename V::T v[8];
    int down;
    __device__ __forceinline__ void load(const typename V::T *row, int col, int cols) {
        down = col + 8 > cols ? col + 8 - cols : 0;
        using At = std::conditional_t<V::kBytes == 4, Words4At4, Words4At2>;
        const At *from = (const At *)(row + (col - down));
        Words4 w[V::kBytes / 2];
#pragma unroll
        for (int k = 0; k < V::kBytes / 2; ++k) w[k] = from[k];
        __builtin_memcpy(v, w, sizeof(w));
    }
    // x = the values, zeros past the row's end
    __device__ __forceinline__ void values(float *x) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (float)v[k];
        if (!__any(down)) return;
#pragma unroll
        for (int step = 8; step; step /= 2)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float here = x[k], after = k + step < 8 ? x[k + step < 8 ? k + step : k] : 0.0f;
                x[k] = (step == 8 ? down >= 8 : (down & step) != 0) ? after : here;
            }
    }
};

// Stores the first `left` of eight values (all of them, if more).
template <typename V, bool STREAM = false>
__device__ __forceinline__ void store8(typename V::T *to, const float *x, int left) {
    if (left >= 8) {
        V::template put8<STREAM>(to, x);
        return;
    }
    int k = 0;
    typename V::T y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (typename V::T)x[e];
    if (left & 4) {
        __builtin_memcpy(to, y, 4 * sizeof(y[0]));
        k = 4;
    }
    if (left & 2) {
        const typename V::T two[2] = {k ? y[4] : y[0], k ? y[5] : y[1]};
        __builtin_memcpy(to + k, two, sizeof(two));
        k += 2;
    }
    if (left & 1) to[k] = k < 4 ? k ? y[2] : y[0] : k == 4 ? y[4] : y[6];
}

// Stores the first `left` of four values (all of them, if more).
template <typename V>
__device__ __forceinline__ void store4(typename V::T *to, const float *x, int left) {
    typename V::T y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (typename V::T)x[e];
    if (left >= 4) {
        __builtin_memcpy(to, y, sizeof(y));
        return;
    }
    if (left & 2) __builtin_memcpy(to, y, 2 * sizeof(y[0]));
    if (left & 1) to[left - 1] = left == 1 ? y[0] : y[2];
}

// Calls f with the type as a constant.
template <typename F> auto with_type(int32_t dtype, F f) {
    if (dtype == OCTNCA_F32) return f(Values<OCTNCA_F32>());
    if (dtype == OCTNCA_F16) return f(Values<OCTNCA_F16>());
    return f(Values<OCTNCA_BF16>());
}

}  // namespace octnca
