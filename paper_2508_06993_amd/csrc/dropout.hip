// Dropout whose mask is drawn where it is used (formulas in octree_nca.h).
#include <algorithm>

#include "launch.h"
#include "values.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kEach = 8;   // elements of a thread: two calls of the generator

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel Random Numbers: As Easy as
// 1, 2, 3", SC 2011): round multipliers and key increments of its Table 2.
__device__ __forceinline__ void philox4x32_10(uint64_t c01, uint64_t c23, uint64_t key,
                                              uint32_t *out) {
    uint32_t c0 = (uint32_t)c01, c1 = (uint32_t)(c01 >> 32);
    uint32_t c2 = (uint32_t)c23, c3 = (uint32_t)(c23 >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

template <typename V>
__global__ __launch_bounds__(kThreads) void dropout(DropArgs a) {
    using T = typename V::T;
    const int64_t n = a.rows * a.cols;
    const uint64_t counter = a.index + (a.step ? (uint64_t)*a.step : 0);
    for (int64_t e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kEach; e < n;
         e += (int64_t)gridDim.x * kThreads * kEach) {
        uint32_t draws[kEach];
        philox4x32_10((uint64_t)e / 4, counter, a.seed, draws);
        philox4x32_10((uint64_t)e / 4 + 1, counter, a.seed, draws + 4);
        int64_t row = e / a.cols, col = e - row * a.cols;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (e + k < n) {
                bool keep = draws[k] >= a.threshold && a.factor > 0.0f;
                if (a.gate)
                    keep = keep && V::get((const T *)a.gate + row * a.gate_stride + col) > 0.0f;
                float y = keep ? V::get((const T *)a.x + row * a.x_stride + col) * a.factor : 0.0f;
                if (a.add) y += V::get((const T *)a.add + row * a.add_stride + col);
                V::put((T *)a.out + row * a.out_stride + col, y);
            }
            if (++col == a.cols) {
                col = 0;
                ++row;
            }
        }
    }
}

}  // namespace

hipError_t launch_dropout(int32_t dtype, const DropArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto type) {
        const int64_t units = (a.rows * a.cols + kThreads * kEach - 1) / (kThreads * kEach);
        dropout<decltype(type)><<<(unsigned)std::min(units, int64_t(1) << 23), kThreads, 0,
                                  stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace octnca
