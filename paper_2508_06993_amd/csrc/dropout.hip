// Dropout whose mask is drawn where it is used (formulas in octree_nca.h).
//
// One pass over memory: 131072 x 4096 bf16 with an addend (3.2 GB) 537 us, 6.0 TB/s;
// 102403 x 517 fp16 gated, rows 520 apart (318 MB), 64 us, 4.9 TB/s.  The generator is
// the 4 x 32 variant because its twenty 32-bit products give four draws, where the fire
// mask's 4 x 64 variant needs eighty for eight: at two bytes an element that would take
// longer than the memory.
#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "values.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;

// a ^ b ^ c in one instruction: bit i of 0x96 is the parity of i's bits.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

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
        c0 = xor3((uint32_t)(q >> 32), c1, k0);
        c1 = (uint32_t)q;
        c2 = xor3((uint32_t)(p >> 32), c3, k1);
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// Elements of a thread, of one row: 32 bytes of an array.
template <typename V> constexpr int kEach = 32 / V::kBytes;

// The elements' draws, from number e on.  A call of the generator gives those of
// four elements from a multiple of four on; where a row starts between (only then),
// one call more is made and the draws move down.
template <int N> __device__ __forceinline__ void draw(uint64_t e, uint64_t counter, uint64_t seed,
                                                      uint32_t *out) {
    uint32_t d[N + 4];
#pragma unroll
    for (int k = 0; k < N; k += 4) philox4x32_10(e / 4 + k / 4, counter, seed, d + k);
    if (e & 3) {
        philox4x32_10(e / 4 + N / 4, counter, seed, d + N);
#pragma unroll
        for (int k = 0; k < N + 2; ++k) {
            const uint32_t here = d[k], after = d[k + 2];
            d[k] = e & 2 ? after : here;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t here = d[k], after = d[k + 1];
            d[k] = e & 1 ? after : here;
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = d[k];
}

// A thread's elements of an array, at any address; `left` of them are in the row.
template <typename V> struct Part {
    using T = typename V::T;
    using At = std::conditional_t<V::kBytes == 4, Words4At4, Words4At2>;
    static constexpr int kN = kEach<V>;
    T v[kN];
    __device__ __forceinline__ void load(const void *p, int64_t at, int64_t left) {
        const T *from = (const T *)p + at;
        if (left >= kN) {
            Words4 w[2] = {((const At *)from)[0], ((const At *)from)[1]};
            __builtin_memcpy(v, w, sizeof(w));
        } else {
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] = from[k < left ? k : 0];
        }
    }
    __device__ __forceinline__ void store(void *p, int64_t at, int64_t left) const {
        T *to = (T *)p + at;
        if (left >= kN) {
            Words4 w[2];
            __builtin_memcpy(w, v, sizeof(w));
            ((At *)to)[0] = w[0];
            ((At *)to)[1] = w[1];
        } else {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                if (k < left) to[k] = v[k];
        }
    }
};

// Workgroup i takes parts 256 i .. of all rows' parts, `parts` to a row.
template <typename V, bool GATE, bool ADD>
__global__ __launch_bounds__(kThreads) void dropout(DropArgs a, int64_t parts, int64_t groups) {
    constexpr int kN = kEach<V>;
    const uint64_t counter = a.index + (a.step ? (uint64_t)*a.step : 0);
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        int64_t row = g * kThreads / parts;
        int64_t part = g * kThreads - row * parts + threadIdx.x;
        if (parts >= kThreads) {   // a workgroup's parts are of two rows at most
            if (part >= parts) part -= parts, ++row;
        } else {
            const uint32_t more = (uint32_t)part / (uint32_t)parts;
            row += more;
            part -= more * (uint32_t)parts;
        }
        if (row >= a.rows) return;
        const int64_t col = part * kN, left = a.cols - col;
        Part<V> x, gate, add, out;
        x.load(a.x, row * a.x_stride + col, left);
        if (GATE) gate.load(a.gate, row * a.gate_stride + col, left);
        if (ADD) add.load(a.add, row * a.add_stride + col, left);
        uint32_t draws[kN];
        draw<kN>((uint64_t)(row * a.cols + col), counter, a.seed, draws);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            bool keep = draws[k] >= a.threshold && a.factor > 0.0f;
            if (GATE) keep = keep && (float)gate.v[k] > 0.0f;
            float y = keep ? (float)x.v[k] * a.factor : 0.0f;
            if (ADD) y += (float)add.v[k];
            out.v[k] = (typename V::T)y;
        }
        out.store(a.out, row * a.out_stride + col, left);
    }
}

template <typename V, bool GATE, bool ADD>
hipError_t run(const DropArgs &a, hipStream_t stream) {
    const int64_t parts = (a.cols + kEach<V> - 1) / kEach<V>;
    const int64_t groups = (a.rows * parts + kThreads - 1) / kThreads;
    dropout<V, GATE, ADD><<<(unsigned)std::min(groups, int64_t(1) << 23), kThreads, 0, stream>>>(
        a, parts, groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int32_t dtype, const DropArgs &args, hipStream_t stream) {
    DropArgs a = args;
    if (a.x_stride == a.cols && a.out_stride == a.cols && (!a.gate || a.gate_stride == a.cols) &&
        (!a.add || a.add_stride == a.cols)) {   // one long row: every part is whole
        a.cols *= a.rows;
        a.rows = 1;
    }
    return with_type(dtype, [&](auto type) {
        using V = decltype(type);
        return a.gate ? a.add ? run<V, true, true>(a, stream) : run<V, true, false>(a, stream)
               : a.add ? run<V, false, true>(a, stream)
                       : run<V, false, false>(a, stream);
    });
}

}  // namespace octnca
