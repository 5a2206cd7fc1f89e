// State cache: states in 8 bits with a scale for each block of cells and
// channel (formulas in octree_nca.h).
#include <algorithm>

#include "launch.h"

namespace octnca {

namespace {

constexpr float kTiny = 0x1p-100f;   // the smallest magnitude that sets a scale

template <typename T> struct Quad;   // four channels of a cell as stored
template <> struct Quad<float> {
    using Raw = uint4;
    static __device__ __forceinline__ void unpack(const Raw &v, float *x) {
        Storage<float>::unpack(v, x);
    }
    static __device__ __forceinline__ Raw pack(const float *x) { return Storage<float>::pack(x); }
};
template <> struct Quad<__half> {
    using Raw = uint2;
    static __device__ __forceinline__ void unpack(const Raw &v, float *x) {
        Storage<__half>::unpack_pair(v.x, x[0], x[1]);
        Storage<__half>::unpack_pair(v.y, x[2], x[3]);
    }
    static __device__ __forceinline__ Raw pack(const float *x) {
        return make_uint2(Storage<__half>::pack_pair(x[0], x[1]),
                          Storage<__half>::pack_pair(x[2], x[3]));
    }
};

// Factor and scale of a block's channel from a = max(A, 2^-100), and the codes
// of four values (lowest byte first) and back.
struct CodeI8 {
    static __device__ __forceinline__ void scale_of(float a, float &inv, float &scale) {
        inv = 127.0f / a;
        scale = a / 127.0f;
    }
    // a finite |x| is at most a, so |x * inv| <= 127 (1 + 2^-23) rounds to 127 at most
    static __device__ __forceinline__ uint32_t one(float x, float inv) {
        const int c = (int)rintf(x * inv);
        return (uint32_t)(__builtin_isfinite(x) ? c : -128) & 0xffu;
    }
    static __device__ __forceinline__ uint32_t encode(const float *x, const float *inv) {
        return one(x[0], inv[0]) | one(x[1], inv[1]) << 8 | one(x[2], inv[2]) << 16 |
               one(x[3], inv[3]) << 24;
    }
    static __device__ __forceinline__ void decode(uint32_t c, const float *scale, float *x) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int v = (int)(int8_t)(c >> (8 * k));
            x[k] = v == -128 ? __builtin_nanf("") : (float)v * scale[k];
        }
    }
};

struct CodeF8 {
    // a = m 2^e with 1 <= m < 2: a / 2^k <= 448 = 1.75 2^8 from k = e - 8 on if
    // m <= 1.75, else from e - 7; the addition carries into the exponent in the
    // second case.  2^-100 <= a, so both exponents are those of normal numbers.
    static __device__ __forceinline__ void scale_of(float a, float &inv, float &scale) {
        const uint32_t e = (__float_as_uint(a) + 0x1fffffu) >> 23;
        scale = __uint_as_float((e - 8) << 23);
        inv = __uint_as_float((262 - e) << 23);
    }
    static __device__ __forceinline__ uint32_t encode(const float *x, const float *inv) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            y[k] = __builtin_isfinite(x[k]) ? x[k] * inv[k] : __builtin_nanf("");
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
    }
    static __device__ __forceinline__ void decode(uint32_t c, const float *scale, float *x) {
        x[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * scale[0];
        x[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * scale[1];
        x[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * scale[2];
        x[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * scale[3];
    }
};

// Slot of state i; whether it is one of the cache's.
__device__ __forceinline__ bool slot_of(const CacheArgs &a, int i, int64_t &slot) {
    slot = a.slots ? a.slots[i] : a.first + i;
    return slot >= 0 && slot < a.n_slots;
}

// One workgroup per block of cells: the channels' largest magnitudes in LDS,
// then the codes.
template <typename T, int C, typename Code>
__global__ __launch_bounds__(256) void cache_write(CacheArgs a, const T *__restrict__ states) {
    constexpr int kQ = C / 4;
    __shared__ uint32_t top[C];
    using Raw = typename Quad<T>::Raw;
    const int64_t blocks = (a.count + a.block - 1) / a.block;
    const int64_t items = blocks * a.n;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = (int)(item / blocks);
        const int64_t b = item - i * blocks;
        const int64_t left = a.count - b * a.block;
        const int quads = (int)(left < a.block ? left : a.block) * kQ;
        int64_t slot;
        bool keep = slot_of(a, i, slot);
        if (a.slots)
            for (int j = i + 1; j < a.n; ++j) keep = keep && a.slots[j] != slot;
        __syncthreads();
        if (threadIdx.x < C) top[threadIdx.x] = __float_as_uint(kTiny);
        __syncthreads();
        if (!keep) continue;
        const Raw *src = (const Raw *)(states + (i * a.count + b * a.block) * C);
        for (int q = threadIdx.x; q < quads; q += 256) {
            float x[4];
            Quad<T>::unpack(src[q], x);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (__builtin_isfinite(x[k]))
                    atomicMax(&top[q % kQ * 4 + k], __float_as_uint(fabsf(x[k])));
        }
        __syncthreads();
        const int64_t cell = a.from + b * a.block;
        uint32_t *dst = (uint32_t *)(a.codes + (slot * a.cells + cell) * C);
        for (int q = threadIdx.x; q < quads; q += 256) {
            float x[4], inv[4], scale[4];
            Quad<T>::unpack(src[q], x);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                Code::scale_of(__uint_as_float(top[q % kQ * 4 + k]), inv[k], scale[k]);
            dst[q] = Code::encode(x, inv);
        }
        if (threadIdx.x < C) {
            float inv, scale;
            Code::scale_of(__uint_as_float(top[threadIdx.x]), inv, scale);
            a.scales[(slot * a.blocks + cell / a.block) * C + threadIdx.x] = scale;
        }
    }
}

// One thread per four channels of a cell.
template <typename T, int C, typename Code>
__global__ __launch_bounds__(256) void cache_read(CacheArgs a, T *__restrict__ states) {
    constexpr int kQ = C / 4;
    using Raw = typename Quad<T>::Raw;
    const int64_t quads = a.count * kQ;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < quads * a.n;
         at += (int64_t)gridDim.x * 256) {
        const int i = (int)(at / quads);
        const int64_t q = at - i * quads;
        const int64_t cell = a.from + q / kQ;
        int64_t slot;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (slot_of(a, i, slot)) {
            const uint32_t c = ((const uint32_t *)(a.codes + (slot * a.cells + a.from) * C))[q];
            const float4 s = *(const float4 *)(a.scales +
                                               (slot * a.blocks + cell / a.block) * C + q % kQ * 4);
            const float scale[4] = {s.x, s.y, s.z, s.w};
            Code::decode(c, scale, x);
        }
        ((Raw *)(states + i * a.count * C))[q] = Quad<T>::pack(x);
    }
}

constexpr int64_t kMaxGrid = 1 << 22;   // workgroups; the kernels loop over the rest

template <typename T, int C, typename Code>
hipError_t run(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    if (write) {
        const int64_t items = (a.count + a.block - 1) / a.block * a.n;
        cache_write<T, C, Code><<<(unsigned)std::min(items, kMaxGrid), 256, 0, stream>>>(
            a, (const T *)states);
    } else {
        const int64_t items = (a.count * (C / 4) * a.n + 255) / 256;
        cache_read<T, C, Code><<<(unsigned)std::min(items, kMaxGrid), 256, 0, stream>>>(
            a, (T *)states);
    }
    return hipGetLastError();
}

template <typename T, int C>
hipError_t run_code(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    return a.f8 ? run<T, C, CodeF8>(a, write, states, stream)
                : run<T, C, CodeI8>(a, write, states, stream);
}

template <typename T>
hipError_t run_channels(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    switch (a.channels) {
        case 12: return run_code<T, 12>(a, write, states, stream);
        case 16: return run_code<T, 16>(a, write, states, stream);
        case 20: return run_code<T, 20>(a, write, states, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_write(Dtype dt, const CacheArgs &a, const void *states,
                              hipStream_t stream) {
    void *s = const_cast<void *>(states);
    return dt == Dtype::F16 ? run_channels<__half>(a, true, s, stream)
                            : run_channels<float>(a, true, s, stream);
}

hipError_t launch_cache_read(Dtype dt, const CacheArgs &a, void *states, hipStream_t stream) {
    return dt == Dtype::F16 ? run_channels<__half>(a, false, states, stream)
                            : run_channels<float>(a, false, states, stream);
}

}  // namespace octnca
