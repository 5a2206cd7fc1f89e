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

constexpr int kWaves = 4;              // per workgroup, each with blocks of its own
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups along x; the kernels loop over the rest

// Work split of both kernels: a wave takes one block of cells (of one state),
// whose channel quads lie one after the other in memory.  Lane l takes quads l,
// l + kLanes, ..: kLanes is a multiple of the quads per cell, so a lane stays
// with one channel quad, and a pass of the wave is contiguous in memory.
template <int C, int B> struct Split {
    static constexpr int kQ = C / 4;
    static constexpr int kLanes = 64 / kQ * kQ;
    static constexpr int kPasses = (B * kQ + kLanes - 1) / kLanes;
    static constexpr int kPeers = kLanes / kQ;   // lanes of one channel quad
};

// Orders a wave's own LDS accesses (a wave runs them in order; the compiler
// must too).
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Largest of the 16 lanes of a row, in every lane: rotations by 1, 2, 4, 8.
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x121, 15, 15, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x122, 15, 15, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x124, 15, 15, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 15, 15, true)));
    return x;
}

// Largest values (4 channels a lane) over the lanes of one channel quad, in
// each of them: every lane leaves its four in LDS by quad, row r of 16 lanes
// reduces quads r, r + 4, .., and each lane fetches its quad's.
template <int Q, int PEERS>
__device__ __forceinline__ void quad_max(float (*peers)[4], float (*top)[4], float *m) {
    const int lane = threadIdx.x & 63;
    if (lane < Q * PEERS)
        *(float4 *)peers[lane % Q * PEERS + lane / Q] = make_float4(m[0], m[1], m[2], m[3]);
    wave_fence();
    for (int q = lane >> 4; q < Q; q += 4) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = lane & 15; k < PEERS; k += 16) {
            const float4 v = *(const float4 *)peers[q * PEERS + k];
            t = make_float4(fmaxf(t.x, v.x), fmaxf(t.y, v.y), fmaxf(t.z, v.z), fmaxf(t.w, v.w));
        }
        t = make_float4(row_max(t.x), row_max(t.y), row_max(t.z), row_max(t.w));
        if ((lane & 15) == 0) *(float4 *)top[q] = t;
    }
    wave_fence();
    const float4 t = *(const float4 *)top[lane % Q];
    m[0] = t.x, m[1] = t.y, m[2] = t.z, m[3] = t.w;
    wave_fence();   // the next block's maxima come after these reads
}

// Slot of state i; whether it is one of the cache's.
__device__ __forceinline__ bool slot_of(const CacheArgs &a, int i, int64_t &slot) {
    slot = a.slots ? a.slots[i] : a.first + i;
    return slot >= 0 && slot < a.n_slots;
}

// Whether a later entry of `slots` names the same slot (then that one is kept).
__device__ __forceinline__ bool written_later(const CacheArgs &a, int i, int64_t slot) {
    if (!a.slots) return false;
    bool found = false;
    for (int j = i + 1 + (threadIdx.x & 63); j < a.n; j += 64) found |= a.slots[j] == slot;
    return __any(found);
}

// The block's values stay in registers between the maxima and the codes.
template <typename T, int C, int B, typename Code>
__global__ __launch_bounds__(64 * kWaves) void cache_write(CacheArgs a,
                                                           const T *__restrict__ states) {
    using S = Split<C, B>;
    using Raw = typename Quad<T>::Raw;
    __shared__ __align__(16) float peers[kWaves][64][4];
    __shared__ __align__(16) float tops[kWaves][S::kQ][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t blocks = (a.count + B - 1) / B;
    for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
        const T *from = states + (int64_t)i * a.count * C;
        for (int64_t b = (int64_t)blockIdx.x * kWaves + wave; b < blocks;
             b += (int64_t)gridDim.x * kWaves) {
            const int64_t left = a.count - b * B;
            const int quads = lane < S::kLanes ? (int)(left < B ? left : B) * S::kQ : 0;
            const Raw *src = (const Raw *)(from + b * B * C);
            float x[S::kPasses][4];
            float m[4] = {kTiny, kTiny, kTiny, kTiny};
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k) {
                const int q = lane + k * S::kLanes;
                Raw r{};
                if (q < quads) r = src[q];
                Quad<T>::unpack(r, x[k]);
            }
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    m[c] = fmaxf(m[c], __builtin_isfinite(x[k][c]) ? fabsf(x[k][c]) : 0.f);
            quad_max<S::kQ, S::kPeers>(peers[wave], tops[wave], m);
            // the slot is looked up behind the block's loads, which do not need it
            int64_t slot;
            if (!slot_of(a, i, slot) || written_later(a, i, slot)) break;
            int8_t *codes = a.codes + (slot * a.cells + a.from) * C;
            float *scales = a.scales + (slot * a.blocks + a.from / B) * C;
            float inv[4], scale[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) Code::scale_of(m[c], inv[c], scale[c]);
            uint32_t *dst = (uint32_t *)(codes + b * B * C);
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k) {
                const int q = lane + k * S::kLanes;
                if (q < quads) dst[q] = Code::encode(x[k], inv);
            }
            if (lane < S::kQ)
                ((float4 *)(scales + b * C))[lane] =
                    make_float4(scale[0], scale[1], scale[2], scale[3]);
        }
    }
}

template <typename T, int C, int B, typename Code>
__global__ __launch_bounds__(64 * kWaves) void cache_read(CacheArgs a, T *__restrict__ states) {
    using S = Split<C, B>;
    using Raw = typename Quad<T>::Raw;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t blocks = (a.count + B - 1) / B;
    for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
        int64_t slot;
        const bool there = slot_of(a, i, slot);
        T *to = states + (int64_t)i * a.count * C;
        const int8_t *codes = a.codes + (slot * a.cells + a.from) * C;
        const float *scales = a.scales + (slot * a.blocks + a.from / B) * C;
        for (int64_t b = (int64_t)blockIdx.x * kWaves + wave; b < blocks;
             b += (int64_t)gridDim.x * kWaves) {
            const int64_t left = a.count - b * B;
            const int quads = lane < S::kLanes ? (int)(left < B ? left : B) * S::kQ : 0;
            uint32_t code[S::kPasses] = {};
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            if (there) {
                const uint32_t *src = (const uint32_t *)(codes + b * B * C);
                s = ((const float4 *)(scales + b * C))[lane % S::kQ];
#pragma unroll
                for (int k = 0; k < S::kPasses; ++k) {
                    const int q = lane + k * S::kLanes;
                    if (q < quads) code[k] = src[q];
                }
            }
            const float scale[4] = {s.x, s.y, s.z, s.w};
            Raw *dst = (Raw *)(to + b * B * C);
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k) {
                const int q = lane + k * S::kLanes;
                float x[4];
                Code::decode(code[k], scale, x);
                if (q < quads) dst[q] = Quad<T>::pack(x);
            }
        }
    }
}

template <typename T, int C, int B, typename Code>
hipError_t run(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    const int64_t groups = ((a.count + B - 1) / B + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)std::min(groups, kMaxGrid), (unsigned)std::min(a.n, 65535));
    if (write)
        cache_write<T, C, B, Code><<<grid, 64 * kWaves, 0, stream>>>(a, (const T *)states);
    else
        cache_read<T, C, B, Code><<<grid, 64 * kWaves, 0, stream>>>(a, (T *)states);
    return hipGetLastError();
}

template <typename T, int C, typename Code>
hipError_t run_block(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    switch (a.block) {
        case 32: return run<T, C, 32, Code>(a, write, states, stream);
        case 64: return run<T, C, 64, Code>(a, write, states, stream);
        case 128: return run<T, C, 128, Code>(a, write, states, stream);
    }
    return hipErrorInvalidValue;
}

template <typename T, int C>
hipError_t run_code(const CacheArgs &a, bool write, void *states, hipStream_t stream) {
    return a.f8 ? run_block<T, C, CodeF8>(a, write, states, stream)
                : run_block<T, C, CodeI8>(a, write, states, stream);
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
