// State cache: states in 8 bits with a scale for each block of cells and
// channel (formulas in octree_nca.h).
//
// Both directions are one pass over memory: a write reads a value once and
// leaves one byte of it, a read the reverse, and a block's scales add 4 bytes per
// channel.  A 184.5M-cell fp32 state (11.8 GB, blocks of 64) is written in 2.43
// ms and read back in 2.49 ms, 6.2 and 6.0 TB/s of these bytes (counters show no
// others); a copy of 8 GB reaches 4.4 TB/s on this card and reading alone 6.3.
// What took the writes there from 3.0 TB/s: the values stay in registers between
// the block's maxima and its codes (one read instead of two), the maxima are
// unsigned maxima of the magnitudes' bits (a comparison for finite values only
// where a block has others), one lane per channel divides, the slot list is on its
// way with the values, and calls larger than the last-level cache go past it.
// Small calls are bound by their launches: a 320 x 320 state 4.5 and 4.3 us.
#include <algorithm>
#include <type_traits>

#include "launch.h"

namespace octnca {

namespace {

constexpr float kTiny = 0x1p-100f;   // the smallest magnitude that sets a scale

typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));

// Loads and stores that go past the last-level cache (STREAM) or through it.
template <bool STREAM, typename R> __device__ __forceinline__ R get(const R *p) {
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}
template <bool STREAM, typename R> __device__ __forceinline__ void put(R *p, R x) {
    if (STREAM)
        __builtin_nontemporal_store(x, p);
    else
        *p = x;
}

// Four channels of a cell as stored; Top keeps the largest magnitudes of four
// channels, as bits (the order of the bits of magnitudes is that of the values,
// with infinities and NaNs above all numbers).
template <typename T> struct Quad;
template <> struct Quad<float> {
    using Raw = Words4;
    static __device__ __forceinline__ void unpack(Raw v, float *x) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(v[k]);
    }
    static __device__ __forceinline__ Raw pack(const float *x) {
        return Raw{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                   __float_as_uint(x[3])};
    }
    struct Top {
        Words4 m = {0, 0, 0, 0};
        __device__ __forceinline__ void add(Raw v) {
            m = __builtin_elementwise_max(m, v & 0x7fffffffu);
        }
        __device__ __forceinline__ Words4 bits() const { return m; }
    };
};
template <> struct Quad<__half> {
    using Raw = Words2;
    static __device__ __forceinline__ void unpack(Raw v, float *x) {
        Storage<__half>::unpack_pair(v.x, x[0], x[1]);
        Storage<__half>::unpack_pair(v.y, x[2], x[3]);
    }
    static __device__ __forceinline__ Raw pack(const float *x) {
        return Raw{Storage<__half>::pack_pair(x[0], x[1]), Storage<__half>::pack_pair(x[2], x[3])};
    }
    struct Top {
        typedef uint16_t Halves __attribute__((ext_vector_type(4)));
        Halves m = {0, 0, 0, 0};
        __device__ __forceinline__ void add(Raw v) {
            m = __builtin_elementwise_max(m, __builtin_bit_cast(Halves, v & 0x7fff7fffu));
        }
        // as fp32 bits
        __device__ __forceinline__ Words4 bits() const {
            float x[4];
            unpack(__builtin_bit_cast(Raw, m), x);
            return Quad<float>::pack(x);
        }
    };
};

constexpr uint32_t kInfBits = 0x7f800000u;

// Factor and scale of a block's channel from a = max(A, 2^-100), and the codes
// of four values (lowest byte first) and back.  ODD: some of the values may not
// be finite.
struct CodeI8 {
    static __device__ __forceinline__ void scale_of(float a, float &inv, float &scale) {
        inv = 127.0f / a;
        scale = a / 127.0f;
    }
    // |x| is at most a, so |x * inv| <= 127 (1 + 2^-23) rounds to 127 at most.
    // Adding 1.5 * 2^23 rounds to an integer, ties to even, and leaves it in
    // the low bits; the product is rounded before (no fused multiply-add).
    static __device__ __forceinline__ uint32_t nearest(float x, float inv) {
#pragma clang fp contract(off)
        return __float_as_uint(x * inv + 0x1.8p23f);
    }
    template <bool ODD> static __device__ __forceinline__ uint32_t encode(const float *x,
                                                                          const float *inv) {
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            c[k] = nearest(x[k], inv[k]);
            if (ODD && !__builtin_isfinite(x[k])) c[k] = 0x80u;
        }
        // the low bytes of the four, in order
        return __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u) |
               __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
    }
    // With the sign bit flipped a byte is code + 128, which has a conversion of
    // its own for each byte.
    static __device__ __forceinline__ void decode(uint32_t c, const float *scale, float *x) {
        const uint32_t u = c ^ 0x80808080u;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = ((float)(u >> (8 * k) & 0xffu) - 128.0f) * scale[k];
        if ((u - 0x01010101u) & ~u & 0x80808080u)   // a byte is 0: code -128
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((u >> (8 * k) & 0xffu) == 0) x[k] = __builtin_nanf("");
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
    template <bool ODD> static __device__ __forceinline__ uint32_t encode(const float *x,
                                                                          const float *inv) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            y[k] = !ODD || __builtin_isfinite(x[k]) ? x[k] * inv[k] : __builtin_nanf("");
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
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
constexpr int64_t kMaxGrid = 1 << 23;  // workgroups along x; the kernels loop over the rest

// Work split of the writes: a wave takes whole blocks of cells of one state,
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
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    x = std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 15, 15, true));
    x = std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 15, 15, true));
    x = std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 15, 15, true));
    return std::max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 15, 15, true));
}

// Largest magnitudes of the channels of N blocks, tops[block][channel], from
// those of each lane's channel quad: every lane leaves its four in LDS by quad,
// and row r of 16 lanes reduces quads r, r + 4, ..
template <int Q, int PEERS, int N>
__device__ __forceinline__ void quad_max(Words4 (*peers)[64], Words4 (*tops)[Q], const Words4 *m) {
    const int lane = threadIdx.x & 63;
    if (lane < Q * PEERS)
#pragma unroll
        for (int b = 0; b < N; ++b) peers[b][lane % Q * PEERS + lane / Q] = m[b];
    wave_fence();
    for (int q = lane >> 4; q < Q; q += 4) {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            Words4 t = {0, 0, 0, 0};
#pragma unroll
            for (int k0 = 0; k0 < PEERS; k0 += 16) {
                const int k = k0 + (lane & 15);
                if (k < PEERS) t = __builtin_elementwise_max(t, peers[b][q * PEERS + k]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) t[c] = row_max(t[c]);
            if ((lane & 15) == 0) tops[b][q] = t;
        }
    }
    wave_fence();
}

// What the caller's list says of state i: its slot, and (writes) the entries
// after it, 64 of them a lane each.  Loaded ahead of the values, used after.
struct SlotEntry {
    int64_t slot, later;

    __device__ __forceinline__ SlotEntry(const int64_t *__restrict__ slots, const CacheArgs &a,
                                         int i, bool write) {
        const int j = i + 1 + (threadIdx.x & 63);
        slot = slots ? slots[i] : a.first + i;
        later = write && slots && j < a.n ? slots[j] : -1;
    }

    __device__ __forceinline__ bool in_cache(const CacheArgs &a) const {
        return slot >= 0 && slot < a.n_slots;
    }

    // Whether a later entry names the same slot (then that one is kept).
    __device__ __forceinline__ bool written_later(const int64_t *__restrict__ slots,
                                                  const CacheArgs &a, int i) const {
        if (!slots) return false;
        bool found = later == slot;
        for (int j = i + 65 + (threadIdx.x & 63); j < a.n; j += 64) found |= slots[j] == slot;
        return __any(found);
    }
};

// Calls f with `flag` as a constant.
template <typename F> __device__ __forceinline__ void with_flag(bool flag, F f) {
    if (flag)
        f(std::true_type());
    else
        f(std::false_type());
}

// Loads, maxima, factors and codes of N consecutive blocks of a state (cells of
// them, src: their first) by one wave; FULL: cells = N B.  LDS of the wave:
// peers, tops.
template <typename T, int C, int B, int N, typename Code, bool FULL, bool STREAM>
__device__ __forceinline__ void write_blocks(const CacheArgs &a, const int64_t *__restrict__ slots,
                                             const SlotEntry &entry, int i, int64_t cell, int cells,
                                             const T *src_cells, Words4 (*peers)[64],
                                             Words4 (*tops)[C / 4]) {
    using S = Split<C, B>;
    using Raw = typename Quad<T>::Raw;
    const int lane = threadIdx.x & 63;
    const Raw *src = (const Raw *)src_cells;
    // whether the lane has a quad in pass k of block b
    const auto has = [&](int b, int k) {
        const int q = lane + k * S::kLanes;
        const bool in = lane < S::kLanes && ((k + 1) * S::kLanes <= B * S::kQ || q < B * S::kQ);
        return FULL ? in : in && q < (cells - b * B) * S::kQ;
    };
    // where it has none, it loads its channels of the block's first cell (of
    // the first block's, if the block is past the end) once more: no branches,
    // and the maxima stay what they are
    Raw raw[N][S::kPasses];
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int k = 0; k < S::kPasses; ++k) {
            const int at = FULL || b * B < cells ? b * B * S::kQ : 0;
            raw[b][k] = get<STREAM>(src + (has(b, k) ? b * B * S::kQ + k * S::kLanes + lane
                                                     : at + lane % S::kQ));
        }
    Words4 m[N];
#pragma unroll
    for (int b = 0; b < N; ++b) {
        typename Quad<T>::Top top;
#pragma unroll
        for (int k = 0; k < S::kPasses; ++k) top.add(raw[b][k]);
        m[b] = top.bits();
    }
    quad_max<S::kQ, S::kPeers, N>(peers, tops, m);
    if (!entry.in_cache(a) || entry.written_later(slots, a, i)) return;
    const int64_t slot = entry.slot;
    float *scales = a.scales + (slot * a.blocks + (a.from + cell) / B) * C;
    // one lane a channel and block: its factor takes its maximum's place
    uint32_t *values = (uint32_t *)tops;
    bool odd = false;
    for (int e = lane; e < N * C; e += 64) odd |= values[e] >= kInfBits;
    odd = __any(odd);
    if (odd) {   // again over the finite values
        wave_fence();
#pragma unroll
        for (int b = 0; b < N; ++b) {
            m[b] = Words4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k) {
                float x[4];
                Quad<T>::unpack(raw[b][k], x);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (__builtin_isfinite(x[c]))
                        m[b][c] = std::max(m[b][c], __float_as_uint(fabsf(x[c])));
            }
        }
        quad_max<S::kQ, S::kPeers, N>(peers, tops, m);
    }
    for (int e = lane; e < N * C; e += 64) {
        float inv, scale;
        Code::scale_of(fmaxf(__uint_as_float(values[e]), kTiny), inv, scale);
        if (FULL || e / C * B < cells) scales[e] = scale;
        values[e] = __float_as_uint(inv);
    }
    wave_fence();
    uint32_t *dst = (uint32_t *)(a.codes + (slot * a.cells + a.from + cell) * C);
    with_flag(odd, [&](auto is_odd) {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            float inv[4];
            Quad<float>::unpack(tops[b][lane % S::kQ], inv);
#pragma unroll
            for (int k = 0; k < S::kPasses; ++k) {
                float x[4];
                Quad<T>::unpack(raw[b][k], x);
                const uint32_t c = Code::template encode<decltype(is_odd)::value>(x, inv);
                if (has(b, k)) put<STREAM>(dst + b * B * S::kQ + k * S::kLanes + lane, c);
            }
        }
    });
    wave_fence();   // the next maxima come after these reads
}

// A wave takes N consecutive blocks at a time, with all their loads in flight.
// The values stay in registers between the maxima and the codes.  A state has
// `full` groups of N B cells and one of `tail` cells (0: none).  Both come as
// arguments: with the group's cells as a 64-bit minimum in the kernel, this
// compiler (ROCm 7.2) selected between them by a carry flag that the comparison
// had not set, and the tail was taken for a full group.
template <typename T, int C, int B, int N, typename Code>
__global__ __launch_bounds__(64 * kWaves) void cache_write(CacheArgs a, uint32_t full, int tail,
                                                           const int64_t *__restrict__ slots,
                                                           const T *__restrict__ states) {
    __shared__ Words4 peers[kWaves][N][64];
    __shared__ Words4 tops[kWaves][N][C / 4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
        const T *from = states + (int64_t)i * a.count * C;
        const uint32_t groups = full + (tail > 0);
        for (uint32_t g = blockIdx.x * kWaves + wave; g < groups; g += gridDim.x * kWaves) {
            const int64_t cell = (int64_t)g * (N * B);
            const SlotEntry entry(slots, a, i, true);
            if (g < full)
                with_flag(a.stream, [&](auto stream) {
                    write_blocks<T, C, B, N, Code, true, decltype(stream)::value>(
                        a, slots, entry, i, cell, N * B, from + cell * C, peers[wave],
                        tops[wave]);
                });
            else
                write_blocks<T, C, B, N, Code, false, false>(
                    a, slots, entry, i, cell, tail, from + cell * C, peers[wave], tops[wave]);
        }
    }
}

// A thread takes channel quads of a state, the workgroup's threads apart: 32
// bytes of the state's values (of one quad a thread fp16 states were read at 3.0
// TB/s, of four at 5.8).  The workgroups do not loop: a grid of 2048 that loop
// over a 184.5M-cell state took 3.1 ms instead of 2.5.
template <typename T> constexpr int kReadQuads = sizeof(T) == 4 ? 2 : 4;
template <typename T, int C, typename Code>
__global__ __launch_bounds__(64 * kWaves) void cache_read(CacheArgs a, int shift, uint32_t full,
                                                          int tail,
                                                          const int64_t *__restrict__ slots,
                                                          T *__restrict__ states) {
    constexpr int kQ = C / 4, kThreads = 64 * kWaves, kN = kReadQuads<T>;
    using Raw = typename Quad<T>::Raw;
    for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
        const SlotEntry entry(slots, a, i, false);
        const bool there = entry.in_cache(a);
        const int64_t slot = there ? entry.slot : 0;
        Raw *to = (Raw *)(states + (int64_t)i * a.count * C);
        const uint32_t *codes = (const uint32_t *)(a.codes + (slot * a.cells + a.from) * C);
        const float4 *scales = (const float4 *)(a.scales + (slot * a.blocks + (a.from >> shift)) * C);
        const uint32_t tiles = full + (tail > 0);   // of kN kThreads quads; the last of `tail`
        for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            const int64_t base = (int64_t)tile * (kN * kThreads);
            const int left = tile < full ? kN * kThreads : tail;
            const int64_t cell = base / kQ;                 // of the first quad, and its place in it
            const int over = (int)(base - cell * kQ);
            // past the tile's end a thread reads its last quad once more: no
            // branches among the loads
            uint32_t code[kN];
            float4 s[kN];
            with_flag(a.stream, [&](auto stream) {
                if (there) {
#pragma unroll
                    for (int k = 0; k < kN; ++k) {
                        const int q = std::min((int)threadIdx.x + k * kThreads, left - 1);
                        code[k] = get<decltype(stream)::value>(codes + base + q);
                        const int c = (q + over) / kQ;
                        s[k] = scales[((cell + c) >> shift) * kQ + (q + over - c * kQ)];
                    }
                }
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int q = threadIdx.x + k * kThreads;
                    const float scale[4] = {s[k].x, s[k].y, s[k].z, s[k].w};
                    float x[4] = {0.f, 0.f, 0.f, 0.f};
                    if (there) Code::decode(code[k], scale, x);
                    if (q < left) put<decltype(stream)::value>(to + base + q, Quad<T>::pack(x));
                }
            });
        }
    }
}

template <typename T, int C, int B, int N, typename Code>
hipError_t launch_write(const CacheArgs &a, const void *states, hipStream_t stream) {
    const int64_t groups = (a.count + (int64_t)B * N * kWaves - 1) / (B * N * kWaves);
    const dim3 grid((unsigned)std::min(groups, kMaxGrid), (unsigned)std::min(a.n, 65535));
    cache_write<T, C, B, N, Code><<<grid, 64 * kWaves, 0, stream>>>(
        a, (uint32_t)(a.count / (N * B)), (int)(a.count % (N * B)), a.slots,
        (const T *)states);
    return hipGetLastError();
}

// Blocks a wave takes at a time: as many as make a lane's loads in flight about
// 64 bytes (32 for fp16: 128 cells), where even so every SIMD gets several
// waves; else one, for the most waves.  Four 2048 x 2048 states (1 GB) with 32
// cells a block, one block and this many: C = 12 fp32 4.2 and 5.5 TB/s, C = 16
// 5.9 and 6.1; fp16 2.7 and 5.0, 4.4 and 5.9.
template <typename T, int C, int B, typename Code>
hipError_t run_write(const CacheArgs &a, const void *states, hipStream_t stream) {
    constexpr int kCells = sizeof(T) == 4 ? 64 : 128;
    if (B < kCells && a.count * a.n >= int64_t(kCells) * 8192)
        return launch_write<T, C, B, (B < kCells ? kCells / B : 1), Code>(a, states, stream);
    return launch_write<T, C, B, 1, Code>(a, states, stream);
}

template <typename T, int C, typename Code>
hipError_t run(CacheArgs a, bool write, void *states, hipStream_t stream) {
    // Past the last-level cache (256 MB) from half its size on: what is wanted next
    // is little of a call of this size.  us past it and through it, of one state
    // again and again (of three in turn): writes of 96 MB 16 and 15 (17, 16), 128 MB
    // 21 and 20 (22, 24), 256 MB 42 and 36 (42, 46), 512 MB 83 and 91 (84, 91); reads
    // of 128 MB 25 and 20 (25, 27), 256 MB 44 and 37 (47, 47), 1 GB 177 and 175.
    a.stream = a.count * a.n * C * (int64_t)(sizeof(T) + 1) >= int64_t(1) << 27;
    if (!write) {
        const int64_t per = kReadQuads<T> * 64 * kWaves;
        const int64_t groups = (a.count * (C / 4) + per - 1) / per;
        const dim3 grid((unsigned)std::min(groups, kMaxGrid), (unsigned)std::min(a.n, 65535));
        const int shift = a.block == 32 ? 5 : a.block == 64 ? 6 : 7;
        cache_read<T, C, Code><<<grid, 64 * kWaves, 0, stream>>>(
            a, shift, (uint32_t)(a.count * (C / 4) / per), (int)(a.count * (C / 4) % per),
            a.slots, (T *)states);
        return hipGetLastError();
    }
    switch (a.block) {
        case 32: return run_write<T, C, 32, Code>(a, states, stream);
        case 64: return run_write<T, C, 64, Code>(a, states, stream);
        case 128: return run_write<T, C, 128, Code>(a, states, stream);
    }
    return hipErrorInvalidValue;
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
