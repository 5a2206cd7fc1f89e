// Gradients of many tensors: global norm, clipping, clipped AdamW (formulas in
// octree_nca.h).  The list's tensors are cut into chunks of at most kParamChunk
// elements, each with a record in the list's table, so that a launch serves any
// number of tensors and a workgroup's addresses come with one scalar load.
//
// Every element depends on all gradients through the norm, so a call is two
// passes: squares (in fp64, added in an order that does not depend on the run),
// then the elements.  Both are bound by memory: 250M bf16 gradients into bf16
// 86 + 168 us (5.8 and 6.0 TB/s), 30M packed fp32 ones 21 + 40 us, an update of
// 100M elements with bf16 gradients and a running average 35 + 5 + 568 us (3.4
// GB, 6.0 TB/s).  Reading alone reaches 6.3 TB/s on this card, a large copy 4.4
// to 5.1.  Small lists are bound by launches and take one (see kSmallUpdate):
// the 25 tensors of a 5-level model 5.2 us clipped, 6.9 us updated.
#include <algorithm>
#include <type_traits>

#include "launch.h"

namespace octnca {

namespace {

constexpr int kThreads = 512;
constexpr int kMaxSums = 2048;   // workgroups that sum squares
constexpr int64_t kMaxGrid = 1 << 22;   // workgroups of a launch; the kernels loop over the rest

// Scratch of a call at the start of the table.
struct Scratch {
    double sums[kMaxSums];     // squares, by workgroup
    double corr1, corr2;       // 1 / (1 - beta^t) of the update
    double total;              // their sum, for updates of large lists
    uint32_t done;             // workgroups that have read *step; 0 between calls
    uint32_t pad[9];
};

// A piece of one tensor.  If its arrays lie alike (all at the same element
// modulo 4 of their aligned groups of four), the pointers are moved back to a
// group's start and the piece is elements first .. end - 1 from there, so that
// all but the edges moves four elements at a time; otherwise first is 0.
struct Chunk {
    const void *grad;
    void *clipped;
    float *param, *m, *v, *ema;
    int32_t first, end;
    int32_t types;             // grad_dtype, clipped_dtype << 8
    int32_t quads;             // whether the arrays lie alike

    __device__ __forceinline__ int grad_dtype() const { return types & 0xff; }
    __device__ __forceinline__ int clipped_dtype() const { return types >> 8; }
};
static_assert(sizeof(Chunk) == 64 && sizeof(Scratch) % 64 == 0, "one record per 64-byte line");

Scratch *scratch_of(void *table) { return (Scratch *)table; }
Chunk *chunks_of(void *table) { return (Chunk *)((char *)table + sizeof(Scratch)); }

// --- the table ---------------------------------------------------------------

constexpr int kFillTensors = 52;   // a launch's tensors travel in its arguments
struct FillArgs {
    octnca_param t[kFillTensors];
    uint32_t at[kFillTensors];   // first record of each, from the launch's first
};
static_assert(sizeof(FillArgs) <= 4096 - 64, "kernel arguments");

__host__ __device__ inline int64_t bytes_of(int32_t dtype) { return dtype == OCTNCA_F32 ? 4 : 2; }

// Element of its group of four that the tensor's arrays start at, -1 if they
// do not agree.
__host__ __device__ inline int lead_of(const octnca_param &t) {
    const int lead = (int)((uintptr_t)t.grad / bytes_of(t.grad_dtype) % 4);
    if (t.clipped && (int)((uintptr_t)t.clipped / bytes_of(t.clipped_dtype) % 4) != lead) return -1;
    const void *f32[] = {t.param, t.m, t.v, t.ema};
    for (const void *p : f32)
        if (p && (int)((uintptr_t)p / 4 % 4) != lead) return -1;
    return lead;
}

__host__ __device__ inline int64_t pieces_of(const octnca_param &t) {
    const int lead = lead_of(t);
    return (t.count + (lead > 0 ? lead : 0) + kParamChunk - 1) / kParamChunk;
}

// Records of the tensors of `f`, one per blockIdx.y, from record `at` on.
__global__ __launch_bounds__(kThreads) void fill_table(FillArgs f, Scratch *scratch, Chunk *chunks,
                                                       int64_t at) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) scratch->done = 0;
    const octnca_param &t = f.t[blockIdx.y];
    if (t.count == 0) return;
    const int lead = lead_of(t);
    const int64_t skip = lead > 0 ? lead : 0;
    const int64_t total = t.count + skip, pieces = pieces_of(t);
    for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < pieces;
         k += (int64_t)gridDim.x * kThreads) {
        const int64_t e = k * kParamChunk - skip;   // the aligned start
        Chunk c;
        c.grad = (const char *)t.grad + e * bytes_of(t.grad_dtype);
        c.clipped = t.clipped ? (char *)t.clipped + e * bytes_of(t.clipped_dtype) : nullptr;
        c.param = t.param ? t.param + e : nullptr;
        c.m = t.m ? t.m + e : nullptr;
        c.v = t.v ? t.v + e : nullptr;
        c.ema = t.ema ? t.ema + e : nullptr;
        c.first = k == 0 ? (int32_t)skip : 0;
        const int64_t left = total - k * kParamChunk;
        c.end = (int32_t)(left < kParamChunk ? left : kParamChunk);
        c.types = t.grad_dtype | (t.clipped ? t.clipped_dtype << 8 : 0);
        c.quads = lead >= 0;
        chunks[at + f.at[blockIdx.y] + k] = c;
    }
}

// --- values ------------------------------------------------------------------

// nearest bf16, ties to even; a NaN stays one
__device__ __forceinline__ uint32_t to_bf16(float x) {
    const uint32_t u = __float_as_uint(x);
    return x != x ? 0x7fc0u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// Addresses read from a table are global ones (the compiler cannot know, and
// flat accesses would wait on the LDS counter too).
#define OCTNCA_GLOBAL __attribute__((address_space(1)))
typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
template <typename T, bool STREAM = false>
__device__ __forceinline__ T get(const void *p, int i) {
    const OCTNCA_GLOBAL T *at = (const OCTNCA_GLOBAL T *)p + i;
    return STREAM ? __builtin_nontemporal_load(at) : *at;
}
template <bool STREAM = false, typename T>
__device__ __forceinline__ void put(void *p, int i, T x) {
    OCTNCA_GLOBAL T *at = (OCTNCA_GLOBAL T *)p + i;
    if (STREAM)
        __builtin_nontemporal_store(x, at);
    else
        *at = x;
}

// An array's elements by type: Raw is a group of four as stored.
template <int DT> struct Array {
    using Raw = Words2;
    static __device__ __forceinline__ float value(uint32_t u) {
        return DT == OCTNCA_BF16 ? __uint_as_float(u << 16)
                                 : __half2float(__ushort_as_half((unsigned short)u));
    }
    static __device__ __forceinline__ uint32_t bits(float x) {
        return DT == OCTNCA_BF16 ? to_bf16(x) : (uint32_t)__half_as_ushort(__float2half_rn(x));
    }
    static __device__ __forceinline__ float load(const void *p, int i) {
        return value(get<uint16_t>(p, i));
    }
    static __device__ __forceinline__ void store(void *p, int i, float x) {
        put(p, i, (uint16_t)bits(x));
    }
    static __device__ __forceinline__ void unpack(Raw u, float *x) {
        x[0] = value(u.x & 0xffffu);
        x[1] = value(u.x >> 16);
        x[2] = value(u.y & 0xffffu);
        x[3] = value(u.y >> 16);
    }
    static __device__ __forceinline__ Raw pack(const float *x) {
        return Raw{bits(x[0]) | bits(x[1]) << 16, bits(x[2]) | bits(x[3]) << 16};
    }
};
template <> struct Array<OCTNCA_F32> {
    using Raw = Words4;
    static __device__ __forceinline__ float load(const void *p, int i) { return get<float>(p, i); }
    static __device__ __forceinline__ void store(void *p, int i, float x) { put(p, i, x); }
    static __device__ __forceinline__ void unpack(Raw u, float *x) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(u[k]);
    }
    static __device__ __forceinline__ Raw pack(const float *x) {
        return Raw{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                   __float_as_uint(x[3])};
    }
};
using F32 = Array<OCTNCA_F32>;

// Calls f with the type of a gradient as a constant.
template <typename F> __device__ __forceinline__ void with_type(int dtype, F f) {
    if (dtype == OCTNCA_F32)
        f(std::integral_constant<int, OCTNCA_F32>());
    else if (dtype == OCTNCA_F16)
        f(std::integral_constant<int, OCTNCA_F16>());
    else
        f(std::integral_constant<int, OCTNCA_BF16>());
}

// Sum of a wave's lanes, in each of them; the same additions in every run.
__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
    return s;
}

// Sum over the workgroup of T threads, in every thread.
template <int T> __device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[T / 64];
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) s += part[w];
    return s;
}

// The whole groups of four of a chunk (group q: elements 4 q .. 4 q + 3 from its
// pointers) by thread t of T, N groups of a thread at a time: load(k, q) of
// all of them before finish(k, q), so that N loads of an array are in flight.
template <int T, int N, typename Load, typename Finish>
__device__ __forceinline__ void for_groups(const Chunk &c, int t, Load load, Finish finish) {
    static_assert(kParamChunk / 4 % (N * T) == 0, "a full chunk is whole rounds of N T groups");
    if (!c.quads) return;
    const int inner = (c.first + 3) / 4, outer = c.end / 4;   // whole ones: inner .. outer - 1
    if (inner == 0 && outer == kParamChunk / 4) {             // a full chunk: no comparisons
#pragma unroll
        for (int q0 = 0; q0 < kParamChunk / 4; q0 += N * T) {
#pragma unroll
            for (int k = 0; k < N; ++k) load(k, q0 + k * T + t);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < N; ++k) finish(k, q0 + k * T + t);
        }
        return;
    }
    for (int q0 = t; q0 < outer; q0 += N * T) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (q0 + k * T >= inner && q0 + k * T < outer) load(k, q0 + k * T);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (q0 + k * T >= inner && q0 + k * T < outer) finish(k, q0 + k * T);
    }
}

// The other elements: at most three before and three after the whole groups,
// or all, lane after lane, where the arrays lie differently.
template <int T, typename Edge>
__device__ __forceinline__ void for_edges(const Chunk &c, int t, Edge edge) {
    if (!c.quads) {
        for (int i = t; i < c.end; i += T) edge(i);
        return;
    }
    const int inner = (c.first + 3) / 4, outer = c.end / 4;
    if (t < 8) {
        const int i = t < 4 ? c.first + t : std::max(outer, inner) * 4 + t - 4;
        const int stop = t < 4 ? std::min(inner * 4, c.end) : c.end;
        if (i < stop) edge(i);
    }
}

// --- sum of squares ----------------------------------------------------------

// A chunk's squares in fp64 (no square of an fp32 value overflows it), by
// thread t of T.
template <int T> __device__ __forceinline__ double chunk_squares(const Chunk &c, int t) {
    constexpr int kN = kParamChunk / 4 / T < 8 ? kParamChunk / 4 / T : 8;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    with_type(c.grad_dtype(), [&](auto type) {
        using G = Array<decltype(type)::value>;
        typename G::Raw g[kN];
        for_groups<T, kN>(
            c, t, [&](int k, int q) { g[k] = get<typename G::Raw>(c.grad, q); },
            [&](int k, int) {
                float x[4];
                G::unpack(g[k], x);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = fma((double)x[i], (double)x[i], s[i]);
            });
        for_edges<T>(c, t, [&](int i) {
            const double x = G::load(c.grad, i);
            s[0] = fma(x, x, s[0]);
        });
    });
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Runs body(chunk) over chunks k, k + step, ..; the next one's record is on its
// way during a chunk.
template <typename Body>
__device__ __forceinline__ void for_chunks(const Chunk *chunks, int64_t n, int64_t k, int64_t step,
                                           Body body) {
    if (k >= n) return;
    Chunk c = chunks[k];
    while (true) {
        k += step;
        const Chunk next = chunks[k < n ? k : 0];
        body(c);
        if (k >= n) return;
        c = next;
    }
}

__device__ __forceinline__ double power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

// First pass of a large list: workgroup b sums chunks b, b + gridDim.x, ..
// With step, workgroup 0 also prepares the update's bias corrections: only
// here, so that *step is read in one launch and written in the next.
__global__ __launch_bounds__(kThreads) void square_sums(Scratch *scratch, const Chunk *chunks,
                                                        int64_t n, const int64_t *step,
                                                        double beta1, double beta2) {
    double s = 0.0;
    for_chunks(chunks, n, blockIdx.x, gridDim.x,
               [&](const Chunk &c) { s += chunk_squares<kThreads>(c, threadIdx.x); });
    s = block_sum<kThreads>(s);
    if (threadIdx.x == 0) scratch->sums[blockIdx.x] = s;
    if (step && blockIdx.x == 0 && threadIdx.x == 0) {
        const int64_t t = *step + 1;
        scratch->corr1 = 1.0 / (1.0 - power(beta1, t));
        scratch->corr2 = 1.0 / (1.0 - power(beta2, t));
    }
}

// scale * sqrt(sum of the first pass's sums), added in the same order by every
// workgroup.
__device__ __forceinline__ double norm_of(const Scratch *scratch, int sums, double scale) {
    double s = 0.0;
    for (int i = threadIdx.x; i < sums; i += kThreads) s += scratch->sums[i];
    return sqrt(block_sum<kThreads>(s)) * scale;
}

__device__ __forceinline__ float clip_factor(double norm, double scale, double max_norm) {
    return (float)(norm <= max_norm ? scale : scale * (max_norm / norm));
}

// The same sum, once for all workgroups of a large update.
__global__ __launch_bounds__(kThreads) void add_sums(Scratch *scratch, int sums) {
    double s = 0.0;
    for (int i = threadIdx.x; i < sums; i += kThreads) s += scratch->sums[i];
    s = block_sum<kThreads>(s);
    if (threadIdx.x == 0) scratch->total = s;
}

__global__ __launch_bounds__(kThreads) void write_norm(const Scratch *scratch, int sums,
                                                       double scale, float *norm) {
    const double n = norm_of(scratch, sums, scale);
    if (threadIdx.x == 0) *norm = (float)n;
}

// --- clipping ----------------------------------------------------------------

template <int T, bool STREAM>
__device__ __forceinline__ void clip_chunk(const Chunk &c, int t, float f) {
    if (c.clipped == c.grad && f == 1.0f) return;
    constexpr int kN = kParamChunk / 4 / T < 8 ? kParamChunk / 4 / T : 8;
    with_type(c.grad_dtype(), [&](auto gt) {
        with_type(c.clipped_dtype(), [&](auto ct) {
            using G = Array<decltype(gt)::value>;
            using O = Array<decltype(ct)::value>;
            typename G::Raw g[kN];
            for_groups<T, kN>(
                c, t, [&](int k, int q) { g[k] = get<typename G::Raw, STREAM>(c.grad, q); },
                [&](int k, int q) {
                    float x[4];
                    G::unpack(g[k], x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] *= f;
                    put<STREAM>(c.clipped, q, O::pack(x));
                });
            for_edges<T>(c, t, [&](int i) { O::store(c.clipped, i, G::load(c.grad, i) * f); });
        });
    });
}

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void clip(const Scratch *scratch, int sums,
                                                 const Chunk *chunks, int64_t n, double scale,
                                                 double max_norm, float *norm) {
    const double len = norm_of(scratch, sums, scale);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)len;
    const float f = clip_factor(len, scale, max_norm);
    for_chunks(chunks, n, blockIdx.x, gridDim.x,
               [&](const Chunk &c) { clip_chunk<kThreads, STREAM>(c, threadIdx.x, f); });
}

// --- update ------------------------------------------------------------------

struct UpdateArgs {
    double scale, max_norm;
    float lr, beta1, beta2, rest1, rest2, eps, decay, ema, ema_rest;
};

// Whether an update is made: by the norm as the caller sees it, in fp32.
__device__ __forceinline__ bool norm_fits(double len) { return __builtin_isfinite((float)len); }

// One element: g already clipped; corr = 1 / (1 - beta^t).
__device__ __forceinline__ void update(const UpdateArgs &u, float corr1, float corr2, float g,
                                       float &p, float &m, float &v) {
    m = u.beta1 * m + u.rest1 * g;
    v = u.beta2 * v + u.rest2 * (g * g);
    const float d = (m * corr1) / (sqrtf(v * corr2) + u.eps) + u.decay * p;
    p = p - u.lr * d;
}

// A group of four elements of an update.
template <int DT, bool STREAM> struct Group {
    typename Array<DT>::Raw g;
    Words4 p, m, v, e;

    __device__ __forceinline__ void load(const Chunk &c, int q) {
        g = get<typename Array<DT>::Raw, STREAM>(c.grad, q);
        p = get<Words4, STREAM>(c.param, q);
        m = get<Words4, STREAM>(c.m, q);
        v = get<Words4, STREAM>(c.v, q);
        if (c.ema) e = get<Words4, STREAM>(c.ema, q);
    }

    __device__ __forceinline__ void finish(const Chunk &c, int q, const UpdateArgs &u, float f,
                                           float corr1, float corr2) {
        float gs[4], ps[4], ms[4], vs[4];
        Array<DT>::unpack(g, gs);
        F32::unpack(p, ps);
        F32::unpack(m, ms);
        F32::unpack(v, vs);
#pragma unroll
        for (int k = 0; k < 4; ++k) update(u, corr1, corr2, gs[k] * f, ps[k], ms[k], vs[k]);
        put<STREAM>(c.m, q, F32::pack(ms));
        put<STREAM>(c.v, q, F32::pack(vs));
        put<STREAM>(c.param, q, F32::pack(ps));
        if (c.ema) {
            float es[4];
            F32::unpack(e, es);
#pragma unroll
            for (int k = 0; k < 4; ++k) es[k] = u.ema * es[k] + u.ema_rest * ps[k];
            put<STREAM>(c.ema, q, F32::pack(es));
        }
    }
};

template <int T, int DT>
__device__ __forceinline__ void update_edges(const Chunk &c, int t, const UpdateArgs &u, float f,
                                             float corr1, float corr2) {
    for_edges<T>(c, t, [&](int i) {
        float p = F32::load(c.param, i), m = F32::load(c.m, i), v = F32::load(c.v, i);
        update(u, corr1, corr2, Array<DT>::load(c.grad, i) * f, p, m, v);
        F32::store(c.m, i, m);
        F32::store(c.v, i, v);
        F32::store(c.param, i, p);
        if (c.ema) F32::store(c.ema, i, u.ema * F32::load(c.ema, i) + u.ema_rest * p);
    });
}

template <int T, bool STREAM>
__device__ __forceinline__ void update_chunk(const Chunk &c, int t, const UpdateArgs &u, float f,
                                             float corr1, float corr2) {
    constexpr int kN = 2;
    with_type(c.grad_dtype(), [&](auto gt) {
        constexpr int DT = decltype(gt)::value;
        Group<DT, STREAM> r[kN];
        for_groups<T, kN>(
            c, t, [&](int k, int q) { r[k].load(c, q); },
            [&](int k, int q) { r[k].finish(c, q, u, f, corr1, corr2); });
        update_edges<T, DT>(c, t, u, f, corr1, corr2);
    });
}

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw(const Scratch *scratch, int sums,
                                                  const Chunk *chunks, int64_t n, UpdateArgs u,
                                                  int64_t *step, float *norm) {
    const double len =
        STREAM ? sqrt(scratch->total) * u.scale : norm_of(scratch, sums, u.scale);
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    if (norm && first) *norm = (float)len;
    if (!norm_fits(len)) return;
    if (first) *step += 1;
    const float f = clip_factor(len, u.scale, u.max_norm);
    const float corr1 = (float)scratch->corr1, corr2 = (float)scratch->corr2;
    for_chunks(chunks, n, blockIdx.x, gridDim.x, [&](const Chunk &c) {
        update_chunk<kThreads, STREAM>(c, threadIdx.x, u, f, corr1, corr2);
    });
}

// --- small lists: one launch --------------------------------------------------

// A small list takes one launch: every workgroup sums all gradients itself (in
// the same order), then does one chunk.  The sum of 16.5k elements costs a
// workgroup less than a second launch would.
constexpr int kSmallThreads = 1024;

// scale * norm of the list; wave w of the workgroup takes chunks w, w + 16, ..
__device__ __forceinline__ double small_norm(const Chunk *chunks, int n, double scale) {
    double s = 0.0;
    for_chunks(chunks, n, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kSmallThreads / 64,
               [&](const Chunk &c) { s += chunk_squares<64>(c, threadIdx.x & 63); });
    return sqrt(block_sum<kSmallThreads>(s)) * scale;
}

__global__ __launch_bounds__(kSmallThreads) void small_write_norm(const Chunk *chunks, int n,
                                                                  double scale, float *norm) {
    const double len = small_norm(chunks, n, scale);
    if (threadIdx.x == 0) *norm = (float)len;
}

// Whether thread t has a whole group of its workgroup's chunk.
__device__ __forceinline__ bool small_group(const Chunk &c, int t) {
    static_assert(kParamChunk / 4 == kSmallThreads, "one group of four a thread");
    return c.quads && t >= (c.first + 3) / 4 && t < c.end / 4;
}

// Not in place: another workgroup may still be summing.  The workgroup's own
// chunk is read before the sum, so that both wait together.
__global__ __launch_bounds__(kSmallThreads) void small_clip(const Chunk *chunks, int n,
                                                            double scale, double max_norm,
                                                            float *norm) {
    Chunk c{};
    if (n > 0) c = chunks[blockIdx.x];
    const int q = threadIdx.x;
    with_type(c.grad_dtype(), [&](auto gt) {
        using G = Array<decltype(gt)::value>;
        const bool whole = small_group(c, q);
        typename G::Raw g{};
        if (whole) g = get<typename G::Raw>(c.grad, q);
        const double len = small_norm(chunks, n, scale);
        if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)len;
        if (n == 0) return;
        const float f = clip_factor(len, scale, max_norm);
        with_type(c.clipped_dtype(), [&](auto ct) {
            using O = Array<decltype(ct)::value>;
            float x[4];
            G::unpack(g, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] *= f;
            if (whole) put(c.clipped, q, O::pack(x));
            for_edges<kSmallThreads>(
                c, q, [&](int i) { O::store(c.clipped, i, G::load(c.grad, i) * f); });
        });
    });
}

__global__ __launch_bounds__(kSmallThreads) void small_adamw(Scratch *scratch, const Chunk *chunks,
                                                             int n, UpdateArgs u, double beta1,
                                                             double beta2, int64_t *step,
                                                             float *norm) {
    // One thread reads *step, before the sum's barrier (the last one: its wave has
    // the least to sum), and leaves it in LDS.
    __shared__ int64_t now;
    if (threadIdx.x == kSmallThreads - 1)
        now = __hip_atomic_load(step, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    Chunk c{};
    if (n > 0) c = chunks[blockIdx.x];
    with_type(c.grad_dtype(), [&](auto type) {
        constexpr int DT = decltype(type)::value;
        const int q = threadIdx.x;
        const bool whole = small_group(c, q);
        Group<DT, false> own;
        if (whole) own.load(c, q);
        const double len = small_norm(chunks, n, u.scale);
        const bool fine = norm_fits(len);
        const int64_t t = now;
        if (threadIdx.x == 0) {
            if (norm && blockIdx.x == 0) *norm = (float)len;
            // The workgroup that counts last writes *step: the others have read
            // it before they counted.
            const uint32_t before = __hip_atomic_fetch_add(&scratch->done, 1u, __ATOMIC_ACQ_REL,
                                                           __HIP_MEMORY_SCOPE_AGENT);
            if (before == gridDim.x - 1) {
                scratch->done = 0;
                if (fine) *step = t;
            }
        }
        if (n == 0 || !fine) return;
        const float f = clip_factor(len, u.scale, u.max_norm);
        const float corr1 = (float)(1.0 / (1.0 - power(beta1, t)));
        const float corr2 = (float)(1.0 / (1.0 - power(beta2, t)));
        if (whole) own.finish(c, q, u, f, corr1, corr2);
        update_edges<kSmallThreads, DT>(c, threadIdx.x, u, f, corr1, corr2);
    });
}

// Lists that take one launch.  Calls in a row take two launches 7.2 to 9.0 us for an
// update, 6.4 to 8.7 for clipping, 6.3 to 7.9 for the norm (by the machine, hardly by
// the list).  One launch:
//   25 tensors of 656 elements   6.8   4.7   3.8 to 4.3
//   37                           7.4   5.3   4.2 to 4.4
//   50                           8.5   6.3   5.1
//   75                          10.2   7.6   6.5
// and, as every workgroup goes through all chunks, of any size,
//   64 tensors of 16 elements    9.4   7.0   5.9
//   128 of 16, or of 192        14.3  11.2  10.2
constexpr int64_t kSmallUpdate = 3 << 13, kSmallNorm = 1 << 15;   // elements
constexpr int64_t kSmallChunks = 64;
bool small(const octnca_param_list &l, int64_t elements) {
    return l.elements <= elements && l.chunks <= kSmallChunks;
}
unsigned small_grid(const octnca_param_list &l) { return (unsigned)std::max<int64_t>(1, l.chunks); }

// Lists whose second pass goes past the last-level cache (256 MB), from half its size
// on: the next call finds little of them there.  us past it and through it, of one
// list again and again (of three in turn), by the bytes of the arrays: clipping of
// 128 MB 31 and 34 (31, 38), 256 MB 57 and 59 (57, 74), 512 MB 114 and 144 (117, 148);
// an update, which then also has a workgroup per chunk, of 96 MB 23 and 21 (24, 22),
// 128 MB 28 and 28 (30, 28), 192 MB 39 and 39 (40, 45), 1 GB 181 and 219 (178, 222).
bool streams(const octnca_param_list &l) { return l.bytes >= (int64_t(1) << 27); }

// Enqueues the first pass; the number of sums it leaves.
int first_pass(const octnca_param_list &l, const int64_t *step, double beta1, double beta2,
               hipStream_t stream) {
    const int sums = (int)std::max<int64_t>(1, std::min<int64_t>(l.chunks, kMaxSums));
    square_sums<<<sums, kThreads, 0, stream>>>(scratch_of(l.table), chunks_of(l.table), l.chunks,
                                               step, beta1, beta2);
    return sums;
}

unsigned second_grid(int64_t chunks) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>(chunks, kMaxSums));
}

}  // namespace

int64_t param_chunks(const octnca_param &t) { return t.count > 0 ? pieces_of(t) : 0; }

size_t param_table_bytes(int64_t chunks) { return sizeof(Scratch) + (size_t)chunks * sizeof(Chunk); }

hipError_t launch_param_table(const octnca_param *params, int n, void *table, hipStream_t stream) {
    int64_t at = 0;
    int i = 0;
    do {   // once at least: an empty list has scratch memory too
        FillArgs f{};
        int64_t pieces = 0, most = 1;
        int m = 0;
        for (; i < n && m < kFillTensors; ++i) {
            if (params[i].count == 0) continue;
            const int64_t own = pieces_of(params[i]);
            f.t[m] = params[i];
            f.at[m++] = (uint32_t)pieces;
            pieces += own;
            most = std::max(most, own);
        }
        const dim3 grid((unsigned)std::min<int64_t>((most + kThreads - 1) / kThreads, 256),
                        (unsigned)std::max(m, 1));
        fill_table<<<grid, kThreads, 0, stream>>>(f, scratch_of(table), chunks_of(table), at);
        at += pieces;
    } while (i < n);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const octnca_param_list &l, double scale, float *norm,
                            hipStream_t stream) {
    if (small(l, kSmallNorm)) {
        small_write_norm<<<1, kSmallThreads, 0, stream>>>(chunks_of(l.table), (int)l.chunks, scale,
                                                          norm);
        return hipGetLastError();
    }
    const int sums = first_pass(l, nullptr, 0.0, 0.0, stream);
    write_norm<<<1, kThreads, 0, stream>>>(scratch_of(l.table), sums, scale, norm);
    return hipGetLastError();
}

hipError_t launch_clip_grads(const octnca_param_list &l, double scale, double max_norm,
                             float *norm, hipStream_t stream) {
    if (small(l, kSmallNorm) && !(l.has & kHasInPlace)) {
        small_clip<<<small_grid(l), kSmallThreads, 0, stream>>>(
            chunks_of(l.table), (int)l.chunks, scale, max_norm, norm);
        return hipGetLastError();
    }
    const int sums = first_pass(l, nullptr, 0.0, 0.0, stream);
    const auto kernel = streams(l) ? clip<true> : clip<false>;
    kernel<<<second_grid(l.chunks), kThreads, 0, stream>>>(scratch_of(l.table), sums,
                                                           chunks_of(l.table), l.chunks, scale,
                                                           max_norm, norm);
    return hipGetLastError();
}

hipError_t launch_adamw(const octnca_param_list &l, const octnca_adamw &h, int64_t *step,
                        float *norm, hipStream_t stream) {
    UpdateArgs u;
    u.scale = h.scale;
    u.max_norm = h.max_norm;
    u.lr = (float)h.lr;
    u.beta1 = (float)h.beta1;
    u.beta2 = (float)h.beta2;
    u.rest1 = (float)(1.0 - h.beta1);
    u.rest2 = (float)(1.0 - h.beta2);
    u.eps = (float)h.eps;
    u.decay = (float)h.weight_decay;
    u.ema = (float)h.ema_decay;
    u.ema_rest = (float)(1.0 - h.ema_decay);
    if (small(l, kSmallUpdate)) {
        small_adamw<<<small_grid(l), kSmallThreads, 0, stream>>>(
            scratch_of(l.table), chunks_of(l.table), (int)l.chunks, u, h.beta1, h.beta2, step,
            norm);
        return hipGetLastError();
    }
    const int sums = first_pass(l, step, h.beta1, h.beta2, stream);
    if (streams(l)) {
        // A workgroup per chunk: a call of 100M elements takes 635 us, with 2048
        // workgroups that loop over the chunks 765.  So many do not each add the sums.
        add_sums<<<1, kThreads, 0, stream>>>(scratch_of(l.table), sums);
        adamw<true><<<(unsigned)std::min(l.chunks, kMaxGrid), kThreads, 0, stream>>>(
            scratch_of(l.table), sums, chunks_of(l.table), l.chunks, u, step, norm);
    } else {
        adamw<false><<<second_grid(l.chunks), kThreads, 0, stream>>>(
            scratch_of(l.table), sums, chunks_of(l.table), l.chunks, u, step, norm);
    }
    return hipGetLastError();
}

}  // namespace octnca
