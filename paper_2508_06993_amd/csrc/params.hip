// Gradients of many tensors: global norm, clipping, clipped AdamW (formulas in
// octree_nca.h).  The list's tensors are cut into chunks of at most kParamChunk
// elements, each with a record in the list's table.
#include <algorithm>

#include "launch.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSums = 2048;   // workgroups of a pass over a large list

// Scratch of a call at the start of the table.
struct Scratch {
    double sums[kMaxSums];     // squares, by workgroup
    double corr1, corr2;       // 1 / (1 - beta^t) of the update
    uint32_t done;             // workgroups that have read *step; 0 between calls
    uint32_t pad[11];
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
    int16_t grad_dtype, clipped_dtype;
    int32_t quads;             // whether the arrays lie alike
};
static_assert(sizeof(Chunk) == 64 && sizeof(Scratch) % 64 == 0, "one record per 64-byte line");

Scratch *scratch_of(void *table) { return (Scratch *)table; }
Chunk *chunks_of(void *table) { return (Chunk *)((char *)table + sizeof(Scratch)); }

// --- the table ---------------------------------------------------------------

constexpr int kFillTensors = 48;   // a launch's tensors travel in its arguments
struct FillArgs {
    octnca_param t[kFillTensors];
    int n;
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

// Records of the tensors of `f`, from record `at` on.
__global__ __launch_bounds__(kThreads) void fill_table(FillArgs f, Scratch *scratch, Chunk *chunks,
                                                       int64_t at) {
    const int64_t thread = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t threads = (int64_t)gridDim.x * kThreads;
    if (thread == 0) scratch->done = 0;
    for (int i = 0; i < f.n; ++i) {
        const octnca_param &t = f.t[i];
        const int lead = lead_of(t);
        const int64_t skip = lead > 0 ? lead : 0;
        const int64_t total = t.count + skip, pieces = pieces_of(t);
        for (int64_t k = thread; k < pieces; k += threads) {
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
            c.grad_dtype = (int16_t)t.grad_dtype;
            c.clipped_dtype = (int16_t)t.clipped_dtype;
            c.quads = lead >= 0;
            chunks[at + k] = c;
        }
        at += pieces;
    }
}

// --- values ------------------------------------------------------------------

// nearest bf16, ties to even; a NaN stays one
__device__ __forceinline__ uint32_t to_bf16(float x) {
    const uint32_t u = __float_as_uint(x);
    return x != x ? 0x7fc0u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// Element and group-of-four access to an array of type DT.
template <int DT> struct Array {
    static __device__ __forceinline__ float value(uint32_t u) {
        return DT == OCTNCA_BF16 ? __uint_as_float(u << 16)
                                 : __half2float(__ushort_as_half((unsigned short)u));
    }
    static __device__ __forceinline__ uint32_t bits(float x) {
        return DT == OCTNCA_BF16 ? to_bf16(x) : (uint32_t)__half_as_ushort(__float2half_rn(x));
    }
    static __device__ __forceinline__ float load(const void *p, int i) {
        return value(((const uint16_t *)p)[i]);
    }
    static __device__ __forceinline__ void store(void *p, int i, float x) {
        ((uint16_t *)p)[i] = (uint16_t)bits(x);
    }
    static __device__ __forceinline__ float4 load4(const void *p, int q) {
        const uint2 u = ((const uint2 *)p)[q];
        return make_float4(value(u.x & 0xffffu), value(u.x >> 16), value(u.y & 0xffffu),
                           value(u.y >> 16));
    }
    static __device__ __forceinline__ void store4(void *p, int q, const float *x) {
        ((uint2 *)p)[q] = make_uint2(bits(x[0]) | bits(x[1]) << 16, bits(x[2]) | bits(x[3]) << 16);
    }
};
template <> struct Array<OCTNCA_F32> {
    static __device__ __forceinline__ float load(const void *p, int i) {
        return ((const float *)p)[i];
    }
    static __device__ __forceinline__ void store(void *p, int i, float x) { ((float *)p)[i] = x; }
    static __device__ __forceinline__ float4 load4(const void *p, int q) {
        return ((const float4 *)p)[q];
    }
    static __device__ __forceinline__ void store4(void *p, int q, const float *x) {
        ((float4 *)p)[q] = make_float4(x[0], x[1], x[2], x[3]);
    }
};

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

// Runs body over the groups of four of a chunk (element index 4 q): `whole`
// for those inside it, `edge` per element for the two partial ones; with
// arrays that lie differently `edge` for every element, lane after lane.
// Thread `t` of T.
template <int T, typename Whole, typename Edge>
__device__ __forceinline__ void for_elements(const Chunk &c, int t, Whole whole, Edge edge) {
    if (!c.quads) {
        for (int i = t; i < c.end; i += T) edge(i);
        return;
    }
    const int inner = (c.first + 3) / 4, outer = c.end / 4;   // whole groups inner .. outer - 1
#pragma unroll
    for (int k = 0; k < kParamChunk / 4 / T; ++k) {
        const int q = t + k * T;
        if (q >= inner && q < outer) whole(q);
    }
    if (t < 8) {   // the elements before and after them, at most three each
        const int i = t < 4 ? c.first + t : std::max(outer, inner) * 4 + t - 4;
        const int stop = t < 4 ? std::min(inner * 4, c.end) : c.end;
        if (i < stop) edge(i);
    }
}

// --- sum of squares ----------------------------------------------------------

// A chunk's squares in fp64 (no square of an fp32 value overflows it), by
// thread t of T.
template <int T> __device__ __forceinline__ double chunk_squares(const Chunk &c, int t) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    with_type(c.grad_dtype, [&](auto type) {
        using G = Array<decltype(type)::value>;
        if (c.quads) {
            constexpr int kN = kParamChunk / 4 / T < 8 ? kParamChunk / 4 / T : 8;
            const int inner = (c.first + 3) / 4, outer = c.end / 4;
            for (int q0 = 0; q0 < kParamChunk / 4; q0 += kN * T) {
                if (q0 >= outer) break;
                float4 g[kN];
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int q = q0 + k * T + t;
                    g[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (q >= inner && q < outer) g[k] = G::load4(c.grad, q);
                }
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const double x = g[k].x, y = g[k].y, z = g[k].z, w = g[k].w;
                    s[0] = fma(x, x, s[0]);
                    s[1] = fma(y, y, s[1]);
                    s[2] = fma(z, z, s[2]);
                    s[3] = fma(w, w, s[3]);
                }
            }
        }
        for_elements<T>(c, t, [](int) {}, [&](int i) {
            const double x = G::load(c.grad, i);
            s[0] = fma(x, x, s[0]);
        });
    });
    return (s[0] + s[1]) + (s[2] + s[3]);
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
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x)
        s += chunk_squares<kThreads>(chunks[k], threadIdx.x);
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

__global__ __launch_bounds__(kThreads) void write_norm(const Scratch *scratch, int sums,
                                                       double scale, float *norm) {
    const double n = norm_of(scratch, sums, scale);
    if (threadIdx.x == 0) *norm = (float)n;
}

// --- clipping ----------------------------------------------------------------

template <int T> __device__ __forceinline__ void clip_chunk(const Chunk &c, int t, float f) {
    with_type(c.grad_dtype, [&](auto gt) {
        with_type(c.clipped_dtype, [&](auto ct) {
            using G = Array<decltype(gt)::value>;
            using O = Array<decltype(ct)::value>;
            for_elements<T>(
                c, t,
                [&](int q) {
                    const float4 g = G::load4(c.grad, q);
                    const float x[4] = {g.x * f, g.y * f, g.z * f, g.w * f};
                    O::store4(c.clipped, q, x);
                },
                [&](int i) { O::store(c.clipped, i, G::load(c.grad, i) * f); });
        });
    });
}

__global__ __launch_bounds__(kThreads) void clip(const Scratch *scratch, int sums,
                                                 const Chunk *chunks, int64_t n, double scale,
                                                 double max_norm, float *norm) {
    const double len = norm_of(scratch, sums, scale);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)len;
    const float f = clip_factor(len, scale, max_norm);
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x)
        clip_chunk<kThreads>(chunks[k], threadIdx.x, f);
}

// --- update ------------------------------------------------------------------

struct UpdateArgs {
    double scale, max_norm;
    float lr, beta1, beta2, rest1, rest2, eps, decay, ema, ema_rest;
};

// One element: g already clipped; corr = 1 / (1 - beta^t).
__device__ __forceinline__ void update(const UpdateArgs &u, float corr1, float corr2, float g,
                                       float &p, float &m, float &v) {
    m = u.beta1 * m + u.rest1 * g;
    v = u.beta2 * v + u.rest2 * (g * g);
    const float d = (m * corr1) / (sqrtf(v * corr2) + u.eps) + u.decay * p;
    p = p - u.lr * d;
}

template <int T>
__device__ __forceinline__ void update_chunk(const Chunk &c, int t, const UpdateArgs &u, float f,
                                             float corr1, float corr2) {
    with_type(c.grad_dtype, [&](auto gt) {
        using G = Array<decltype(gt)::value>;
        using F = Array<OCTNCA_F32>;
        for_elements<T>(
            c, t,
            [&](int q) {
                const float4 g4 = G::load4(c.grad, q), p4 = F::load4(c.param, q),
                             m4 = F::load4(c.m, q), v4 = F::load4(c.v, q);
                float4 e4 = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c.ema) e4 = F::load4(c.ema, q);
                const float g[4] = {g4.x, g4.y, g4.z, g4.w};
                float p[4] = {p4.x, p4.y, p4.z, p4.w}, m[4] = {m4.x, m4.y, m4.z, m4.w};
                float v[4] = {v4.x, v4.y, v4.z, v4.w}, e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    update(u, corr1, corr2, g[k] * f, p[k], m[k], v[k]);
                    e[k] = u.ema * e[k] + u.ema_rest * p[k];
                }
                F::store4(c.m, q, m);
                F::store4(c.v, q, v);
                F::store4(c.param, q, p);
                if (c.ema) F::store4(c.ema, q, e);
            },
            [&](int i) {
                float p = c.param[i], m = c.m[i], v = c.v[i];
                update(u, corr1, corr2, G::load(c.grad, i) * f, p, m, v);
                c.m[i] = m;
                c.v[i] = v;
                c.param[i] = p;
                if (c.ema) c.ema[i] = u.ema * c.ema[i] + u.ema_rest * p;
            });
    });
}

__global__ __launch_bounds__(kThreads) void adamw(const Scratch *scratch, int sums,
                                                  const Chunk *chunks, int64_t n, UpdateArgs u,
                                                  int64_t *step, float *norm) {
    const double len = norm_of(scratch, sums, u.scale);
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    if (norm && first) *norm = (float)len;
    if (!__builtin_isfinite(len)) return;
    if (first) *step += 1;
    const float f = clip_factor(len, u.scale, u.max_norm);
    const float corr1 = (float)scratch->corr1, corr2 = (float)scratch->corr2;
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x)
        update_chunk<kThreads>(chunks[k], threadIdx.x, u, f, corr1, corr2);
}

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
        FillArgs f;
        int64_t pieces = 0;
        for (f.n = 0; i < n && f.n < kFillTensors; ++i) {
            if (params[i].count == 0) continue;
            f.t[f.n++] = params[i];
            pieces += pieces_of(params[i]);
        }
        const unsigned grid =
            (unsigned)std::min<int64_t>((pieces + kThreads) / kThreads, 256);
        fill_table<<<grid, kThreads, 0, stream>>>(f, scratch_of(table), chunks_of(table), at);
        at += pieces;
    } while (i < n);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const octnca_param_list &l, double scale, float *norm,
                            hipStream_t stream) {
    const int sums = first_pass(l, nullptr, 0.0, 0.0, stream);
    write_norm<<<1, kThreads, 0, stream>>>(scratch_of(l.table), sums, scale, norm);
    return hipGetLastError();
}

hipError_t launch_clip_grads(const octnca_param_list &l, double scale, double max_norm,
                             float *norm, hipStream_t stream) {
    const int sums = first_pass(l, nullptr, 0.0, 0.0, stream);
    clip<<<second_grid(l.chunks), kThreads, 0, stream>>>(scratch_of(l.table), sums,
                                                         chunks_of(l.table), l.chunks, scale,
                                                         max_norm, norm);
    return hipGetLastError();
}

hipError_t launch_adamw(const octnca_param_list &l, const octnca_adamw &h, int64_t *step,
                        float *norm, hipStream_t stream) {
    const int sums = first_pass(l, step, h.beta1, h.beta2, stream);
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
    adamw<<<second_grid(l.chunks), kThreads, 0, stream>>>(scratch_of(l.table), sums,
                                                          chunks_of(l.table), l.chunks, u, step,
                                                          norm);
    return hipGetLastError();
}

}  // namespace octnca
