// Gradients of many tensors: global norm, clipping, clipped AdamW (formulas in
// octree_nca.h).  The list's tensors are cut into chunks of at most kParamChunk
// elements, each with a record in the list's table.
#include <algorithm>

#include "launch.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSums = 2048;   // workgroups of the norm's first pass

// Scratch of a call at the start of the table.
struct Scratch {
    double sums[kMaxSums];     // squares, by workgroup
    double corr1, corr2;       // 1 / (1 - beta^t) of the update
};

struct Chunk {
    const void *grad;
    void *clipped;
    float *param, *m, *v, *ema;
    int32_t count;
    int32_t grad_dtype, clipped_dtype, pad;
};
static_assert(sizeof(Chunk) == 64, "one record per 64-byte line");

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

// Records of the tensors of `f`, from record `at` on.
__global__ __launch_bounds__(kThreads) void fill_table(FillArgs f, Chunk *chunks, int64_t at) {
    const int64_t thread = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t threads = (int64_t)gridDim.x * kThreads;
    for (int i = 0; i < f.n; ++i) {
        const octnca_param &t = f.t[i];
        const int64_t pieces = (t.count + kParamChunk - 1) / kParamChunk;
        for (int64_t k = thread; k < pieces; k += threads) {
            const int64_t e = k * kParamChunk;
            Chunk c;
            c.grad = (const char *)t.grad + e * bytes_of(t.grad_dtype);
            c.clipped = t.clipped ? (char *)t.clipped + e * bytes_of(t.clipped_dtype) : nullptr;
            c.param = t.param ? t.param + e : nullptr;
            c.m = t.m ? t.m + e : nullptr;
            c.v = t.v ? t.v + e : nullptr;
            c.ema = t.ema ? t.ema + e : nullptr;
            c.count = (int32_t)(t.count - e < kParamChunk ? t.count - e : kParamChunk);
            c.grad_dtype = t.grad_dtype;
            c.clipped_dtype = t.clipped_dtype;
            c.pad = 0;
            chunks[at + k] = c;
        }
        at += pieces;
    }
}

// --- values ------------------------------------------------------------------

__device__ __forceinline__ float load(const void *p, int32_t dtype, int i) {
    if (dtype == OCTNCA_F32) return ((const float *)p)[i];
    const uint16_t u = ((const uint16_t *)p)[i];
    if (dtype == OCTNCA_BF16) return __uint_as_float((uint32_t)u << 16);
    return __half2float(__ushort_as_half(u));
}

// nearest bf16, ties to even; a NaN stays one
__device__ __forceinline__ uint16_t to_bf16(float x) {
    const uint32_t u = __float_as_uint(x);
    if (x != x) return 0x7fc0;
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

__device__ __forceinline__ void store(void *p, int32_t dtype, int i, float x) {
    if (dtype == OCTNCA_F32)
        ((float *)p)[i] = x;
    else if (dtype == OCTNCA_BF16)
        ((uint16_t *)p)[i] = to_bf16(x);
    else
        ((uint16_t *)p)[i] = __half_as_ushort(__float2half_rn(x));
}

// Sum over the workgroup, the same in every thread and in every run.
__device__ double block_sum(double s) {
    __shared__ double part[kThreads];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int k = kThreads / 2; k > 0; k >>= 1) {
        if ((int)threadIdx.x < k) part[threadIdx.x] += part[threadIdx.x + k];
        __syncthreads();
    }
    return part[0];
}

// --- first pass: squares -----------------------------------------------------

// Workgroup b sums chunks b, b + gridDim.x, .. in fp64 (no square of an fp32
// value overflows it).  With step, workgroup 0 also prepares the update's bias
// corrections: only here, so that *step is read in one launch and written in
// the next.
__global__ __launch_bounds__(kThreads) void square_sums(Scratch *scratch, const Chunk *chunks,
                                                        int64_t n, const int64_t *step,
                                                        double beta1, double beta2) {
    double s = 0.0;
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x) {
        const Chunk c = chunks[k];
        for (int i = threadIdx.x; i < c.count; i += kThreads) {
            const double g = load(c.grad, c.grad_dtype, i);
            s += g * g;
        }
    }
    s = block_sum(s);
    if (threadIdx.x == 0) scratch->sums[blockIdx.x] = s;
    if (step && blockIdx.x == 0 && threadIdx.x == 0) {
        const double t = (double)(*step + 1);
        scratch->corr1 = 1.0 / (1.0 - pow(beta1, t));
        scratch->corr2 = 1.0 / (1.0 - pow(beta2, t));
    }
}

// --- second pass -------------------------------------------------------------

// scale * sqrt(sum of the first pass's sums), added in the same order by every
// workgroup.
__device__ double norm_of(const Scratch *scratch, int sums, double scale) {
    double s = 0.0;
    for (int i = threadIdx.x; i < sums; i += kThreads) s += scratch->sums[i];
    return sqrt(block_sum(s)) * scale;
}

__device__ float clip_factor(double norm, double scale, double max_norm) {
    return (float)(norm <= max_norm ? scale : scale * (max_norm / norm));
}

__global__ __launch_bounds__(kThreads) void write_norm(const Scratch *scratch, int sums,
                                                       double scale, float *norm) {
    const double n = norm_of(scratch, sums, scale);
    if (threadIdx.x == 0) *norm = (float)n;
}

__global__ __launch_bounds__(kThreads) void clip(const Scratch *scratch, int sums,
                                                 const Chunk *chunks, int64_t n, double scale,
                                                 double max_norm, float *norm) {
    const double len = norm_of(scratch, sums, scale);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)len;
    const float f = clip_factor(len, scale, max_norm);
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x) {
        const Chunk c = chunks[k];
        for (int i = threadIdx.x; i < c.count; i += kThreads)
            store(c.clipped, c.clipped_dtype, i, load(c.grad, c.grad_dtype, i) * f);
    }
}

struct UpdateArgs {
    double scale, max_norm;
    float lr, beta1, beta2, rest1, rest2, eps, decay, ema, ema_rest;
};

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
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x) {
        const Chunk c = chunks[k];
        for (int i = threadIdx.x; i < c.count; i += kThreads) {
            const float g = load(c.grad, c.grad_dtype, i) * f;
            const float m = u.beta1 * c.m[i] + u.rest1 * g;
            const float v = u.beta2 * c.v[i] + u.rest2 * (g * g);
            const float p0 = c.param[i];
            const float d = (m * corr1) / (sqrtf(v * corr2) + u.eps) + u.decay * p0;
            const float p = p0 - u.lr * d;
            c.m[i] = m;
            c.v[i] = v;
            c.param[i] = p;
            if (c.ema) c.ema[i] = u.ema * c.ema[i] + u.ema_rest * p;
        }
    }
}

int sums_of(int64_t chunks) { return (int)std::min<int64_t>(chunks, kMaxSums); }

// Enqueues the first pass; the number of sums it leaves.
int first_pass(const octnca_param_list &l, const int64_t *step, double beta1, double beta2,
               hipStream_t stream) {
    const int sums = std::max(1, sums_of(l.chunks));
    square_sums<<<sums, kThreads, 0, stream>>>(scratch_of(l.table), chunks_of(l.table), l.chunks,
                                               step, beta1, beta2);
    return sums;
}

unsigned second_grid(int64_t chunks) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>(chunks, kMaxSums));
}

}  // namespace

size_t param_table_bytes(int64_t chunks) { return sizeof(Scratch) + (size_t)chunks * sizeof(Chunk); }

hipError_t launch_param_table(const octnca_param *params, int n, void *table, hipStream_t stream) {
    int64_t at = 0;
    for (int i = 0; i < n;) {
        FillArgs f;
        int64_t pieces = 0;
        for (f.n = 0; i < n && f.n < kFillTensors; ++i) {
            if (params[i].count == 0) continue;
            f.t[f.n++] = params[i];
            pieces += (params[i].count + kParamChunk - 1) / kParamChunk;
        }
        if (pieces == 0) continue;
        const unsigned grid = (unsigned)std::min<int64_t>((pieces + kThreads - 1) / kThreads, 256);
        fill_table<<<grid, kThreads, 0, stream>>>(f, chunks_of(table), at);
        at += pieces;
    }
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
