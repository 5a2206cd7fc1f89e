// C ABI of the OctreeNCA inference library (include/octree_nca.h): argument
// checks, buffer planning and the launch sequence of the octree inference
// (Sec. 3.2; supplement S6, Listing 3).  Every entry point validates all of its
// arguments before it enqueues any work, allocates nothing and never
// synchronises the host.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <cmath>
#include <algorithm>
#include <mutex>
#include <new>
#include <utility>
#include <vector>
#include "launch.h"
#include "octree_nca.h"

using namespace octnca;

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 30;      // per axis (kernels index with int)
constexpr int64_t kMaxCells = int64_t(1) << 36;    // per level
constexpr int kMaxLevels = 16;
constexpr int64_t kMaxCacheBytes = int64_t(1) << 60;
constexpr int32_t kMaxCacheStates = INT32_MAX - (1 << 17);   // of a call (steps of int past them)
constexpr int kMaxGroup = 64;   // images of a batch that run together at most
constexpr size_t kAlign = 256;

size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

int check_model(const octnca_model *m) {
    if (m == nullptr) return OCTNCA_EINVAL;
    if (m->ndim != 2 && m->ndim != 3) return OCTNCA_EUNSUPPORTED;
    // C / H: the paper's 16 / 64 and the 12 / 48 and 20 / 100 of its ablation
    // (supplement S10); every size runs on the matrix cores (the specialised
    // kernels for 16 / 64 and, in most cases, 12 / 48, a generic kernel
    // otherwise) and on the vector kernel
    const bool size_ok = (m->channels == 16 && m->hidden == 64) ||
                         (m->channels == 12 && m->hidden == 48) ||
                         (m->channels == 20 && m->hidden == 100);
    if (!size_ok) return OCTNCA_EUNSUPPORTED;
    if (m->n_in != 1 && m->n_in != 3) return OCTNCA_EUNSUPPORTED;
    if (m->state_dtype != OCTNCA_F32 && m->state_dtype != OCTNCA_F16) return OCTNCA_EUNSUPPORTED;
    // step kernel choice
    if (m->mlp < OCTNCA_MLP_AUTO || m->mlp > OCTNCA_MLP_VALU) return OCTNCA_EINVAL;
    if (m->layout2d < OCTNCA_LAYOUT_AUTO || m->layout2d > OCTNCA_LAYOUT_TILES) return OCTNCA_EINVAL;
    if (m->steps_per_launch != 0 && m->steps_per_launch != 1) return OCTNCA_EINVAL;
    if (!(m->channels == 16 && m->hidden == 64) && m->mlp != OCTNCA_MLP_AUTO &&
        m->mlp != OCTNCA_MLP_VALU)
        return OCTNCA_EUNSUPPORTED;   // only the vector kernel serves the other sizes
    if (m->mlp == OCTNCA_MLP_F16 && m->state_dtype != OCTNCA_F16) return OCTNCA_EUNSUPPORTED;
    if (m->mlp == OCTNCA_MLP_F16S && m->state_dtype != OCTNCA_F32) return OCTNCA_EUNSUPPORTED;
    return OCTNCA_OK;
}

// The caller's step-kernel choice (fields checked by check_model).
KernelChoice kernel_choice(const octnca_model *m) {
    KernelChoice k;
    k.valu = m->mlp == OCTNCA_MLP_VALU;
    k.pairs = m->steps_per_launch == 0;
    switch (m->mlp) {
        case OCTNCA_MLP_F32: k.mlp = MfmaMlp::F32; break;
        case OCTNCA_MLP_BF16X3: k.mlp = MfmaMlp::Bf16x3; break;
        case OCTNCA_MLP_F16: k.mlp = MfmaMlp::F16; break;
        case OCTNCA_MLP_F16S: k.mlp = MfmaMlp::F16S; break;
        default: k.mlp = MfmaMlp::Default; break;
    }
    k.layout = m->layout2d == OCTNCA_LAYOUT_ROWS    ? Layout2d::Rows
               : m->layout2d == OCTNCA_LAYOUT_TILES ? Layout2d::Tiles
                                                    : Layout2d::Auto;
    return k;
}

int check_extent(const octnca_model *m, const octnca_extent &e) {
    if (e.d <= 0 || e.h <= 0 || e.w <= 0) return OCTNCA_ESHAPE;
    if (e.d > kMaxDim || e.h > kMaxDim || e.w > kMaxDim) return OCTNCA_ESHAPE;
    if (m->ndim == 2 && e.d != 1) return OCTNCA_ESHAPE;
    // d * h <= 2^60 cannot overflow; the cell count is bounded by division
    // (d * h * w itself could reach 2^90)
    if (e.d * e.h > kMaxCells || e.w > kMaxCells / (e.d * e.h)) return OCTNCA_ESHAPE;
    return OCTNCA_OK;
}

int check_factor(const octnca_model *m, const int32_t *f) {
    for (int a = 0; a < 3; ++a)
        if (f[a] < 1 || f[a] > 8) return OCTNCA_ESHAPE;
    if (m->ndim == 2 && f[0] != 1) return OCTNCA_ESHAPE;
    return OCTNCA_OK;
}

// fire_rate in [0, 1] (NaN rejected); threshold = min(2^32, floor(rate * 2^32)).
bool fire_threshold(float rate, uint64_t *out) {
    if (!(rate >= 0.0f && rate <= 1.0f)) return false;
    const double t = floor((double)rate * 4294967296.0);
    *out = t >= 4294967296.0 ? (uint64_t(1) << 32) : (uint64_t)t;
    return true;
}

size_t elem_bytes(const octnca_model *m) { return m->state_dtype == OCTNCA_F16 ? 2 : 4; }

Extent3 ext3(const octnca_extent &e) { return Extent3{e.d, e.h, e.w}; }

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    return pa < pb + nb && pb < pa + na;
}

int hip_status(hipError_t e) { return e == hipSuccess ? OCTNCA_OK : OCTNCA_EHIP; }

// Level extents, finest first; ESHAPE when a factor does not divide.
int level_extents(const octnca_model *m, octnca_extent finest, int32_t levels,
                  const int32_t *factors, octnca_extent *out) {
    if (levels < 1 || levels > kMaxLevels) return OCTNCA_EINVAL;
    if (levels > 1 && factors == nullptr) return OCTNCA_EINVAL;
    int st = check_extent(m, finest);
    if (st) return st;
    out[0] = finest;
    for (int l = 1; l < levels; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        if ((st = check_factor(m, f))) return st;
        const octnca_extent &p = out[l - 1];
        if (p.d % f[0] || p.h % f[1] || p.w % f[2]) return OCTNCA_ESHAPE;
        out[l] = octnca_extent{p.d / f[0], p.h / f[1], p.w / f[2]};
    }
    return OCTNCA_OK;
}

bool weights_ok(const octnca_level_weights *w) {
    return w != nullptr && w->conv_w && w->conv_b && w->w1 && w->b1 && w->w2;
}

LevelWeightsDev to_dev(const octnca_level_weights *w) {
    return LevelWeightsDev{w->conv_w, w->conv_b, w->w1, w->b1, w->w2};
}

Dtype dtype_of(const octnca_model *m) { return m->state_dtype == OCTNCA_F16 ? Dtype::F16 : Dtype::F32; }

StepArgs step_args(const octnca_model *m, const octnca_extent &e, const octnca_level_weights *w,
                   int32_t level, uint64_t seed, uint64_t threshold, uint32_t batch) {
    StepArgs a;
    a.batch = batch;
    a.dtype = dtype_of(m);
    a.ndim = m->ndim;
    a.n_in = m->n_in;
    a.ext = ext3(e);
    a.w = to_dev(w);
    a.level = (uint32_t)level;
    a.step = 0;
    a.seed = seed;
    a.threshold = threshold;
    a.channels = m->channels;
    a.hidden = m->hidden;
    a.kc = kernel_choice(m);
    return a;
}

// Launches that run steps t0 .. t1-1 of a level: one per step, or one per two
// steps where the two-step kernel applies (a trailing odd step runs alone).
// (Small 2D levels are planned by step_block_plan instead; in the count of
// octree_nca_infer_launches they take one unit per step.)
int32_t level_launches(const StepArgs &a, int32_t t0, int32_t t1) {
    if (t1 <= t0) return 0;
    return step_pairs(a) ? (t1 - t0 + 1) / 2 : t1 - t0;
}

// Steps run by a level's first launch when it is fused with the upsample: two
// where the two-step kernel applies and the level has two steps, else one; 0
// when the first step is not fused.
int32_t fused_up_steps(const StepArgs &a, bool fused, int32_t steps) {
    if (!fused) return 0;
    return steps >= 2 && step_pairs(a) ? 2 : 1;
}

// Enqueue steps t0 .. t1-1 of a level; launch k reads bufs[k % 2] and writes
// bufs[(k + 1) % 2], so the result is in bufs[level_launches(..) % 2].
// seg_last: the last launch also writes the readout of its result there (null:
// no readout); the caller passes it only where that launch's kernel can.
// max_pairs caps the two-step launches (the remaining steps run one per
// launch); it is unlimited by default.
int run_steps(const octnca_model *m, void *b0, void *b1, const octnca_extent &e,
              const octnca_level_weights *w, int32_t level, int32_t t0, int32_t t1,
              uint64_t seed, uint64_t threshold, hipStream_t stream, uint32_t batch = 0,
              uint8_t *seg_last = nullptr, int32_t max_pairs = INT32_MAX) {
    StepArgs a = step_args(m, e, w, level, seed, threshold, batch);
    void *bufs[2] = {b0, b1};
    const bool pairs = step_pairs(a);
    int k = 0;
    int32_t pairs_left = max_pairs;
    for (int32_t t = t0; t < t1; k ^= 1) {
        a.step = (uint32_t)t;
        hipError_t err;
        if (pairs && pairs_left > 0 && t + 1 < t1) {
            --pairs_left;
            a.seg = t + 2 == t1 ? seg_last : nullptr;
            err = launch_step_pair(a, bufs[k], bufs[k ^ 1], stream);
            a.seg = nullptr;
            t += 2;
        } else {
            a.seg = t + 1 == t1 ? seg_last : nullptr;
            err = launch_step(a, bufs[k], bufs[k ^ 1], stream);
            a.seg = nullptr;
            t += 1;
        }
        if (err != hipSuccess) return OCTNCA_EHIP;
    }
    return OCTNCA_OK;
}

// Enqueue steps 0 .. steps-1 of a small 2D level as `plan` divides them over
// launches; launch k reads bufs[k % 2] and writes bufs[(k + 1) % 2], the first
// one with its state formed as `in` says (src: the coarse state, null for a
// seed).  seg: readout of the last state, or null.
int run_block_steps(StepArgs a, const StepBlockPlan &plan, const void *src, void *b0, void *b1,
                    StepBlockInput in, int32_t steps, uint8_t *seg, hipStream_t stream) {
    void *bufs[2] = {b0, b1};
    uint32_t t = 0;
    for (int i = 0; i < plan.launches; ++i) {
        const int n = plan.steps_of(i, steps);
        a.step = t;
        a.seg = i + 1 == plan.launches ? seg : nullptr;
        if (launch_step_block(a, false, plan.tile, n, i == 0 ? src : bufs[i & 1],
                              bufs[(i + 1) & 1], in, stream) != hipSuccess)
            return OCTNCA_EHIP;
        in.img = nullptr;   // the later launches read a state of the level
        in.src_stride = in.dst_stride;
        t += (uint32_t)n;
    }
    return OCTNCA_OK;
}

struct Plan {
    octnca_extent ext[kMaxLevels];
    size_t image_off[kMaxLevels];   // workspace offsets of level images 1..L-1
    size_t state_off[2];            // workspace offsets of the state buffers it holds
    size_t bytes;
};

int make_plan(const octnca_model *m, octnca_extent finest, int32_t levels, const int32_t *factors,
              bool with_final_state, Plan *p) {
    int st = check_model(m);
    if (st) return st;
    if ((st = level_extents(m, finest, levels, factors, p->ext))) return st;
    const size_t eb = elem_bytes(m);
    size_t off = 0;
    p->image_off[0] = 0;
    for (int l = 1; l < levels; ++l) {
        p->image_off[l] = off;
        off += align_up((size_t)(p->ext[l].d * p->ext[l].h * p->ext[l].w) * m->n_in * eb);
    }
    const size_t state_bytes = align_up((size_t)(finest.d * finest.h * finest.w) * m->channels * eb);
    p->state_off[0] = off;
    off += state_bytes;
    p->state_off[1] = off;
    if (!with_final_state) off += state_bytes;
    p->bytes = off;
    return OCTNCA_OK;
}

}  // namespace

extern "C" {

int octree_nca_abi_version(void) { return OCTNCA_ABI_VERSION; }

const char *octree_nca_strerror(int status) {
    switch (status) {
        case OCTNCA_OK: return "ok";
        case OCTNCA_EINVAL: return "invalid argument";
        case OCTNCA_EUNSUPPORTED: return "model configuration not compiled into this library";
        case OCTNCA_ESHAPE: return "invalid extent or pooling factor";
        case OCTNCA_EHIP: return "HIP runtime error";
        case OCTNCA_ESPACE: return "workspace too small";
        default: return "unknown status";
    }
}

int octree_nca_build_pyramid(const octnca_model *model, const void *image, octnca_extent finest,
                             int32_t levels, const int32_t *factors, void *const *level_images,
                             void *stream) {
    int st = check_model(model);
    if (st) return st;
    octnca_extent ext[kMaxLevels];
    if ((st = level_extents(model, finest, levels, factors, ext))) return st;
    if (image == nullptr || (levels > 1 && level_images == nullptr)) return OCTNCA_EINVAL;
    for (int l = 1; l < levels; ++l)
        if (level_images[l - 1] == nullptr) return OCTNCA_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    const void *prev = image;
    for (int l = 1; l < levels; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        const hipError_t e = launch_pool(dtype_of(model), prev, ext3(ext[l]), level_images[l - 1],
                                         f[0], f[1], f[2], model->n_in, s);
        if (e != hipSuccess) return OCTNCA_EHIP;
        prev = level_images[l - 1];
    }
    return OCTNCA_OK;
}

int octree_nca_upsample(const octnca_model *model, const void *coarse_state, octnca_extent coarse,
                        const int32_t *factor, const void *fine_image, void *fine_state,
                        void *stream) {
    int st = check_model(model);
    if (st) return st;
    if (factor == nullptr || coarse_state == nullptr || fine_image == nullptr ||
        fine_state == nullptr)
        return OCTNCA_EINVAL;
    if ((st = check_extent(model, coarse)) || (st = check_factor(model, factor))) return st;
    const octnca_extent fine{coarse.d * factor[0], coarse.h * factor[1], coarse.w * factor[2]};
    if ((st = check_extent(model, fine))) return st;
    const size_t eb = elem_bytes(model);
    const size_t fine_bytes = (size_t)(fine.d * fine.h * fine.w) * model->channels * eb;
    if (overlap(fine_state, fine_bytes, coarse_state,
                (size_t)(coarse.d * coarse.h * coarse.w) * model->channels * eb) ||
        overlap(fine_state, fine_bytes, fine_image,
                (size_t)(fine.d * fine.h * fine.w) * model->n_in * eb))
        return OCTNCA_EINVAL;
    return hip_status(launch_upsample(dtype_of(model), coarse_state, ext3(fine), factor[0],
                                      factor[1], factor[2], fine_image, fine_state, model->n_in,
                                      model->channels, (hipStream_t)stream));
}

int octree_nca_run_level(const octnca_model *model, void *buf0, void *buf1, octnca_extent extent,
                         const octnca_level_weights *weights, int32_t level, int32_t steps,
                         float fire_rate, uint64_t seed, int32_t *result_in_buf1, void *stream) {
    int st = check_model(model);
    if (st) return st;
    if ((st = check_extent(model, extent))) return st;
    uint64_t threshold;
    if (buf0 == nullptr || buf1 == nullptr || !weights_ok(weights) || level < 0 || steps < 0 ||
        !fire_threshold(fire_rate, &threshold))
        return OCTNCA_EINVAL;
    const size_t bytes =
        (size_t)(extent.d * extent.h * extent.w) * model->channels * elem_bytes(model);
    if (overlap(buf0, bytes, buf1, bytes)) return OCTNCA_EINVAL;
    // The number of launches has the parity of `steps`, so that the result is
    // in buf1 exactly when steps is odd, whichever kernels run: an even number
    // of two-step launches (the rest one step each), or on small levels the best
    // division over launches among those of that parity.  (The best of all with
    // a launch added ran two steps of 512^2 cells in 30 us, one launch per step
    // in 21.)
    const StepArgs a = step_args(model, extent, weights, level, seed, threshold, 0);
    StepBlockPlan blocks;
    if (step_block_plan(a, false, steps, 1, &blocks, true)) {
        st = run_block_steps(a, blocks, buf0, buf0, buf1, StepBlockInput{}, steps, nullptr,
                             (hipStream_t)stream);
        if (st) return st;
        if (result_in_buf1) *result_in_buf1 = steps & 1;
        return OCTNCA_OK;
    }
    st = run_steps(model, buf0, buf1, extent, weights, level, 0, steps, seed, threshold,
                   (hipStream_t)stream, 0, nullptr, steps / 4 * 2);
    if (st) return st;
    if (result_in_buf1) *result_in_buf1 = steps & 1;
    return OCTNCA_OK;
}

int octree_nca_readout(const octnca_model *model, const void *state, octnca_extent extent,
                       uint8_t *seg, void *stream) {
    int st = check_model(model);
    if (st) return st;
    if ((st = check_extent(model, extent))) return st;
    if (state == nullptr || seg == nullptr) return OCTNCA_EINVAL;
    return hip_status(launch_readout(dtype_of(model), state, extent.d * extent.h * extent.w,
                                     model->channels, seg, (hipStream_t)stream));
}

int octree_nca_readout_classes(const octnca_model *model, const void *state, octnca_extent extent,
                               int32_t classes, uint8_t *seg, void *stream) {
    int st = check_model(model);
    if (st) return st;
    if ((st = check_extent(model, extent))) return st;
    if (state == nullptr || seg == nullptr || classes < 2 || classes > model->channels - model->n_in)
        return OCTNCA_EINVAL;
    return hip_status(launch_readout_classes(dtype_of(model), state,
                                             extent.d * extent.h * extent.w, model->channels,
                                             classes, seg, (hipStream_t)stream));
}

int32_t octree_nca_first_level_steps(float alpha0, octnca_extent coarsest) {
    if (!(alpha0 >= 0.f) || !std::isfinite(alpha0)) return -1;
    if (coarsest.d <= 0 || coarsest.h <= 0 || coarsest.w <= 0) return -1;
    const int64_t m = std::max(coarsest.d, std::max(coarsest.h, coarsest.w));
    const double steps = std::floor((double)alpha0 * (double)m);
    if (steps > (double)INT32_MAX) return -1;
    return (int32_t)steps;
}

int octree_nca_fire_mask(uint64_t seed, int32_t level, int32_t step, octnca_extent extent,
                         float fire_rate, uint8_t *mask, void *stream) {
    uint64_t threshold;
    if (mask == nullptr || level < 0 || step < 0 || !fire_threshold(fire_rate, &threshold))
        return OCTNCA_EINVAL;
    if (extent.d <= 0 || extent.h <= 0 || extent.w <= 0 || extent.d > kMaxDim ||
        extent.h > kMaxDim || extent.w > kMaxDim || extent.d * extent.h > kMaxCells ||
        extent.d * extent.h * extent.w > kMaxCells)
        return OCTNCA_ESHAPE;
    return hip_status(launch_fire_mask(seed, (uint32_t)level, (uint32_t)step,
                                       extent.d * extent.h * extent.w, threshold, mask,
                                       (hipStream_t)stream));
}

size_t octree_nca_workspace_bytes(const octnca_model *model, octnca_extent finest, int32_t levels,
                                  const int32_t *factors, int32_t with_final_state) {
    Plan p;
    if (make_plan(model, finest, levels, factors, with_final_state != 0, &p)) return 0;
    return p.bytes;
}

int octree_nca_infer_launches(const octnca_model *model, octnca_extent finest, int32_t levels,
                              const int32_t *factors, const int32_t *steps, int32_t *launches) {
    Plan p;
    const int st = make_plan(model, finest, levels, factors, true, &p);
    if (st) return st;
    if (steps == nullptr || launches == nullptr) return OCTNCA_EINVAL;
    for (int l = 0; l < levels; ++l)
        if (steps[l] < 0) return OCTNCA_EINVAL;
    const octnca_level_weights none{};
    for (int l = 0; l < levels; ++l) {
        const StepArgs a = step_args(model, p.ext[l], &none, l, 0, 0, 0);
        const bool fused = l + 1 < levels && steps[l] >= 1 && step_fuses_upsample(a);
        launches[l] = (fused ? 1 : 0) + level_launches(a, fused_up_steps(a, fused, steps[l]),
                                                       steps[l]);
    }
    return OCTNCA_OK;
}

}  // extern "C"

namespace {

// An inference whose levels above `level` have run already: it starts with the
// upsample from `coarse`, the state of level `level` + 1.
struct Resume {
    int32_t level;
    const void *coarse;
};

int infer_impl(const octnca_model *model, const void *image, octnca_extent finest,
               int32_t levels, const int32_t *factors, const octnca_level_weights *weights,
               const int32_t *steps, float fire_rate, uint64_t seed, void *workspace,
               size_t workspace_bytes, void *final_state, uint8_t *seg,
               void *const *level_events, void *stream, uint32_t batch, bool check_only,
               const Resume *resume = nullptr) {
    Plan p;
    int st = make_plan(model, finest, levels, factors, final_state != nullptr, &p);
    if (st) return st;
    uint64_t threshold;
    if (image == nullptr || weights == nullptr || steps == nullptr || workspace == nullptr ||
        !fire_threshold(fire_rate, &threshold))
        return OCTNCA_EINVAL;
    for (int l = 0; l < levels; ++l)
        if (!weights_ok(&weights[l]) || steps[l] < 0) return OCTNCA_EINVAL;
    if (workspace_bytes < p.bytes) return OCTNCA_ESPACE;
    const size_t eb = elem_bytes(model);
    const size_t state_bytes = (size_t)(finest.d * finest.h * finest.w) * model->channels * eb;
    char *ws = (char *)workspace;
    if (final_state != nullptr &&
        (overlap(final_state, state_bytes, workspace, p.bytes) ||
         overlap(final_state, state_bytes, image,
                 (size_t)(finest.d * finest.h * finest.w) * model->n_in * eb)))
        return OCTNCA_EINVAL;
    if (overlap(workspace, p.bytes, image,
                (size_t)(finest.d * finest.h * finest.w) * model->n_in * eb))
        return OCTNCA_EINVAL;
    if (check_only) return OCTNCA_OK;

    // bufs[0] ends up holding the final state: the coarsest seed goes to the
    // buffer that makes the parity of (upsamples + steps) land there.
    void *bufs[2];
    bufs[0] = final_state != nullptr ? final_state : (void *)(ws + p.state_off[1]);
    bufs[1] = (void *)(ws + p.state_off[0]);
    const void *img[kMaxLevels];
    img[0] = image;
    for (int l = 1; l < levels; ++l) img[l] = ws + p.image_off[l];

    const hipStream_t s = (hipStream_t)stream;
    const Dtype dt = dtype_of(model);
    // Levels whose first step reads the next coarser state directly (upsample
    // + inject fused into the step): that transition flips no buffer.
    // Buffer flips: one per unfused upsample and one per step launch.  Small
    // levels run several steps per launch, the first fused with the upsample
    // or, on the coarsest level, with the seed.
    bool fused[kMaxLevels] = {};
    bool block[kMaxLevels] = {};
    StepBlockPlan blocks[kMaxLevels];
    int64_t flips = 0;
    const int32_t top = resume ? resume->level : levels - 1;   // first level to run
    for (int l = 0; l <= top; ++l) {
        const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch);
        block[l] = step_block_plan(a, false, steps[l], 1, &blocks[l]);
        if (block[l]) {
            flips += blocks[l].launches;
            continue;
        }
        if (l + 1 < levels && steps[l] >= 1) fused[l] = step_fuses_upsample(a);
        const int32_t t0 = fused_up_steps(a, fused[l], steps[l]);
        flips += (l + 1 < levels ? 1 : 0) + level_launches(a, t0, steps[l]);
    }
    for (int l = 1; l <= top; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        if (launch_pool(dt, img[l - 1], ext3(p.ext[l]), (void *)img[l], f[0], f[1], f[2],
                        model->n_in, s) != hipSuccess)
            return OCTNCA_EHIP;
    }
    int cur = (int)(flips & 1);
    // the state that level l + 1 left, read by level l's upsample
    const void *coarse = resume ? resume->coarse : bufs[cur];
    if (resume && cur == 1 && overlap(coarse, 1, final_state, state_bytes)) {
        // the first launch writes the buffer that holds the coarse state: move that
        const octnca_extent &e = p.ext[top + 1];
        if (hipMemcpyAsync(bufs[1], coarse, (size_t)(e.d * e.h * e.w) * model->channels * eb,
                           hipMemcpyDeviceToDevice, s) != hipSuccess)
            return OCTNCA_EHIP;
        coarse = bufs[1];
    }
    if (!resume && !block[levels - 1] &&
        launch_upsample(dt, nullptr, ext3(p.ext[levels - 1]), 1, 1, 1, img[levels - 1], bufs[cur],
                        model->n_in, model->channels, s) != hipSuccess)
        return OCTNCA_EHIP;
    bool seg_fused = false;
    for (int l = top; l >= 0; --l) {
        const int32_t *f = factors + 3 * l;
        if (l != top || !resume) coarse = bufs[cur];
        if (l < levels - 1 && !fused[l] && !block[l]) {
            if (launch_upsample(dt, coarse, ext3(p.ext[l]), f[0], f[1], f[2], img[l],
                                bufs[cur ^ 1], model->n_in, model->channels, s) != hipSuccess)
                return OCTNCA_EHIP;
            cur ^= 1;
        }
        if (level_events && level_events[2 * l] &&
            hipEventRecord((hipEvent_t)level_events[2 * l], s) != hipSuccess)
            return OCTNCA_EHIP;
        if (block[l]) {
            const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch);
            StepBlockInput in;
            in.img = img[l];
            if (l < levels - 1) {
                in.coarse_w = (int)p.ext[l + 1].w;
                in.fy = f[1];
                in.fx = f[2];
            }
            seg_fused = l == 0 && seg != nullptr;
            st = run_block_steps(a, blocks[l], l < levels - 1 ? coarse : nullptr, bufs[cur],
                                 bufs[cur ^ 1], in, steps[l], l == 0 ? seg : nullptr, s);
            if (st) return st;
            cur ^= blocks[l].launches & 1;
            if (level_events && level_events[2 * l + 1] &&
                hipEventRecord((hipEvent_t)level_events[2 * l + 1], s) != hipSuccess)
                return OCTNCA_EHIP;
            continue;
        }
        // The finest level's last launch writes the readout too when it is a
        // two-step launch; otherwise the readout kernel runs at the end.
        uint8_t *seg_last = nullptr;
        if (l == 0 && seg != nullptr) {
            const StepArgs a = step_args(model, p.ext[0], &weights[0], 0, seed, threshold, batch);
            const int32_t first = fused_up_steps(a, fused[0], steps[0]);
            const int32_t rest = steps[0] - first;
            bool ok;
            if (step_pairs(a))   // the last launch runs two steps
                ok = rest % 2 == 0 && (rest > 0 || first == 2);
            else                 // the last launch is a single step after the first
                ok = rest >= 1 && step_single_fuses_readout(a);
            if (ok) seg_last = seg;
            seg_fused = ok;
        }
        int32_t t0 = 0;
        if (fused[l]) {
            // step 0 (or steps 0 and 1) from the coarse state (level l + 1)
            // and image l
            StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch);
            t0 = fused_up_steps(a, true, steps[l]);
            if (t0 == steps[l]) a.seg = seg_last;   // this launch is the level's last
            const hipError_t err =
                t0 == 2 ? launch_step_pair_up(a, coarse, (int)p.ext[l + 1].w, f[0], f[1], f[2],
                                              img[l], bufs[cur ^ 1], s)
                        : launch_step_up(a, coarse, (int)p.ext[l + 1].h, (int)p.ext[l + 1].w,
                                         f[0], f[1], f[2], img[l], bufs[cur ^ 1], s);
            if (err != hipSuccess) return OCTNCA_EHIP;
            cur ^= 1;
        }
        st = run_steps(model, bufs[cur], bufs[cur ^ 1], p.ext[l], &weights[l], l, t0, steps[l],
                       seed, threshold, s, batch, seg_last);
        if (st) return st;
        cur ^= level_launches(step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch),
                              t0, steps[l]) & 1;
        if (level_events && level_events[2 * l + 1] &&
            hipEventRecord((hipEvent_t)level_events[2 * l + 1], s) != hipSuccess)
            return OCTNCA_EHIP;
    }
    // cur == 0 here by construction of the seed buffer
    if (seg != nullptr && !seg_fused &&
        launch_readout(dt, bufs[cur], finest.d * finest.h * finest.w, model->channels, seg, s) !=
            hipSuccess)
        return OCTNCA_EHIP;
    return OCTNCA_OK;
}

}  // namespace

extern "C" {

int octree_nca_infer(const octnca_model *model, const void *image, octnca_extent finest,
                     int32_t levels, const int32_t *factors, const octnca_level_weights *weights,
                     const int32_t *steps, float fire_rate, uint64_t seed, void *workspace,
                     size_t workspace_bytes, void *final_state, uint8_t *seg,
                     void *const *level_events, void *stream) {
    return infer_impl(model, image, finest, levels, factors, weights, steps, fire_rate, seed,
                      workspace, workspace_bytes, final_state, seg, level_events, stream, 0,
                      false);
}

// ---------------------------------------------------------------------------
// Inference without allocation: the workspace is a static device array.
// ---------------------------------------------------------------------------

}  // extern "C"

namespace {

// A batch is run in groups.  The small levels of one image leave most of the
// chip idle, so the coarse levels of a group's images run in the same launches,
// with their level states in the group's own final states, which hold nothing
// yet.  Images of a group: as many as have room for their pyramid images in the
// workspace, the batch divided evenly; 1 where the groups would not apply.
int32_t batch_group(const octnca_model *m, const Plan &p, int32_t batch, int32_t levels,
                    size_t workspace_bytes, bool with_final_states) {
    if (batch < 2 || m->ndim != 2 || !with_final_states) return 1;
    const size_t eb = elem_bytes(m);
    size_t pyramid = 0;   // n images' levels need at most n times this
    for (int l = 1; l < levels; ++l)
        pyramid += align_up((size_t)(p.ext[l].h * p.ext[l].w) * m->n_in * eb);
    int64_t n = std::min<int64_t>(batch, kMaxGroup);
    if (pyramid > 0) n = std::min<int64_t>(n, (int64_t)(workspace_bytes / pyramid));
    if (n < 2) return 1;
    const int64_t groups = (batch + n - 1) / n;
    return (int32_t)((batch + groups - 1) / groups);
}

// The finest level from which a group of n images runs together up to the
// coarsest one (levels: none does).  The levels are those that the multi-step
// launches take; two buffers of the finest of them, or of level 1 where level
// 0 is among them, have to fit the final states.  Levels finer than those are
// pooled for the group, to reach the coarse ones, and again image by image
// (their place in the workspace is the second state buffer), so the group has
// to save more than that: two images of 4096^2 with levels of 512^2 and below
// together took 1750 us for one step a level instead of 1646, for 20 steps 21.2
// ms instead of 21.6.
int32_t group_levels(const octnca_model *m, const Plan &p, int32_t n, int32_t levels,
                     const octnca_level_weights *weights, const int32_t *steps) {
    constexpr double kPoolLaunchUs = 2.5, kPoolBytesPerUs = 6.5e6;   // measured
    int32_t from = levels;
    double saved = (double)(n - 1) * (levels - 1) * kPoolLaunchUs;
    double gain[kMaxLevels + 1] = {};   // with the levels from l on together
    StepBlockPlan blocks;
    while (from > 0) {
        const StepArgs a = step_args(m, p.ext[from - 1], &weights[from - 1], from - 1, 0, 0, 0);
        if (!step_block_plan(a, false, steps[from - 1], n, &blocks)) break;
        saved -= blocks.us;
        step_block_plan(a, false, steps[from - 1], 1, &blocks);
        saved += n * blocks.us;
        gain[--from] = saved;
    }
    const int64_t cells = p.ext[0].h * p.ext[0].w;
    auto fits = [&](int l) { return 2 * p.ext[l].h * p.ext[l].w <= cells; };
    if (from == 0 && levels > 1 && !fits(1)) from = 1;
    while (from > 0 && from < levels && !fits(from)) ++from;
    int32_t best = levels;
    double again = 0, most = 0;
    for (int32_t l = 0; l < levels; ++l) {
        if (l > 1) {   // level l - 1 is pooled twice
            const int64_t values = p.ext[l - 2].h * p.ext[l - 2].w + p.ext[l - 1].h * p.ext[l - 1].w;
            again += n * (kPoolLaunchUs + values * m->n_in * elem_bytes(m) / kPoolBytesPerUs);
        }
        if (l >= from && gain[l] - again > most) {
            most = gain[l] - again;
            best = l;
        }
    }
    return best;
}

// A group of n images (their first one is image `batch` of the call): levels
// from `together` up run for all images at once, the finer ones image by image
// (the finest, where it runs together, in as large parts as leave a second
// buffer).  The arguments have been checked.
int infer_group(const octnca_model *model, const void *images, int32_t n, octnca_extent finest,
                int32_t levels, const int32_t *factors, const octnca_level_weights *weights,
                const int32_t *steps, float fire_rate, uint64_t seed, void *workspace,
                size_t workspace_bytes, void *final_states, uint8_t *segs, void *stream,
                uint32_t batch, int32_t together) {
    Plan p;
    int st = make_plan(model, finest, levels, factors, true, &p);
    if (st) return st;
    uint64_t threshold;
    if (!fire_threshold(fire_rate, &threshold)) return OCTNCA_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    const Dtype dt = dtype_of(model);
    const size_t eb = elem_bytes(model);
    const int64_t c = model->channels;
    auto cells_of = [&](int l) { return p.ext[l].h * p.ext[l].w; };
    const size_t state_bytes = (size_t)(cells_of(0) * c) * eb;
    const size_t image_bytes = (size_t)(cells_of(0) * model->n_in) * eb;
    char *const out = (char *)final_states;

    // Pyramids of the group, [n][h][w] per level: the batch as a z axis.  Only
    // the levels that run together need them.
    const int32_t shared = std::max(together, 1);   // finest level of the shared coarse part
    const void *img[kMaxLevels];
    img[0] = images;
    size_t off = 0;
    for (int l = 1; l < levels; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        void *dst = (char *)workspace + off;
        const Extent3 e{n, p.ext[l].h, p.ext[l].w};
        if (launch_pool(dt, img[l - 1], e, dst, f[0], f[1], f[2], model->n_in, s) != hipSuccess)
            return OCTNCA_EHIP;
        img[l] = dst;
        off += align_up((size_t)(n * cells_of(l) * model->n_in) * eb);
    }

    // Coarse levels of all images: two buffers at the end of the group's final
    // states, image i's state of a level at i states of that level.  The last
    // level's result lands in the one at the very end.
    const void *coarse = nullptr;
    const size_t shared_bytes = shared < levels ? (size_t)(cells_of(shared) * c) * eb : 0;
    if (shared < levels) {
        void *bufs[2] = {out + n * (state_bytes - shared_bytes),
                         out + n * (state_bytes - 2 * shared_bytes)};
        StepBlockPlan blocks[kMaxLevels];
        int flips = 0;
        for (int l = shared; l < levels; ++l) {
            const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch);
            if (!step_block_plan(a, false, steps[l], n, &blocks[l])) return OCTNCA_EINVAL;
            flips += blocks[l].launches;
        }
        int cur = flips & 1;
        for (int l = levels - 1; l >= shared; --l) {
            const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, batch);
            StepBlockInput in;
            in.images = n;
            in.img = img[l];
            in.img_stride = cells_of(l) * model->n_in;
            in.dst_stride = cells_of(l) * c;
            if (l < levels - 1) {
                in.coarse_w = (int)p.ext[l + 1].w;
                in.fy = factors[3 * l + 1];
                in.fx = factors[3 * l + 2];
                in.src_stride = cells_of(l + 1) * c;
            }
            st = run_block_steps(a, blocks[l], l < levels - 1 ? bufs[cur] : nullptr, bufs[cur],
                                 bufs[cur ^ 1], in, steps[l], nullptr, s);
            if (st) return st;
            cur ^= blocks[l].launches & 1;
        }
        coarse = bufs[0];
    }

    for (int32_t b = 0; b < n;) {
        // Images b .. b + k - 1: their final states and as many further ones as
        // a second buffer, short of the coarse states still to be read.
        const int64_t left = n - b;
        int32_t k = 1;
        StepBlockPlan blocks;
        StepArgs a = step_args(model, p.ext[0], &weights[0], 0, seed, threshold, batch + b);
        if (together == 0)
            k = (int32_t)std::max<int64_t>(
                1, left * (int64_t)(state_bytes - shared_bytes) / (int64_t)(2 * state_bytes));
        const void *from =
            coarse ? (const void *)((const char *)coarse + b * shared_bytes) : nullptr;
        const void *image = (const char *)images + b * image_bytes;
        uint8_t *seg = segs ? segs + b * cells_of(0) : nullptr;
        if (k > 1 && step_block_plan(a, false, steps[0], k, &blocks)) {
            StepBlockInput in;
            in.images = k;
            in.img = image;
            in.img_stride = cells_of(0) * model->n_in;
            in.dst_stride = cells_of(0) * c;
            if (from) {
                in.coarse_w = (int)p.ext[1].w;
                in.fy = factors[1];
                in.fx = factors[2];
                in.src_stride = cells_of(1) * c;
            }
            void *mine = out + b * state_bytes, *other = out + (b + k) * state_bytes;
            const bool odd = blocks.launches & 1;
            st = run_block_steps(a, blocks, from, odd ? other : mine, odd ? mine : other, in,
                                 steps[0], seg, s);
        } else {
            k = 1;
            const Resume resume{shared - 1, from};
            st = infer_impl(model, image, finest, levels, factors, weights, steps, fire_rate, seed,
                            workspace, workspace_bytes, out + b * state_bytes, seg, nullptr,
                            stream, batch + (uint32_t)b, false, from ? &resume : nullptr);
        }
        if (st) return st;
        b += k;
    }
    return OCTNCA_OK;
}

// Static scratch of octree_nca_infer_static: the pyramid images and the second
// state buffer of one inference.  Each device the library runs on holds its
// own copy until the process ends.  In host code `scratch` only names the
// symbol; its device address comes from hipGetSymbolAddress, per device.
__device__ __align__(256) unsigned char scratch[OCTNCA_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;

// Device address of the current device's scratch, looked up once per device
// (with that device current) and kept; nullptr if the lookup failed.
void *scratch_ptr() {
    static std::mutex mu;
    static void *ptrs[kMaxDevices] = {};
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (ptrs[dev] == nullptr) {
        void *p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr)
            return nullptr;
        ptrs[dev] = p;
    }
    return ptrs[dev];
}

}  // namespace

extern "C" {

int octree_nca_infer_static(const octnca_model *model, const void *image, octnca_extent finest,
                            int32_t levels, const int32_t *factors,
                            const octnca_level_weights *weights, const int32_t *steps,
                            float fire_rate, uint64_t seed, void *final_state, uint8_t *seg,
                            void *stream) {
    Plan p;
    int st = make_plan(model, finest, levels, factors, true, &p);
    if (st) return st;
    if (final_state == nullptr) return OCTNCA_EINVAL;
    if (p.bytes > (size_t)OCTNCA_STATIC_SCRATCH_BYTES) return OCTNCA_ESPACE;
    void *ws = scratch_ptr();
    if (ws == nullptr) return OCTNCA_EHIP;
    // Nothing in the workspace needs to start at zero: every pyramid image is
    // written by the pooling and the state buffer by the seed or a step before
    // it is read.
    return infer_impl(model, image, finest, levels, factors, weights, steps, fire_rate, seed, ws,
                      (size_t)OCTNCA_STATIC_SCRATCH_BYTES, final_state, seg, nullptr, stream, 0,
                      false);
}

int octree_nca_infer_batch(const octnca_model *model, const void *images, int32_t batch,
                           octnca_extent finest, int32_t levels, const int32_t *factors,
                           const octnca_level_weights *weights, const int32_t *steps,
                           float fire_rate, uint64_t seed, void *workspace,
                           size_t workspace_bytes, void *final_states, uint8_t *segs,
                           void *stream) {
    int st = check_model(model);
    if (st) return st;
    if (images == nullptr || batch < 1) return OCTNCA_EINVAL;
    if ((st = check_extent(model, finest))) return st;
    const size_t cells = (size_t)(finest.d * finest.h * finest.w);
    const size_t eb = elem_bytes(model);
    const size_t image_bytes = cells * model->n_in * eb;
    const size_t state_bytes = cells * model->channels * eb;
    // the byte counts below (state_bytes * batch at most) stay far from 2^64
    if ((uint64_t)batch > (uint64_t(1) << 48) / state_bytes) return OCTNCA_EINVAL;
    // the batch's outputs must not overlap its inputs or the workspace
    if (final_states != nullptr &&
        (overlap(final_states, state_bytes * batch, images, image_bytes * batch) ||
         (workspace != nullptr &&
          overlap(final_states, state_bytes * batch, workspace, workspace_bytes))))
        return OCTNCA_EINVAL;
    if (segs != nullptr &&
        (overlap(segs, cells * batch, images, image_bytes * batch) ||
         (final_states != nullptr && overlap(segs, cells * batch, final_states,
                                             state_bytes * batch)) ||
         (workspace != nullptr && overlap(segs, cells * batch, workspace, workspace_bytes))))
        return OCTNCA_EINVAL;
    if (workspace != nullptr && overlap(workspace, workspace_bytes, images, image_bytes * batch))
        return OCTNCA_EINVAL;
    auto image_of = [&](int32_t b) { return (const char *)images + image_bytes * b; };
    auto state_of = [&](int32_t b) {
        return final_states ? (void *)((char *)final_states + state_bytes * b) : nullptr;
    };
    auto seg_of = [&](int32_t b) { return segs ? segs + cells * b : nullptr; };
    // every image's arguments are checked before anything is enqueued
    for (int32_t b = 0; b < batch; ++b) {
        st = infer_impl(model, image_of(b), finest, levels, factors, weights, steps, fire_rate,
                        seed, workspace, workspace_bytes, state_of(b), seg_of(b), nullptr, stream,
                        (uint32_t)b, true);
        if (st) return st;
    }
    // groups of images whose coarse levels run together, the others one by one
    Plan p;
    if ((st = make_plan(model, finest, levels, factors, final_states != nullptr, &p))) return st;
    const int32_t group = batch_group(model, p, batch, levels, workspace_bytes,
                                      final_states != nullptr);
    for (int32_t b = 0, n; b < batch; b += n) {
        n = std::min(group, batch - b);
        const int32_t together = n > 1 ? group_levels(model, p, n, levels, weights, steps) : levels;
        if (together < levels) {
            st = infer_group(model, image_of(b), n, finest, levels, factors, weights, steps,
                             fire_rate, seed, workspace, workspace_bytes, state_of(b), seg_of(b),
                             stream, (uint32_t)b, together);
        } else {
            n = 1;
            st = infer_impl(model, image_of(b), finest, levels, factors, weights, steps, fire_rate,
                            seed, workspace, workspace_bytes, state_of(b), seg_of(b), nullptr,
                            stream, (uint32_t)b, false);
        }
        if (st) return st;
    }
    return OCTNCA_OK;
}

// ---------------------------------------------------------------------------
// Training (fp32 states): backward of a step, of the upsample, a readout MSE
// and the whole training step (Sec. 3.2 efficient training; supplement S7).
// ---------------------------------------------------------------------------

size_t octree_nca_step_backward_workspace_bytes(const octnca_model *model, octnca_extent extent) {
    if (check_model(model) || check_extent(model, extent)) return 0;
    return step_backward_workspace_floats(model->ndim, model->channels, model->hidden,
                                          ext3(extent)) *
           sizeof(float);
}

int octree_nca_step_backward(const octnca_model *model, const void *state, const void *grad_out,
                             octnca_extent extent, const octnca_level_weights *weights,
                             int32_t level, int32_t step, float fire_rate, uint64_t seed,
                             void *grad_in, const octnca_level_grads *grads, void *workspace,
                             size_t workspace_bytes, void *stream) {
    int st = check_model(model);
    if (st) return st;
    if (model->state_dtype != OCTNCA_F32) return OCTNCA_EUNSUPPORTED;
    if ((st = check_extent(model, extent))) return st;
    uint64_t threshold;
    if (state == nullptr || grad_out == nullptr || grad_in == nullptr || workspace == nullptr ||
        !weights_ok(weights) || grads == nullptr || !grads->conv_w || !grads->conv_b ||
        !grads->w1 || !grads->b1 || !grads->w2 || level < 0 || step < 0 ||
        !fire_threshold(fire_rate, &threshold))
        return OCTNCA_EINVAL;
    const size_t need = octree_nca_step_backward_workspace_bytes(model, extent);
    if (workspace_bytes < need) return OCTNCA_ESPACE;
    const size_t bytes = (size_t)(extent.d * extent.h * extent.w) * model->channels * sizeof(float);
    if (overlap(grad_in, bytes, state, bytes) || overlap(workspace, need, state, bytes) ||
        overlap(workspace, need, grad_in, bytes) || overlap(workspace, need, grad_out, bytes))
        return OCTNCA_EINVAL;
    if (grad_in != grad_out && overlap(grad_in, bytes, grad_out, bytes)) return OCTNCA_EINVAL;
    StepArgs a = step_args(model, extent, weights, level, seed, threshold, 0);
    a.step = (uint32_t)step;
    const LevelGradsDev g{grads->conv_w, grads->conv_b, grads->w1, grads->b1, grads->w2};
    return hip_status(launch_step_backward(a, (const float *)state, (const float *)grad_out,
                                           (float *)grad_in, g, (float *)workspace,
                                           (hipStream_t)stream));
}

int octree_nca_upsample_backward(const octnca_model *model, const void *grad_fine,
                                 octnca_extent coarse, const int32_t *factor, void *grad_coarse,
                                 void *stream) {
    int st = check_model(model);
    if (st) return st;
    if (model->state_dtype != OCTNCA_F32) return OCTNCA_EUNSUPPORTED;
    if (grad_fine == nullptr || grad_coarse == nullptr || factor == nullptr) return OCTNCA_EINVAL;
    if ((st = check_extent(model, coarse)) || (st = check_factor(model, factor))) return st;
    const octnca_extent fine{coarse.d * factor[0], coarse.h * factor[1], coarse.w * factor[2]};
    if ((st = check_extent(model, fine))) return st;
    if (overlap(grad_coarse, (size_t)(coarse.d * coarse.h * coarse.w) * model->channels * 4,
                grad_fine, (size_t)(fine.d * fine.h * fine.w) * model->channels * 4))
        return OCTNCA_EINVAL;
    return hip_status(launch_upsample_adjoint((const float *)grad_fine, ext3(coarse), factor[0],
                                              factor[1], factor[2], model->n_in, model->channels,
                                              (float *)grad_coarse, (hipStream_t)stream));
}

size_t octree_nca_readout_mse_workspace_bytes(octnca_extent extent) {
    if (extent.d <= 0 || extent.h <= 0 || extent.w <= 0) return 0;
    return mse_workspace_doubles(extent.d * extent.h * extent.w) * sizeof(double);
}

int octree_nca_readout_mse(const octnca_model *model, const void *state, const float *target,
                           octnca_extent extent, void *grad, double *loss, void *workspace,
                           size_t workspace_bytes, void *stream) {
    int st = check_model(model);
    if (st) return st;
    if (model->state_dtype != OCTNCA_F32) return OCTNCA_EUNSUPPORTED;
    if ((st = check_extent(model, extent))) return st;
    if (state == nullptr || target == nullptr || grad == nullptr || loss == nullptr ||
        workspace == nullptr)
        return OCTNCA_EINVAL;
    const int64_t cells = extent.d * extent.h * extent.w;
    if (workspace_bytes < octree_nca_readout_mse_workspace_bytes(extent)) return OCTNCA_ESPACE;
    const size_t bytes = (size_t)cells * model->channels * sizeof(float);
    if (overlap(grad, bytes, state, bytes) || overlap(grad, bytes, target, (size_t)cells * 8) ||
        overlap(workspace, workspace_bytes, grad, bytes))
        return OCTNCA_EINVAL;
    return hip_status(launch_readout_mse((const float *)state, target, cells, model->channels,
                                         (float *)grad, loss, (double *)workspace,
                                         (hipStream_t)stream));
}

}  // extern "C"

namespace {

// Workspace of a training step: pyramid images 1..L-1, the states of every
// level (before each step and after the last), two finest-size gradient
// buffers, the level-backward workspace (finest size) and the loss partials.
struct TrainPlan {
    octnca_extent ext[kMaxLevels];
    size_t image_off[kMaxLevels];
    size_t tape_off[kMaxLevels];    // state t of level l at tape_off[l] + t * state bytes of l
    size_t grad_off[2], bwd_off, mse_off, bytes;
};

int make_train_plan(const octnca_model *m, octnca_extent finest, int32_t levels,
                    const int32_t *factors, const int32_t *steps, TrainPlan *p) {
    int st = check_model(m);
    if (st) return st;
    if (m->state_dtype != OCTNCA_F32) return OCTNCA_EUNSUPPORTED;
    if ((st = level_extents(m, finest, levels, factors, p->ext))) return st;
    if (steps == nullptr) return OCTNCA_EINVAL;
    for (int l = 0; l < levels; ++l)
        if (steps[l] < 0) return OCTNCA_EINVAL;
    size_t off = 0;
    p->image_off[0] = 0;
    for (int l = 1; l < levels; ++l) {
        p->image_off[l] = off;
        off += align_up((size_t)(p->ext[l].d * p->ext[l].h * p->ext[l].w) * m->n_in * 4);
    }
    for (int l = 0; l < levels; ++l) {
        p->tape_off[l] = off;
        const size_t sb = (size_t)(p->ext[l].d * p->ext[l].h * p->ext[l].w) * m->channels * 4;
        off += align_up(sb * ((size_t)steps[l] + 1));
    }
    const int64_t cells = finest.d * finest.h * finest.w;
    const size_t gb = align_up((size_t)cells * m->channels * 4);
    p->grad_off[0] = off;
    off += gb;
    p->grad_off[1] = off;
    off += gb;
    p->bwd_off = off;
    // the finest level needs the most (every level's extent is at most the finest's)
    off += align_up(level_backward_workspace_floats(m->ndim, m->channels, m->hidden, ext3(finest)) *
                    4);
    p->mse_off = off;
    off += align_up(mse_workspace_doubles(cells) * sizeof(double));
    p->bytes = off;
    return OCTNCA_OK;
}

// Forward step of a training pass: split-bf16 MLP operands on the
// matrix-core kernel for C = 16, H = 64 (each product to about 2^-16, three
// bf16 products instead of one fp32 one: a fifth of the matrix-core time),
// fp32 FMAs on the vector kernel otherwise.
hipError_t train_forward_step(const StepArgs &a, const void *src, void *dst, hipStream_t s) {
    if (a.channels == kC && a.hidden == kH)
        return launch_step_mfma(a, MfmaMlp::Bf16x3, Layout2d::Auto, src, dst, s);
    return launch_step_valu(a, src, dst, s);
}

hipError_t clear_grads(const octnca_model *m, const octnca_level_grads &g, hipStream_t s) {
    const int64_t c = m->channels, h = m->hidden;
    float *at[] = {g.conv_w, g.conv_b, g.w1, g.b1, g.w2};
    const int64_t n[] = {c * (m->ndim == 3 ? 27 : 9), c, h * 2 * c, h, c * h};
    for (int i = 0; i < 5; ++i) {
        const hipError_t e = launch_fill_zero(at[i], n[i], s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Forward steps t0 .. t0 + n - 1 of a level: the state after step t goes to
// dst + (t - t0) states; src is the state before step t0, outside those.
hipError_t train_forward_run(StepArgs a, int32_t t0, int32_t n, const float *src, float *dst,
                             hipStream_t s) {
    const size_t state = (size_t)a.ext.cells() * a.channels;
    StepBlockPlan blocks;
    if (step_block_plan(a, true, n, 1, &blocks)) {
        for (int i = 0, t = 0; i < blocks.launches; ++i) {
            const int k = blocks.steps_of(i, n);
            a.step = (uint32_t)(t0 + t);
            const hipError_t e =
                launch_step_block(a, true, blocks.tile, k, t == 0 ? src : dst + (t - 1) * state,
                                  dst + t * state, StepBlockInput{}, s);
            if (e != hipSuccess) return e;
            t += k;
        }
        return hipSuccess;
    }
    for (int32_t t = 0; t < n; ++t) {
        a.step = (uint32_t)(t0 + t);
        const hipError_t e =
            train_forward_step(a, t == 0 ? src : dst + (t - 1) * state, dst + t * state, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

extern "C" {

size_t octree_nca_train_workspace_bytes(const octnca_model *model, octnca_extent finest,
                                        int32_t levels, const int32_t *factors,
                                        const int32_t *steps) {
    TrainPlan p;
    return make_train_plan(model, finest, levels, factors, steps, &p) ? 0 : p.bytes;
}

int octree_nca_train_step(const octnca_model *model, const void *image, octnca_extent finest,
                          int32_t levels, const int32_t *factors,
                          const octnca_level_weights *weights, const int32_t *steps,
                          float fire_rate, uint64_t seed, const float *target, void *workspace,
                          size_t workspace_bytes, const octnca_level_grads *grads, double *loss,
                          void *final_state, void *stream) {
    TrainPlan p;
    int st = make_train_plan(model, finest, levels, factors, steps, &p);
    if (st) return st;
    uint64_t threshold;
    if (image == nullptr || weights == nullptr || target == nullptr || workspace == nullptr ||
        grads == nullptr || loss == nullptr || !fire_threshold(fire_rate, &threshold))
        return OCTNCA_EINVAL;
    for (int l = 0; l < levels; ++l)
        if (!weights_ok(&weights[l]) || !grads[l].conv_w || !grads[l].conv_b || !grads[l].w1 ||
            !grads[l].b1 || !grads[l].w2)
            return OCTNCA_EINVAL;
    if (workspace_bytes < p.bytes) return OCTNCA_ESPACE;
    const int64_t cells = finest.d * finest.h * finest.w;
    const size_t state_bytes = (size_t)cells * model->channels * 4;
    if (overlap(workspace, p.bytes, image, (size_t)cells * model->n_in * 4) ||
        overlap(workspace, p.bytes, target, (size_t)cells * 8) ||
        (final_state && overlap(workspace, p.bytes, final_state, state_bytes)))
        return OCTNCA_EINVAL;

    const hipStream_t s = (hipStream_t)stream;
    char *ws = (char *)workspace;
    auto img = [&](int l) { return l == 0 ? image : (const void *)(ws + p.image_off[l]); };
    auto cells_of = [&](int l) { return p.ext[l].d * p.ext[l].h * p.ext[l].w; };
    auto tape = [&](int l, int t) {
        return (float *)(ws + p.tape_off[l]) + (size_t)t * cells_of(l) * model->channels;
    };
    auto ok = [](hipError_t e) { return e == hipSuccess; };

    // forward, keeping every state
    for (int l = 1; l < levels; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        if (!ok(launch_pool(Dtype::F32, img(l - 1), ext3(p.ext[l]), ws + p.image_off[l], f[0],
                            f[1], f[2], model->n_in, s)))
            return OCTNCA_EHIP;
    }
    for (int l = levels - 1; l >= 0; --l) {
        const hipError_t e =
            l == levels - 1
                ? launch_upsample(Dtype::F32, nullptr, ext3(p.ext[l]), 1, 1, 1, img(l), tape(l, 0),
                                  model->n_in, model->channels, s)
                : launch_upsample(Dtype::F32, tape(l + 1, steps[l + 1]), ext3(p.ext[l]),
                                  factors[3 * l], factors[3 * l + 1], factors[3 * l + 2], img(l),
                                  tape(l, 0), model->n_in, model->channels, s);
        if (!ok(e)) return OCTNCA_EHIP;
        const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, 0);
        if (!ok(train_forward_run(a, 0, steps[l], tape(l, 0), tape(l, 1), s))) return OCTNCA_EHIP;
    }
    const float *final_fine = tape(0, steps[0]);
    float *g = (float *)(ws + p.grad_off[0]);
    float *g_other = (float *)(ws + p.grad_off[1]);
    if (!ok(launch_readout_mse(final_fine, target, cells, model->channels, g, loss,
                               (double *)(ws + p.mse_off), s)))
        return OCTNCA_EHIP;
    if (final_state &&
        !ok(hipMemcpyAsync(final_state, final_fine, state_bytes, hipMemcpyDeviceToDevice, s)))
        return OCTNCA_EHIP;

    // backward, finest level first; a level's backward writes its weight
    // gradients, so only levels without steps are cleared here
    for (int l = 0; l < levels; ++l)
        if (steps[l] == 0 && !ok(clear_grads(model, grads[l], s))) return OCTNCA_EHIP;
    for (int l = 0; l < levels; ++l) {
        StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, 0);
        const LevelGradsDev gd{grads[l].conv_w, grads[l].conv_b, grads[l].w1, grads[l].b1,
                               grads[l].w2};
        // all steps of the level, last first (dL/dS of its first state lands
        // in the other gradient buffer)
        if (steps[l] > 0) {
            if (!ok(launch_level_backward(a, steps[l], false, tape(l, 0), g, g_other, gd,
                                          (float *)(ws + p.bwd_off), s)))
                return OCTNCA_EHIP;
            std::swap(g, g_other);
        }
        if (l + 1 < levels) {
            if (!ok(launch_upsample_adjoint(g, ext3(p.ext[l + 1]), factors[3 * l],
                                            factors[3 * l + 1], factors[3 * l + 2], model->n_in,
                                            model->channels, g_other, s)))
                return OCTNCA_EHIP;
            std::swap(g, g_other);
        }
    }
    return OCTNCA_OK;
}

}  // extern "C"

namespace {

// Workspace of a training step whose states are kept in 8 bits: pyramid images
// 1..L-1, every level's codes and scales, a window of fp32 states, and the
// gradient buffers and scratch of TrainPlan.
struct KeptPlan {
    octnca_extent ext[kMaxLevels];
    size_t image_off[kMaxLevels];
    CacheArgs cache[kMaxLevels];      // offsets in codes / scales until placed
    size_t code_off[kMaxLevels], scale_off[kMaxLevels];
    int32_t window[kMaxLevels];       // states of a level that the window holds, even
    size_t window_off, grad_off[2], bwd_off, mse_off, bytes;
};

// The window holds kWindowStates of the finest level, and so more of the coarser
// ones.  A level's forward uses its halves in turn (a run of steps reads the last
// state of the other half), its backward all of it.
constexpr int32_t kWindowStates = 4;
constexpr int32_t kMaxWindow = 32;

int make_kept_plan(const octnca_model *m, octnca_extent finest, int32_t levels,
                   const int32_t *factors, const int32_t *steps, const octnca_keep *keep,
                   KeptPlan *p) {
    TrainPlan t;
    int st = make_train_plan(m, finest, levels, factors, steps, &t);
    if (st) return st;
    if (keep == nullptr || (keep->code != OCTNCA_CODE_I8 && keep->code != OCTNCA_CODE_F8) ||
        (keep->block != 32 && keep->block != 64 && keep->block != 128))
        return OCTNCA_EINVAL;
    const int64_t finest_cells = finest.d * finest.h * finest.w;
    size_t off = 0;
    for (int l = 0; l < levels; ++l) {
        p->ext[l] = t.ext[l];
        p->image_off[l] = off;
        const int64_t cells = t.ext[l].d * t.ext[l].h * t.ext[l].w;
        if (l > 0) off += align_up((size_t)cells * m->n_in * 4);
        const int64_t room = kWindowStates * (finest_cells / cells);
        p->window[l] = (int32_t)std::min<int64_t>(room, kMaxWindow) / 2 * 2;
    }
    for (int l = 0; l < levels; ++l) {
        const int64_t cells = t.ext[l].d * t.ext[l].h * t.ext[l].w;
        // no sum of the sizes below leaves 64 bits
        if (steps[l] > kMaxCacheBytes / kMaxLevels / (cells * m->channels * 5)) return OCTNCA_ESHAPE;
        CacheArgs a{};
        a.n_slots = steps[l];
        a.cells = a.count = cells;
        a.blocks = (cells + keep->block - 1) / keep->block;
        a.block = keep->block;
        a.channels = m->channels;
        a.f8 = keep->code == OCTNCA_CODE_F8;
        p->cache[l] = a;
        p->code_off[l] = off;
        off += align_up((size_t)steps[l] * cells * m->channels);
        p->scale_off[l] = off;
        off += align_up((size_t)steps[l] * a.blocks * m->channels * 4);
    }
    p->window_off = off;
    off += align_up((size_t)kWindowStates * finest_cells * m->channels * 4);
    // what the other training step has behind its states, unchanged
    const size_t base = t.grad_off[0];
    for (int i = 0; i < 2; ++i) p->grad_off[i] = off + (t.grad_off[i] - base);
    p->bwd_off = off + (t.bwd_off - base);
    p->mse_off = off + (t.mse_off - base);
    p->bytes = off + (t.bytes - base);
    return OCTNCA_OK;
}

}  // namespace

extern "C" {

size_t octree_nca_train_kept_workspace_bytes(const octnca_model *model, octnca_extent finest,
                                             int32_t levels, const int32_t *factors,
                                             const int32_t *steps, const octnca_keep *keep) {
    KeptPlan p;
    return make_kept_plan(model, finest, levels, factors, steps, keep, &p) ? 0 : p.bytes;
}

int octree_nca_train_step_kept(const octnca_model *model, const void *image, octnca_extent finest,
                               int32_t levels, const int32_t *factors,
                               const octnca_level_weights *weights, const int32_t *steps,
                               float fire_rate, uint64_t seed, const float *target,
                               const octnca_keep *keep, void *workspace, size_t workspace_bytes,
                               const octnca_level_grads *grads, double *loss, void *final_state,
                               void *stream) {
    KeptPlan p;
    const int st = make_kept_plan(model, finest, levels, factors, steps, keep, &p);
    if (st) return st;
    uint64_t threshold;
    if (image == nullptr || weights == nullptr || target == nullptr || workspace == nullptr ||
        grads == nullptr || loss == nullptr || !fire_threshold(fire_rate, &threshold) ||
        (uintptr_t)workspace % 16)
        return OCTNCA_EINVAL;
    for (int l = 0; l < levels; ++l)
        if (!weights_ok(&weights[l]) || !grads[l].conv_w || !grads[l].conv_b || !grads[l].w1 ||
            !grads[l].b1 || !grads[l].w2)
            return OCTNCA_EINVAL;
    if (workspace_bytes < p.bytes) return OCTNCA_ESPACE;
    const int64_t cells = finest.d * finest.h * finest.w;
    const size_t state_bytes = (size_t)cells * model->channels * 4;
    if (overlap(workspace, p.bytes, image, (size_t)cells * model->n_in * 4) ||
        overlap(workspace, p.bytes, target, (size_t)cells * 8) ||
        (final_state && overlap(workspace, p.bytes, final_state, state_bytes)))
        return OCTNCA_EINVAL;

    const hipStream_t s = (hipStream_t)stream;
    char *ws = (char *)workspace;
    auto img = [&](int l) { return l == 0 ? image : (const void *)(ws + p.image_off[l]); };
    auto ok = [](hipError_t e) { return e == hipSuccess; };
    float *const window = (float *)(ws + p.window_off);
    float *const buf[2] = {(float *)(ws + p.grad_off[0]), (float *)(ws + p.grad_off[1])};
    for (int l = 0; l < levels; ++l) {
        p.cache[l].codes = (int8_t *)(ws + p.code_off[l]);
        p.cache[l].scales = (float *)(ws + p.scale_off[l]);
    }
    // n states of level l from or to slots first, first + 1, ..
    auto write = [&](int l, const float *states, int32_t first, int32_t n) {
        CacheArgs a = p.cache[l];
        a.first = first;
        a.n = n;
        return n == 0 || ok(launch_cache_write(Dtype::F32, a, states, s));
    };
    auto read = [&](int l, float *states, int32_t first, int32_t n) {
        CacheArgs a = p.cache[l];
        a.first = first;
        a.n = n;
        return ok(launch_cache_read(Dtype::F32, a, states, s));
    };

    // forward: the states before each step go to the cache.  A level starts in
    // one of the gradient buffers, which are free until the loss; the next level
    // up starts in the other one, as this one's steps may be none.
    for (int l = 1; l < levels; ++l) {
        const int32_t *f = factors + 3 * (l - 1);
        if (!ok(launch_pool(Dtype::F32, img(l - 1), ext3(p.ext[l]), ws + p.image_off[l], f[0],
                            f[1], f[2], model->n_in, s)))
            return OCTNCA_EHIP;
    }
    const float *cur = nullptr;   // the last level's last state
    for (int l = levels - 1; l >= 0; --l) {
        float *const begin = buf[l & 1];
        const bool coarsest = l == levels - 1;
        const int32_t *f = factors + 3 * l;
        if (!ok(launch_upsample(Dtype::F32, cur, ext3(p.ext[l]), coarsest ? 1 : f[0],
                                coarsest ? 1 : f[1], coarsest ? 1 : f[2], img(l), begin,
                                model->n_in, model->channels, s)))
            return OCTNCA_EHIP;
        cur = begin;
        if (steps[l] > 0 && !write(l, begin, 0, 1)) return OCTNCA_EHIP;
        const StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, 0);
        const size_t state = (size_t)a.ext.cells() * model->channels;
        const int32_t half = p.window[l] / 2;
        for (int32_t t = 0, side = 0; t < steps[l]; t += half, side ^= 1) {
            const int32_t n = std::min(half, steps[l] - t);
            float *const dst = window + side * half * state;
            if (!ok(train_forward_run(a, t, n, cur, dst, s)) ||
                !write(l, dst, t + 1, t + n == steps[l] ? n - 1 : n))   // not the last state
                return OCTNCA_EHIP;
            cur = dst + (n - 1) * state;
        }
    }
    float *g = cur == buf[0] ? buf[1] : buf[0];
    float *g_other = g == buf[0] ? buf[1] : buf[0];
    if (!ok(launch_readout_mse(cur, target, cells, model->channels, g, loss,
                               (double *)(ws + p.mse_off), s)))
        return OCTNCA_EHIP;
    if (final_state &&
        !ok(hipMemcpyAsync(final_state, cur, state_bytes, hipMemcpyDeviceToDevice, s)))
        return OCTNCA_EHIP;

    // backward, finest level first, each level's steps in windows from the last
    for (int l = 0; l < levels; ++l) {
        StepArgs a = step_args(model, p.ext[l], &weights[l], l, seed, threshold, 0);
        const LevelGradsDev gd{grads[l].conv_w, grads[l].conv_b, grads[l].w1, grads[l].b1,
                               grads[l].w2};
        if (steps[l] == 0 && !ok(clear_grads(model, grads[l], s))) return OCTNCA_EHIP;
        for (int32_t end = steps[l]; end > 0;) {
            const int32_t n = std::min(p.window[l], end);
            a.step = (uint32_t)(end - n);
            if (!read(l, window, end - n, n) ||
                !ok(launch_level_backward(a, n, end < steps[l], window, g, g_other, gd,
                                          (float *)(ws + p.bwd_off), s)))
                return OCTNCA_EHIP;
            std::swap(g, g_other);
            end -= n;
        }
        if (l + 1 < levels) {
            if (!ok(launch_upsample_adjoint(g, ext3(p.ext[l + 1]), factors[3 * l],
                                            factors[3 * l + 1], factors[3 * l + 2], model->n_in,
                                            model->channels, g_other, s)))
                return OCTNCA_EHIP;
            std::swap(g, g_other);
        }
    }
    return OCTNCA_OK;
}

}  // extern "C"

namespace {

// Checks a cache and a call's range; fills the kernels' arguments.
int make_cache_args(const octnca_model *m, const octnca_state_cache *c, const void *states,
                    int64_t from, int64_t count, int32_t n, const int64_t *slots, int64_t first,
                    bool write, CacheArgs *a) {
    const int st = check_model(m);
    if (st) return st;
    if (c == nullptr || n < 0 || from < 0 || count < 0) return OCTNCA_EINVAL;
    if (n > kMaxCacheStates) return OCTNCA_ESHAPE;
    if (c->code != OCTNCA_CODE_I8 && c->code != OCTNCA_CODE_F8) return OCTNCA_EINVAL;
    if (c->block != 32 && c->block != 64 && c->block != 128) return OCTNCA_EINVAL;
    if (c->slots < 0 || c->cells < 1 || c->cells > kMaxCells) return OCTNCA_ESHAPE;
    const int64_t blocks = (c->cells + c->block - 1) / c->block;
    const int64_t slot_bytes = c->cells * m->channels;            // <= 2^36 * 20
    if (c->slots > kMaxCacheBytes / (slot_bytes + 4 * blocks * m->channels)) return OCTNCA_ESHAPE;
    if (from % c->block != 0) return OCTNCA_EINVAL;
    if (from > c->cells || count > c->cells - from) return OCTNCA_ESHAPE;
    if (write && count % c->block != 0 && from + count != c->cells) return OCTNCA_EINVAL;
    if (slots == nullptr && n > 0 && (first < 0 || first > c->slots || n > c->slots - first))
        return OCTNCA_ESHAPE;
    a->n = n;
    a->count = count;
    if (n == 0 || count == 0) return OCTNCA_OK;
    const uintptr_t state_align = 4 * elem_bytes(m);
    const bool no_cache = c->slots == 0;   // every entry of `slots` is outside
    if (states == nullptr || (!no_cache && (c->codes == nullptr || c->scales == nullptr)) ||
        (uintptr_t)states % state_align || (uintptr_t)c->codes % 4 || (uintptr_t)c->scales % 16 ||
        (uintptr_t)slots % 8)
        return OCTNCA_EINVAL;
    if (count > kMaxCacheBytes / n / m->channels / 4) return OCTNCA_ESHAPE;
    const size_t state_bytes = (size_t)(count * n) * m->channels * elem_bytes(m);
    const size_t code_bytes = (size_t)(slot_bytes * c->slots);
    const size_t scale_bytes = (size_t)(4 * blocks * m->channels * c->slots);
    if (overlap(states, state_bytes, c->codes, code_bytes) ||
        overlap(states, state_bytes, c->scales, scale_bytes) ||
        overlap(c->codes, code_bytes, c->scales, scale_bytes) ||
        (slots && overlap(states, state_bytes, slots, (size_t)n * 8)))
        return OCTNCA_EINVAL;
    // a write's workgroups read the list while others write codes and scales
    if (write && slots &&
        (overlap(slots, (size_t)n * 8, c->codes, code_bytes) ||
         overlap(slots, (size_t)n * 8, c->scales, scale_bytes)))
        return OCTNCA_EINVAL;
    a->codes = (int8_t *)c->codes;
    a->scales = c->scales;
    a->n_slots = c->slots;
    a->cells = c->cells;
    a->blocks = blocks;
    a->from = from;
    a->slots = slots;
    a->first = first;
    a->block = c->block;
    a->channels = m->channels;
    a->f8 = c->code == OCTNCA_CODE_F8;
    return OCTNCA_OK;
}

// A contiguous array of a parameter list, for the overlap check.
struct Range {
    uintptr_t begin, end;
    bool written;
};

size_t dtype_bytes(int32_t t) { return t == OCTNCA_F32 ? 4 : 2; }
bool grad_type(int32_t t) { return t == OCTNCA_F32 || t == OCTNCA_F16 || t == OCTNCA_BF16; }
bool misaligned(const void *p, size_t to) { return (uintptr_t)p % to != 0; }

// Chunks, elements and arrays of a list (octnca_param_list without its table).
int check_params(const octnca_param *params, int32_t n, octnca_param_list *l) {
    if (n < 0 || (n > 0 && params == nullptr)) return OCTNCA_EINVAL;
    l->table = nullptr;
    l->chunks = l->elements = l->bytes = 0;
    l->has = 0;
    bool any = false;
    for (int32_t i = 0; i < n; ++i) {
        const octnca_param &t = params[i];
        if (t.count < 0 || t.count > kMaxCells) return OCTNCA_ESHAPE;
        if (t.count == 0) continue;
        if (t.grad == nullptr || !grad_type(t.grad_dtype) ||
            misaligned(t.grad, dtype_bytes(t.grad_dtype)))
            return OCTNCA_EINVAL;
        if (t.clipped && (!grad_type(t.clipped_dtype) ||
                          misaligned(t.clipped, dtype_bytes(t.clipped_dtype))))
            return OCTNCA_EINVAL;
        const int given = (t.param != nullptr) + (t.m != nullptr) + (t.v != nullptr);
        if ((given != 0 && given != 3) || (t.ema && given == 0)) return OCTNCA_EINVAL;
        if (misaligned(t.param, 4) || misaligned(t.m, 4) || misaligned(t.v, 4) ||
            misaligned(t.ema, 4))
            return OCTNCA_EINVAL;
        const int32_t has = (t.clipped ? kHasClipped : 0) | (t.param ? kHasParam : 0) |
                            (t.ema ? kHasEma : 0);
        if (any && has != (l->has & ~kHasInPlace)) return OCTNCA_EINVAL;
        any = true;
        l->has |= has | (t.clipped == t.grad ? kHasInPlace : 0);
        l->elements += t.count;
        l->bytes += t.count * (int64_t)(dtype_bytes(t.grad_dtype) +
                                        (t.clipped ? dtype_bytes(t.clipped_dtype) : 0) +
                                        (t.param ? 12 : 0) + (t.ema ? 4 : 0));
        l->chunks += param_chunks(t);
        if (l->elements > kMaxCells) return OCTNCA_ESHAPE;
    }
    return OCTNCA_OK;
}

// Whether an array that a call writes overlaps another one of the list.
bool params_overlap(const octnca_param *params, int32_t n) {
    std::vector<Range> r;
    r.reserve((size_t)n * 6);
    for (int32_t i = 0; i < n; ++i) {
        const octnca_param &t = params[i];
        if (t.count == 0) continue;
        auto add = [&](const void *p, size_t bytes, bool written) {
            if (p) r.push_back({(uintptr_t)p, (uintptr_t)p + bytes * (size_t)t.count, written});
        };
        const bool in_place = t.clipped == t.grad && t.clipped_dtype == t.grad_dtype;
        add(t.grad, dtype_bytes(t.grad_dtype), in_place);
        if (!in_place) add(t.clipped, dtype_bytes(t.clipped_dtype), true);
        add(t.param, 4, true);
        add(t.m, 4, true);
        add(t.v, 4, true);
        add(t.ema, 4, true);
    }
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uintptr_t read_end = 0, write_end = 0;   // of the ranges so far
    for (const Range &x : r) {
        if (x.begin < write_end || (x.written && x.begin < read_end)) return true;
        (x.written ? write_end : read_end) = std::max(x.written ? write_end : read_end, x.end);
    }
    return false;
}

bool list_ok(const octnca_param_list *l, int32_t need) {
    if (l == nullptr || l->table == nullptr || l->chunks < 0) return false;
    return l->chunks == 0 || (l->has & need) == need;
}

bool positive(double x) { return x > 0.0 && x < HUGE_VAL; }

// --- cell layers -------------------------------------------------------------

constexpr int64_t kMaxLayerRows = int64_t(1) << 29;
constexpr int64_t kMaxLayerCols = int64_t(1) << 20;
constexpr int64_t kMaxElements = int64_t(1) << 44;

// A matrix of values or of codes in memory: `rows` runs of `row_bytes`, `stride`
// bytes apart.
struct Span {
    const void *data;
    size_t rows, row_bytes, stride;
    size_t bytes() const { return rows ? (rows - 1) * stride + row_bytes : 0; }
};

Span span_of(const octnca_rows *x, int64_t rows, int64_t cols) {
    const size_t size = dtype_bytes(x->dtype);
    return Span{x->data, (size_t)rows, (size_t)cols * size,
                rows > 1 ? (size_t)x->stride * size : (size_t)cols * size};
}
Span span_of(const void *p, size_t bytes) { return Span{p, bytes ? 1u : 0u, bytes, bytes}; }

// Whether two matrices share bytes.  Of equal strides (two sets of columns of one
// buffer) the columns decide, of others the memory from first to last byte.
bool overlap(const Span &a, const Span &b) {
    if (a.rows == 0 || b.rows == 0 || !overlap(a.data, a.bytes(), b.data, b.bytes())) return false;
    if (a.rows > 1 && a.stride == b.stride) {
        const uintptr_t pa = (uintptr_t)a.data, pb = (uintptr_t)b.data;
        // where b's columns begin after a's, modulo the stride
        const size_t at = pb >= pa ? (pb - pa) % a.stride
                                   : (a.stride - (pa - pb) % a.stride) % a.stride;
        return at < a.row_bytes || at + b.row_bytes > a.stride;
    }
    return true;
}

int check_rows(const octnca_rows *x, int64_t rows, int64_t cols) {
    if (x == nullptr || !grad_type(x->dtype)) return OCTNCA_EINVAL;
    if (rows == 0) return OCTNCA_OK;
    if (x->data == nullptr || misaligned(x->data, dtype_bytes(x->dtype))) return OCTNCA_EINVAL;
    if (rows > 1 && (x->stride < cols || x->stride > kMaxCacheBytes / 4 / rows)) return OCTNCA_ESHAPE;
    return OCTNCA_OK;
}

bool mx4_size_ok(int64_t rows, int64_t cols) {
    return rows >= 0 && rows <= kMaxLayerRows && cols >= 1 && cols <= kMaxLayerCols;
}

size_t mx4_code_bytes(int64_t rows, int64_t cols) {
    return (size_t)((rows + 15) / 16 * mx4_blocks(cols)) * 256;
}

int check_mx4(const octnca_mx4 *m) {
    if (m == nullptr) return OCTNCA_EINVAL;
    if (!mx4_size_ok(m->rows, m->cols)) return OCTNCA_ESHAPE;
    if (m->rows == 0) return OCTNCA_OK;
    if (m->codes == nullptr || m->scales == nullptr || misaligned(m->codes, 16) ||
        misaligned(m->scales, 16))
        return OCTNCA_EINVAL;
    const size_t bytes = mx4_code_bytes(m->rows, m->cols);
    return overlap(m->codes, bytes, m->scales, bytes / 16) ? OCTNCA_EINVAL : OCTNCA_OK;
}

bool overlap(const octnca_mx4 *m, const Span &x) {
    const size_t bytes = mx4_code_bytes(m->rows, m->cols);
    return overlap(span_of(m->codes, bytes), x) || overlap(span_of(m->scales, bytes / 16), x);
}

bool overlap(const octnca_mx4 *a, const octnca_mx4 *b) {
    const size_t bytes = mx4_code_bytes(b->rows, b->cols);
    return overlap(a, span_of(b->codes, bytes)) || overlap(a, span_of(b->scales, bytes / 16));
}

// Arguments of a product of a [rows][cols] with w, its result apart.
int check_product(const octnca_mx4 *a, const octnca_mx4 *w, const float *bias,
                  const octnca_rows *out) {
    int st = check_mx4(a);
    if (st == OCTNCA_OK) st = check_mx4(w);
    if (st) return st;
    if (w->cols != a->cols || w->rows > kMaxLayerCols) return OCTNCA_ESHAPE;
    if (misaligned(bias, 4)) return OCTNCA_EINVAL;
    if (w->rows == 0) return out && grad_type(out->dtype) ? OCTNCA_OK : OCTNCA_EINVAL;
    if ((st = check_rows(out, a->rows, w->rows))) return st;
    const Span o = span_of(out, a->rows, w->rows);
    if (overlap(a, o) || overlap(w, o) || (bias && overlap(span_of(bias, (size_t)w->rows * 4), o)))
        return OCTNCA_EINVAL;
    return OCTNCA_OK;
}

}  // namespace

extern "C" {

int octree_nca_state_cache_write(const octnca_model *model, const octnca_state_cache *cache,
                                 const void *states, int64_t from, int64_t count, int32_t n,
                                 const int64_t *slots, int64_t first, void *stream) {
    CacheArgs a{};
    const int st = make_cache_args(model, cache, states, from, count, n, slots, first, true, &a);
    if (st || n == 0 || count == 0) return st;
    return hip_status(launch_cache_write((Dtype)model->state_dtype, a, states,
                                         (hipStream_t)stream));
}

int octree_nca_state_cache_read(const octnca_model *model, const octnca_state_cache *cache,
                                void *states, int64_t from, int64_t count, int32_t n,
                                const int64_t *slots, int64_t first, void *stream) {
    CacheArgs a{};
    const int st = make_cache_args(model, cache, states, from, count, n, slots, first, false, &a);
    if (st || n == 0 || count == 0) return st;
    return hip_status(launch_cache_read((Dtype)model->state_dtype, a, states,
                                        (hipStream_t)stream));
}

size_t octree_nca_param_table_bytes(const octnca_param *params, int32_t n) {
    octnca_param_list l;
    return check_params(params, n, &l) ? 0 : param_table_bytes(l.chunks);
}

int octree_nca_param_table(const octnca_param *params, int32_t n, void *table, size_t table_bytes,
                           octnca_param_list *list, void *stream) {
    octnca_param_list l;
    const int st = check_params(params, n, &l);
    if (st) return st;
    if (table == nullptr || list == nullptr || misaligned(table, 16)) return OCTNCA_EINVAL;
    try {   // the check's own list may run out of memory
        if (params_overlap(params, n)) return OCTNCA_EINVAL;
    } catch (const std::bad_alloc &) {
        return OCTNCA_ESPACE;
    }
    const size_t need = param_table_bytes(l.chunks);
    if (table_bytes < need) return OCTNCA_ESPACE;
    for (int32_t i = 0; i < n; ++i) {
        const octnca_param &t = params[i];
        const size_t c = (size_t)t.count;
        if (c == 0) continue;
        if (overlap(table, need, t.grad, c * dtype_bytes(t.grad_dtype)) ||
            (t.clipped && overlap(table, need, t.clipped, c * dtype_bytes(t.clipped_dtype))) ||
            (t.param && (overlap(table, need, t.param, c * 4) || overlap(table, need, t.m, c * 4) ||
                         overlap(table, need, t.v, c * 4))) ||
            (t.ema && overlap(table, need, t.ema, c * 4)))
            return OCTNCA_EINVAL;
    }
    if (launch_param_table(params, n, table, (hipStream_t)stream) != hipSuccess)
        return OCTNCA_EHIP;
    l.table = table;
    *list = l;
    return OCTNCA_OK;
}

int octree_nca_grad_norm(const octnca_param_list *list, float scale, float *norm, void *stream) {
    if (!list_ok(list, 0) || !positive(scale) || norm == nullptr || misaligned(norm, 4))
        return OCTNCA_EINVAL;
    return hip_status(launch_grad_norm(*list, scale, norm, (hipStream_t)stream));
}

int octree_nca_clip_grads(const octnca_param_list *list, float scale, float max_norm, float *norm,
                          void *stream) {
    if (!list_ok(list, kHasClipped) || !positive(scale) || !(max_norm > 0.0f) ||
        misaligned(norm, 4))
        return OCTNCA_EINVAL;
    return hip_status(launch_clip_grads(*list, scale, max_norm, norm, (hipStream_t)stream));
}

int octree_nca_adamw(const octnca_param_list *list, const octnca_adamw *settings, int64_t *step,
                     float *norm, void *stream) {
    if (!list_ok(list, kHasParam) || settings == nullptr || step == nullptr ||
        misaligned(step, 8) || misaligned(norm, 4))
        return OCTNCA_EINVAL;
    const octnca_adamw &h = *settings;
    auto beta_ok = [](double b) { return b >= 0.0 && b < 1.0; };
    // the kernels use these in fp32
    auto not_negative = [](double x) { return x >= 0.0 && (float)x < HUGE_VALF; };
    if (!not_negative(h.lr) || !beta_ok(h.beta1) || !beta_ok(h.beta2) || !positive((float)h.eps) ||
        !not_negative(h.weight_decay) || !(h.max_norm > 0.0) || !positive((float)h.scale) ||
        !(h.ema_decay >= 0.0 && h.ema_decay <= 1.0))
        return OCTNCA_EINVAL;
    return hip_status(launch_adamw(*list, h, step, norm, (hipStream_t)stream));
}

size_t octree_nca_mx4_code_bytes(int64_t rows, int64_t cols) {
    return mx4_size_ok(rows, cols) ? mx4_code_bytes(rows, cols) : 0;
}

int octree_nca_mx4_quantise(const octnca_rows *x, const octnca_mx4 *m, void *stream) {
    int st = check_mx4(m);
    if (st == OCTNCA_OK) st = check_rows(x, m->rows, m->cols);
    if (st || m->rows == 0) return st;
    if (overlap(m, span_of(x, m->rows, m->cols))) return OCTNCA_EINVAL;
    return hip_status(launch_mx4_quantise(*x, *m, (hipStream_t)stream));
}

int octree_nca_mx4_dequantise(const octnca_mx4 *m, const octnca_rows *x, void *stream) {
    int st = check_mx4(m);
    if (st == OCTNCA_OK) st = check_rows(x, m->rows, m->cols);
    if (st || m->rows == 0) return st;
    if (overlap(m, span_of(x, m->rows, m->cols))) return OCTNCA_EINVAL;
    return hip_status(launch_mx4_dequantise(*m, *x, (hipStream_t)stream));
}

int octree_nca_mx4_product(const octnca_mx4 *a, const octnca_mx4 *w, const float *bias,
                           int32_t relu, const octnca_rows *out, void *stream) {
    const int st = check_product(a, w, bias, out);
    if (st || a->rows == 0 || w->rows == 0) return st;
    return hip_status(launch_mx4_product(*a, *w, bias, relu != 0, *out, (hipStream_t)stream));
}

int octree_nca_mx4_linear(const octnca_rows *x, const octnca_mx4 *kept, const octnca_mx4 *w,
                          const float *bias, int32_t relu, const octnca_rows *out, void *stream) {
    int st = check_product(kept, w, bias, out);
    if (st == OCTNCA_OK) st = check_rows(x, kept->rows, kept->cols);
    if (st || kept->rows == 0) return st;
    const Span in = span_of(x, kept->rows, kept->cols);
    if (overlap(kept, in) || overlap(kept, w) ||
        (bias && overlap(kept, span_of(bias, (size_t)w->rows * 4))) ||
        (w->rows && overlap(span_of(out, kept->rows, w->rows), in)))
        return OCTNCA_EINVAL;
    if (w->rows == 0) return hip_status(launch_mx4_quantise(*x, *kept, (hipStream_t)stream));
    return hip_status(launch_mx4_linear(*x, *kept, *w, bias, relu != 0, *out,
                                        (hipStream_t)stream));
}

size_t octree_nca_mx4_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t outs) {
    if (!mx4_size_ok(rows, cols) || outs < 1 || outs > kMaxLayerCols) return 0;
    return mx4_backward_bytes(rows, cols, outs);
}

int octree_nca_mx4_backward(const octnca_rows *grad_out, const octnca_mx4 *a, const octnca_mx4 *w,
                            const octnca_rows *grad_in, float *grad_weight, float *grad_bias,
                            void *workspace, size_t workspace_bytes, void *stream) {
    int st = check_mx4(a);
    if (st == OCTNCA_OK) st = check_mx4(w);
    if (st) return st;
    const int64_t rows = a->rows, cols = a->cols, outs = w->rows;
    if (w->cols != cols || outs < 1 || outs > kMaxLayerCols) return OCTNCA_ESHAPE;
    if ((st = check_rows(grad_out, rows, outs))) return st;
    if (grad_in && (st = check_rows(grad_in, rows, cols))) return st;
    if (grad_in && grad_in->dtype != grad_out->dtype) return OCTNCA_EINVAL;
    if (misaligned(grad_weight, 4) || misaligned(grad_bias, 4) || misaligned(workspace, 16))
        return OCTNCA_EINVAL;
    const bool sums = grad_weight != nullptr || grad_bias != nullptr;
    const size_t need = sums ? mx4_backward_bytes(rows, cols, outs) : 0;
    if (sums && workspace == nullptr) return OCTNCA_EINVAL;
    if (workspace_bytes < need) return OCTNCA_ESPACE;
    // what is written, apart from each other and from what is read
    const Span written[] = {grad_in ? span_of(grad_in, rows, cols) : Span{},
                            span_of(grad_weight, grad_weight ? (size_t)(outs * cols) * 4 : 0),
                            span_of(grad_bias, grad_bias ? (size_t)outs * 4 : 0),
                            span_of(workspace, need)};
    const Span grad = span_of(grad_out, rows, outs);
    for (int i = 0; i < 4; ++i) {
        if (overlap(written[i], grad) || overlap(a, written[i]) || overlap(w, written[i]))
            return OCTNCA_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(written[i], written[j])) return OCTNCA_EINVAL;
    }
    return hip_status(launch_mx4_backward(*grad_out, *a, *w, grad_in, grad_weight, grad_bias,
                                          workspace, (hipStream_t)stream));
}

int octree_nca_dropout(const octnca_dropout *dropout, const octnca_rows *x, const octnca_rows *gate,
                       const octnca_rows *add, const octnca_rows *out, int64_t rows, int64_t cols,
                       void *stream) {
    uint64_t threshold;
    if (dropout == nullptr || !fire_threshold(dropout->rate, &threshold) ||
        misaligned(dropout->step, 8))
        return OCTNCA_EINVAL;
    if (rows < 0 || cols < 0) return OCTNCA_ESHAPE;
    if (rows == 0 || cols == 0) return x && out ? OCTNCA_OK : OCTNCA_EINVAL;
    if (rows > kMaxElements / cols) return OCTNCA_ESHAPE;
    const octnca_rows *all[] = {x, gate, add, out};
    for (int i = 0; i < 4; ++i) {
        if (all[i] == nullptr && (i == 1 || i == 2)) continue;
        const int st = check_rows(all[i], rows, cols);
        if (st) return st;
        if (all[i]->dtype != x->dtype) return OCTNCA_EINVAL;
    }
    const Span o = span_of(out, rows, cols);
    for (int i = 0; i < 3; ++i) {
        if (all[i] == nullptr) continue;
        const Span s = span_of(all[i], rows, cols);
        if (overlap(o, s) && !(s.data == o.data && s.stride == o.stride)) return OCTNCA_EINVAL;
    }
    if (dropout->step && overlap(o, span_of(dropout->step, 8))) return OCTNCA_EINVAL;
    DropArgs d{};
    d.x = x->data;
    d.gate = gate ? gate->data : nullptr;
    d.add = add ? add->data : nullptr;
    d.out = out->data;
    // one row has any stride
    const auto stride = [&](const octnca_rows *r) { return r == nullptr || rows == 1 ? cols : r->stride; };
    d.x_stride = stride(x);
    d.gate_stride = stride(gate);
    d.add_stride = stride(add);
    d.out_stride = stride(out);
    d.rows = rows;
    d.cols = cols;
    d.seed = dropout->seed;
    d.index = dropout->index;
    d.step = dropout->step;
    d.threshold = (uint32_t)threshold;   // 2^32: nothing is kept, by the factor
    d.factor = threshold >> 32 ? 0.0f : (float)(4294967296.0 / (4294967296.0 - (double)threshold));
    return hip_status(launch_dropout(x->dtype, d, (hipStream_t)stream));
}

}  // extern "C"

namespace octnca {
// The step kernel comes with the arguments (StepArgs::kc, filled from the
// caller's octnca_model); nothing here reads the environment.
hipError_t launch_step(const StepArgs &a, const void *src, void *dst, hipStream_t stream) {
    if (a.kc.valu) return launch_step_valu(a, src, dst, stream);
    // the specialised matrix-core kernels serve C = 16, H = 64 and most steps of
    // C = 12, H = 48; the other steps of the ablation's sizes run on the generic
    // matrix-core kernel
    if (!step_mfma_serves(a, a.kc.layout)) return launch_step_gen(a, src, dst, stream);
    return launch_step_mfma(a, a.kc.mlp, a.kc.layout, src, dst, stream);
}

bool step_single_fuses_readout(const StepArgs &a) {
    return !a.kc.valu && step_mfma_single_readout(a, a.kc.mlp);
}

bool step_pairs(const StepArgs &a) {
    return !a.kc.valu && a.kc.pairs && step_mfma_pairs(a, a.kc.mlp, a.kc.layout);
}

hipError_t launch_step_pair(const StepArgs &a, const void *src, void *dst, hipStream_t stream) {
    if (!step_pairs(a)) return hipErrorInvalidValue;
    return launch_step2_mfma(a, a.kc.mlp, a.kc.layout, src, dst, stream);
}

hipError_t launch_step_pair_up(const StepArgs &a, const void *coarse, int coarse_w, int fz,
                               int fy, int fx, const void *img, void *dst, hipStream_t stream) {
    if (fz != 1 || !step_pairs(a) || !step_fuses_upsample(a)) return hipErrorInvalidValue;
    return launch_step2_mfma_up(a, a.kc.mlp, a.kc.layout, coarse, coarse_w, fy, fx, img, dst,
                                stream);
}

bool step_fuses_upsample(const StepArgs &a) {
    return !a.kc.valu && step_mfma_fuses_upsample(a, a.kc.mlp, a.kc.layout);
}

hipError_t launch_step_up(const StepArgs &a, const void *coarse, int coarse_h, int coarse_w,
                          int fz, int fy, int fx, const void *img, void *dst,
                          hipStream_t stream) {
    if (!step_fuses_upsample(a)) return hipErrorInvalidValue;
    return launch_step_mfma_up(a, a.kc.layout, coarse, coarse_h, coarse_w, fz, fy, fx, img, dst,
                               stream);
}
}  // namespace octnca
