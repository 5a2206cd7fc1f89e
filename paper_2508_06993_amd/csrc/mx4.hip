// Matrices in microscaled 4 bits: quantisation and product (formulas and layout
// in octree_nca.h).
//
// The layout is that of the matrix instruction's operands: 16 rows of a block are 256
// bytes in a row, four blocks of them the 1 KB that a wave multiplies at once, whether
// it comes from memory or LDS.
//
// Quantisation and reading back are one pass over memory: 65536 x 4096 bf16 (679 MB)
// 117 us and 111, 5.8 and 6.1 TB/s.  Products: 16384 x 8192 -> 8192 in 647 us, 3.4
// PFLOP/s (the 32 x 32 instruction alone does 7.0 with random codes; a library's
// bf16 product 1.34), bound by what a wave issues between its products: with its loads
// left out the kernel takes 0.76 of the time, with its LDS traffic too 0.51.  One row
// is bound by the weights' bytes: 1 x 16384 -> 16384 6.2 TB/s, 1 x 4096 -> 4096 4.3 us.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "launch.h"
#include "mx4.h"

namespace octnca {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 23;

template <typename V, bool NARROW>
__global__ __launch_bounds__(kThreads) void quantise(const typename V::T *__restrict__ x,
                                                     int64_t stride, int cols, Mx4View m,
                                                     int64_t units) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t u = ((int64_t)blockIdx.x * (kThreads / 64) + wave) * kUnits; u < units;
         u += (int64_t)gridDim.x * (kThreads / 64) * kUnits) {
        const Place p = place_of(u, m.blocks);
        Eight<V> raw[kPasses];
        load_units<V, NARROW>(x, stride, cols, m.rows, p, raw);
        uint32_t c[kPasses], scale[kPasses];
        quantise_units(raw, c, scale);
#pragma unroll
        for (int k = 0; k < kPasses; ++k)
            if (p.row + 4 * k < m.rows)
                ((uint32_t *)m.codes)[p.unit * 64 + (4 * k + lane / 16) * 4 + lane % 4] = c[k];
        // lane q of a block's four stores the scale of pass q's row
        const int q = lane % 4;
        if (p.row + 4 * q < m.rows)
            m.scales[p.unit * kMxGroup + 4 * q + lane / 16] = (uint8_t)quad_pick(scale);
    }
}

template <typename V, bool STREAM>
__global__ __launch_bounds__(kThreads) void dequantise(Mx4View m, typename V::T *__restrict__ x,
                                                       int64_t stride, int cols, int64_t units) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t u = ((int64_t)blockIdx.x * (kThreads / 64) + wave) * kUnits; u < units;
         u += (int64_t)gridDim.x * (kThreads / 64) * kUnits) {
        const Place p = place_of(u, m.blocks);
        const int64_t unit = std::min(p.unit, units - 1);
        uint32_t c[kPasses];
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int64_t at = unit * 64 + (4 * k + lane / 16) * 4;
            if (V::kBytes == 4) {   // fours 4 q and 16 + 4 q: 64 bytes in a row a store
                const uint16_t *from = (const uint16_t *)((const uint32_t *)m.codes + at);
                c[k] = from[lane % 4] | (uint32_t)from[4 + lane % 4] << 16;
            } else {
                c[k] = ((const uint32_t *)m.codes)[at + lane % 4];
            }
        }
        // lane q of a block's four has the scale of pass q's row
        const uint32_t s = m.scales[unit * kMxGroup + lane % 4 * 4 + lane / 16];
        const uint32_t scale[kPasses] = {quad_lane<0>(s), quad_lane<1>(s), quad_lane<2>(s),
                                         quad_lane<3>(s)};
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            float v[8];
            mx4_values(c[k], v);
            const float factor = mx4_scale_value(scale[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            if (p.row + 4 * k >= m.rows) continue;
            typename V::T *row = x + (p.row + 4 * k) * stride;
            if (V::kBytes == 4) {
                const int col = p.col - lane % 4 * 4;
                if (col < cols) store4<V>(row + col, v, cols - col);
                if (col + 16 < cols) store4<V>(row + col + 16, v + 4, cols - col - 16);
            } else if (p.col < cols) {
                store8<V, STREAM>(row + p.col, v, cols - p.col);
            }
        }
    }
}

// Values of few rows that every workgroup quantises for itself at most: as many as
// that takes less time than a launch (4 us).
constexpr int kFewValues = 16384;

struct ProductArgs {
    Mx4View a, w;
    const float *bias;   // or null
    bool relu;
    void *out;
    int64_t stride;
};

// Few rows.  A workgroup takes 16 outputs times 16 G rows, its waves a part of the
// columns each: what there is to read, the weights, is on its way at once.  The waves'
// sums are added in order.  X: type of the values that are quantised on the way (one
// row group, few values: every workgroup does it for itself), or int: codes.
constexpr int kAhead = 4;   // steps of four blocks that are loaded together
template <typename V, typename X, int G, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_rows(ProductArgs p, const void *x,
                                                       int64_t x_stride, int cols) {
    constexpr bool kValues = !std::is_same<X, int>::value;
    __shared__ float sums[WAVES][G][256];
    __shared__ Words4 codes[kValues ? kFewValues / 32 : 1];   // [block][row]
    __shared__ uint8_t scales[kValues ? kFewValues / 32 : 1];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blocks = p.a.blocks, rows = (int)p.a.rows;
    const int64_t group0 = (int64_t)blockIdx.y * G, last = (p.a.rows + kMxGroup - 1) / kMxGroup - 1;
    const int steps = (blocks + 3) / 4, each = (steps + WAVES - 1) / WAVES;
    const int begin = wave * each, end = std::min(steps, begin + each);
    const Words4 *w_codes = (const Words4 *)p.w.codes + (int64_t)blockIdx.x * blocks * kMxGroup;
    const uint8_t *w_scales = p.w.scales + (int64_t)blockIdx.x * blocks * kMxGroup;

    Mx4Operand w[kAhead];
    const auto load_w = [&](int step) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = std::min((step + k) * 64 + lane, blocks * kMxGroup - 1);
            w[k] = Mx4Operand{w_codes[at], w_scales[at]};
        }
    };
    load_w(std::min(begin, steps - 1));
    if constexpr (kValues) {
        // four lanes a block, eight values each
        const int parts = blocks * 4;
        for (int e = threadIdx.x; e < (rows * parts + 63) / 64 * 64; e += 64 * WAVES) {
            const int row = std::min(e / parts, rows - 1), col = (e - e / parts * parts) * 8;
            const auto from = (const typename X::T *)x + row * x_stride;
            Eight<X> raw;
            if (cols < 8) {
                raw.down = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    raw.v[k] = col + k < cols ? from[col + k] : (typename X::T)0.0f;
            } else {
                raw.load(from, col, cols);
            }
            uint32_t c, s;
            quantise_eight(raw, c, s);
            if (e < rows * parts) {
                const int at = col / kMxBlock * rows + row;
                ((uint32_t *)codes)[at * 4 + col % kMxBlock / 8] = c;
                if (col % kMxBlock == 0) scales[at] = (uint8_t)s;
                if (blockIdx.x == 0) {
                    const int kept = col / kMxBlock * kMxGroup + row;
                    ((uint32_t *)p.a.codes)[kept * 4 + col % kMxBlock / 8] = c;
                    if (col % kMxBlock == 0) p.a.scales[kept] = (uint8_t)s;
                }
            }
        }
        __syncthreads();
    }
    v4f32 acc[G] = {};
    for (int step = begin; step < end; step += kAhead) {
        Mx4Operand a[kAhead][G];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int block = std::min((step + k) * 4 + lane / 16, blocks - 1);
                if constexpr (kValues) {
                    const int at = block * rows + std::min(lane % 16, rows - 1);
                    a[k][g] = Mx4Operand{codes[at], scales[at]};
                } else {
                    const int64_t at = (std::min(group0 + g, last) * blocks + block) * kMxGroup + lane % 16;
                    a[k][g] = Mx4Operand{((const Words4 *)p.a.codes)[at], p.a.scales[at]};
                }
            }
        Mx4Operand now[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool in = step + k < end && (step + k) * 4 + lane / 16 < blocks;
            now[k] = Mx4Operand{w[k].codes & (in ? ~0u : 0u), in ? w[k].scale : 127u};
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (!in) a[k][g].scale = 127;
        }
        load_w(std::min(step + kAhead, steps - 1));
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g) acc[g] = mx4_mfma(now[k], a[k][g], acc[g]);
    }
    // [output][row] of a row group
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][g][(lane / 16 * 4 + i) * 16 + lane % 16] = acc[g][i];
    __syncthreads();
    for (int e = threadIdx.x; e < G * 256; e += 64 * WAVES) {
        const int g = e / 256, r = e % 256 / 16, n = e % 16;
        const int64_t row = (group0 + g) * kMxGroup + r, out = (int64_t)blockIdx.x * kMxGroup + n;
        if (row >= p.a.rows || out >= p.w.rows) continue;
        float y = sums[0][g][n * 16 + r];
        for (int v = 1; v < WAVES; ++v) y += sums[v][g][n * 16 + r];
        if (p.bias) y += p.bias[out];
        if (p.relu && y < 0.0f) y = 0.0f;
        V::put((typename V::T *)p.out + row * p.stride + out, y);
    }
}

// Tile of a workgroup among row_tiles x col_tiles.  Workgroups go round the eight dies,
// each with its own L2: a die takes tiles in a row, which run down eight row tiles
// before they go to the next columns.  us with this and with tiles in plain order, 1024 x
// 4096 -> 4096: 26 and 27; large tiles: no difference.
struct Tile {
    int row, col;
};
__device__ __forceinline__ Tile die_tile(int id, int row_tiles, int col_tiles) {
    const int each = row_tiles * col_tiles / 8;
    if (id < each * 8) id = id % 8 * each + id / 8;
    const int band = id / (8 * col_tiles), left = row_tiles - band * 8, deep = left < 8 ? left : 8;
    const int in_band = id - band * 8 * col_tiles;
    return Tile{band * 8 + in_band % deep, in_band / deep};
}

// Large products.  A workgroup takes 32 S rows times 32 S outputs, a wave a quarter of
// them with its sums in registers.  A step takes 4 U blocks (256 columns) through LDS: the
// next one's are loaded during the first half of its products and go to the other half of
// LDS during the second.  Blocks past the last come as codes 0 with scale 1.  The weights'
// rows go to the operands so that a lane ends up with 16 bytes of outputs in a row, and the
// two lanes of a row with 32.
template <typename V, int S, int U>
__global__ __launch_bounds__(kThreads) void product_tiles(ProductArgs p, int row_tiles,
                                                          int out_tiles) {
    constexpr int kGroups = 2 * S, kLoads = kGroups / 4;   // row groups of a side
    constexpr int kEach = 16 / V::kBytes;                  // outputs of a lane in a row
    __shared__ Words4 codes[2][U][2][kGroups][64];
    __shared__ uint32_t scales[2][U][2][kGroups][16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Tile tile = die_tile(blockIdx.x, row_tiles, out_tiles);
    const int64_t group0[2] = {(int64_t)tile.row * kGroups, (int64_t)tile.col * kGroups};
    const Mx4View side[2] = {p.a, p.w};
    const int blocks = p.a.blocks;

    struct Next {
        Words4 codes[2][kLoads];
        uint32_t scales[2];
        bool codes_in, scales_in;   // applied when the values are stored: no wait before
    };
    const int last[2] = {(int)((p.a.rows + kMxGroup - 1) / kMxGroup) - 1,
                         (int)((p.w.rows + kMxGroup - 1) / kMxGroup) - 1};
    const auto load_codes = [&](Next &x, int from_block, int s, int k) {
        x.codes_in = from_block + lane / kMxGroup < blocks;
        const int64_t group = std::min((int)group0[s] + k * 4 + wave, last[s]);
        const Words4 *from = (const Words4 *)side[s].codes +
                             (group * blocks + std::min(from_block, blocks - 1)) * kMxGroup;
        x.codes[s][k] = from[x.codes_in ? lane : 0];
    };
    const auto load_scales = [&](Next &x, int from_block) {
        const int part = threadIdx.x % 16;   // a thread takes four rows' scales of a block
        x.scales_in = from_block + part / 4 < blocks;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t group = std::min((int)group0[s] + (int)threadIdx.x / 16, last[s]);
            const uint32_t *from = (const uint32_t *)side[s].scales +
                                   (group * blocks + std::min(from_block, blocks - 1)) * 4;
            x.scales[s] = from[x.scales_in ? part : 0];
        }
    };
    // Where row r of a group goes: the weights' bits 2 and 3 change places where a lane
    // is to have eight outputs in a row.
    const auto place = [&](int s, int r) {
        return s == 0 || kEach == 4 ? r : (r & 3) | (r & 4) << 1 | (r & 8) >> 1;
    };
    // Codes k of a side; past the end zeros of one side do, with scales that are numbers.
    const auto store_codes = [&](const Next &x, int buffer, int u, int s, int k) {
        const int at = lane / kMxGroup * kMxGroup + place(s, lane % kMxGroup);
        codes[buffer][u][s][k * 4 + wave][at] =
            s == 0 ? x.codes[s][k] & (x.codes_in ? ~0u : 0u) : x.codes[s][k];
    };
    const auto store_scales = [&](const Next &x, int buffer, int u) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = threadIdx.x % 16 / 4 * 4 + place(s, threadIdx.x % 4 * 4) / 4;
            if (kGroups == 16 || threadIdx.x < kGroups * 16)
                scales[buffer][u][s][threadIdx.x / 16][at] = x.scales_in ? x.scales[s] : 0x7f7f7f7fu;
        }
    };
    constexpr int kT = S / 2;   // tiles of 32 of a wave, each way
    const int ga = wave % 2 * S, gw = wave / 2 * S;
    const auto operand = [&](int buffer, int u, int s, int group, int half) {
        const int g = group + lane % 32 / 16, at = (2 * half + lane / 32) * 16 + lane % 16;
        return Mx4Operand{codes[buffer][u][s][g][at],
                          ((const uint8_t *)scales[buffer][u][s][g])[at]};
    };
    v16f32 acc[kT][kT] = {};
    Next next[U];
    // Piece x of what is loaded and stored for the next step
    constexpr int kPieces = U * (2 * kLoads + 1), kTurns = U * 2 * kT;
    const auto load = [&](int block, int x) {
        const int u = x / (2 * kLoads + 1), piece = x % (2 * kLoads + 1);
        if (piece < 2 * kLoads)
            load_codes(next[u], block + 4 * u, piece / kLoads, piece % kLoads);
        else
            load_scales(next[u], block + 4 * u);
    };
    const auto store = [&](int buffer, int x) {
        const int u = x / (2 * kLoads + 1), piece = x % (2 * kLoads + 1);
        if (piece < 2 * kLoads)
            store_codes(next[u], buffer, u, piece / kLoads, piece % kLoads);
        else
            store_scales(next[u], buffer, u);
    };
#pragma unroll
    for (int x = 0; x < kPieces; ++x) load(0, x);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) store(0, x);
    int buffer = 0;
    for (int block = 0; block < blocks; block += 4 * U, buffer ^= 1) {
        __syncthreads();
        // kT products a turn, with the next operands on their way from LDS.  The next
        // step's pieces are loaded in the first half of the turns and go to LDS in the
        // second: a wave's instructions wait for each other where many of a kind follow.
        Mx4Operand w[2][kT], a = operand(buffer, 0, 0, ga, 0);
#pragma unroll
        for (int t = 0; t < kT; ++t) w[0][t] = operand(buffer, 0, 1, gw + 2 * t, 0);
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            const int pass = turn / kT, i = turn % kT;   // a pass: two blocks
            Mx4Operand after = a;
            if (turn + 1 < kTurns) {
                const int then = (turn + 1) / kT;
                after = operand(buffer, then / 2, 0, ga + 2 * ((turn + 1) % kT), then % 2);
            }
            if (pass + 1 < 2 * U)
                w[(pass + 1) % 2][i] =
                    operand(buffer, (pass + 1) / 2, 1, gw + 2 * i, (pass + 1) % 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < kT; ++t) acc[i][t] = mx4_mfma32(w[pass % 2][t], a, acc[i][t]);
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {
                if (x * (kTurns / 2) / kPieces == turn) load(block + 4 * U, x);
                if (kTurns / 2 + x * (kTurns / 2) / kPieces == turn) store(buffer ^ 1, x);
            }
            a = after;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // kEach outputs of row lane % 32 of each tile, from n on; the next ones 2 kEach on
    constexpr int kRuns = 16 / kEach;
    const int64_t n = (group0[1] + gw) * kMxGroup + lane / 32 * kEach;
    float bias[kT][16];
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int64_t at = n + t * 32 + k / kEach * (2 * kEach) + k % kEach;
            bias[t][k] = p.bias ? p.bias[std::min(at, p.w.rows - 1)] : 0.0f;
        }
#pragma unroll
    for (int i = 0; i < kT; ++i) {
        const int64_t row = (group0[0] + ga + 2 * i) * kMxGroup + lane % 32;
        if (row >= p.a.rows) continue;
        typename V::T *to = (typename V::T *)p.out + row * p.stride + n;
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                float y[kEach];
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    y[k] = acc[i][t][r * kEach + k] + bias[t][r * kEach + k];
                    if (p.relu && y[k] < 0.0f) y[k] = 0.0f;
                }
                const int off = t * 32 + r * 2 * kEach;
                const int64_t left = p.w.rows - n - off;
                if (left <= 0) continue;
                if constexpr (kEach == 8)
                    store8<V>(to + off, y, (int)std::min<int64_t>(left, 8));
                else
                    store4<V>(to + off, y, (int)std::min<int64_t>(left, 4));
            }
    }
}

// Whether a matrix is so large (half the last-level cache) that its values are written
// past it.  us through it and past it: 1.2M x 128 fp16 72 and 58, 65536 x 4096 bf16
// 121 and 111.  Not where a store has less than 128 bytes in a row or lines stay half
// written: 600 thousand x 100 fp32 71 and 107, 30000 x 4100 fp16 74 and 89.
bool streams(const octnca_rows &x, int64_t rows, int64_t cols) {
    return rows * cols * (x.dtype == OCTNCA_F32 ? 4 : 2) >= int64_t(1) << 27;
}

bool rows_aligned(const octnca_rows &x, int to) {
    return (uintptr_t)x.data % to == 0 && x.stride * (x.dtype == OCTNCA_F32 ? 4 : 2) % to == 0;
}

}  // namespace

hipError_t launch_mx4_quantise(const octnca_rows &x, const octnca_mx4 &m, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const int64_t grid = (units + kUnits * 4 - 1) / (kUnits * 4);
        const auto from = (const typename V::T *)x.data;
        const unsigned n = (unsigned)std::min(grid, kMaxGrid);
        const auto run = [&](auto kernel) {
            kernel<<<n, kThreads, 0, stream>>>(from, x.stride, (int)m.cols, v, units);
        };
        if (m.cols < 8)
            run(quantise<V, true>);
        else
            run(quantise<V, false>);
        return hipGetLastError();
    });
}

hipError_t launch_mx4_dequantise(const octnca_mx4 &m, const octnca_rows &x, hipStream_t stream) {
    return with_type(x.dtype, [&](auto type) {
        using V = decltype(type);
        const Mx4View v = mx4_view(m);
        const int64_t units = (m.rows + kMxGroup - 1) / kMxGroup * v.blocks;
        const int64_t grid = (units + kUnits * 4 - 1) / (kUnits * 4);
        const auto run = [&](auto kernel) {
            kernel<<<(unsigned)std::min(grid, kMaxGrid), kThreads, 0, stream>>>(
                v, (typename V::T *)x.data, x.stride, (int)m.cols, units);
        };
        const bool whole = x.stride == m.cols && m.cols * V::kBytes % 16 == 0 && rows_aligned(x, 16);
        if (V::kBytes == 2 && whole && streams(x, m.rows, m.cols))
            run(dequantise<V, true>);
        else
            run(dequantise<V, false>);
        return hipGetLastError();
    });
}

namespace {

// Which kernel serves a product that is not narrow: large tiles; for more than 64 rows 128 of
// the tiles of 128 x 128 and more (160 for up to 1024 rows of more than 48 blocks); else a
// few rows at a time with the columns split, where each die reads all rows for itself.  us of
// tiles and of few rows: 512 x 300 -> 4096 (128 tiles) 8.4 and 9.9, 384 x 300 (96) 8.1 and
// 7.3; 512 x 4096 -> 4096 24.1 and 20.7, 640 x 4096 (160) 24.5 and 24.9, 768 x 4096 24.9 and
// 28.2; 16384 x 4096 -> 128 (128) 24.8 and 43.6, 10300 -> 128 (81) 23.9 and 30.0, 8000 -> 128 (63)
// 23.7 and 23.1, 12000 -> 16 (94) 22 and 8; 65 x 4096 -> 16384 24.2 and 20.0, 64 rows 23.9 and
// 13.2, 64 x 4096 -> 32768 (256) 25.9 and 21.9.
bool takes_tiles(int64_t rows, int blocks, int64_t tiles) {
    return rows > 64 && tiles >= (rows <= 1024 && blocks > 48 ? 160 : 128);
}

template <typename V, typename X, int G>
hipError_t run_few(const ProductArgs &p, const octnca_rows *x, int cols, hipStream_t stream) {
    const dim3 grid((unsigned)((p.w.rows + kMxGroup - 1) / kMxGroup),
                    (unsigned)((p.a.rows + kMxGroup * G - 1) / (kMxGroup * G)));
    const void *from = x ? x->data : nullptr;
    const int64_t stride = x ? x->stride : 0;
    constexpr bool kValues = !std::is_same<X, int>::value;
    // Sixteen waves where a workgroup has much to read or to quantise and there are no
    // more workgroups than compute units, two where it has little.  us with sixteen, four
    // and two.  Codes, -> 1024: 1 x 4096 3.5, 3.1, 3.5, 1 x 8192 3.5, 4.1, 4.9; 64 x 8192 8.8,
    // 7.8, 10.3, 64 x 32768 22.3, 24.4, 33.8; 1000 x 517 -> 1003 20.2, 7.7, 6.7, 1 x 1100 3.1,
    // 2.5, 2.8.  Values: 1 x 1024 -> 300 3.3, 3.1, 3.0, 1 x 2048 -> 1024 3.6, 3.2, 3.7, 1 x 4096
    // 3.8, 3.9, 5.2, 16 x 1024 -> 4096 5.2, 6.4, 9.8 and -> 16384 (1024 workgroups) 14.0, 10.0,
    // 10.5.
    const int64_t work = kValues ? p.a.rows * p.a.blocks : p.a.blocks;
    if ((int64_t)grid.x * grid.y <= 256 && work >= (kValues ? 80 : G == 4 ? 512 : 192))
        few_rows<V, X, G, 16><<<grid, 64 * 16, 0, stream>>>(p, from, stride, cols);
    else if (work <= 32)
        few_rows<V, X, G, 2><<<grid, 64 * 2, 0, stream>>>(p, from, stride, cols);
    else
        few_rows<V, X, G, 4><<<grid, 64 * 4, 0, stream>>>(p, from, stride, cols);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_product(const octnca_mx4 &a, const octnca_mx4 &w, const float *bias,
                              bool relu, const octnca_rows &out, hipStream_t stream) {
    if (mx4_narrow_serves(a.cols, w.rows))
        return launch_mx4_narrow(nullptr, a, w, bias, relu, out, stream);
    return with_type(out.dtype, [&](auto type) {
        using V = decltype(type);
        const ProductArgs p{mx4_view(a), mx4_view(w), bias, relu, out.data, out.stride};
        const auto tiles = [&](int64_t side) {
            return std::make_pair((a.rows + side - 1) / side, (w.rows + side - 1) / side);
        };
        const auto large = tiles(256), small = tiles(128);
        if (mx4_large_tiles(a.rows, w.rows)) {
            product_tiles<V, 8, 2><<<(unsigned)(large.first * large.second), kThreads, 0, stream>>>(
                p, (int)large.first, (int)large.second);
            return hipGetLastError();
        }
        if (takes_tiles(a.rows, p.a.blocks, small.first * small.second)) {
            product_tiles<V, 4, 2><<<(unsigned)(small.first * small.second), kThreads, 0, stream>>>(
                p, (int)small.first, (int)small.second);
            return hipGetLastError();
        }
        return a.rows <= 16   ? run_few<V, int, 1>(p, nullptr, (int)a.cols, stream)
               : a.rows <= 32 ? run_few<V, int, 2>(p, nullptr, (int)a.cols, stream)
                              : run_few<V, int, 4>(p, nullptr, (int)a.cols, stream);
    });
}

hipError_t launch_mx4_linear(const octnca_rows &x, const octnca_mx4 &kept, const octnca_mx4 &w,
                             const float *bias, bool relu, const octnca_rows &out,
                             hipStream_t stream) {
    if (mx4_narrow_serves(kept.cols, w.rows))
        return launch_mx4_narrow(&x, kept, w, bias, relu, out, stream);
    if (kept.rows <= kMxGroup && kept.rows * mx4_blocks(kept.cols) * kMxBlock <= kFewValues)
        return with_type(out.dtype, [&](auto type) {
            return with_type(x.dtype, [&](auto x_type) {
                const ProductArgs p{mx4_view(kept), mx4_view(w), bias, relu, out.data, out.stride};
                return run_few<decltype(type), decltype(x_type), 1>(p, &x, (int)kept.cols, stream);
            });
        });
    const hipError_t e = launch_mx4_quantise(x, kept, stream);
    return e == hipSuccess ? launch_mx4_product(kept, w, bias, relu, out, stream) : e;
}

}  // namespace octnca
