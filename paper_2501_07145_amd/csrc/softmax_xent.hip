// Softmax cross entropy of linear scores and its gradients (rfsf_softmax_xent):
//   l[n, c] = sum_k Phi[n, k] W[c, k],   loss[n] = log sum_c exp l[n, c] - l[n, y_n],
//   G[n, c] = s_n (exp l[n, c] / sum - [c = y_n]),   dPhi = G W,   dW = G^T Phi.
//
// Three products of 2 N K C flop, everything else is of the order of N C and bound by memory. float32 operands cost three 16-bit products each, bfloat16 ones
// one for the scores and two for a gradient, G being two terms. The operands are packed once for
// the matrix instructions (plane_pack.h), W and Phi by rows for the scores, their transposes for the gradients, so that
// all three products are of one kind (plane_product.h). The scores of a tile give their maximum and sum of exponentials per row before
// they leave the registers; without gradients they are never written. For gradients the rows are taken in blocks, and the
// scores of a block stay in the workspace from their product to the pass that turns them into G (both layouts), in as
// few rows at a time as fill the GPU, so that the last-level cache holds them.
#include "plane_pack.h"
#include "xent_direct.h"

#include <algorithm>

#include "../../include/rfsf_ts.h"

namespace rfsf {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
// (The rounding of x log2 e is a relative error of |x| 2^-24, that of a score of size |x| rounded to 32 bits.)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Rows that count, of all blocks.
__global__ __launch_bounds__(256) void count_kernel(const int64_t *labels, int64_t N, uint32_t *count)
{
    uint32_t mine = 0;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < N; n += (int64_t)gridDim.x * 256) mine += labels[n] >= 0 ? 1 : 0;
#pragma unroll
    for (int o = 32; o > 0; o /= 2) mine += (uint32_t)__shfl_xor((int)mine, o);
    if ((threadIdx.x & 63) == 0 && mine != 0) atomicAdd(count, mine);
}
__global__ void zero_kernel(uint32_t *p) { *p = 0; }

template <typename T>
__global__ __launch_bounds__(256) void clear_rows_kernel(T *rows, int64_t count, int64_t columns, int64_t ld)
{
    for (int64_t r = blockIdx.x; r < count; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < columns; c += 256) rows[r * ld + c] = 0;
}

// Of the scores of some classes: their maximum, the sum of exponentials from there, and the largest exponential times 2^exponent(the
// class's weights), as a power of two, which bounds G[n, c] 2^exponent(W[c, :]). All from the maximum: nothing of it is lost where
// the scores are large.
struct Partial { float top, sum, reach; };
__device__ __forceinline__ Partial joined(const Partial &a, const Partial &b)
{
    const float m = fmaxf(a.top, b.top), from = m == -INFINITY ? 0.f : m;
    const float ta = (a.top - from) * kLog2e, tb = (b.top - from) * kLog2e;
    return {m, a.sum * __builtin_amdgcn_exp2f(ta) + b.sum * __builtin_amdgcn_exp2f(tb), fmaxf(a.reach + ta, b.reach + tb)};
}

// Scores: classes along the tile's rows, sequences along its columns, so that a lane holds many classes of one sequence and
// nearly all of the maximum and the sum is taken inside it.
// Bound by the product; where the scores are written, by that after it, as a CU holds one tile and all of them end together. Tiles of 256: 10000 x
// 5121, 5003 classes, float32, losses alone 1.46 to 1.50 ms (1030 to 1050 TFLOP/s of 16-bit products; 800 tiles are 3.1 rounds of the CUs, paid as four); 1024 x 2049, 32768 classes, bfloat16, with 134 MB of scores
// 157 us (875 TFLOP/s).
struct Scores {
    const uint32_t *largest_w, *largest_phi;    // per class, per sequence of the block
    int64_t C, rows;                            // classes; sequences of this launch
    const int64_t *labels;                      // of its first sequence on
    Partial *partial;                           // [class tiles][rows_ld]
    int64_t rows_ld;
    float *target;                              // the label's score
    float *scores;                              // [rows][ld], or null
    int64_t ld;
    bool with_reach;

    template <typename T>
    __device__ __forceinline__ void operator()(T &t) const
    {
        constexpr int BN = T::BN, CLASSES = T::ROWS + (T::HAS_EXTRA ? 32 : 0);
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        const int64_t c0 = t.tile_i * T::ROWS;
        // the classes' powers of two (of a class without weights, whose scores are zero, the smallest)
        int *powers = reinterpret_cast<int *>(t.lds);
        __syncthreads();
        for (int i = threadIdx.x; i < CLASSES; i += blockDim.x) powers[i] = exponent_of(c0 + i < C ? largest_w[c0 + i] : 0) - kTopBit;
        __syncthreads();
        float top[BN], sum[BN], reach[BN], from[BN];
        int shift_n[BN], label[BN];                         // the label's place in this tile
#pragma unroll
        for (int b = 0; b < BN; ++b) {
            const int64_t n = t.j0 + 32 * b + col, y = n < rows ? labels[n] - c0 : -1;
            shift_n[b] = n < rows ? shift_of(largest_phi[n]) : 0;
            label[b] = y >= 0 && y < CLASSES ? (int)y : -1;
            top[b] = reach[b] = -INFINITY;
            sum[b] = 0.f;
        }
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int4 p = *reinterpret_cast<const int4 *>(powers + (int)(first - c0) + 8 * q + 4 * half);
                acc[4 * q] = ldexpf(acc[4 * q], p.x - shift_n[b]);
                acc[4 * q + 1] = ldexpf(acc[4 * q + 1], p.y - shift_n[b]);
                acc[4 * q + 2] = ldexpf(acc[4 * q + 2], p.z - shift_n[b]);
                acc[4 * q + 3] = ldexpf(acc[4 * q + 3], p.w - shift_n[b]);
            }
        });
        if (c0 + CLASSES > C)
            t.each_block([&](auto &acc, int64_t first, int) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (first + 8 * (e / 4) + 4 * half + e % 4 >= C) acc[e] = -INFINITY;
            });
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
            const int64_t n = t.j0 + 32 * b + col;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = (int)(first - c0) + 8 * q + 4 * half, y = label[b] - i;
                if (y >= 0 && y < 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (y == e) target[n] = acc[4 * q + e];
                }
                top[b] = fmaxf(top[b], fmaxf(fmaxf(acc[4 * q], acc[4 * q + 1]), fmaxf(acc[4 * q + 2], acc[4 * q + 3])));
                if (scores && n < rows && c0 + i < C)             // (ld is a multiple of four: numbers beyond C are nobody's)
                    *reinterpret_cast<float4 *>(scores + n * ld + c0 + i) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
            }
        });
#pragma unroll
        for (int b = 0; b < BN; ++b) {
            top[b] = fmaxf(top[b], __shfl_xor(top[b], 32));
            from[b] = top[b] == -INFINITY ? 0.f : top[b];
        }
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = (acc[e] - from[b]) * kLog2e;
            if (with_reach) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int4 p = *reinterpret_cast<const int4 *>(powers + (int)(first - c0) + 8 * q + 4 * half);
                    const float r0 = fmaxf(acc[4 * q] + (float)p.x, acc[4 * q + 1] + (float)p.y), r1 = fmaxf(acc[4 * q + 2] + (float)p.z, acc[4 * q + 3] + (float)p.w);
                    reach[b] = fmaxf(reach[b], fmaxf(r0, r1) + (float)kTopBit);
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[b] += __builtin_amdgcn_exp2f(acc[e]);
        });
#pragma unroll
        for (int b = 0; b < BN; ++b) {
            sum[b] += __shfl_xor(sum[b], 32);
            reach[b] = fmaxf(reach[b], __shfl_xor(reach[b], 32));
        }
        // the wavefronts that hold other classes of the same sequences
        Partial *shared = reinterpret_cast<Partial *>(t.lds);
        constexpr int WIDE = T::COLUMNS, ROWS = T::WAVES_I;
        __syncthreads();
        if (half == 0) {
#pragma unroll
            for (int b = 0; b < BN; ++b) shared[t.wave_i * WIDE + t.wave_j * (32 * BN) + 32 * b + col] = {top[b], sum[b], reach[b]};
        }
        __syncthreads();
        const int64_t first = t.tile_j * WIDE;
        for (int j = threadIdx.x; j < WIDE; j += blockDim.x) {
            if (first + j >= rows) break;
            Partial v = shared[j];
#pragma unroll
            for (int w = 1; w < ROWS; ++w) v = joined(v, shared[w * WIDE + j]);
            partial[t.tile_i * rows_ld + first + j] = v;
        }
    }
};

// Joins the class tiles' parts: the loss, and for the gradients the maximum, 1 / sum, the row's scale and the exponent that bounds
// G[n, c] 2^exponent(W[c, :]).
struct __attribute__((aligned(16))) RowTerms { float top, inverse, scale; int32_t reach; };
constexpr int32_t kLeftOut = 4096;                  // as the exponent (others are within 512): the row's dPhi is 0, also where W holds infinities
struct JoinJob {
    const Partial *partial;
    int64_t tiles, rows_ld, rows, C;
    const int64_t *labels;
    const float *weight;
    const uint32_t *count, *largest_w;
    const float *target;
    float *loss;
    RowTerms *terms;                // null without gradients
};
// What follows from the statistics of all classes; `write`: the loss and the terms are written.
__device__ __forceinline__ RowTerms finish(const JoinJob &job, int64_t n, const Partial &v, bool write)
{
    const float from = v.top == -INFINITY ? 0.f : v.top, s = v.sum;
    const int64_t label = job.labels[n];
    const bool known = label >= 0 && label < job.C;
    if (write) job.loss[n] = label < 0 ? 0.f : known ? logf(s) + (from - job.target[n]) : NAN;
    float bound = v.reach - log2f(s);
    if (known) bound = fmaxf(bound, (float)exponent_of(job.largest_w[label]));
    const RowTerms t = {from, 1.0f / s, label < 0 ? 0.f : job.weight ? job.weight[n] : job.terms ? 1.0f / (float)*job.count : 0.f,
                        label < 0 ? kLeftOut : (int32_t)ceilf(fminf(fmaxf(bound, -512.f), 512.f))};
    if (write && job.terms) job.terms[n] = t;
    return t;
}
// 16 rows a workgroup, whose 16 groups of threads share out the tiles. Bound by latency: 6.3 us for 1024 rows of 128 tiles.
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(256) void join_kernel(JoinJob job)
{
    __shared__ Partial part[16][kJoinRows];
    const int r = threadIdx.x % kJoinRows, group = threadIdx.x / kJoinRows;
    const int64_t n = (int64_t)blockIdx.x * kJoinRows + r;
    Partial v = {-INFINITY, 0.f, -INFINITY};
    if (n < job.rows)
        for (int64_t t = group; t < job.tiles; t += 16) v = joined(v, job.partial[t * job.rows_ld + n]);
    part[group][r] = v;
    __syncthreads();
    if (group != 0 || n >= job.rows) return;
    for (int g = 1; g < 16; ++g) v = joined(v, part[g][r]);
    finish(job, n, v, true);
}

// From the scores of `rows` sequences to G as operand, in tiles of 64 x 64. By rows, for the product with W^T, whose columns are scaled by
// the classes' powers of two: (p - [c = y]) 2^exponent(W[c, :]), brought to 2^14 by the row's own exponent; the rows' scales
// enter at the end of the product, so that rows of small scale lose nothing. Transposed, for the product with Phi^T: the same with
// the rows' scales and exponents, brought to 2^14 by the largest of all.
// Bound by memory (scores read, two operands of two terms written), the scores coming from the last-level cache: 1024 x 32768 98 us for 403 MB (4.1 TB/s).
struct GradientJob {
    const float *scores;
    int64_t ld, rows, C;
    const int64_t *labels;
    const float *weight;
    const RowStats *stats;
    const RowTerms *terms;
    const uint32_t *largest_w, *largest_phi;
    char *by_row, *by_class;        // either may be null; by_class from the first sequence's column on
    int64_t pitch_row, pitch_class;
    JoinJob join;                   // JOIN: the class tiles' parts, of which the terms are made here; the first tiles of classes write them
};
template <bool JOIN>
__global__ __launch_bounds__(256) void gradient_kernel(GradientJob job)
{
    __shared__ float tile[64][65];
    const int64_t c0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
    const int at = threadIdx.x >> 3, group = threadIdx.x & 7;
    const int shift = job.by_class ? kTopBit - ((int)job.stats->top - kTopBias) : 0;
    __shared__ RowTerms made[JOIN ? 64 : 1];
    if constexpr (JOIN) {
        const int64_t n = n0 + threadIdx.x / 4;
        Partial v = {-INFINITY, 0.f, -INFINITY};
        if (n < job.rows) {
#pragma unroll 4
            for (int64_t t = threadIdx.x % 4; t < job.join.tiles; t += 4) v = joined(v, job.join.partial[t * job.join.rows_ld + n]);
        }
#pragma unroll
        for (int o = 1; o < 4; o *= 2) {
            const Partial w = {__shfl_xor(v.top, o), __shfl_xor(v.sum, o), __shfl_xor(v.reach, o)};
            v = joined(v, w);
        }
        if (threadIdx.x % 4 == 0 && n < job.rows) made[threadIdx.x / 4] = finish(job.join, n, v, blockIdx.x == 0);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 64; u += 32) {
        const int64_t n = n0 + at + u, c = c0 + 8 * group;
        float g[8], scale = 0.f;
        if (n < job.rows) {
            const RowTerms t = JOIN ? made[at + u] : job.terms[n];
            const int64_t label = job.labels[n];
            scale = ldexpf(job.weight ? t.scale : 1.0f, shift + exponent_of(job.largest_phi[n]));
            float v[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4 f = c + 4 * q < job.C ? *reinterpret_cast<const float4 *>(job.scores + n * job.ld + c + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[4 * q] = f.x;
                v[4 * q + 1] = f.y;
                v[4 * q + 2] = f.z;
                v[4 * q + 3] = f.w;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = exp_of(v[e] - t.top) * t.inverse;
                if (c + e == label) g[e] -= 1.0f;
                if (label < 0 || c + e >= job.C) g[e] = 0.f;
                else if (label >= job.C) g[e] = NAN;
            }
            if (job.by_row) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = c + e < job.C ? ldexpf(g[e], exponent_of(job.largest_w[c + e]) + kTopBit - t.reach) : 0.f;
                plane::store_terms<true>(job.by_row + n * job.pitch_row, c, plane::terms_of<true>(x));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) tile[at + u][8 * group + e] = g[e] == 0.f ? 0.f : g[e] * scale;
    }
    if (!job.by_class) return;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 64; u += 32) {
        const int64_t c = c0 + at + u;
        if (c >= job.C) continue;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = tile[8 * group + e][at + u];
        plane::store_terms<true>(job.by_class + c * job.pitch_class, n0 + 8 * group, plane::terms_of<true>(x));
    }
}

// A gradient: rows of the tile along the contiguous axis of the result. Both gradients share a launch, so that the second one's tiles fill the CUs
// that the first one's leave. 8192 x 2049, 32768 classes, bfloat16: 3.55 to 3.61
// ms (1220 to 1240 TFLOP/s of 16-bit products; with G as one term of 11 bits 1.95 ms, and dPhi 3.4e-4 from the rounded exact result instead of 0.9e-4); 1000 x 1025, 1000
// classes, float32 32 us.
struct Gradient {
    void *out;
    int64_t ld, rows_i, cols_j;
    bool bf16;                          // type of out
    const RowTerms *terms;              // dPhi: the rows' scales and exponents. Null (dW):
    const RowStats *stats;              // ... one exponent
    const uint32_t *count;              // ... and, without weights (else null), one scale
    const float *add;                   // [cols_j][add_ld] of the blocks before, or null
    int64_t add_ld;
    int64_t cut_stride;                 // numbers from one part of a cut sum to the next

    template <typename T>
    __device__ __forceinline__ void operator()(T &t) const
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        const int all = terms ? 0 : (int)stats->top - kTopBias;
        const float mean = count ? 1.0f / (float)max(*count, 1u) : 1.0f;
        const int64_t first_of_cut = t.cut * cut_stride;
        t.each_block([&](const auto &acc, int64_t first, int b) __attribute__((always_inline)) {
            const int64_t j = t.j0 + 32 * b + col;
            if (j >= cols_j) return;
            const int64_t row = first_of_cut + j * ld;
            const float scale = terms ? terms[j].scale : mean;
            const int exponent = terms ? terms[j].reach : all, shift = exponent - 2 * kTopBit;
            const bool left_out = terms && exponent == kLeftOut;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t i = first + 8 * q + 4 * half;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = left_out ? 0.f : ldexpf(acc[4 * q + e], shift) * scale;
                    if (add && i + e < rows_i) v[e] += add[j * add_ld + i + e];
                }
                if (i < rows_i) store(row + i, rows_i - i, v);
            }
        });
    }
    __device__ __forceinline__ void store(int64_t at, int64_t left, const float (&v)[4]) const
    {
        struct __attribute__((packed, aligned(4))) Float4u { float x, y, z, w; };
        struct __attribute__((packed, aligned(2))) Bf16x4u { __bf16 x, y, z, w; };
        if (bf16) {
            __bf16 *dst = static_cast<__bf16 *>(out) + at;
            if (left >= 4) {
                *reinterpret_cast<Bf16x4u *>(dst) = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            } else {
                for (int e = 0; e < 4; ++e)
                    if (e < left) dst[e] = (__bf16)v[e];
            }
        } else {
            float *dst = static_cast<float *>(out) + at;
            if (left >= 4) {
                *reinterpret_cast<Float4u *>(dst) = {v[0], v[1], v[2], v[3]};
            } else {
                for (int e = 0; e < 4; ++e)
                    if (e < left) dst[e] = v[e];
            }
        }
    }
};

// Adds the parts of cut sums up. Bound by memory.
struct CutSum {
    const float *parts;                 // [cuts][numbers / K][K]
    void *out;
    const float *add;                   // or null
    int64_t ld, add_ld, numbers, cuts, bf16;
};
// (A sum is chosen as a whole, by whole words: flags of a byte, indexed in the arguments beside longer fields, have been read with scalar loads from addresses
// that are no multiples of four, whose last bits these ignore.)
struct AddJob {
    CutSum first, second;
    int64_t K;
    unsigned groups_of_first;
};
__global__ __launch_bounds__(256) void add_kernel(AddJob job)
{
    const bool is_first = blockIdx.x < job.groups_of_first;
    const CutSum s = is_first ? job.first : job.second;
    const int64_t m = (int64_t)(blockIdx.x - (is_first ? 0 : job.groups_of_first)) * 256 + threadIdx.x;
    if (m >= s.numbers) return;
    float sum = 0.f;
#pragma unroll 4
    for (int64_t c = 0; c < s.cuts; ++c) sum += s.parts[c * s.numbers + m];
    const int64_t j = m / job.K, i = m - j * job.K;
    if (s.add) sum += s.add[j * s.add_ld + i];
    if (s.bf16) static_cast<__bf16 *>(s.out)[j * s.ld + i] = (__bf16)sum;
    else static_cast<float *>(s.out)[j * s.ld + i] = sum;
}

// ---------------------------------------------------------------------------------------------------------------
// Workspace and order of work.
// How the gradients' products of a block of rows are made: the tiles' edge, and the parts of their sums (dPhi, dW), by the steps' time. A long sum of few tiles
// leaves CUs without work; cut, it costs its parts' way through memory and a launch. (us a call, whole and cut: 7487 x 316, 365 classes, float32, dW
// 105 and 56; 1209 x 88, 7765, float32, dPhi 129 and 81; 9000 x 4000, 300, bfloat16, both 282 and 263; 8638 x
// 3613, 172, float32, dPhi, is not cut. Of 60 shapes with 65 to 10000 rows and 65 to 33000 classes the geometric mean is 1.11.)
struct GradientPlan { int edge, cuts[2]; };
constexpr double kPartRate = 3e6, kAddTime = 5.0;                  // bytes a us, written and read; us
constexpr int64_t kMostPartBytes = (int64_t)256 << 20;
constexpr int kStartSteps = 4;                                     // what a tile costs besides its steps, in steps
GradientPlan plan_gradients(bool d_phi, bool d_w, int64_t rows, int64_t K, int64_t C, bool may_cut)
{
    const bool asked[2] = {d_phi, d_w};
    const int64_t steps[2] = {d_phi ? plane_steps(C, true) : 0, d_w ? plane_steps(rows, true) : 0}, across[2] = {rows, C};
    GradientPlan best = {0, {1, 1}};
    double least = 0.0;
    for (const PlaneWay &way : kPlaneWays) {
        const double tiles[2] = {d_phi ? (double)plane_tiles(K, rows, way.edge) : 0.0, d_w ? (double)plane_tiles(K, C, way.edge) : 0.0};
        int most[2];
        for (int p = 0; p < 2; ++p) {
            most[p] = 1;
            while (may_cut && asked[p] && 2 * most[p] <= 32 && tiles[p] * most[p] < way.slots && steps[p] / (2 * most[p]) >= 8 &&
                   4 * K * across[p] * 2 * most[p] <= kMostPartBytes)
                most[p] *= 2;
        }
        for (int a = 1; a <= most[0]; a *= 2)
            for (int b = 1; b <= most[1]; b *= 2) {
                const double s0 = asked[0] ? (double)steps[0] / a + kStartSteps : 0.0, s1 = asked[1] ? (double)steps[1] / b + kStartSteps : 0.0;
                const double longest = std::max(s0, s1), count = (tiles[0] * a * s0 + tiles[1] * b * s1) / longest;
                double time = plane_step_time(way, count) * longest;
                if (a > 1 || b > 1) time += kAddTime + 8.0 * (double)K * ((a > 1 ? (double)a * (double)rows : 0.0) + (b > 1 ? (double)b * (double)C : 0.0)) / kPartRate;
                if (best.edge == 0 || time < least) {
                    best = {way.edge, {a, b}};
                    least = time;
                }
            }
    }
    return best;
}
constexpr int64_t kUnit = 64;                           // rows of a block are counted in these
// Tiles of classes whose parts the pass to G joins by itself, every workgroup those of its rows, which saves a launch; with more of them they are read
// too often. (us a call, apart and here: 4454 x 257, 468 classes, bfloat16, dPhi 49.2 and 45.4; 1000 x 1025, 1000, float32, both 67.3 and 65.5; 1432 x
// 1999, 2885, 12 tiles, float32, both 293.0 and 293.8. Of 44 shapes with 302 to 4541 classes the geometric mean is 1.016, the worst 0.990.)
constexpr int64_t kJoinHere = 32;
constexpr size_t kScoreBytes = (size_t)128 << 20;       // of scores in flight: half of the last-level cache
constexpr size_t kBlockBytes = (size_t)8 << 30;         // recommended, of what grows with the rows of a block
constexpr int64_t kMostBlockRows = 3500000 / kUnit * kUnit;

size_t up(size_t v) { return (v + 255) / 256 * 256; }
int64_t units(int64_t rows) { return (rows + kUnit - 1) / kUnit * kUnit; }

struct Sizes {
    bool two, d_phi, d_w;
    int64_t N, K, C, ld_scores, class_tiles;
    explicit Sizes(const rfsf_xent_shape &s)
        : two(s.bf16 == 0), d_phi((s.gradients & RFSF_XENT_DPHI) != 0), d_w((s.gradients & RFSF_XENT_DW) != 0), N(s.N), K(s.K), C(s.C),
          ld_scores((s.C + 3) / 4 * 4), class_tiles((s.C + kUnit - 1) / kUnit)
    {
    }
    // of the call: W both ways, the magnitudes, the rows' statistics
    size_t fixed() const
    {
        return up((size_t)C * plane_pitch(K, two)) + (d_phi ? up((size_t)K * plane_pitch(C, two)) : 0) + up(sizeof(RowStats)) + up(4) + up(4 * (size_t)C) + 256;
    }
    // of a block of `rows` rows (a multiple of kUnit)
    size_t block(int64_t rows) const
    {
        size_t b = up((size_t)rows * plane_pitch(K, two)) + up(4 * (size_t)rows) + up(4 * (size_t)rows) + up(sizeof(RowTerms) * (size_t)rows) +
                   up(sizeof(Partial) * (size_t)class_tiles * (size_t)rows);
        if (d_phi) b += up((size_t)rows * plane_pitch(C, true));
        if (d_w) b += up((size_t)C * plane_pitch(rows, true)) + up((size_t)K * plane_pitch(rows, two));
        if (d_w && !two && rows < N) b += up(4 * (size_t)C * (size_t)K);        // sums of the blocks before
        if (d_phi || d_w) {
            const GradientPlan plan = gradients(rows);
            b += parts(plan.cuts[0], rows) + parts(plan.cuts[1], C);
        }
        return b;
    }
    // (a workspace for small blocks only has none for parts either)
    GradientPlan gradients(int64_t rows) const { return plan_gradients(d_phi, d_w, rows, K, C, rows >= std::min<int64_t>(N, 1024)); }
    size_t parts(int cuts, int64_t across) const { return cuts > 1 ? up(4 * (size_t)cuts * (size_t)K * (size_t)across) : 0; }
    size_t scores(int64_t rows) const { return d_phi || d_w ? up(4 * (size_t)rows * (size_t)ld_scores) : 0; }
    int64_t score_rows(int64_t rows) const
    {
        int64_t n = (int64_t)(kScoreBytes / (4 * (size_t)ld_scores)) / 256 * 256;
        n = std::max<int64_t>(n, 256);
        return std::min(n, rows);
    }
    int64_t recommended_rows() const
    {
        int64_t rows = std::min(units(std::max<int64_t>(N, 1)), kMostBlockRows);
        while (rows > 4096 && block(rows) > kBlockBytes) rows = units(rows / 2);
        return rows;
    }
};

struct Plan { int64_t rows, score_rows; };
// The largest blocks that the workspace holds.
bool plan_of(const Sizes &z, size_t bytes, Plan *plan)
{
    if (bytes < z.fixed()) return false;
    const size_t room = bytes - z.fixed();
    int64_t rows = std::min(units(z.N), kMostBlockRows);
    for (;; rows = units(rows / 2)) {
        int64_t s = z.score_rows(rows);
        for (;; s = units(s / 2)) {
            if (z.block(rows) + z.scores(s) <= room) {
                *plan = {rows, s};
                return true;
            }
            if (s <= kUnit) break;
        }
        if (rows <= kUnit) return false;
    }
}

struct Carve {
    char *at;
    template <typename T>
    T *take(size_t bytes)
    {
        T *p = reinterpret_cast<T *>(at);
        at += up(bytes);
        return p;
    }
};

}  // namespace

void softmax_xent_bytes(const rfsf_xent_shape &shape, size_t *recommended, size_t *minimum)
{
    if (xent_direct(shape)) {
        *recommended = *minimum = xent_direct_bytes(shape);
        return;
    }
    const Sizes z(shape);
    const int64_t rows = z.recommended_rows();
    *recommended = z.fixed() + z.block(rows) + z.scores(z.score_rows(rows));
    // (blocks of the fewest rows need room to add dW up, which all rows at once may not)
    *minimum = std::min(*recommended, z.fixed() + z.block(kUnit) + z.scores(kUnit));
}

hipError_t launch_clear_rows(void *rows, int64_t count, int64_t columns, int64_t ld, bool bf16, hipStream_t stream)
{
    const dim3 grid((unsigned)std::min<int64_t>(count, 65536));
    if (bf16) clear_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<uint16_t *>(rows), count, columns, ld);
    else clear_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<uint32_t *>(rows), count, columns, ld);
    return hipGetLastError();
}

#define RFSF_TRY(call)                                   \
    do {                                                 \
        const hipError_t e_ = (call);                    \
        if (e_ != hipSuccess) return e_;                 \
    } while (0)

template <PlaneMode MODE>
hipError_t xent_blocks(const rfsf_xent_shape &shape, const void *Phi, const void *W, const int64_t *labels, const float *weight, float *loss, void *dPhi,
                       void *dW, void *workspace, size_t bytes, hipStream_t stream)
{
    const Sizes z(shape);
    Plan plan;
    if (!plan_of(z, bytes, &plan)) return hipErrorInvalidValue;
    const bool bf16 = !z.two, gradients = z.d_phi || z.d_w;
    const size_t element = bf16 ? 2 : 4;
    const int64_t pitch_k = plane_pitch(z.K, z.two), pitch_c = plane_pitch(z.C, z.two), pitch_n = plane_pitch(plan.rows, z.two);
    const int64_t pitch_gc = plane_pitch(z.C, true), pitch_gn = plane_pitch(plan.rows, true);            // of G's two terms
    const int64_t N = z.N, K = z.K, C = z.C;

    const size_t mis = (size_t)(reinterpret_cast<uintptr_t>(workspace) % 256);
    Carve ws{static_cast<char *>(workspace) + (mis ? 256 - mis : 0)};
    char *w_rows = ws.take<char>((size_t)C * pitch_k);
    char *w_columns = z.d_phi ? ws.take<char>((size_t)K * pitch_c) : nullptr;
    RowStats *stats = ws.take<RowStats>(sizeof(RowStats));
    uint32_t *total = ws.take<uint32_t>(4);
    uint32_t *largest_w = ws.take<uint32_t>(4 * (size_t)C);
    uint32_t *largest_phi = ws.take<uint32_t>(4 * (size_t)plan.rows);
    float *target = ws.take<float>(4 * (size_t)plan.rows);
    RowTerms *terms = ws.take<RowTerms>(sizeof(RowTerms) * (size_t)plan.rows);
    Partial *partial = ws.take<Partial>(sizeof(Partial) * (size_t)z.class_tiles * (size_t)plan.rows);
    char *phi_rows = ws.take<char>((size_t)plan.rows * pitch_k);
    char *g_rows = z.d_phi ? ws.take<char>((size_t)plan.rows * pitch_gc) : nullptr;
    char *g_classes = z.d_w ? ws.take<char>((size_t)C * pitch_gn) : nullptr;
    char *phi_columns = z.d_w ? ws.take<char>((size_t)K * pitch_n) : nullptr;
    float *sums = z.d_w && bf16 && plan.rows < N ? ws.take<float>(4 * (size_t)C * (size_t)K) : nullptr;
    const GradientPlan how = gradients ? z.gradients(plan.rows) : GradientPlan{64, {1, 1}};
    float *parts_phi = ws.take<float>(z.parts(how.cuts[0], plan.rows)), *parts_w = ws.take<float>(z.parts(how.cuts[1], C));
    float *scores = gradients ? ws.take<float>(4 * (size_t)plan.score_rows * (size_t)z.ld_scores) : nullptr;

    // the scale of rows without weights is known from the rows' packing, unless they are packed in several blocks
    const uint32_t *count = weight ? nullptr : plan.rows < N ? total : &stats->count;
    if (gradients && count == total) {
        zero_kernel<<<1, 1, 0, stream>>>(total);
        count_kernel<<<dim3((unsigned)std::min<int64_t>((N + 1023) / 1024, 256)), dim3(256), 0, stream>>>(labels, N, total);
        RFSF_TRY(hipGetLastError());
    }
    const PackJob pack_w = {W, C, K, shape.ld_w, nullptr, largest_w, w_rows, w_columns, pitch_k, pitch_c};
    for (int64_t n0 = 0; n0 < N; n0 += plan.rows) {
        const int64_t rows = std::min(plan.rows, N - n0);
        const PackJob pack_phi = {static_cast<const char *>(Phi) + (size_t)n0 * shape.ld_phi * element, rows, K, shape.ld_phi, labels + n0, largest_phi,
                                  phi_rows, phi_columns, pitch_k, pitch_n};
        PackPair pair = {{pack_w, pack_phi}, gradients ? stats : nullptr, weight ? weight + n0 : nullptr};
        if (n0 > 0) pair.job[0].R = 0;
        if (!gradients && K <= kPackRowsColumns) {
            RFSF_TRY(launch_pack_rows(pair, bf16, stream));
        } else {
            RFSF_TRY(launch_largest(pair, bf16, stream));
            RFSF_TRY(launch_pack(pair, bf16, stream));
        }
        const int64_t step = gradients ? plan.score_rows : rows;
        for (int64_t m0 = 0; m0 < rows; m0 += step) {
            const int64_t part = std::min(step, rows - m0);
            const int edge = plane_tile(C, part);
            const Scores epilogue = {largest_w, largest_phi + m0, C, part, labels + n0 + m0, partial, plan.rows, target, scores, z.ld_scores, z.d_phi};
            RFSF_TRY(launch_plane_product<MODE>(Planes{w_rows, pitch_k, C}, Planes{phi_rows + m0 * pitch_k, pitch_k, part}, plane_steps(K, z.two), edge,
                                                epilogue, stream));
            const JoinJob join = {partial, plane_tiles_a(C, edge), plan.rows, part, C, labels + n0 + m0, weight ? weight + n0 + m0 : nullptr, count, largest_w,
                                  target, loss + n0 + m0, gradients ? terms + m0 : nullptr};
            const bool join_apart = !gradients || join.tiles > kJoinHere;
            if (join_apart) {
                join_kernel<<<dim3((unsigned)((part + kJoinRows - 1) / kJoinRows)), dim3(256), 0, stream>>>(join);
                RFSF_TRY(hipGetLastError());
            }
            if (!gradients) continue;
            const GradientJob job = {scores, z.ld_scores, part, C, labels + n0 + m0, weight, stats, terms + m0, largest_w, largest_phi + m0, g_rows ? g_rows + m0 * pitch_gc : nullptr,
                                     g_classes ? g_classes + (m0 / 64) * (2 * kStepBytes) : nullptr, pitch_gc, pitch_gn, join};
            const dim3 grid((unsigned)((C + 63) / 64), (unsigned)((part + 63) / 64));
            if (join_apart) gradient_kernel<false><<<grid, dim3(256), 0, stream>>>(job);
            else gradient_kernel<true><<<grid, dim3(256), 0, stream>>>(job);
            RFSF_TRY(hipGetLastError());
        }
        if (!gradients) continue;
        Product<Gradient> products[2];
        AddJob sum = {};
        int count_of_products = 0, cut_sums = 0;
        // a product whose sum is cut writes parts, which are added up to what it would have written
        auto cut = [&](Product<Gradient> &p, int cuts, float *parts) {
            p.per_cut = (p.steps + cuts - 1) / cuts;
            if (p.cuts() == 1) return;
            Gradient &g = p.epilogue;
            (cut_sums++ == 0 ? sum.first : sum.second) = {parts, g.out, g.add, g.ld, g.add_ld, K * g.cols_j, p.cuts(), g.bf16};
            g.out = parts;
            g.ld = K;
            g.bf16 = false;
            g.add = nullptr;
            g.cut_stride = K * g.cols_j;
        };
        if (z.d_phi) {
            products[count_of_products] = {Planes{w_columns, pitch_c, K}, Planes{g_rows, pitch_gc, rows}, plane_steps(C, true),
                                           Gradient{static_cast<char *>(dPhi) + (size_t)n0 * shape.ld_dphi * element, shape.ld_dphi, K, rows, bf16,
                                                    terms, nullptr, nullptr, nullptr, 0, 0}, 0};
            cut(products[count_of_products++], how.cuts[0], parts_phi);
        }
        if (z.d_w) {
            const bool to_sums = sums && n0 + rows < N;
            const float *add = n0 == 0 ? nullptr : sums ? sums : static_cast<const float *>(dW);
            products[count_of_products] = {Planes{phi_columns, pitch_n, K}, Planes{g_classes, pitch_gn, C}, plane_steps(rows, true),
                                           Gradient{to_sums ? static_cast<void *>(sums) : dW, to_sums ? K : shape.ld_dw, K, C, bf16 && !to_sums, nullptr,
                                                    stats, count, add, sums ? K : shape.ld_dw, 0}, 0};
            cut(products[count_of_products++], how.cuts[1], parts_w);
        }
        // the longer tiles first, so that the others fill up behind them
        if (count_of_products == 2 && products[1].per_cut > products[0].per_cut) std::swap(products[0], products[1]);
        RFSF_TRY(launch_plane_products<MODE == kHalf ? kHalfByTwo : MODE>(products, count_of_products, how.edge, stream));
        if (cut_sums > 0) {
            sum.K = K;
            sum.groups_of_first = (unsigned)((sum.first.numbers + 255) / 256);
            const unsigned groups = sum.groups_of_first + (unsigned)((sum.second.numbers + 255) / 256);
            add_kernel<<<dim3(groups), dim3(256), 0, stream>>>(sum);
            RFSF_TRY(hipGetLastError());
        }
    }
    return hipSuccess;
}

hipError_t launch_softmax_xent(const rfsf_xent_shape &shape, const void *Phi, const void *W, const int64_t *labels, const float *weight, float *loss,
                               void *dPhi, void *dW, void *workspace, size_t bytes, hipStream_t stream)
{
    if (xent_direct(shape)) return launch_xent_direct(shape, Phi, W, labels, weight, loss, dPhi, dW, workspace, stream);
    return shape.bf16 ? xent_blocks<kHalf>(shape, Phi, W, labels, weight, loss, dPhi, dW, workspace, bytes, stream)
                      : xent_blocks<kHalfTwo>(shape, Phi, W, labels, weight, loss, dPhi, dW, workspace, bytes, stream);
}

}  // namespace rfsf
