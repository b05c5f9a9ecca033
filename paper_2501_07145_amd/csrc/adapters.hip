// Scores of a linear classifier with low-rank adapters of many requests at once (rfsf_adapted_scores):
//   out[n, c] = x_n . w_c + sum_r s[n, r] B[a][c, r],   s[n, r] = scale[a] (A[a][r] . x_n),   a the row's adapter
//
// Weights and adapters lie packed as operands of plane_product.h, the rows of X are packed by each call. Rows are put in the order of their adapters, so that
// rows that are worked on together share few of them; the inner products s go through matrix instructions in tiles of 16 rows, one
// adapter of the tile after another; the shared product's epilogue adds B's part to its accumulators, again one
// adapter of a block of 32 rows after another. What belongs to a row of another adapter is left out by a choice between registers, never by a factor of 0, which
// infinities and NaN would get through.
#include "plane_product.h"

#include <algorithm>

#include "../../include/rfsf_ts.h"
#include "plane_pack.h"
#include "rows8.h"

#define RFSF_TRY(call)                       \
    do {                                     \
        const hipError_t e_ = (call);        \
        if (e_ != hipSuccess) return e_;     \
    } while (0)

namespace rfsf {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A number as the sum of three of bfloat16, cut off and not rounded, so that none of them is infinite unless it is.
struct Terms3 { uint16_t v[3]; };
__device__ __forceinline__ Terms3 terms3(float x)
{
    Terms3 t;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const uint32_t top = __float_as_uint(x) & 0xffff0000u;
        t.v[i] = (uint16_t)(top >> 16);
        x -= __uint_as_float(top);
    }
    return t;
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// The caller's memory: W's rows, those of the adapters' A (ranks rounded up to 16, zeros beyond), each with their largest numbers, then B in its own type
// (ranks rounded up to 16 bytes, zeros beyond), and the scales.
struct Layout {
    int64_t pitch;                      // bytes of a packed row
    int ranks, ranks_b;                 // rows of an adapter's A, numbers of a row of its B
    size_t w, largest_w, a, largest_a, b, scale, bytes;
};
Layout layout_of(const rfsf_adapters_shape &s)
{
    Layout z;
    z.pitch = plane_pitch(s.K, !s.bf16);
    z.ranks = (int)((s.rank + 15) / 16 * 16);
    z.ranks_b = (int)(s.bf16 ? (s.rank + 7) / 8 * 8 : (s.rank + 3) / 4 * 4);
    z.w = 0;
    z.largest_w = z.w + up((size_t)s.C * z.pitch);
    z.a = z.largest_w + up((size_t)s.C * 4);
    z.largest_a = z.a + up((size_t)s.count * z.ranks * z.pitch);
    z.b = z.largest_a + up((size_t)s.count * z.ranks * 4);
    z.scale = z.b + up((size_t)s.count * s.C * z.ranks_b * (s.bf16 ? 2 : 4));
    z.bytes = z.scale + up((size_t)s.count * 4);
    return z;
}

hipError_t pack(const PackJob &job, bool bf16, hipStream_t stream)
{
    PackPair pair = {};
    pair.job[0] = job;
    if (job.K <= kPackRowsColumns) return launch_pack_rows(pair, bf16, stream);
    RFSF_TRY(launch_largest(pair, bf16, stream));
    return launch_pack(pair, bf16, stream);
}

// An adapter's B with rows of `ranks_b` numbers, its scale, and zeros for the rows of its A beyond the rank. Replacing an adapter is this launch and the packing of its A, bound by
// latency: 1025 columns, 1000 classes, rank 8 4.7 us, 5121, 10000, 16 5.5, 2049, 32768, 32 8.3 (float32; floor 1.8), beyond 12288 columns, packed in two launches, 15. Laying out
// W is bound by memory: 10000 x 5121, float32 75 us, 32768 x 2049 105; 50000 x 12300, read twice, 1320 (floor 992).
template <typename T>
__global__ __launch_bounds__(256) void set_kernel(const T *B, int64_t ld_b, int64_t C, int rank, int ranks_b, T *to, char *a_rest, int64_t rest_bytes,
                                                  uint32_t *largest_rest, int rest, float *scale_at, float scale)
{
    const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = first; i < C * ranks_b; i += step) {
        const int64_t c = i / ranks_b;
        const int r = (int)(i - c * ranks_b);
        to[i] = r < rank ? B[c * ld_b + r] : (T)0;
    }
    for (int64_t i = first; i < rest_bytes / 16; i += step) reinterpret_cast<uint4 *>(a_rest)[i] = make_uint4(0, 0, 0, 0);
    for (int64_t i = first; i < rest; i += step) largest_rest[i] = 0;
    if (first == 0) *scale_at = scale;
}

// The rows in the order of their adapters: each row's place is the number of rows that come before it, those with a lower adapter, or the same one and a lower
// number. Two lanes have a row, 16 wavefronts share the rows it is compared with. Bound by reading the keys from LDS: 8192 rows 11 us.
constexpr int kMostRows = 8192;             // at a time: 13 bits beside the adapter's number, of which there are fewer than 2^18
constexpr int kNone = -1, kUnknown = -2;    // who: rows without an adapter, and with one that does not exist
constexpr int kOrderWaves = 16, kOrderRows = 32;
__device__ __forceinline__ int code_of(int64_t adapter, int64_t count) { return adapter < 0 ? 0 : adapter < count ? (int)adapter + 1 : (int)count + 1; }
__device__ __forceinline__ int who_of(int64_t adapter, int64_t count) { return adapter < 0 ? kNone : adapter < count ? (int)adapter : kUnknown; }
__global__ __launch_bounds__(64 * kOrderWaves) void order_kernel(const int64_t *adapters, int rows, int64_t count, int32_t *order, int32_t *who)
{
    __shared__ __attribute__((aligned(16))) uint32_t keys[kMostRows];
    __shared__ int part[2 * kOrderWaves][kOrderRows];
    const int lane = threadIdx.x % kOrderRows, group = threadIdx.x / kOrderRows, row = blockIdx.x * kOrderRows + lane;
    const int fours = (rows + 3) / 4;
#pragma unroll 4
    for (int m = threadIdx.x; m < 4 * fours; m += 64 * kOrderWaves) keys[m] = m < rows ? (uint32_t)code_of(adapters[m], count) << 13 | (uint32_t)m : ~0u;
    __syncthreads();
    const uint32_t mine = row < rows ? keys[row] : 0;
    int before = 0;
#pragma unroll 8
    for (int f = group; f < fours; f += 2 * kOrderWaves) {
        const uint4 k = *reinterpret_cast<const uint4 *>(keys + 4 * f);
        before += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
    }
    part[group][lane] = before;
    __syncthreads();
    if (group != 0 || row >= rows) return;
    before = 0;
#pragma unroll
    for (int w = 0; w < 2 * kOrderWaves; ++w) before += part[w][lane];
    order[before] = row;
    who[before] = who_of(adapters[row], count);
}

// Order and packing in one launch, for some hundred rows that fit into registers: a workgroup packs a row, and compares it with all others on the way. Bound by latency:
// 333 x 5121, bfloat16 5.2 us (order_kernel and packing 9.1).
constexpr int kPlaceThreads = 512;
constexpr int64_t kPlaceRows = 1024, kPlaceColumns = 3 * 8 * kPlaceThreads;
struct PlaceJob {
    const void *X;
    int64_t ld_x, K, count;
    const int64_t *adapters;
    int rows;
    char *x;                            // packed, in the order of the adapters
    int64_t pitch;
    uint32_t *largest_x;
    int32_t *order, *who;
};
template <bool TWO, int HELD>
__global__ __launch_bounds__(kPlaceThreads) void place_kernel(PlaceJob job)
{
    typedef std::conditional_t<TWO, float, uint16_t> Number;
    constexpr int WAVES = kPlaceThreads / 64;
    __shared__ uint32_t part_largest[WAVES];
    __shared__ int part_before[WAVES];
    const int row = blockIdx.x;
    const Number *from = static_cast<const Number *>(job.X) + row * job.ld_x;
    float x[HELD][8];
#pragma unroll
    for (int u = 0; u < HELD; ++u) rows8::load(from, 8 * (int64_t)(threadIdx.x + u * kPlaceThreads), job.K, x[u]);
    const int64_t adapter = job.adapters[row];
    const int mine = code_of(adapter, job.count);
    int before = 0;
    for (int m = threadIdx.x; m < job.rows; m += kPlaceThreads) {
        const int other = code_of(job.adapters[m], job.count);
        before += other < mine || (other == mine && m < row);
    }
    uint32_t largest = 0;
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(x[u][e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) {
        largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
        before += __shfl_xor(before, o);
    }
    if ((threadIdx.x & 63) == 0) {
        part_largest[threadIdx.x >> 6] = largest;
        part_before[threadIdx.x >> 6] = before;
    }
    __syncthreads();
    largest = 0;
    before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        largest = max(largest, part_largest[w]);
        before += part_before[w];
    }
    if (threadIdx.x == 0) {
        job.largest_x[before] = largest;
        job.order[before] = row;
        job.who[before] = who_of(adapter, job.count);
    }
    const int shift = shift_of(largest);
    char *to = job.x + before * job.pitch;
    const int64_t end = (job.K + 63) / 64 * 64;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
        const int64_t k = 8 * (int64_t)(threadIdx.x + u * kPlaceThreads);
        if (k >= end) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = ldexpf(x[u][e], shift);
        plane::store_terms<TWO>(to, k, plane::terms_of<TWO>(x[u]));
    }
}

// A step of products of 16 rows of each of `fa` and 16 of each of `fx`.
template <bool TWO, int BM, int NB>
__device__ __forceinline__ void multiply_step(const halfx8 (&fa)[BM][2], const halfx8 (&fx)[NB][2], floatx4 (&acc)[BM][NB])
{
#pragma unroll
    for (int m = 0; m < BM; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            if (TWO) {
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[m][1], fx[n][0], acc[m][n], 0, 0, 0);
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[m][0], fx[n][1], acc[m][n], 0, 0, 0);
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[m][0], fx[n][0], acc[m][n], 0, 0, 0);
            } else {
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[m][0], fx[n][0], acc[m][n], 0, 0, 0);
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[m][1], fx[n][1], acc[m][n], 0, 0, 0);
            }
        }
}

// Sums of products of 16 rows of `a` (lane l: row l % 16, already advanced to its quarter of 64 bytes) and 16 of each of NB groups of `x`, over steps first,
// first + stride, ..: AHEAD steps under way at a time.
template <bool TWO, int BM, int NB, int AHEAD>
__device__ __forceinline__ void multiply_steps(const char *const (&a)[BM], const char *const (&x)[NB], int first, int stride, int steps, floatx4 (&acc)[BM][NB])
{
    auto load = [&](int s, halfx8 (&fa)[BM][2], halfx8 (&fx)[NB][2]) {
        const int64_t at = (int64_t)s * kStepBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int m = 0; m < BM; ++m) fa[m][h] = *reinterpret_cast<const halfx8 *>(a[m] + at + 64 * h);
#pragma unroll
            for (int n = 0; n < NB; ++n) fx[n][h] = *reinterpret_cast<const halfx8 *>(x[n] + at + 64 * h);
        }
    };
    int s = first;
    for (; s + (AHEAD - 1) * stride < steps; s += AHEAD * stride) {
        halfx8 fa[AHEAD][BM][2], fx[AHEAD][NB][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(s + u * stride, fa[u], fx[u]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) multiply_step<TWO>(fa[u], fx[u], acc);
    }
    for (; s < steps; s += stride) {
        halfx8 fa[BM][2], fx[NB][2];
        load(s, fa, fx);
        multiply_step<TWO>(fa, fx, acc);
    }
}

// Inner products, and for few rows the shared ones, straight from the packed rows. A workgroup has 16 rows of an adapter's A and 16 of X, of which it keeps what belongs to
// rows of this adapter, or 16 BM rows of W, and a cut of the columns; its wavefronts share the steps. Slot s of a tile of 16 rows takes the adapters number s, s + slots, ..
// of those that its rows have. What is left are sums of products as they are, which are scaled and added up where they are used. Bound by reading W and the
// adapters once: 16 x 5121, 5003 classes, adapters of rank 16, float32 23.5 us (4.8 TB/s; with 16 rows of W a workgroup, which read X twice as often, 38); 8 x 10241, 50000
// classes, all launches, 410 us (5.1 TB/s).
constexpr int64_t kFewGroups = 512;
constexpr int kFewWaves = 4, kFewAhead = 2, kFewBlocks = 4, kFewRows = 16 * kFewBlocks, kWide = 2;
// LOCAL: up to four rows of X that have few numbers altogether are packed by every workgroup for itself into LDS: a launch less (1 x 1025, 1000 classes 13.0 -> 9.6 us;
// seven rows 11.2 -> 12.3), all numbers at once (1 x 8192, 1000 classes, float32 14.4 us; a wavefront a row, in turns, 25.4).
constexpr int kMostRank = 256;              // that is accepted
constexpr int kLocal = 8192, kLocalRows = kFewWaves, kLocalPad = 16;        // numbers, rows; bytes between rows, for their banks
constexpr size_t local_bytes(bool two) { return kLocal * (two ? 4 : 2) + kLocalRows * (kStepBytes + kLocalPad); }
// Packs the rows into `local`, all wavefronts together, some to a row: every number is loaded once, all loads are under way at the same time. largest: in LDS, the
// wavefronts' largest numbers of a row (largest_in), there when this returns. meanwhile(): called when the loads are under way, which come back in their order.
template <int WAVES>
__device__ __forceinline__ uint32_t largest_in(const uint32_t (&largest)[WAVES])
{
    uint32_t v = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = max(v, largest[w]);
    return v;
}
template <bool TWO, int WAVES, typename F>
__device__ __forceinline__ void pack_local(const void *X, int64_t ld_x, int64_t K, int rows, int steps, int64_t pitch, char *local, uint32_t (&largest)[kLocalRows][WAVES],
                                           const F &meanwhile)
{
    typedef std::conditional_t<TWO, float, uint16_t> Number;
    constexpr int EIGHTS = TWO ? 4 : 8, HELD = (kLocal / 8 / 3 + EIGHTS + 16 * WAVES - 1) / (16 * WAVES);        // eights of a step; of a lane at most: three rows, a wavefront in four each
    static_assert(kLocalRows == 4 && HELD * 64 * WAVES >= kLocal / 8 + EIGHTS, "");
    const int each = steps * EIGHTS, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), sharing = rows == 1 ? WAVES : rows == 2 ? WAVES / 2 : WAVES / 4;
    const int row = wave / sharing, first = wave % sharing * 64 + (int)(threadIdx.x & 63);
    float v[HELD][8];
    if (row < rows) {
#pragma unroll
        for (int u = 0; u < HELD; ++u)
            if (first + u * sharing * 64 < each) rows8::load(static_cast<const Number *>(X) + row * ld_x, 8 * (first + u * sharing * 64), K, v[u]);
    }
    __builtin_amdgcn_sched_barrier(0);
    meanwhile();
    __builtin_amdgcn_sched_barrier(0);
    if (row < rows) {
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < HELD; ++u)
            if (first + u * sharing * 64 < each)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[u][e]) & 0x7fffffffu);
#pragma unroll
        for (int o = 32; o > 0; o /= 2) most = max(most, (uint32_t)__shfl_xor((int)most, o));
        for (int w = wave % sharing; w < WAVES; w += sharing) largest[row][w] = most;
    }
    __syncthreads();
    if (row < rows) {
        const int shift = shift_of(largest_in(largest[row]));
#pragma unroll
        for (int u = 0; u < HELD; ++u)
            if (first + u * sharing * 64 < each) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = ldexpf(v[u][e], shift);
                plane::store_terms<TWO>(local + row * pitch, 8 * (first + u * sharing * 64), plane::terms_of<TWO>(v[u]));
            }
    }
    __syncthreads();
}
struct FewJob {
    const char *x, *w, *a;              // packed
    const void *X;                      // LOCAL: as they are, ld_x numbers apart
    int64_t ld_x, K;
    uint32_t *largest_x;                // LOCAL: written for join_kernel
    int64_t pitch, C;
    const int64_t *adapters;
    const int32_t *who;                 // in their place, if not null
    int64_t count;
    float *shared, *inner;              // [cuts][rows][ld], [cuts_inner][rows][ranks]
    int64_t ld;
    int rows, ranks, rank_blocks, slots, steps, cuts, per_cut, cuts_inner, per_cut_inner;
    unsigned inner_groups;
};
template <bool TWO, int BM, int NB, bool LOCAL>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(FewJob job)
{
    static_assert(!LOCAL || NB == 1, "");
    __shared__ float part[kFewWaves][BM * NB * 4][64];
    __shared__ __attribute__((aligned(16))) char local[LOCAL ? local_bytes(TWO) : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
    const int64_t pitch_x = LOCAL ? job.steps * kStepBytes + kLocalPad : job.pitch;
    const char *rows_x = LOCAL ? local : job.x;
    if constexpr (LOCAL) {
        __shared__ uint32_t largest[kLocalRows][kFewWaves];
        pack_local<TWO>(job.X, job.ld_x, job.K, job.rows, job.steps, pitch_x, local, largest, [] {});
        if (blockIdx.x == 0 && (int)threadIdx.x < job.rows) job.largest_x[threadIdx.x] = largest_in(largest[threadIdx.x]);
    }
    if (blockIdx.x < job.inner_groups) {
        int id = blockIdx.x;
        const int cut = id % job.cuts_inner;
        id /= job.cuts_inner;
        const int slot = id % job.slots;
        id /= job.slots;
        const int block = id % job.rank_blocks, n = id / job.rank_blocks * 16 + col;
        const int mine = n >= job.rows ? kNone : job.who ? job.who[n] : who_of(job.adapters[n], job.count);
        const char *x = rows_x + (n < job.rows ? n : job.rows - 1) * pitch_x + 16 * quarter;
        const int last = std::min(job.steps, (cut + 1) * job.per_cut_inner);
        uint32_t left = (uint32_t)(__ballot(mine >= 0) & 0xffff);
        for (int number = 0; left != 0; ++number) {
            const int adapter = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
            const bool its = mine == adapter;
            left &= ~(uint32_t)(__ballot(its) & 0xffff);
            if (number % job.slots != slot) continue;
            const char *a = job.a + ((int64_t)adapter * job.ranks + 16 * block + col) * job.pitch + 16 * quarter;
            floatx4 acc[1][1] = {{{0.f, 0.f, 0.f, 0.f}}};
            multiply_steps<TWO, 1, 1, kFewAhead>({a}, {x}, cut * job.per_cut_inner + wave, kFewWaves, last, acc);
            __syncthreads();                // (what was read before has been)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][e][lane] = acc[0][0][e];
            __syncthreads();
            static_assert(kFewWaves == 4, "a wavefront for each element of a lane");
            if (its) {                      // element `wave` of every lane
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) sum += part[w][wave][lane];
                job.inner[((int64_t)cut * job.rows + n) * job.ranks + 16 * block + 4 * quarter + wave] = sum;
            }
        }
        return;
    }
    const unsigned id = blockIdx.x - job.inner_groups;
    const int cut = (int)(id % job.cuts), last = std::min(job.steps, (cut + 1) * job.per_cut);
    const int64_t c0 = (int64_t)(id / job.cuts) * (16 * BM);
    const char *w[BM], *x[NB];
#pragma unroll
    for (int m = 0; m < BM; ++m) w[m] = job.w + std::min<int64_t>(c0 + 16 * m + col, job.C - 1) * job.pitch + 16 * quarter;
#pragma unroll
    for (int n = 0; n < NB; ++n) x[n] = rows_x + std::min(16 * n + col, job.rows - 1) * pitch_x + 16 * quarter;
    floatx4 acc[BM][NB];
#pragma unroll
    for (int m = 0; m < BM; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    multiply_steps<TWO, BM, NB, kFewAhead>(w, x, cut * job.per_cut + wave, kFewWaves, last, acc);
#pragma unroll
    for (int m = 0; m < BM; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][(n * 4 + e) * BM + m][lane] = acc[m][n][e];
    __syncthreads();
    // (n, class) places, classes fastest: 16 BM of them are together in memory
    for (int at = threadIdx.x; at < BM * NB * 4 * 64; at += 64 * kFewWaves) {
        const int c = at % (16 * BM), row = at / (16 * BM), m = c / 16, r = c % 16;
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) sum += part[v][((row / 16) * 4 + r % 4) * BM + m][16 * (r / 4) + row % 16];
        if (row < job.rows && c0 + c < job.C) job.shared[((int64_t)cut * job.rows + row) * job.ld + c0 + c] = sum;
    }
}

// The sums of the cuts, scaled, and B's part, by multiply-adds: a lane has a class, and goes through some of the rows. Bound by latency where rows are few (16 rows, 5003
// classes 6 us), by its reads and writes where not.
struct JoinJob {
    const float *shared, *inner;
    const uint32_t *largest_x, *largest_w, *largest_a;
    const float *scale;
    const int64_t *adapters;
    const int32_t *order, *who;         // of rows that are in another order; or both null
    int64_t count, C, ld_shared, ld;
    const void *B;
    float *out;
    int rows, rows_each, ranks, ranks_b, cuts, cuts_inner;
};
constexpr int kJoinThreads = 256;
template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(JoinJob job)
{
    __shared__ __attribute__((aligned(16))) float s[kMostRank];
    const int64_t c = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int first = blockIdx.y * job.rows_each, last = std::min(job.rows, first + job.rows_each);
    const int shift_w = c < job.C ? shift_of(job.largest_w[c]) : 0;
    for (int n = first; n < last; ++n) {
        const int adapter = job.who ? job.who[n] : who_of(job.adapters[n], job.count), shift_x = shift_of(job.largest_x[n]);
        float v = 0.f;
        if (c < job.C) {
#pragma unroll 4
            for (int p = 0; p < job.cuts; ++p) v += job.shared[((int64_t)p * job.rows + n) * job.ld_shared + c];
            v = ldexpf(v, -shift_x - shift_w);
        }
        if (adapter >= 0) {
            __syncthreads();                // (what was read before has been)
            for (int r = threadIdx.x; r < job.ranks; r += kJoinThreads) {
                float sum = 0.f;
#pragma unroll 8
                for (int p = 0; p < job.cuts_inner; ++p) sum += job.inner[((int64_t)p * job.rows + n) * job.ranks + r];
                s[r] = ldexpf(sum, -shift_x - shift_of(job.largest_a[(int64_t)adapter * job.ranks + r])) * job.scale[adapter];
            }
            __syncthreads();
            if (c < job.C) {
                float sum = 0.f;
                const int64_t row = ((int64_t)adapter * job.C + c) * job.ranks_b;
                if constexpr (BF16) {
                    for (int r = 0; r < job.ranks_b; r += 8) {
                        float b[8];
                        rows8::load(static_cast<const uint16_t *>(job.B) + row + r, 0, 8, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum = fmaf(s[r + e], b[e], sum);
                    }
                } else {
                    for (int r = 0; r < job.ranks_b; r += 4) {
                        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(job.B) + row + r);
                        sum = fmaf(s[r], b.x, sum);
                        sum = fmaf(s[r + 1], b.y, sum);
                        sum = fmaf(s[r + 2], b.z, sum);
                        sum = fmaf(s[r + 3], b.w, sum);
                    }
                }
                v += sum;
            }
        }
        if (c < job.C) job.out[(int64_t)(job.order ? job.order[n] : n) * job.ld + c] = adapter == kUnknown ? NAN : v;
    }
}

// One request, up to 16 ranks, and so few classes and columns that latency is all that counts: everything in one launch. A workgroup has 16 classes, packs the row and forms
// its adapter's inner products for itself, its wavefronts sharing the steps. All that it reads is under way before the row is packed. 1 x 1025, 1000 classes, rank 8: float32
// 7.8 us a call (few_kernel and join_kernel 9.6; replayed in a graph 7.9 and 8.5), bfloat16 8.0 (9.6; 8.0 and 8.2).
constexpr int kOneWaves = 16, kOneSteps = 3, kCus = 256;         // steps of a wavefront at most
struct OneJob {
    const char *w, *a;                  // packed
    const void *X, *B;
    int64_t K, pitch, C, count;
    const int64_t *adapters;
    const uint32_t *largest_w, *largest_a;
    const float *scale;
    float *out;
    int ranks_b, steps;
};
template <bool TWO>
__global__ __launch_bounds__(64 * kOneWaves) void one_kernel(OneJob job)
{
    constexpr int SIXTEEN = TWO ? 4 : 2;
    __shared__ float part[kOneWaves][32];                   // shared products of 16 classes, inner ones of 16 ranks
    __shared__ __attribute__((aligned(16))) char local[local_bytes(TWO)];
    __shared__ uint32_t largest[kLocalRows][kOneWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
    const int64_t c0 = (int64_t)blockIdx.x * 16, c = std::min(c0 + col, job.C - 1);
    halfx8 f[kOneSteps][2][2];
    auto load = [&](int m, const char *row) {
#pragma unroll
        for (int u = 0; u < kOneSteps; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                f[u][m][h] = *reinterpret_cast<const halfx8 *>(row + (int64_t)std::min(wave + u * kOneWaves, job.steps - 1) * kStepBytes + 16 * quarter + 64 * h);
    };
    // the first wavefront writes the results: class l % 16 and rank l % 16 in all four quarters
    int adapter = kNone, shift = 0;
    uint4 b[SIXTEEN];
    float scale = 0.f;
    pack_local<TWO>(job.X, 0, job.K, 1, job.steps, 0, local, largest, [&] {
        load(0, job.w + c * job.pitch);
        adapter = who_of(job.adapters[0], job.count);
        load(1, adapter >= 0 ? job.a + ((int64_t)adapter * 16 + col) * job.pitch : job.w + c * job.pitch);
        if (wave != 0) return;
        shift = -shift_of(lane & 16 ? (adapter >= 0 ? job.largest_a[(int64_t)adapter * 16 + col] : 0u) : job.largest_w[c]);
        if (adapter < 0) return;
        scale = job.scale[adapter];
        const char *b_row = static_cast<const char *>(job.B) + ((int64_t)adapter * job.C + c) * job.ranks_b * (TWO ? 4 : 2);
#pragma unroll
        for (int i = 0; i < SIXTEEN; ++i) b[i] = i * 16 < job.ranks_b * (TWO ? 4 : 2) ? *reinterpret_cast<const uint4 *>(b_row + 16 * i) : make_uint4(0, 0, 0, 0);
    });
    floatx4 acc[2][1] = {{{0.f, 0.f, 0.f, 0.f}}, {{0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
    for (int u = 0; u < kOneSteps; ++u) {
        const int step = wave + u * kOneWaves;
        if (step >= job.steps) break;
        halfx8 x[1][2];                                     // (the row, for all columns of the product)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[0][h] = *reinterpret_cast<const halfx8 *>(local + step * kStepBytes + 64 * h + 16 * quarter);
        multiply_step<TWO>(f[u], x, acc);
    }
    if (col == 0) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][16 * m + 4 * quarter + e] = acc[m][0][e];
    }
    __syncthreads();
    if (wave != 0) return;
    float sum = 0.f;                                        // of half the wavefronts: lanes 0 to 15 and 32 to 47 a class, the others a rank
#pragma unroll
    for (int v = 0; v < kOneWaves / 2; ++v) sum += part[lane / 32 * (kOneWaves / 2) + v][lane % 32];
    sum = ldexpf(sum + __shfl_xor(sum, 32), shift - shift_of(largest_in(largest[0])));
    if (adapter >= 0) {
        const float inner = sum * scale;
        float added = 0.f;
#pragma unroll
        for (int r0 = 0; r0 < 16; r0 += 8) {
            float v[8];
            if constexpr (TWO) __builtin_memcpy(v, b + r0 / 4, 32);
            else rows8::load(reinterpret_cast<const uint16_t *>(b + r0 / 8), 0, 8, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) added = fmaf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inner), 16 + r0 + e)), v[e], added);
        }
        sum += added;
    }
    if (lane < 16 && c0 + col < job.C) job.out[c0 + col] = adapter == kUnknown ? NAN : sum;
}

// Inner products from the sums of their cuts, scaled, as three terms for Adapted.
struct FinishJob {
    const float *inner;
    const uint32_t *largest_x, *largest_a;
    const float *scale;
    const int32_t *who;
    uint16_t *terms;
    int rows, ranks, cuts;
};
__global__ __launch_bounds__(256) void finish_kernel(FinishJob job)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int n = (int)(at / job.ranks), r = (int)(at % job.ranks);
    if (n >= job.rows || job.who[n] < 0) return;
    const int adapter = job.who[n];
    float sum = 0.f;
#pragma unroll 8
    for (int p = 0; p < job.cuts; ++p) sum += job.inner[((int64_t)p * job.rows + n) * job.ranks + r];
    const Terms3 t = terms3(ldexpf(sum, -shift_of(job.largest_x[n]) - shift_of(job.largest_a[(int64_t)adapter * job.ranks + r])) * job.scale[adapter]);
#pragma unroll
    for (int i = 0; i < 3; ++i) job.terms[((int64_t)n * 3 + i) * job.ranks + r] = t.v[i];
}

// The shared product's epilogue where the sum over columns is cut: the accumulators as they are, for join_kernel.
struct Parts {
    float *shared;              // [cuts][rows][ld]
    int64_t ld, C;
    int rows;

    template <typename T>
    __device__ __forceinline__ void operator()(T &t) const
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
            const int64_t n = t.j0 + 32 * b + col;
            if (n >= rows) return;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t i = first + 8 * q + 4 * half;
                if (i < C)              // (ld is a multiple of four: numbers beyond C are nobody's)
                    *reinterpret_cast<float4 *>(shared + ((int64_t)t.cut * rows + n) * ld + i) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
            }
        });
    }
};

// The shared product's epilogue, which adds to the accumulators the sums over ranks of a block of 32 classes and 32 rows, for one adapter of the rows after the
// other, and keeps the sums of the rows that have it. v_mfma_f32_32x32x16_bf16: lane l holds eight ranks of class (row) l % 32. B enters as it is (bfloat16) or as
// three terms, of whose products with those of the inner products the three smallest are left out (below 2^-21 of the product). 32-bit matrix instructions took 240 us
// instead of 50 to 80 of 8192 x 2049, 32768 classes, rank 32, whose product takes 1170 us without adapters (0.94 PFLOP/s; a library product of these matrices 1078).
template <bool BF16>
struct Adapted {
    const uint32_t *largest_w, *largest_x;
    int64_t C;
    int rows;                   // of this launch, in the order of their adapters
    const int32_t *order, *who;
    const uint16_t *terms;      // [rows][3][ranks], of finish_kernel
    const void *B;
    int ranks, ranks_b;
    float *out;
    int64_t ld;

    static constexpr int TERMS = BF16 ? 1 : 3, WORDS = BF16 ? 4 : 8;
    // Eight ranks of a class of an adapter, as they lie in memory.
    __device__ __forceinline__ void load_b(int64_t row, int r, uint32_t (&v)[WORDS]) const
    {
        const char *from = static_cast<const char *>(B) + (row * ranks_b + r) * (BF16 ? 2 : 4);
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
            const uint4 w = r + (BF16 ? 0 : i) < ranks_b ? *reinterpret_cast<const uint4 *>(from + 4 * i) : make_uint4(0, 0, 0, 0);
            v[i] = w.x;
            v[i + 1] = w.y;
            v[i + 2] = w.z;
            v[i + 3] = w.w;
        }
    }
    static __device__ __forceinline__ void three_terms(const float (&v)[8], bf16x8 (&f)[3])
    {
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Terms3 lo = terms3(v[2 * i]), hi = terms3(v[2 * i + 1]);
#pragma unroll
            for (int k = 0; k < 3; ++k) w[k][i] = lo.v[k] | (uint32_t)hi.v[k] << 16;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) f[k] = __builtin_bit_cast(bf16x8, make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]));
    }
    static __device__ __forceinline__ void terms_of_b(const uint32_t (&v)[WORDS], bf16x8 (&f)[TERMS])
    {
        if constexpr (BF16) {
            f[0] = __builtin_bit_cast(bf16x8, make_uint4(v[0], v[1], v[2], v[3]));
        } else {
            float x[8];
            __builtin_memcpy(x, v, 32);
            three_terms(x, f);
        }
    }
    template <typename T>
    __device__ __forceinline__ void operator()(T &t) const
    {
        struct __attribute__((packed, aligned(4))) Float4u { float x, y, z, w; };
        constexpr int CLASSES = T::ROWS + (T::HAS_EXTRA ? 32 : 0), BN = T::BN, BM = T::BM;
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        const int64_t c0 = t.tile_i * T::ROWS;
        int *powers = reinterpret_cast<int *>(t.lds);
        __syncthreads();
        for (int i = threadIdx.x; i < CLASSES; i += blockDim.x) powers[i] = -shift_of(c0 + i < C ? largest_w[c0 + i] : 0);
        __syncthreads();
        int mine[BN], shift[BN];
#pragma unroll
        for (int b = 0; b < BN; ++b) {
            const int64_t n = t.j0 + 32 * b + col;
            mine[b] = n < rows ? who[n] : kNone;
            shift[b] = n < rows ? shift_of(largest_x[n]) : 0;
        }
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int4 p = *reinterpret_cast<const int4 *>(powers + (int)(first - c0) + 8 * q + 4 * half);
                acc[4 * q] = ldexpf(acc[4 * q], p.x - shift[b]);
                acc[4 * q + 1] = ldexpf(acc[4 * q + 1], p.y - shift[b]);
                acc[4 * q + 2] = ldexpf(acc[4 * q + 2], p.z - shift[b]);
                acc[4 * q + 3] = ldexpf(acc[4 * q + 3], p.w - shift[b]);
            }
        });
#pragma unroll
        for (int b = 0; b < BN; ++b) {
            const uint64_t with = __ballot(mine[b] >= 0);
            if (with == 0) continue;
            const int64_t n = std::min<int64_t>(t.j0 + 32 * b + col, rows - 1);
            const uint16_t *from = terms + n * 3 * ranks + 8 * half;
            for (int r0 = 0; r0 < ranks; r0 += 16) {
                bf16x8 s[3];
#pragma unroll
                for (int i = 0; i < 3; ++i) s[i] = *reinterpret_cast<const bf16x8 *>(from + i * ranks + r0);
                // (in small tiles the next adapter's part of B is under way while the present one's is multiplied: 100 x 257, 50000 classes, 30 adapters 85 -> 63 us;
                // in large ones, of which more rows are of one adapter, its registers are not there)
                constexpr bool AHEAD = BM <= 2;
                constexpr int GROUP = T::HAS_EXTRA || !BF16 ? 1 : 4;            // blocks of large tiles whose parts of B are loaded together, where registers allow
                uint32_t next[BM][WORDS];
                auto load = [&](uint64_t of, int a, int64_t first) __attribute__((always_inline)) {
                    const int64_t adapter = (int64_t)__builtin_amdgcn_readlane(mine[b], __builtin_ctzll(of)) * C;
                    load_b(adapter + std::min(first + col, C - 1), r0 + 8 * half, next[a]);
                };
                if constexpr (AHEAD) {
#pragma unroll
                    for (int a = 0; a < BM; ++a) load(with, a, t.i0 + 32 * a);
                }
                for (uint64_t left = with; left != 0;) {
                    const uint64_t now = left;
                    const bool its = mine[b] == __builtin_amdgcn_readlane(mine[b], __builtin_ctzll(now));
                    left &= ~__ballot(its);
                    bf16x8 f[BM][TERMS];
                    if constexpr (AHEAD) {
#pragma unroll
                        for (int a = 0; a < BM; ++a) terms_of_b(next[a], f[a]);
                        if (left != 0) {
#pragma unroll
                            for (int a = 0; a < BM; ++a) load(left, a, t.i0 + 32 * a);
                        }
                    }
                    auto add = [&](auto &acc, const bf16x8 (&f)[TERMS]) __attribute__((always_inline)) {
                        floatx16 sum = {};
                        if constexpr (!BF16) {
                            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[2], s[0], sum, 0, 0, 0);
                            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1], s[1], sum, 0, 0, 0);
                        }
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], s[2], sum, 0, 0, 0);
                        if constexpr (!BF16) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1], s[0], sum, 0, 0, 0);
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], s[1], sum, 0, 0, 0);
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], s[0], sum, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[e] += its ? sum[e] : 0.f;
                    };
#pragma unroll
                    for (int a = 0; a < BM; ++a) {
                        if constexpr (!AHEAD) {
                            if (GROUP == 1 && t.i0 + 32 * a >= C) continue;
                            if (a % GROUP == 0) {
#pragma unroll
                                for (int i = a; i < a + GROUP; ++i) load(now, i, t.i0 + 32 * i);
                            }
                            terms_of_b(next[a], f[a]);
                        }
                        add(t.acc[a][b], f[a]);
                    }
                    if constexpr (T::HAS_EXTRA) {
                        static_assert(!AHEAD, "");
                        if (b == t.wave_i) {
                            load(now, 0, t.extra_i);
                            terms_of_b(next[0], f[0]);
                            add(t.extra, f[0]);
                        }
                    }
                }
            }
        }
        t.each_block([&](auto &acc, int64_t first, int b) __attribute__((always_inline)) {
            const int64_t n = t.j0 + 32 * b + col;
            if (n >= rows) return;
            float *row = out + (int64_t)order[n] * ld;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t i = first + 8 * q + 4 * half;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mine[b] == kUnknown ? NAN : acc[4 * q + e];
                if (i + 3 < C) {
                    *reinterpret_cast<Float4u *>(row + i) = {v[0], v[1], v[2], v[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < C) row[i + e] = v[e];
                }
            }
        });
    }
};

// How a number of rows is worked on. Sums over columns may be cut into parts, which join_kernel adds up, so that there are workgroups enough: those of few rows
// straight from their packed form, those of more rows as tiles.
struct Way { bool split; int edge, cuts; };             // edge of tiles, or 0: straight
struct Plan {
    Way way;
    int blocks, wide;                                   // straight: groups of 16 rows of X, of W a workgroup
    int per_cut, slots, cuts_inner, per_cut_inner;
    int64_t groups, inner_groups, ld;
    size_t x, largest_x, order, who, inner, shared, terms, bytes;       // (the last two: of a sum that is cut, and of one that is not)
};
int blocks_of(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : kFewBlocks; }
int wide_of(int64_t C) { return C >= 16 * kWide ? kWide : 1; }
Plan plan_of(const rfsf_adapters_shape &s, const Layout &z, int64_t rows, const Way &way)
{
    Plan f;
    const int64_t steps = plane_steps(s.K, !s.bf16);
    auto cut = [&](int64_t wanted, int *cuts_, int *per_cut) {
        const int64_t most = std::max<int64_t>(1, std::min(steps / (kFewAhead * kFewWaves), wanted));
        *per_cut = (int)((steps + most - 1) / most);
        *cuts_ = (int)((steps + *per_cut - 1) / *per_cut);
    };
    f.way = way;
    f.blocks = f.wide = 0;
    f.groups = 0;
    if (way.edge == 0) {
        f.blocks = blocks_of(rows);
        f.wide = wide_of(s.C);
        f.groups = (s.C + 16 * f.wide - 1) / (16 * f.wide);
        cut(kFewGroups / f.groups, &f.way.cuts, &f.per_cut);
        f.groups *= f.way.cuts;
    } else {
        f.per_cut = (int)((steps + way.cuts - 1) / way.cuts);
        f.way.cuts = (int)((steps + f.per_cut - 1) / f.per_cut);
    }
    // slots for the adapters that a tile of 16 rows has on average, or for all of them where that makes few workgroups; those without an adapter end at once
    const int64_t tiles = (rows + 15) / 16 * (z.ranks / 16), most = std::min<int64_t>(16, std::min(s.count, rows));
    const int64_t average = way.edge == 0 ? most : std::min(most, 16 * std::min(s.count, rows) / rows + 1);
    f.slots = (int)average;
    cut(kFewGroups / (tiles * average), &f.cuts_inner, &f.per_cut_inner);
    f.inner_groups = tiles * f.slots * f.cuts_inner;
    f.ld = (s.C + 3) / 4 * 4;
    f.x = 0;
    f.largest_x = f.x + up((size_t)rows * z.pitch);
    f.order = f.largest_x + up((size_t)rows * 4);
    f.who = f.order + up((size_t)rows * 4);
    f.inner = f.who + up((size_t)rows * 4);
    f.shared = f.inner + up((size_t)f.cuts_inner * rows * z.ranks * 4);
    f.terms = f.shared;
    f.bytes = f.shared + up(way.split ? (size_t)f.way.cuts * rows * f.ld * 4 : (size_t)rows * 3 * z.ranks * 2) + 256;
    return f;
}

// The way of a number of rows, by estimates of its time in us: straight, bound by what the L2s deliver to the CUs (rows of W and X); tiles with B's part in their
// epilogue, which costs them some us each, the more the more adapters the rows of a block have; tiles whose sums are cut where they would not fill the CUs; and
// join_kernel, bound by its reads and writes. Of the 160 calls of 8 to 1000 rows that the constants were fitted to the choice takes at most 1.25 times what the best way takes,
// more than 1.1 times in 5; of 300 others at most 1.17, more than 1.1 in 3 (profiles/adapters_ways.txt).
// (Straight, tiles, cut tiles, us, float32: 20 x 5121, 5003 classes, 50 adapters of rank 16 39, 67, 37; 64 rows 59, 71, 41; 330 rows -, 95, 115; 64 x 1025, 1000
// classes 17, 27, 18; 64 x 1025, 30000 classes 74, 42, 57; 180 x 2049, 2000 classes, 100 adapters of rank 32 -, 58, 41; bfloat16: 20 x 257, 50000 classes 28, 34, 34.)
Way way_of(const rfsf_adapters_shape &s, const Layout &z, int64_t rows)
{
    const int64_t steps = plane_steps(s.K, !s.bf16);
    auto join = [&](int cuts) { return (double)rows * (double)s.C * (4.0 * cuts + 4.0 + (s.bf16 ? 2 : 4) * z.ranks_b) / 2.8e6; };
    Way best = {false, 0, 0};
    double least = 0.0;
    const double base = rows <= kPlaceRows && s.K <= kPlaceColumns ? 14.0 : 18.0;
    auto consider = [&](bool split, int edge, int cuts, double time) {
        if (best.cuts == 0 || time < least) {
            best = {split, edge, cuts};
            least = time;
        }
    };
    if (rows <= kFewRows) {
        const Plan f = plan_of(s, z, rows, {true, 0, 0});
        const int cuts = f.way.cuts;
        const double moved = ((double)f.groups / cuts * 16.0 * (f.wide + f.blocks) + (double)f.inner_groups / f.cuts_inner * 32.0) * (double)steps * kStepBytes;
        consider(true, 0, cuts, (f.blocks == 1 ? 8.0 : 11.0) + moved / (f.blocks == 1 ? 9.0e6 : f.blocks == 2 ? 8.0e6 : 7.0e6) + join(cuts));
    }
    // (adapters that the 32 rows of a block have)
    const double runs = std::min(32.0, 1.0 + 32.0 * (double)std::min(s.count, rows) / (double)rows), epilogue = (0.3 + 0.07 * runs) * (z.ranks / 16);
    for (const PlaneWay &way : kPlaneWays) {
        const double tiles = (double)plane_tiles(s.C, rows, way.edge);
        consider(false, way.edge, 1, base + 3.0 + plane_step_time(way, tiles) * (double)steps + epilogue * (way.edge == 256 ? 18.0 : way.edge == 128 ? 9.0 : 4.0) * std::max(1.0, tiles / way.slots));
        for (int cuts : {2, 3, 4, 5, 6, 8, 10, 12, 16})
            if (steps / cuts >= 8) consider(true, way.edge, cuts, base + plane_step_time(way, tiles * cuts) * (double)((steps + cuts - 1) / cuts) + join(cuts));
    }
    return best;
}
Plan plan_of(const rfsf_adapters_shape &s, const Layout &z, int64_t rows) { return plan_of(s, z, rows, way_of(s, z, rows)); }

// Whether one_kernel works on a row that fits into LDS: as long as every workgroup has a CU to itself (1 x 1025, 5003 classes, float32 15 us instead of 11) and every wavefront
// has all of its steps' loads under way at once.
bool one_launch(const rfsf_adapters_shape &s, const Layout &z, int64_t rows)
{
    return rows == 1 && z.ranks == 16 && s.C <= 16 * kCus && plane_steps(s.K, !s.bf16) <= kOneWaves * kOneSteps;
}

// (f: of as many rows or more)
hipError_t launch_rows(const Plan &f, const rfsf_adapters_shape &s, const Layout &z, const char *lay, const void *X, int64_t rows, int64_t ld_x, const int64_t *adapters,
                       float *out, int64_t ld_out, char *ws, hipStream_t stream)
{
    const bool bf16 = s.bf16 != 0, straight = f.way.edge == 0;
    const int64_t steps = plane_steps(s.K, !bf16);
    uint32_t *largest_x = reinterpret_cast<uint32_t *>(ws + f.largest_x);
    float *shared = reinterpret_cast<float *>(ws + f.shared), *inner = reinterpret_cast<float *>(ws + f.inner);
    const uint32_t *largest_w = reinterpret_cast<const uint32_t *>(lay + z.largest_w), *largest_a = reinterpret_cast<const uint32_t *>(lay + z.largest_a);
    const float *scale = reinterpret_cast<const float *>(lay + z.scale);
    int32_t *order = nullptr, *who = nullptr;
    bool packed = straight && rows <= kLocalRows && f.blocks == 1 && rows * s.K <= kLocal;
    const bool local = packed;
    if (local && one_launch(s, z, rows)) {
        const OneJob job = {lay + z.w, lay + z.a, X, lay + z.b, s.K, z.pitch, s.C, s.count, adapters, largest_w, largest_a, scale, out, z.ranks_b, (int)steps};
        const dim3 grid((unsigned)((s.C + 15) / 16));
        if (bf16) one_kernel<false><<<grid, 64 * kOneWaves, 0, stream>>>(job);
        else one_kernel<true><<<grid, 64 * kOneWaves, 0, stream>>>(job);
        return hipGetLastError();
    }
    if (!straight) {
        order = reinterpret_cast<int32_t *>(ws + f.order);
        who = reinterpret_cast<int32_t *>(ws + f.who);
    }
    if (!straight && rows <= kPlaceRows && s.K <= kPlaceColumns) {
        const PlaceJob job = {X, ld_x, s.K, s.count, adapters, (int)rows, ws + f.x, z.pitch, largest_x, order, who};
        auto launch = [&](auto kernel) { kernel<<<dim3((unsigned)rows), kPlaceThreads, 0, stream>>>(job); };
        if (s.K <= 8 * kPlaceThreads) bf16 ? launch(place_kernel<false, 1>) : launch(place_kernel<true, 1>);
        else bf16 ? launch(place_kernel<false, 3>) : launch(place_kernel<true, 3>);
        RFSF_TRY(hipGetLastError());
        packed = true;
    } else if (!straight) {
        order_kernel<<<dim3((unsigned)((rows + kOrderRows - 1) / kOrderRows)), 64 * kOrderWaves, 0, stream>>>(adapters, (int)rows, s.count, order, who);
        RFSF_TRY(hipGetLastError());
    }
    if (!packed) RFSF_TRY(pack(PackJob{X, rows, s.K, ld_x, nullptr, largest_x, ws + f.x, nullptr, z.pitch, 0, order}, bf16, stream));
    const FewJob job = {ws + f.x, lay + z.w, lay + z.a, X, ld_x, s.K, largest_x, z.pitch, s.C, adapters, who, s.count, shared, inner, f.ld, (int)rows, z.ranks, z.ranks / 16, f.slots, (int)steps,
                        f.way.cuts, f.per_cut, f.cuts_inner, f.per_cut_inner, (unsigned)f.inner_groups};
    auto launch = [&](auto kernel) { kernel<<<dim3((unsigned)(f.groups + f.inner_groups)), 64 * kFewWaves, 0, stream>>>(job); };
    auto launch_blocks = [&](auto two) {
        constexpr bool TWO = decltype(two)::value;
        auto launch_wide = [&](auto wide) {
            constexpr int BM = decltype(wide)::value;
            if (f.blocks <= 1) local ? launch(few_kernel<TWO, BM, 1, true>) : launch(few_kernel<TWO, BM, 1, false>);
            else f.blocks == 2 ? launch(few_kernel<TWO, BM, 2, false>) : launch(few_kernel<TWO, BM, 4, false>);
        };
        if (f.wide == kWide) launch_wide(std::integral_constant<int, kWide>());
        else launch_wide(std::integral_constant<int, 1>());
    };
    if (bf16) launch_blocks(std::false_type());
    else launch_blocks(std::true_type());
    RFSF_TRY(hipGetLastError());
    const Planes w_rows = {lay + z.w, z.pitch, s.C}, x_rows = {ws + f.x, z.pitch, rows};
    if (!f.way.split) {
        uint16_t *terms = reinterpret_cast<uint16_t *>(ws + f.terms);
        finish_kernel<<<dim3((unsigned)((rows * z.ranks + 255) / 256)), 256, 0, stream>>>(FinishJob{inner, largest_x, largest_a, scale, who, terms, (int)rows, z.ranks,
                                                                                                   f.cuts_inner});
        RFSF_TRY(hipGetLastError());
        auto product = [&](auto is_bf16) {
            constexpr bool BF16 = decltype(is_bf16)::value;
            const Adapted<BF16> epilogue = {largest_w, largest_x, s.C, (int)rows, order, who, terms, lay + z.b, z.ranks, z.ranks_b, out, ld_out};
            return launch_plane_product<BF16 ? kHalf : kHalfTwo>(w_rows, x_rows, steps, f.way.edge, epilogue, stream);
        };
        return bf16 ? product(std::true_type()) : product(std::false_type());
    }
    if (!straight) {
        const Product<Parts> p = {w_rows, x_rows, steps, {shared, f.ld, s.C, (int)rows}, f.per_cut};
        RFSF_TRY(bf16 ? launch_plane_products<kHalf>(&p, 1, f.way.edge, stream) : launch_plane_products<kHalfTwo>(&p, 1, f.way.edge, stream));
    }
    const int64_t across = (s.C + kJoinThreads - 1) / kJoinThreads;
    const int each = (int)std::max<int64_t>(1, rows * across / (4 * kFewGroups));
    const JoinJob join = {shared, inner, largest_x, largest_w, largest_a, scale, adapters, order, who, s.count, s.C, f.ld, ld_out, lay + z.b, out, (int)rows, each, z.ranks,
                          z.ranks_b, f.way.cuts, f.cuts_inner};
    const dim3 grid((unsigned)across, (unsigned)((rows + each - 1) / each));
    if (bf16) join_kernel<true><<<grid, kJoinThreads, 0, stream>>>(join);
    else join_kernel<false><<<grid, kJoinThreads, 0, stream>>>(join);
    return hipGetLastError();
}

}  // namespace

size_t adapters_layout_bytes(const rfsf_adapters_shape &s) { return layout_of(s).bytes; }

void adapted_scores_bytes(const rfsf_adapters_shape &s, int64_t N, size_t *recommended, size_t *minimum)
{
    const Layout z = layout_of(s);
    // (a smaller workspace means fewer rows at a time, which may need more than more rows do: parts of few rows are kept apart)
    *minimum = plan_of(s, z, 1).bytes;
    *recommended = std::max(*minimum, plan_of(s, z, std::min<int64_t>(std::max<int64_t>(N, 1), kMostRows)).bytes);
}

hipError_t launch_adapters_weights(const rfsf_adapters_shape &s, const void *W, int64_t ld_w, void *layout, hipStream_t stream)
{
    const Layout z = layout_of(s);
    char *to = static_cast<char *>(layout);
    return pack(PackJob{W, s.C, s.K, ld_w, nullptr, reinterpret_cast<uint32_t *>(to + z.largest_w), to + z.w, nullptr, z.pitch, 0}, s.bf16 != 0, stream);
}

hipError_t launch_adapters_set(const rfsf_adapters_shape &s, int64_t index, const void *A, int64_t ld_a, const void *B, int64_t ld_b, float scale, void *layout,
                               hipStream_t stream)
{
    const Layout z = layout_of(s);
    char *to = static_cast<char *>(layout), *a = to + z.a + (size_t)index * z.ranks * z.pitch;
    uint32_t *largest = reinterpret_cast<uint32_t *>(to + z.largest_a) + index * z.ranks;
    RFSF_TRY(pack(PackJob{A, s.rank, s.K, ld_a, nullptr, largest, a, nullptr, z.pitch, 0}, s.bf16 != 0, stream));
    const int rest = z.ranks - (int)s.rank;
    const size_t at_b = (size_t)index * s.C * z.ranks_b;
    const dim3 grid((unsigned)std::min<int64_t>(1024, (s.C * z.ranks_b + 255) / 256));
    float *scale_at = reinterpret_cast<float *>(to + z.scale) + index;
    auto launch = [&](auto *b, const auto *from) {
        set_kernel<<<grid, 256, 0, stream>>>(from, ld_b, s.C, (int)s.rank, z.ranks_b, b + at_b, a + s.rank * z.pitch, rest * z.pitch, largest + s.rank, rest, scale_at, scale);
    };
    if (s.bf16) launch(reinterpret_cast<uint16_t *>(to + z.b), static_cast<const uint16_t *>(B));
    else launch(reinterpret_cast<float *>(to + z.b), static_cast<const float *>(B));
    return hipGetLastError();
}

hipError_t launch_adapted_scores(const rfsf_adapters_shape &s, const void *layout, const void *X, int64_t N, int64_t ld_x, const int64_t *adapters, float *out,
                                 int64_t ld_out, void *workspace, size_t bytes, hipStream_t stream)
{
    const Layout z = layout_of(s);
    int64_t most = std::min<int64_t>(N, kMostRows);
    Plan plan = plan_of(s, z, most);
    while (most > 1 && plan.bytes > bytes) {
        most = (most + 1) / 2;
        plan = plan_of(s, z, most);
    }
    const size_t mis = (size_t)(reinterpret_cast<uintptr_t>(workspace) % 256);
    char *ws = static_cast<char *>(workspace) + (mis ? 256 - mis : 0);
    for (int64_t n0 = 0; n0 < N; n0 += most) {
        const int64_t rows = std::min(N - n0, most);
        if (rows < most) {          // the last ones, which may need more room than more rows do: their way is taken if there is that
            const Plan last = plan_of(s, z, rows);
            if (last.bytes <= bytes) plan = last;
        }
        RFSF_TRY(launch_rows(plan, s, z, static_cast<const char *>(layout), static_cast<const char *>(X) + (size_t)n0 * ld_x * (s.bf16 ? 2 : 4), rows, ld_x, adapters + n0,
                             out + n0 * ld_out, ld_out, ws, stream));
    }
    return hipSuccess;
}

}  // namespace rfsf
