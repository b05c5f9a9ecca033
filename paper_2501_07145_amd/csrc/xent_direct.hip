// The softmax cross entropy of few rows, classes or columns, straight from the matrices as they lie in memory (softmax_xent.hip packs
// them first, which pays where its products are large). What bounds it is reading Phi and W and writing the gradients, and the
// number of launches: one for up to 16 classes and 2048 columns, two for up to 64 classes, three for more, and one more where a gradient's sum is cut.
//
// Products: 32-bit numbers as three terms of bfloat16 (8 significand bits each, 24 in all, with the range of 32-bit numbers), six
// products of pairs of terms, smallest first; bfloat16 operands as they are, G then as two terms. Sums in 32 bits. A tile's summed index is
// shared out among the wavefronts of a workgroup and their parts are added up in LDS; operands go from memory to registers.
// Gradients of up to 16 rows or 16 classes take no matrix instructions: one pass over the many of the two, in 32-bit multiply-adds.
#include "xent_direct.h"

#include <algorithm>
#include <type_traits>

namespace rfsf {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float number(float x) { return x; }
__device__ __forceinline__ float number(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ floatx16 mfma(const bf16x8 &a, const bf16x8 &b, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma(const bf16x8 &a, const bf16x8 &b, const floatx4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t round_pair(float a, float b)
{
    const floatx2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// Eight numbers as TERMS terms. The first one is cut off rather than rounded, so that the largest numbers stay finite.
template <int TERMS>
struct Split { bf16x8 t[TERMS]; };
template <int TERMS>
__device__ __forceinline__ Split<TERMS> split(const float (&x)[8])
{
    uint32_t w[TERMS][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
        w[0][i] = (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u);
        if constexpr (TERMS > 1) {
            a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
#pragma unroll
            for (int t = 1; t < TERMS; ++t) {
                w[t][i] = round_pair(a, b);
                a -= __uint_as_float(w[t][i] << 16);
                b -= __uint_as_float(w[t][i] & 0xffff0000u);
            }
        }
    }
    Split<TERMS> s;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) s.t[t] = __builtin_bit_cast(bf16x8, make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]));
    return s;
}
// c += a b, of all pairs of terms whose orders come to less than the larger number of terms, smallest first.
template <int TA, int TB, typename Acc>
__device__ __forceinline__ Acc multiply(const Split<TA> &a, const Split<TB> &b, Acc c)
{
    constexpr int MOST = (TA > TB ? TA : TB) - 1;
#pragma unroll
    for (int order = MOST; order >= 0; --order)
#pragma unroll
        for (int k = 0; k < TA; ++k)
            if (order - k >= 0 && order - k < TB) c = mfma(a.t[k], b.t[order - k < 0 ? 0 : order - k < TB ? order - k : TB - 1], c);
    return c;
}

// 16 of the 64 numbers of a row from k on: 16 bytes at a time, so that the four lanes that share a row read 64 bytes together.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Chunk { T v[16 / sizeof(T)]; };
template <typename T>
__device__ __forceinline__ void load16(const T *row, int64_t k, int quarter, int64_t K, bool there, float (&x)[16])
{
    constexpr int PER = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 16 / PER; ++j) {
        const int64_t at = k + 4 * PER * j + PER * quarter;
        if (at + PER <= K) {
            const Chunk<T> c = *reinterpret_cast<const Chunk<T> *>(row + at);
#pragma unroll
            for (int e = 0; e < PER; ++e) x[PER * j + e] = there ? number(c.v[e]) : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) x[PER * j + e] = there && at + e < K ? number(row[at + e]) : 0.f;
        }
    }
}

// Adds the wavefronts' parts of BM blocks up: block b is then whole in the registers of wavefront b (of its first ones).
template <int BM, int NW, int PER, typename Acc>
__device__ __forceinline__ Acc add_up(const Acc (&acc)[BM], float *shared, int wave, int lane)
{
#pragma unroll
    for (int a = 0; a < BM; ++a)
#pragma unroll
        for (int e = 0; e < PER; ++e) shared[((a * NW + wave) * PER + e) * 64 + lane] = acc[a][e];
    __syncthreads();
    Acc sum;
    const int block = wave < BM ? wave : 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s += shared[((block * NW + w) * PER + e) * 64 + lane];
        sum[e] = s;
    }
    return sum;
}

// Scores of 16 rows and 16 BM classes, in blocks of 16 x 16. FUSED (all classes in one tile): the softmax, the loss and G = weight
// (p - [c = y]) follow in registers; otherwise the scores are written. Wavefronts share out the columns, 64 at a time: lane l holds a
// quarter of row l % 16 of each block. Bound by reading Phi and by latency: 7494 x 1001, 10 classes, float32 11.6 us (2.6 TB/s), loss alone or before few_kernel.
constexpr int kRows = 16;
constexpr int64_t kCountedRows = 32768;          // of more, the rows that count are counted by a launch of its own, into kCountTiles numbers
constexpr int kCountTiles = 256;
template <typename T, int BM, int NW, bool FUSED>
__global__ __launch_bounds__(64 * NW) void scores_kernel(XentDirect job)
{
    constexpr int TERMS = sizeof(T) == 4 ? 3 : 1;
    static_assert(BM <= NW, "a wavefront for every block");
    __shared__ float shared[BM * NW * 4 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
    const int64_t n0 = (int64_t)blockIdx.x * kRows, c0 = (int64_t)blockIdx.y * (16 * BM), n = n0 + col;
    const bool row_there = n < job.N;
    const int64_t label = row_there ? job.labels[n] : -1;
    const bool there = label >= 0;
    const T *phi = static_cast<const T *>(job.Phi) + (row_there ? n : job.N - 1) * job.ld_phi;
    const T *w[BM];
#pragma unroll
    for (int a = 0; a < BM; ++a) w[a] = static_cast<const T *>(job.W) + std::min(c0 + 16 * a + col, job.C - 1) * job.ld_w;
    floatx4 acc[BM];
#pragma unroll
    for (int a = 0; a < BM; ++a) acc[a] = floatx4{0.f, 0.f, 0.f, 0.f};
    float xb[16], xa[BM][16];
    auto fetch = [&](int64_t k) {
        load16(phi, k, quarter, job.K, there, xb);
#pragma unroll
        for (int a = 0; a < BM; ++a) load16(w[a], k, quarter, job.K, true, xa[a]);
    };
    const int64_t begin = FUSED ? 0 : blockIdx.z * job.columns_per_cut, end = FUSED ? job.K : std::min(begin + job.columns_per_cut, job.K);
    int64_t k = begin + 64 * wave;
    if (k < end) fetch(k);
    while (k < end) {
        float b[2][8], a8[BM][2][8];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            b[e / 8][e % 8] = xb[e];
#pragma unroll
            for (int a = 0; a < BM; ++a) a8[a][e / 8][e % 8] = xa[a][e];
        }
        k += 64 * NW;
        if (k < end) fetch(k);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Split<TERMS> sb = split<TERMS>(b[u]);
#pragma unroll
            for (int a = 0; a < BM; ++a) acc[a] = multiply(split<TERMS>(a8[a][u]), sb, acc[a]);
        }
    }
    floatx4 sum = add_up<BM, NW, 4>(acc, shared, wave, lane);
    // rows that count, of each tile of rows
    if (blockIdx.y == 0 && blockIdx.z == 0 && wave == 0 && job.N <= kCountedRows) {
        const uint64_t counting = __ballot(there && quarter == 0);
        if (lane == 0) job.counts[blockIdx.x] = (uint32_t)__popcll(counting);
    }
    const int64_t first = c0 + 16 * wave + 4 * quarter;          // class of element e: first + e
    if constexpr (!FUSED) {
        if (wave < BM && row_there && first < job.C)
            *reinterpret_cast<float4 *>(job.scores + ((int64_t)blockIdx.z * job.N + n) * job.ld_scores + first) = make_float4(sum[0], sum[1], sum[2], sum[3]);
        if (!job.partial || wave >= BM) return;
        float top = -INFINITY, s = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e < job.C) top = fmaxf(top, sum[e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int e = 0; e < 4; ++e) s += first + e < job.C ? exp_of(sum[e] - from) : 0.f;
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (quarter == 0 && row_there) job.partial[((int64_t)blockIdx.y * BM + wave) * job.N + n] = make_float2(top, s);
        return;
    }
    __syncthreads();                                             // everybody has read its parts
    float *tops = shared, *sums = shared + 16 * BM, *target = shared + 32 * BM;
    float top = -INFINITY;
    if (wave < BM) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e < job.C) top = fmaxf(top, sum[e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (quarter == 0) tops[16 * wave + col] = top;
    }
    __syncthreads();
    top = tops[col];
#pragma unroll
    for (int a = 1; a < BM; ++a) top = fmaxf(top, tops[16 * a + col]);
    const float from = top == -INFINITY ? 0.f : top;
    if (wave < BM) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (first + e == label) target[col] = sum[e];
            sum[e] = first + e < job.C ? exp_of(sum[e] - from) : 0.f;
            s += sum[e];
        }
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (quarter == 0) sums[16 * wave + col] = s;
    }
    __syncthreads();
    if (!row_there || wave >= BM) return;
    float total = sums[col];
#pragma unroll
    for (int a = 1; a < BM; ++a) total += sums[16 * a + col];
    const bool known = label < job.C;
    if (wave == 0 && quarter == 0) job.loss[n] = !there ? 0.f : known ? logf(total) + (from - target[col]) : NAN;
    if (!job.gradients || first >= job.C) return;
    const float scale = job.weight && there ? job.weight[n] : 1.0f, inverse = 1.0f / total;
    float g[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        g[e] = sum[e] * inverse;
        if (first + e == label) g[e] -= 1.0f;
        g[e] = !there || first + e >= job.C ? 0.f : known ? g[e] * scale : NAN;
    }
    if (job.by_class) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e < job.C) job.G[(first + e) * job.ld_g + n] = g[e];
    } else {
        *reinterpret_cast<float4 *>(job.G + n * job.ld_g + first) = make_float4(g[0], g[1], g[2], g[3]);
    }
}

__global__ __launch_bounds__(256) void count_kernel(XentDirect job)
{
    __shared__ uint32_t part[4];
    uint32_t count = 0;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < job.N; n += 256 * kCountTiles) count += job.labels[n] >= 0 ? 1 : 0;
#pragma unroll
    for (int o = 32; o > 0; o /= 2) count += (uint32_t)__shfl_xor((int)count, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = count;
    __syncthreads();
    if (threadIdx.x == 0) job.counts[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// Scores to loss and G, a workgroup per row, and with many classes (job.partial: the maxima and sums of 16 classes each are known) per
// kPart classes of it. Scores cut in columns are added up on the way.
// THREADS a row, and rows of few classes several to a workgroup of 256. Bound by latency: 12 x 9000 9.3 us, 100 x 300 4.7.
constexpr int kSoftmaxThreads = 512, kAhead = 4, kPart = 4 * kAhead * kSoftmaxThreads;
template <int THREADS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void softmax_kernel(XentDirect job)
{
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1, STEP = 4 * kAhead * THREADS;
    static_assert(THREADS == 64 || ROWS == 1, "a wavefront or a workgroup for a row");
    __shared__ float2 part[THREADS / 64];
    __shared__ float label_scores[ROWS];
    const int thread = threadIdx.x % THREADS;
    float &label_score = label_scores[threadIdx.x / THREADS];
    const int64_t n = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    if (n >= job.N) return;                              // (whole wavefronts that meet no barrier)
    const int64_t label = job.labels[n];
    const float *row = job.scores + n * job.ld_scores;
    const int lane = threadIdx.x & 63, wave = thread >> 6;
    const int64_t begin = job.partial ? (int64_t)blockIdx.y * kPart : 0, end = job.partial ? std::min(begin + kPart, job.C) : job.C;
    // four classes of G, in the row's place, or one after the other in rows of the classes
    auto store = [&](int64_t c, const float (&g)[4]) {
        if (job.by_class) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < job.C) job.G[(c + e) * job.ld_g + n] = g[e];
        } else {
            *reinterpret_cast<float4 *>(job.G + n * job.ld_g + c) = make_float4(g[0], g[1], g[2], g[3]);
        }
    };
    const bool mine = label >= begin && label < end, first = begin == 0;       // the loss is written where the label's score is
    if (label < 0) {
        const float none[4] = {0.f, 0.f, 0.f, 0.f};
        if (thread == 0 && first) job.loss[n] = 0.f;
        if (job.gradients)
            for (int64_t c = begin + 4 * (int64_t)thread; c < end; c += 4 * THREADS) store(c, none);
        return;
    }
    auto load = [&](int64_t c) {
        float4 f = *reinterpret_cast<const float4 *>(row + c);
        for (unsigned k = 1; k < job.column_cuts; ++k) {
            const float4 o = *reinterpret_cast<const float4 *>(row + (int64_t)k * job.N * job.ld_scores + c);
            f = make_float4(f.x + o.x, f.y + o.y, f.z + o.z, f.w + o.w);
        }
        return f;
    };
    auto add = [](float2 a, float2 b) {
        const float m = fmaxf(a.x, b.x), from = m == -INFINITY ? 0.f : m;
        return make_float2(m, a.y * exp_of(a.x - from) + b.y * exp_of(b.x - from));
    };
    float2 v = make_float2(-INFINITY, 0.f);
    if (job.partial) {
        for (int64_t t = thread; t < (job.C + 15) / 16; t += THREADS) v = add(v, job.partial[t * job.N + n]);
        if (thread == 0 && mine && label < job.C) label_score = row[label];           // (before G takes its place)
    } else {
        for (int64_t c0 = 4 * (int64_t)thread; c0 < job.C; c0 += STEP) {
            float4 f[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t c = c0 + 4 * u * THREADS;
                f[u] = c < job.C ? load(c) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (job.column_cuts > 1 && c < job.C) *const_cast<float4 *>(reinterpret_cast<const float4 *>(row + c)) = f[u];
            }
            float m = v.x;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t c = c0 + 4 * u * THREADS;
                float x[4] = {f[u].x, f[u].y, f[u].z, f[u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (c + e >= job.C) x[e] = -INFINITY;
                    if (c + e == label) label_score = x[e];
                    m = fmaxf(m, x[e]);
                }
                f[u] = make_float4(x[0], x[1], x[2], x[3]);
            }
            const float from = m == -INFINITY ? 0.f : m;
            v.y *= exp_of(v.x - from);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v.y += (exp_of(f[u].x - from) + exp_of(f[u].y - from)) + (exp_of(f[u].z - from) + exp_of(f[u].w - from));
            v.x = m;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) v = add(v, make_float2(__shfl_xor(v.x, o), __shfl_xor(v.y, o)));
    if constexpr (THREADS > 64) {
        if (lane == 0) part[wave] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = add(v, part[w]);
    } else {
        __builtin_amdgcn_wave_barrier();                 // (label_score: written and read by one wavefront)
    }
    const float from = v.x == -INFINITY ? 0.f : v.x;
    const bool known = label < job.C;
    if (thread == 0 && (mine || (!known && first))) job.loss[n] = known ? logf(v.y) + (from - label_score) : NAN;
    if (!job.gradients) return;
    const float inverse = 1.0f / v.y, scale = job.weight ? job.weight[n] : 1.0f;
    for (int64_t c0 = begin + 4 * (int64_t)thread; c0 < end; c0 += STEP) {
        float4 f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t c = c0 + 4 * u * THREADS;
            f[u] = c < end ? *reinterpret_cast<const float4 *>(row + c) : make_float4(0.f, 0.f, 0.f, 0.f);       // (a thread's own, added up above)
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t c = c0 + 4 * u * THREADS;
            if (c >= end) break;
            float g[4] = {f[u].x, f[u].y, f[u].z, f[u].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] = exp_of(g[e] - from) * inverse;
                if (c + e == label) g[e] -= 1.0f;
                g[e] = known ? g[e] * scale : NAN;
            }
            store(c, g);
        }
    }
}

__device__ __forceinline__ float mean_scale(const XentDirect &job)
{
    if (job.weight) return 1.0f;
    uint32_t count = 0;
    for (int t = threadIdx.x & 63; t < job.count_tiles; t += 256) {
#pragma unroll
        for (int u = 0; u < 4; ++u) count += t + 64 * u < job.count_tiles ? job.counts[t + 64 * u] : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) count += (uint32_t)__shfl_xor((int)count, o);
    return 1.0f / (float)max(count, 1u);
}
template <typename T>
__device__ __forceinline__ void store(T *dst, float v)
{
    if constexpr (sizeof(T) == 4) *dst = v;
    else *reinterpret_cast<__bf16 *>(dst) = (__bf16)v;
}

// Gradients of few (up to FEW) rows and many classes, or of few classes and many rows: with G[m][f], the many by the few, one pass over the
// many gives  of_many[m, :] = sum_f G[m][f] small[f, :]  and  of_few[f, :] += G[m][f] big[m, :].  A lane has four columns of K, in which it
// keeps the few rows of `small` and the sums; G's rows are the same for all lanes and come from LDS, kFewTile at a time, of which each
// wavefront takes every fourth. The wavefronts' sums are added up in LDS; the many are cut among workgroups.
// What bounds it is reading `big` and writing of_many. 12 x 2000, 9000 classes, float32, both gradients 44 us (144 MB, 3.3 TB/s), with 32-bit multiply-adds
// of 11 us; 7494 x 3001, 10 classes, dW 35 us (90 MB, 2.6 TB/s).
constexpr int kFewWaves = 4, kFewColumns = 256, kFewTile = 64;
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; };
template <typename T, int FEW, bool OF_MANY, bool OF_FEW>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(XentDirect job)
{
    __shared__ float4 parts[OF_FEW ? kFewWaves / 2 : 1][FEW][64];
    __shared__ __attribute__((aligned(16))) float g_tile[kFewTile][FEW];
    __shared__ bool counts[kFewTile];
    const bool rows_are_few = job.by_class;
    const DirectGradient &of_few = rows_are_few ? job.dphi : job.dw, &of_many = rows_are_few ? job.dw : job.dphi;
    const int64_t few = rows_are_few ? job.N : job.C, many = rows_are_few ? job.C : job.N;
    const T *small = static_cast<const T *>(rows_are_few ? job.Phi : job.W), *big = static_cast<const T *>(rows_are_few ? job.W : job.Phi);
    const int64_t ld_small = rows_are_few ? job.ld_phi : job.ld_w, ld_big = rows_are_few ? job.ld_w : job.ld_phi;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const unsigned across = (unsigned)((job.K + kFewColumns - 1) / kFewColumns), cut = blockIdx.x / across;
    const int64_t k = (int64_t)(blockIdx.x % across) * kFewColumns + 4 * lane;
    const int64_t begin = (int64_t)cut * of_few.per_cut, end = std::min(begin + of_few.per_cut, many);
    const uint64_t few_left_out = __ballot(rows_are_few && lane < few && job.labels[lane] < 0);
    const bool whole = k + 4 <= job.K;
    auto load4 = [&](const T *row, float (&x)[4]) {
        if (whole) {
            const Four<T> f = *reinterpret_cast<const Four<T> *>(row + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = number(f.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = k + e < job.K ? number(row[k + e]) : 0.f;
        }
    };
    float s[OF_MANY ? FEW : 1][4], sums[OF_FEW ? FEW : 1][4];
    if constexpr (OF_MANY) {
#pragma unroll
        for (int f = 0; f < FEW; ++f) {
            if (f < few && (few_left_out >> f & 1) == 0) {          // rows left out may hold anything
                load4(small + f * ld_small, s[f]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[f][e] = 0.f;
            }
        }
    }
    if constexpr (OF_FEW) {
#pragma unroll
        for (int f = 0; f < FEW; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[f][e] = 0.f;
    }
    const float scale = OF_MANY || of_few.cuts == 1 ? mean_scale(job) : 1.0f;
    constexpr int AHEAD = 4;
    for (int64_t tile = begin; tile < end; tile += kFewTile) {
        __syncthreads();
        for (int i = threadIdx.x; i < kFewTile * FEW / 4; i += 64 * kFewWaves) {
            const int r = i / (FEW / 4), f = 4 * (i % (FEW / 4));
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (tile + r < end && f < few) {                   // (rows are a multiple of four numbers; what lies beyond the few is nobody's)
                v = *reinterpret_cast<const float4 *>(job.G + (tile + r) * job.ld_g + f);
                if (f + 1 >= few) v.y = 0.f;
                if (f + 2 >= few) v.z = 0.f;
                if (f + 3 >= few) v.w = 0.f;
            }
            *reinterpret_cast<float4 *>(&g_tile[r][f]) = v;
        }
        if (threadIdx.x < kFewTile) {
            const int64_t m = tile + threadIdx.x;
            counts[threadIdx.x] = m < end && (rows_are_few || job.labels[m] >= 0);          // rows left out may hold anything, and have no gradient whatever W holds
        }
        __syncthreads();
        for (int r0 = wave; r0 < kFewTile && tile + r0 < end; r0 += AHEAD * kFewWaves) {
            float x[AHEAD][4];
            if constexpr (OF_FEW) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int r = r0 + u * kFewWaves;
                    if (counts[r]) {
                        load4(big + (tile + r) * ld_big, x[u]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[u][e] = 0.f;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int r = r0 + u * kFewWaves;
                const int64_t m = tile + r;
                if (m >= end) break;
                float g[FEW];
#pragma unroll
                for (int f = 0; f < FEW; f += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(&g_tile[r][f]);
                    g[f] = v.x;
                    g[f + 1] = v.y;
                    g[f + 2] = v.z;
                    g[f + 3] = v.w;
                }
                if constexpr (OF_FEW) {
#pragma unroll
                    for (int f = 0; f < FEW; ++f)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sums[f][e] = fmaf(g[f], x[u][e], sums[f][e]);
                }
                if constexpr (OF_MANY) {
                    float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int f = 0; f < FEW; ++f)
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = fmaf(g[f], s[f][e], y[e]);
                    if (!counts[r]) y[0] = y[1] = y[2] = y[3] = 0.f;
                    T *dst = static_cast<T *>(of_many.out) + m * of_many.ld + k;
                    if (whole) {
                        Four<T> v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) store(&v.v[e], y[e] * scale);
                        *reinterpret_cast<Four<T> *>(dst) = v;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (k + e < job.K) store(dst + e, y[e] * scale);
                    }
                }
            }
        }
    }
    if constexpr (OF_FEW) {
        // the wavefronts' sums: 2 and 3 to 0 and 1, then 1 to 0
        static_assert(kFewWaves == 4, "");
#pragma unroll
        for (int half = 2; half > 0; half /= 2) {
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int f = 0; f < FEW; ++f) parts[wave - half][f][lane] = make_float4(sums[f][0], sums[f][1], sums[f][2], sums[f][3]);
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int f = 0; f < FEW; ++f) {
                    const float4 o = parts[wave][f][lane];
                    sums[f][0] += o.x;
                    sums[f][1] += o.y;
                    sums[f][2] += o.z;
                    sums[f][3] += o.w;
                }
            }
            __syncthreads();
        }
        if (wave != 0) return;
#pragma unroll
        for (int f = 0; f < FEW; ++f) {
            if (f >= few) break;
            if (few_left_out >> f & 1) sums[f][0] = sums[f][1] = sums[f][2] = sums[f][3] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (k + e >= job.K) break;
                if (of_few.cuts > 1) of_few.parts[((int64_t)cut * few + f) * job.K + k + e] = sums[f][e];
                else store(static_cast<T *>(of_few.out) + f * of_few.ld + k + e, sums[f][e] * scale);
            }
        }
    }
}

// Up to 16 classes and 2048 columns: scores, softmax and both gradients in one pass over Phi. A lane has four columns of K: of the classes' weights
// and of their sums dW, which stay in registers, and of the R rows that its wavefront is at, which are read once, while the rows before are worked on.
// CW wavefronts share a row's columns; 8 / CW groups of them take rows of their own and add their sums up in LDS at the end.
// A wavefront's R FEW sums over its columns are spread over its lanes as they are added up: at each step a lane keeps one half of
// them and gives the other half to the lane that keeps that one, about 2 R FEW steps instead of 6 R FEW. The gradients are outer products, which 4 x 4 x 1
// matrix instructions of 32 bits make in half the time of multiply-adds, from the registers as they lie.
// What bounds it is the chain of a tile: of its 9400 cycles (the clock read in the kernel) the scores take 3500, adding up and the softmax 3400, dW 2500; two
// wavefronts a SIMD wait 45 % of their time (counters), and the matrix instructions are busy 9 %. Then reading Phi. 7494 x 1001, 10 classes, float32, dW: 18.7 us (1.6 TB/s) and 5.4 for adding up 235 parts, 22.7 the call; with multiply-adds for the gradients 20.6;
// scores and gradients in two launches 11.6 + 16.2, 31.7 the call. 16 x 193, 10 classes: 7.8 us, where nearly all is latency; 11.7 with the four
// classes that do not exist and the rows that other groups would have worked on, and three rounds of adding up.
constexpr int kOnePassWaves = 8, kOnePassColumns = 256 * kOnePassWaves, kOnePassFew = 16;
constexpr int64_t kCountHere = 8192;             // rows that a workgroup counts by itself, 64 KB of labels out of a cache, rather than in a launch before it
constexpr int one_pass_at_a_time(int few, bool of_phi) { return few <= 4 ? 16 : few <= 8 || !of_phi ? 8 : 4; }        // rows of a wavefront; registers
constexpr int one_pass_least(int few, int groups, bool of_phi) { return (kOnePassWaves + groups) * one_pass_at_a_time(few, of_phi) * few + 8; }
template <int CTRL>
__device__ __forceinline__ float from_lane(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140, kRotate8 = 0x128;
// The sum of a over the pair of lanes that STEP stands for in the lower one, that of b in the other.
template <int STEP>
__device__ __forceinline__ float shared_sum(float a, float b, int lane)
{
    if constexpr (STEP >= 16) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        if constexpr (STEP == 32) {
            const auto s = __builtin_amdgcn_permlane32_swap(x, y, false, false);
            return __uint_as_float(s[0]) + __uint_as_float(s[1]);
        } else {
            const auto s = __builtin_amdgcn_permlane16_swap(x, y, false, false);
            return __uint_as_float(s[0]) + __uint_as_float(s[1]);
        }
    } else {
        const bool upper = (lane & STEP) != 0;
        const float keep = upper ? b : a, give = upper ? a : b;
        return keep + from_lane<STEP == 8 ? kRotate8 : STEP == 4 ? kMirror8 : STEP == 2 ? kXor2 : kXor1>(give);
    }
}
// The sums over all lanes of COUNT numbers, spread over the lanes: the first half of them to the lanes whose bit STEP is not set, and so on.
template <int COUNT, int STEP>
__device__ __forceinline__ void spread_sums(float *v, int lane)
{
    if constexpr (COUNT > 1 && STEP > 0) {
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) v[i] = shared_sum<STEP>(v[i], v[i + COUNT / 2], lane);
        spread_sums<COUNT / 2, STEP / 2>(v, lane);
    }
}
template <int FEW, bool MAX>
__device__ __forceinline__ float among_few(float v)
{
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    v = join(v, from_lane<kXor1>(v));
    v = join(v, from_lane<kXor2>(v));
    if constexpr (FEW >= 8) v = join(v, from_lane<kMirror8>(v));
    if constexpr (FEW >= 16) v = join(v, from_lane<kMirror16>(v));
    return v;
}
template <typename T, int FEW, int CW, bool OF_PHI>
__global__ __launch_bounds__(64 * kOnePassWaves, 2) void one_pass_kernel(XentDirect job)
{
    constexpr int GROUPS = kOnePassWaves / CW, R = one_pass_at_a_time(FEW, OF_PHI), VALUES = R * FEW, PER = VALUES / 64, LEAST = one_pass_least(FEW, GROUPS, OF_PHI);
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), group = wave / CW, part = wave % CW;
    float *parts = shared + group * CW * VALUES, *g_rows = shared + kOnePassWaves * VALUES + group * VALUES;
    uint32_t *counted = reinterpret_cast<uint32_t *>(shared + (kOnePassWaves + GROUPS) * VALUES);
    const int64_t begin = (int64_t)blockIdx.x * job.dw.per_cut, end = std::min(begin + job.dw.per_cut, job.N);
    const int K = (int)job.K, C = (int)job.C;
    // The last numbers of a row are read together with some before them, and shifted to their place.
    const unsigned k = 256 * part + 4 * lane, from_k = std::min((int)k, K - 4), shift = k - from_k;
    const bool all_whole = 256 * part + 256 <= K;
    auto load4 = [&](const T *row) { return *reinterpret_cast<const Four<T> *>(row + from_k); };
    auto placed = [&](float (&x)[4]) __attribute__((always_inline)) {
        if (all_whole) return;
        const bool one = (shift & 1) != 0, two = (shift & 2) != 0, gone = shift >= 4;
        const float a[4] = {one ? x[1] : x[0], one ? x[2] : x[1], one ? x[3] : x[2], one ? 0.f : x[3]};
        x[0] = gone ? 0.f : two ? a[2] : a[0];
        x[1] = gone ? 0.f : two ? a[3] : a[1];
        x[2] = gone || two ? 0.f : a[2];
        x[3] = gone || two ? 0.f : a[3];
    };
    auto store4 = [&](auto *row, const float (&x)[4], float by) __attribute__((always_inline)) {
        typedef std::remove_reference_t<decltype(*row)> O;
        if (shift == 0) {
            Four<O> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) store(&v.v[e], x[e] * by);
            *reinterpret_cast<Four<O> *>(row + k) = v;
        } else if (shift < 4) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if ((int)k + e < K) store(row + k + e, x[e] * by);
        }
    };
    constexpr int FOURS = FEW / 4;
    float w[FEW][4];
    floatx4 sums[4][FOURS];                          // [column][four classes]
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < FOURS; ++q) sums[e][q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < FEW; ++f) {
        const Four<T> v = load4(static_cast<const T *>(job.W) + std::min(f, C - 1) * job.ld_w);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[f][e] = number(v.v[e]);
    }
    Four<T> next[R];
    int next_label;
    float next_weight;
    auto fetch = [&](int64_t first) {
        const int64_t mine = first + (lane & (R - 1));
        const int64_t label = mine < end ? job.labels[mine] : -1;
        next_label = label < 0 ? -1 : label < C ? (int)label : C;
        next_weight = job.weight && mine < end ? job.weight[mine] : 1.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) next[r] = load4(static_cast<const T *>(job.Phi) + std::min(first + r, job.N - 1) * job.ld_phi);
    };
    int64_t first = begin + group * R;
    fetch(first);
#pragma unroll
    for (int f = 0; f < FEW; ++f) placed(w[f]);                    // (of classes that do not exist, the last one's, which only meets G = 0)
    float scale = 1.0f;
    uint32_t all_rows = 0;
    if (job.count_here) {
        for (int64_t n = threadIdx.x; n < job.N; n += 64 * kOnePassWaves) all_rows += job.labels[n] >= 0 ? 1 : 0;
#pragma unroll
        for (int o = 32; o > 0; o /= 2) all_rows += (uint32_t)__shfl_xor((int)all_rows, o);
        if (lane == 0) counted[wave] = all_rows;
        __syncthreads();
        all_rows = 0;
#pragma unroll
        for (int i = 0; i < kOnePassWaves; ++i) all_rows += counted[i];
        __syncthreads();
        scale = 1.0f / (float)max(all_rows, 1u);
        if (blockIdx.x == 0 && threadIdx.x == 0) job.counts[0] = all_rows;
    } else if (OF_PHI) {
        scale = mean_scale(job);
    }
    uint32_t rows_here = 0;
    for (int64_t tile = begin; tile < end; tile += GROUPS * R, first += GROUPS * R) {
        const int label_of = next_label;
        const float weight_of = next_weight;
        const uint64_t there = __ballot(lane < R && label_of >= 0);
        rows_here += (uint32_t)__popcll(there);
        float x[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[r][e] = (there >> r & 1) != 0 ? number(next[r].v[e]) : 0.f;          // rows left out may hold anything
#pragma unroll
        for (int r = 0; r < R; ++r) placed(x[r]);
        if (tile + GROUPS * R < end) fetch(first + GROUPS * R);
        float of_class[FEW];                     // of the row that the lane's upper bits say
#pragma unroll
        for (int f = 0; f < FEW; ++f) of_class[f] = 0.f;
#pragma unroll
        for (int f = 0; f < FEW; ++f) {
            if (there == 0 || (f >= 4 && f / 4 * 4 >= C)) continue;          // (no rows, or four classes that do not exist)
            float v[R];
#pragma unroll
            for (int r = 0; r < R; ++r) v[r] = fmaf(x[r][3], w[f][3], fmaf(x[r][2], w[f][2], fmaf(x[r][1], w[f][1], x[r][0] * w[f][0])));
            spread_sums<R, 32>(v, lane);
            of_class[f] = v[0];
            // one class after the other: all products at a time would not fit the registers
            if (f + 1 < FEW) asm volatile("" : "+v"(of_class[f]), "+v"(w[f + 1][0]), "+v"(w[f + 1][1]), "+v"(w[f + 1][2]), "+v"(w[f + 1][3]));
        }
        spread_sums<FEW, 32 / R>(of_class, lane);
#pragma unroll
        for (int p = 0; p < PER; ++p) parts[part * VALUES + PER * lane + p] = of_class[p];
        __syncthreads();
#pragma unroll
        for (int v0 = 0; v0 < VALUES; v0 += 64 * CW) {
            const int v = v0 + 64 * part + lane, f = v % FEW, r = v / FEW;
            if (VALUES % (64 * CW) != 0 && v >= VALUES) continue;               // (whole wavefronts)
            float score = 0.f;
#pragma unroll
            for (int i = 0; i < CW; ++i) score += parts[i * VALUES + v];
            const int label = __shfl(label_of, r);
            const float weight = __shfl(weight_of, r), top = among_few<FEW, true>(f < C ? score : -INFINITY), from = top == -INFINITY ? 0.f : top;
            const float share = f < C ? exp_of(score - from) : 0.f, total = among_few<FEW, false>(share);
            if (first + r < end) {
                if (f == label && f < C) job.loss[first + r] = logf(total) + (from - score);          // (one lane writes a loss)
                if (f == 0 && label < 0) job.loss[first + r] = 0.f;
                if (f == 0 && label == C) job.loss[first + r] = NAN;
            }
            float g = share * (1.0f / total);
            if (f == label) g -= 1.0f;
            g_rows[v] = label < 0 || f >= C ? 0.f : label < C ? g * weight : NAN;
        }
        __syncthreads();
        if (there == 0 && !OF_PHI) continue;
        // dW[f][k] += G[r][f] x[r][k]: lane l gives column k of its own and class l % 4 of four (4 x 4 x 1 matrix instructions, 16 of which lie
        // next to each other in a wavefront), and has column k of all four classes.
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int q = 0; q < FOURS; ++q) {
                if (q > 0 && 4 * q >= C) break;
                const float g = g_rows[r * FEW + 4 * q + (lane & 3)];
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[e][q] = __builtin_amdgcn_mfma_f32_4x4x1f32(g, x[r][e], sums[e][q], 0, 0, 0);
            }
        }
        if constexpr (OF_PHI) {
            // dPhi[r][k] = sum_f G[r][f] w[f][k], four rows at a time in the same way
#pragma unroll
            for (int r0 = 0; r0 < R; r0 += 4) {
                floatx4 y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < FEW; ++f) {
                    if (f >= 4 && f / 4 * 4 >= C) continue;
                    const float g = g_rows[(r0 + (lane & 3)) * FEW + f];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_mfma_f32_4x4x1f32(g, w[f][e], y[e], 0, 0, 0);
                }
#pragma unroll
                for (int r = r0; r < r0 + 4; ++r) {
                    float row[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) row[e] = (there >> r & 1) != 0 ? y[e][r - r0] : 0.f;             // (whatever W holds)
                    if (first + r < end) store4(static_cast<T *>(job.dphi.out) + (first + r) * job.dphi.ld, row, scale);
                }
            }
        }
    }
    if (!job.dw.out) return;
    // The groups' sums add up: class f is for group f % GROUPS to add and to store.
    const bool cut = job.dw.cuts > 1, counts = !job.weight && !job.count_here && !OF_PHI;
    float4 *all = reinterpret_cast<float4 *>(shared + LEAST);                          // [wave][class][lane]
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int f = 0; f < FEW; ++f)
            if (f < C) all[(wave * C + f) * 64 + lane] = make_float4(sums[0][f / 4][f % 4], sums[1][f / 4][f % 4], sums[2][f / 4][f % 4], sums[3][f / 4][f % 4]);
    }
    if (counts && lane == 0) counted[wave] = part == 0 ? rows_here : 0;
    __syncthreads();
    if (counts) {
        // the rows that count, of this workgroup: all there are if it is the only one
        all_rows = 0;
#pragma unroll
        for (int i = 0; i < kOnePassWaves; ++i) all_rows += counted[i];
        if (!cut) scale = 1.0f / (float)max(all_rows, 1u);
        else if (threadIdx.x == 0) job.counts[blockIdx.x] = all_rows;
    }
    float *part_out = job.dw.parts + (int64_t)blockIdx.x * C * K;
    auto store_sums = [&](int f, const float (&row)[4]) __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 4) {
            store4((cut ? part_out : static_cast<T *>(job.dw.out)) + f * (cut ? K : job.dw.ld), row, cut ? 1.0f : scale);
        } else {
            if (cut) store4(part_out + f * K, row, 1.0f);
            else store4(static_cast<T *>(job.dw.out) + f * job.dw.ld, row, scale);
        }
    };
    if constexpr (GROUPS > 1) {
        for (int f = group; f < C; f += GROUPS) {                                       // (part is its own)
            float row[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const float4 v = all[((g * CW + part) * C + f) * 64 + lane];
                row[0] += v.x;
                row[1] += v.y;
                row[2] += v.z;
                row[3] += v.w;
            }
            store_sums(f, row);
        }
    } else {
#pragma unroll
        for (int f = 0; f < FEW; ++f) {
            const float row[4] = {sums[0][f / 4][f % 4], sums[1][f / 4][f % 4], sums[2][f / 4][f % 4], sums[3][f / 4][f % 4]};
            if (f < C) store_sums(f, row);
        }
    }
}
// Both gradients of more of either, in tiles of 32 rows (sequences, summed over classes, or classes, summed over sequences) x 64 columns of K,
// in blocks of 32 x 32. The wavefronts of a workgroup share out the sum, or (OWN: sums of up to 64 numbers) have tiles of their own next to each
// other. A lane's column of the result is its number in the wavefront, so that 32 lanes write 128 bytes of a row. Bound by latency, and where there are many
// tiles by splitting 32-bit numbers into terms: 3000 x 500, 40 classes, float32 dPhi 12.7 us, dW 15.8; 100 x 500, 300 classes, both 13.1.
constexpr int kWide = 64, kSumWaves = 4;
template <typename T, bool OWN>
__global__ __launch_bounds__(64 * kSumWaves) void gradients_kernel(XentDirect job)
{
    constexpr int TA = sizeof(T) == 4 ? 3 : 1, TB = sizeof(T) == 4 ? 3 : 2;
    __shared__ float shared[OWN ? 1 : 2 * kSumWaves * 16 * 64];
    const bool is_w = blockIdx.x >= job.blocks_phi;
    const DirectGradient &g = is_w ? job.dw : job.dphi;
    unsigned id = blockIdx.x - (is_w ? job.blocks_phi : 0);
    constexpr int WIDE = OWN ? kWide * kSumWaves : kWide;
    const unsigned across = (unsigned)((job.K + WIDE - 1) / WIDE), cut = id % g.cuts;
    id /= g.cuts;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5, col = lane & 31;
    const int64_t i0 = (int64_t)(id % across) * WIDE + (OWN ? kWide * wave : 0), j0 = (int64_t)(id / across) * 32;
    if (OWN && i0 >= job.K) return;
    const int64_t rows = is_w ? job.C : job.N, summed = is_w ? job.N : job.C;
    const int64_t begin = (int64_t)cut * g.per_cut, end = std::min(begin + g.per_cut, summed);
    const T *A = static_cast<const T *>(is_w ? job.Phi : job.W);
    const int64_t ld_a = is_w ? job.ld_phi : job.ld_w;
    // features beyond K and columns beyond the rows are read as the last ones
    const int64_t ia[2] = {std::min(i0 + col, job.K - 1), std::min(i0 + 32 + col, job.K - 1)};
    const int64_t jb = std::min(j0 + col, rows - 1);
    const int64_t label = is_w ? 0 : job.labels[jb];
    floatx16 acc[2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[a][e] = 0.f;
    float xa[2][8], xb[8];
    auto fetch = [&](int64_t s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t m = s + 8 * half + e, at = std::min(m, summed - 1);
            bool there = m < end;
            xb[e] = there ? job.G[is_w ? at * job.ld_g + jb : jb * job.ld_g + at] : 0.f;
            if (is_w) there = there && job.labels[at] >= 0;          // rows left out may hold anything
            xa[0][e] = there ? number(A[at * ld_a + ia[0]]) : 0.f;
            xa[1][e] = there ? number(A[at * ld_a + ia[1]]) : 0.f;
        }
    };
    int64_t s = begin + (OWN ? 0 : 16 * wave);
    if (s < end) fetch(s);
    while (s < end) {
        float a0[8], a1[8], b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a0[e] = xa[0][e];
            a1[e] = xa[1][e];
            b[e] = xb[e];
        }
        s += OWN ? 16 : 16 * kSumWaves;
        if (s < end) fetch(s);
        const Split<TB> sb = split<TB>(b);
        acc[0] = multiply(sb, split<TA>(a0), acc[0]);
        acc[1] = multiply(sb, split<TA>(a1), acc[1]);
    }
    const float scale = g.cuts == 1 ? mean_scale(job) : 1.0f;
    const uint64_t left_out = __ballot(label < 0);          // rows left out have no gradient whatever W holds
    auto store_block = [&](const floatx16 &sum, int64_t first) {
        const int64_t i = first + col;
        if (i >= job.K) return;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int64_t r = j0 + 8 * (e / 4) + 4 * half + e % 4;
            if (r >= rows) continue;
            const float v = (left_out >> (r - j0) & 1) == 0 ? sum[e] : 0.f;
            if (g.cuts > 1) g.parts[((int64_t)cut * rows + r) * job.K + i] = v;
            else store(static_cast<T *>(g.out) + r * g.ld + i, v * scale);
        }
    };
    if constexpr (OWN) {
        store_block(acc[0], i0);
        store_block(acc[1], i0 + 32);
    } else {
        const floatx16 sum = add_up<2, kSumWaves, 16>(acc, shared, wave, lane);
        if (wave < 2) store_block(sum, i0 + 32 * wave);
    }
}

// Adds the parts of the cut sums up: 64 numbers a workgroup, whose wavefronts take parts in turn. Bound by latency: 235 parts of 10010 numbers 5.5 us
// (1.7 TB/s; as long with four wavefronts and 118 parts), few parts 3.7.
template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void add_parts_kernel(XentDirect job)
{
    __shared__ float shared[NW][64];
    const int64_t of_phi = job.dphi.cuts > 1 ? job.N * job.K : 0, of_w = job.dw.cuts > 1 ? job.C * job.K : 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float scale = mean_scale(job);
    const unsigned groups_phi = (unsigned)((of_phi + 63) / 64), groups = groups_phi + (unsigned)((of_w + 63) / 64);
    for (unsigned group = blockIdx.x; group < groups; group += gridDim.x) {
        const bool is_w = group >= groups_phi;
        const DirectGradient &g = is_w ? job.dw : job.dphi;
        const int64_t m = (int64_t)(group - (is_w ? groups_phi : 0)) * 64 + lane, all = is_w ? of_w : of_phi;
        float sum = 0.f;
        if (m < all) {
#pragma unroll 8
            for (unsigned c = wave; c < g.cuts; c += NW) sum += g.parts[(int64_t)c * all + m];
        }
        shared[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && m < all) {
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) sum += shared[w][lane];
            const int64_t r = m / job.K;
            store(static_cast<T *>(g.out) + r * g.ld + (m - r * job.K), sum * scale);
        }
        __syncthreads();
    }
}

constexpr int64_t kWorkgroups = 768;         // three for every CU
constexpr int64_t kLeastSummed = 128;        // of a cut
constexpr int64_t kFew = 16, kOwn = 64, kWaveClasses = 256;

size_t up(size_t v) { return (v + 255) / 256 * 256; }
// How a gradient's sum is cut: into as many parts as fill the GPU.
DirectGradient cut_of(int64_t tiles, int64_t summed, int64_t unit)
{
    DirectGradient g = {};
    int64_t cuts = std::min(kWorkgroups / tiles, summed / kLeastSummed);
    if (cuts < 2) cuts = 1;
    g.per_cut = ((summed + cuts - 1) / cuts + unit - 1) / unit * unit;
    g.cuts = (uint32_t)((summed + g.per_cut - 1) / g.per_cut);
    return g;
}
bool is_few(const rfsf_xent_shape &s) { return std::min(s.N, s.C) <= kFew; }
// All in one pass: where a gradient is asked for, unless it is dPhi alone, of more than 8 classes (4 rows of a wavefront at a time) and many rows.
// us, in two passes and in one, float32 but where said: 50 x 70, 2 classes, dW 12.0 and 6.6; 1000 x 1025, 16, both 30.1 and 23.5; 10000 x 70, 7,
// both 30.3 and 16.5; 10000 x 2000, 7, dW 51.4 and 31.8; 40000 x 1000, 2, dW 86.9 and 38.5, 16, both 159 and 112. dPhi alone: 50 x 2000, 16,
// bfloat16 21.1 and 8.9; 1000 x 300, 16 13.9 and 9.4, 2 10.4 and 11.6; 10000 x 513, 7 22.8 and 23.3; but, left to two, 10000 x 513, 16 26.6 and 30.7;
// 40000 x 1000, 16, bfloat16 69.2 and 92.5. Of 81 shapes in these ranges 77 are taken, 1.50 times faster on average; the worst 0.88 times.
constexpr int64_t kOnePassRowsOfPhi = 4096;
bool is_one_pass(const rfsf_xent_shape &s)
{
    if (!s.gradients || s.C > kOnePassFew || s.K < 4 || s.K > kOnePassColumns) return false;
    return (s.gradients & RFSF_XENT_DW) || s.C <= 8 || s.N <= kOnePassRowsOfPhi;
}
int one_pass_wide(int64_t K) { return K <= 256 ? 1 : K <= 512 ? 2 : K <= 1024 ? 4 : 8; }           // wavefronts that share a row
int64_t one_pass_rows(const rfsf_xent_shape &s)                       // of a workgroup, at a time
{
    return kOnePassWaves / one_pass_wide(s.K) * one_pass_at_a_time((int)s.C, (s.gradients & RFSF_XENT_DPHI) != 0);
}
// The few of the two: rows (G then lies by classes), or classes.
bool rows_are_few(const rfsf_xent_shape &s) { return is_few(s) && s.N < s.C && !is_one_pass(s); }
constexpr int64_t kOnePassCuts = 256;                          // workgroups: one for every CU
constexpr int64_t kLeastMany = 16, kMostParts = 128;           // rows of a workgroup of few_kernel; parts to add up
void cuts_of(const rfsf_xent_shape &s, DirectGradient *dphi, DirectGradient *dw)
{
    if (is_one_pass(s)) {
        const int64_t at_a_time = one_pass_rows(s), tiles = (s.N + at_a_time - 1) / at_a_time, each = (tiles + kOnePassCuts - 1) / kOnePassCuts;
        DirectGradient g = {};
        g.per_cut = each * at_a_time;
        g.cuts = (uint32_t)((s.N + g.per_cut - 1) / g.per_cut);
        *dphi = *dw = g;
        dphi->cuts = 1;
    } else if (is_few(s)) {
        const int64_t many = std::max(s.N, s.C), across = (s.K + kFewColumns - 1) / kFewColumns;
        const int64_t cuts = std::max<int64_t>(std::min(std::min((std::min(s.N, s.C) > 8 ? 512 : kWorkgroups) / across, kMostParts), many / kLeastMany), 1);
        DirectGradient g = {};
        g.per_cut = (many + cuts - 1) / cuts;
        g.cuts = (uint32_t)((many + g.per_cut - 1) / g.per_cut);
        *dphi = *dw = g;
        (rows_are_few(s) ? *dw : *dphi).cuts = 1;                      // (of the many: no sums to add up)
    } else {
        const int64_t across = (s.K + kWide - 1) / kWide;
        *dphi = cut_of((s.N + 31) / 32 * across, s.C, 64);             // (sums of up to kOwn numbers are whole)
        *dw = cut_of((s.C + 31) / 32 * across, s.N, 64);
    }
    if (!(s.gradients & RFSF_XENT_DPHI)) dphi->cuts = 1;
    if (!(s.gradients & RFSF_XENT_DW)) dw->cuts = 1;
}

template <typename T, int FEW>
void launch_few(const XentDirect &job, unsigned blocks, hipStream_t stream)
{
    const bool of_few = (job.by_class ? job.dphi.out : job.dw.out) != nullptr, of_many = (job.by_class ? job.dw.out : job.dphi.out) != nullptr;
    if (of_few && of_many) few_kernel<T, FEW, true, true><<<dim3(blocks), 64 * kFewWaves, 0, stream>>>(job);
    else if (of_few) few_kernel<T, FEW, false, true><<<dim3(blocks), 64 * kFewWaves, 0, stream>>>(job);
    else few_kernel<T, FEW, true, false><<<dim3(blocks), 64 * kFewWaves, 0, stream>>>(job);
}

template <typename T, int FEW, int CW, bool OF_PHI>
hipError_t launch_one_pass(const XentDirect &job, unsigned blocks, hipStream_t stream)
{
    constexpr int GROUPS = kOnePassWaves / CW;
    const size_t sums = GROUPS > 1 && job.dw.out ? (size_t)job.C * kOnePassWaves * 64 * sizeof(float4) : 0;
    const size_t lds = sizeof(float) * one_pass_least(FEW, GROUPS, OF_PHI) + sums;
    static LdsLimit limit;
    const hipError_t e = allow_lds(limit, reinterpret_cast<const void *>(one_pass_kernel<T, FEW, CW, OF_PHI>), lds);
    if (e != hipSuccess) return e;
    one_pass_kernel<T, FEW, CW, OF_PHI><<<dim3(blocks), 64 * kOnePassWaves, lds, stream>>>(job);
    return hipGetLastError();
}
template <typename T, int FEW>
hipError_t launch_one_pass(const XentDirect &job, unsigned blocks, hipStream_t stream)
{
    const int wide = one_pass_wide(job.K);
    auto launch = [&](auto of_phi) {
        constexpr bool PHI = decltype(of_phi)::value;
        return wide == 1   ? launch_one_pass<T, FEW, 1, PHI>(job, blocks, stream)
               : wide == 2 ? launch_one_pass<T, FEW, 2, PHI>(job, blocks, stream)
               : wide == 4 ? launch_one_pass<T, FEW, 4, PHI>(job, blocks, stream)
                           : launch_one_pass<T, FEW, 8, PHI>(job, blocks, stream);
    };
    return job.dphi.out ? launch(std::true_type{}) : launch(std::false_type{});
}
template <typename T>
hipError_t add_parts(const XentDirect &job, hipStream_t stream)
{
    const int64_t numbers = (job.dphi.cuts > 1 ? job.N * job.K : 0) + (job.dw.cuts > 1 ? job.C * job.K : 0);
    if (numbers == 0) return hipSuccess;
    const unsigned groups = (unsigned)std::min<int64_t>((numbers + 63) / 64 + 1, 4096);
    if (std::max(job.dphi.cuts, job.dw.cuts) > 32) add_parts_kernel<T, 16><<<dim3(groups), 1024, 0, stream>>>(job);
    else add_parts_kernel<T, 4><<<dim3(groups), 256, 0, stream>>>(job);
    return hipGetLastError();
}

template <typename T, int BM>
void launch_fused(const XentDirect &job, unsigned tiles, hipStream_t stream)
{
    // wavefronts to share out the columns: more where there are few workgroups
    constexpr int MOST = BM == 1 ? 16 : 8;              // (registers)
    if (tiles <= 256 && job.K > 4 * 64) scores_kernel<T, BM, MOST, true><<<dim3(tiles), 64 * MOST, 0, stream>>>(job);
    else scores_kernel<T, BM, 4, true><<<dim3(tiles), 256, 0, stream>>>(job);
}

template <typename T>
hipError_t run(const XentDirect &job, bool few, hipStream_t stream)
{
    const unsigned tiles_n = (unsigned)((job.N + kRows - 1) / kRows);
    if (job.one_pass) {
        if (job.dphi.out && !job.weight && !job.count_here) count_kernel<<<dim3(kCountTiles), 256, 0, stream>>>(job);
        const unsigned blocks = (unsigned)((job.N + job.dw.per_cut - 1) / job.dw.per_cut);
        const hipError_t e = job.C <= 4   ? launch_one_pass<T, 4>(job, blocks, stream)
                             : job.C <= 8 ? launch_one_pass<T, 8>(job, blocks, stream)
                                          : launch_one_pass<T, 16>(job, blocks, stream);
        return e != hipSuccess ? e : add_parts<T>(job, stream);
    }
    if (job.fused && job.C <= 16) {
        launch_fused<T, 1>(job, tiles_n, stream);
    } else if (job.fused && job.C <= 32) {
        launch_fused<T, 2>(job, tiles_n, stream);
    } else if (job.fused) {
        launch_fused<T, 4>(job, tiles_n, stream);
    } else {
        scores_kernel<T, 2, 4, false><<<dim3(tiles_n, (unsigned)((job.C + 31) / 32), job.column_cuts), 256, 0, stream>>>(job);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (job.C <= kWaveClasses) softmax_kernel<64><<<dim3((unsigned)((job.N + 3) / 4)), 256, 0, stream>>>(job);
        else softmax_kernel<kSoftmaxThreads><<<dim3((unsigned)job.N, job.partial ? (unsigned)((job.C + kPart - 1) / kPart) : 1), kSoftmaxThreads, 0, stream>>>(job);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !job.gradients) return e;
    if (job.N > kCountedRows && !job.weight) count_kernel<<<dim3(kCountTiles), 256, 0, stream>>>(job);
    if (few) {
        const int64_t few_of = std::min(job.N, job.C), cuts = (std::max(job.N, job.C) + job.dphi.per_cut - 1) / job.dphi.per_cut;
        const unsigned blocks = (unsigned)((job.K + kFewColumns - 1) / kFewColumns * cuts);
        if (few_of <= 4) launch_few<T, 4>(job, blocks, stream);
        else if (few_of <= 8) launch_few<T, 8>(job, blocks, stream);
        else launch_few<T, 16>(job, blocks, stream);
    } else {
        // each gradient in its own way: a launch has one of them
        XentDirect one = job;
        auto launch = [&](bool own, bool is_w) {
            const int64_t wide = own ? kWide * kSumWaves : kWide, across = (job.K + wide - 1) / wide;
            const int64_t blocks = ((is_w ? job.C : job.N) + 31) / 32 * across * (is_w ? job.dw.cuts : job.dphi.cuts);
            one.blocks_phi = is_w ? 0 : (unsigned)blocks;
            if (own) gradients_kernel<T, true><<<dim3((unsigned)blocks), 64 * kSumWaves, 0, stream>>>(one);
            else gradients_kernel<T, false><<<dim3((unsigned)blocks), 64 * kSumWaves, 0, stream>>>(one);
        };
        const bool own_phi = job.C <= kOwn, own_w = job.N <= kOwn;
        if (job.dphi.out && job.dw.out && !own_phi && !own_w) {
            const int64_t across = (job.K + kWide - 1) / kWide;
            one.blocks_phi = (unsigned)((job.N + 31) / 32 * across * job.dphi.cuts);
            gradients_kernel<T, false><<<dim3((unsigned)(one.blocks_phi + (job.C + 31) / 32 * across * job.dw.cuts)), 64 * kSumWaves, 0, stream>>>(one);
        } else {
            if (job.dphi.out) launch(own_phi, false);
            if (job.dw.out) launch(own_w, true);
        }
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    return add_parts<T>(job, stream);
}

// How the scores are made: with up to 64 classes in one launch with the softmax, unless few rows of many columns leave CUs without work;
// otherwise cut in columns where there are few tiles, and with the softmax' parts where a row has many classes.
struct ScorePlan { bool fused, partial; uint32_t cuts; int64_t per_cut; };
constexpr int64_t kFusedTiles = 128, kFusedColumns = 1024, kColumnTiles = 512, kLeastColumns = 512;
ScorePlan score_plan(const rfsf_xent_shape &s)
{
    const int64_t tiles_n = (s.N + kRows - 1) / kRows;
    if (s.C <= 64 && (tiles_n >= kFusedTiles || s.K <= kFusedColumns)) return {true, false, 1, s.K};
    if (s.C > kPart) return {false, true, 1, s.K};
    const int64_t tiles = tiles_n * ((s.C + 31) / 32);
    int64_t cuts = std::min(kColumnTiles / tiles, s.K / kLeastColumns);
    if (cuts < 2) return {false, false, 1, s.K};
    const int64_t per = ((s.K + cuts - 1) / cuts + 63) / 64 * 64;
    return {false, false, (uint32_t)((s.K + per - 1) / per), per};
}
struct Places { size_t g, scores, partial, counts, parts_phi, parts_w, all; };
int64_t four(int64_t v) { return (v + 3) / 4 * 4; }
Places places_of(const rfsf_xent_shape &s, const DirectGradient &dphi, const DirectGradient &dw)
{
    Places p;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    const ScorePlan plan = score_plan(s);
    // scores that leave the registers, and G in their place unless it lies by classes; one pass holds neither
    const bool scores = !is_one_pass(s) && !plan.fused, g = !is_one_pass(s) && s.gradients, by_class = rows_are_few(s);
    p.scores = p.g = take(scores || (g && !by_class) ? 4 * (size_t)s.N * (size_t)four(s.C) * plan.cuts : 0);
    if (g && by_class) p.g = take(4 * (size_t)s.C * (size_t)four(s.N));
    p.partial = take(plan.partial ? sizeof(float2) * (size_t)s.N * (size_t)((s.C + 31) / 32 * 2) : 0);
    p.counts = take(4 * (size_t)(kCountedRows / kRows));
    p.parts_phi = take(dphi.cuts > 1 ? 4 * (size_t)dphi.cuts * (size_t)s.N * (size_t)s.K : 0);
    p.parts_w = take(dw.cuts > 1 ? 4 * (size_t)dw.cuts * (size_t)s.C * (size_t)s.K : 0);
    p.all = at + 256;
    return p;
}

}  // namespace

// Where this way is the faster one: for up to 16 rows or classes everywhere, otherwise by the products N K C, of which each gradient weighs four times as
// much as before it (the packed way packs and makes scores in any case), and by h = N C / (N + C), their ratio to what the packed way reads and
// writes beside them. Of 150 shapes with 17 to 10000 rows, 65 to 10241 columns and 17 to 50000 classes, N K C from 3e7 to 6e9, both types and
// any gradients, all timed both ways, the way chosen takes 1.8 % longer than the better one on average; fitted to half of them, 3.4 % with the other
// half. (That was with G of one term in the packed bfloat16 way; with two, the 65 of bfloat16 with gradients come to 1.5 %.) Beyond N C = 2^26 all are packed, few classes
// at a loss: 6.5e6 x 65, 10 classes, dW 2.1 ms here, 6.8e6 rows packed 8.1; losses alone 1.5 and 4.3. (us, packed and here: 30 x 7544, 158 classes, float32, losses 81 and 13; 2845 x 6843, 47, float32, dPhi 153 and 102; 375 x 4022, 283,
// bfloat16, losses 40 and 21; but 8161 x 4507, 42, bfloat16, both 199 and 332; 129 x 1805, 4490, bfloat16, dW 66 and 169; 222 x 565, 34570, bfloat16,
// both 202 and 642.)
bool xent_direct(const rfsf_xent_shape &s)
{
    const double n = (double)s.N, c = (double)s.C;
    if (s.N < 1 || s.C > 1000000 || n * c > 1 << 26) return false;
    if (is_few(s)) return true;
    const double h = n * c / (n + c);
    double products = n * c * (double)s.K;
    if (s.gradients & RFSF_XENT_DPHI) products *= 4;
    if (s.gradients & RFSF_XENT_DW) products *= 4;
    return products <= (h <= 64 ? 4e9 : h <= 128 ? 1.5e9 : h <= 256 ? 3e8 : 6e7);
}

size_t xent_direct_bytes(const rfsf_xent_shape &s)
{
    DirectGradient dphi, dw;
    cuts_of(s, &dphi, &dw);
    return places_of(s, dphi, dw).all;
}

hipError_t launch_xent_direct(const rfsf_xent_shape &s, const void *Phi, const void *W, const int64_t *labels, const float *weight, float *loss, void *dPhi,
                              void *dW, void *workspace, hipStream_t stream)
{
    XentDirect job = {};
    job.Phi = Phi;
    job.W = W;
    job.labels = labels;
    job.weight = weight;
    job.loss = loss;
    job.N = s.N;
    job.K = s.K;
    job.C = s.C;
    job.ld_phi = s.ld_phi;
    job.ld_w = s.ld_w;
    job.gradients = s.gradients;
    cuts_of(s, &job.dphi, &job.dw);
    const Places p = places_of(s, job.dphi, job.dw);
    const size_t mis = (size_t)(reinterpret_cast<uintptr_t>(workspace) % 256);
    char *ws = static_cast<char *>(workspace) + (mis ? 256 - mis : 0);
    job.by_class = rows_are_few(s);
    job.scores = reinterpret_cast<float *>(ws + p.scores);
    job.ld_scores = four(s.C);
    const ScorePlan plan = score_plan(s);
    job.fused = plan.fused;
    job.column_cuts = plan.cuts;
    job.columns_per_cut = plan.per_cut;
    job.partial = plan.partial ? reinterpret_cast<float2 *>(ws + p.partial) : nullptr;
    job.G = reinterpret_cast<float *>(ws + p.g);
    job.ld_g = four(job.by_class ? s.N : s.C);
    job.counts = reinterpret_cast<uint32_t *>(ws + p.counts);
    job.count_tiles = s.N > kCountedRows ? kCountTiles : (int32_t)((s.N + kRows - 1) / kRows);
    job.one_pass = is_one_pass(s);
    if (job.one_pass) {
        job.count_here = (s.gradients & RFSF_XENT_DPHI) && !weight && s.N <= kCountHere;
        job.count_tiles = job.count_here ? 1 : (s.gradients & RFSF_XENT_DPHI) ? kCountTiles : (int32_t)job.dw.cuts;
    }
    job.dphi.parts = reinterpret_cast<float *>(ws + p.parts_phi);
    job.dw.parts = reinterpret_cast<float *>(ws + p.parts_w);
    job.dphi.ld = s.ld_dphi;
    job.dw.ld = s.ld_dw;
    job.dphi.out = (s.gradients & RFSF_XENT_DPHI) ? dPhi : nullptr;
    job.dw.out = (s.gradients & RFSF_XENT_DW) ? dW : nullptr;
    return s.bf16 ? run<uint16_t>(job, is_few(s), stream) : run<float>(job, is_few(s), stream);
}

}  // namespace rfsf
