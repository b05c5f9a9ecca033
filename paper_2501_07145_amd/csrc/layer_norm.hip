// Layer norm of feature rows, with dropout behind it, and its backward pass.
//
//   z = (x - mean) rstd,  rstd = 1 / sqrt(var + eps),  y = dropout(z gain + offset)
//   h = dropout(dy),  g = h gain,  dx = rstd (g - mean(g) - z mean(g z)),  dgain = sum over rows of h z,  doffset = sum over rows of h
#include <algorithm>
#include <type_traits>

#include "../../include/rfsf_ts.h"
#include "dropout.h"
#include "rows8.h"

namespace rfsf {
namespace {

constexpr int64_t kMostHeld = 512 * 5 * 8, kLeastHeld = 8;      // columns of rows that stay in registers; that loads of whole eights need
constexpr int64_t kManyRows = 2048;
constexpr bool is_held(int64_t K) { return K <= kMostHeld; }
constexpr int kCus = 256;

struct NormJob {
    const void *X;
    void *Y;
    const float *gain, *offset;
    float *mean, *rstd;
    int64_t N, K, ldx, ldy;
    float eps;
    DropoutJob dropout;
};
struct BackJob {
    const void *X, *dY;
    void *dX;
    const float *mean, *rstd, *gain;
    float *sums;                // [workgroups along the rows][2][K rounded up to eight], dgain's and doffset's; unused where there is one workgroup
    float *dgain, *doffset;
    int64_t N, K, ldx, ldy, ldd;
    DropoutJob dropout;
};

// Sums of numbers over the THREADS lanes of a row. `part`: LDS of rows of more than a wavefront, not used again before the next barrier.
template <int THREADS, typename S, int COUNT>
__device__ __forceinline__ void add_up(S (&v)[COUNT], S (*part)[COUNT])
{
#pragma unroll
    for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o /= 2)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += __shfl_xor(v[i], o);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) part[threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = part[0][i];
#pragma unroll
            for (int w = 1; w < THREADS / 64; ++w) v[i] += part[w][i];
        }
    }
}

__device__ __forceinline__ void load_or(const float *p, int64_t k, int64_t K, float otherwise, float (&x)[8])
{
    if (p) {
        rows8::load(p, k, K, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = otherwise;
    }
}

// Rows are added up in 64 bits, eight numbers of bfloat16 first in 32 (exact as long as they lie within 2^13 of each other), so that the mean is rounded once; what that
// leaves over is known, and taken off the differences to it, and its square off their mean square. Rows far from zero lose nothing. (Eighths of the numbers, which have
// no error, the smallest one's being 2^-136, and whose sum is finite. FEW: of rows that wait for each other, as products and sums apart, 1 x 1025 with dropout 7.1 us, the
// other way 7.5; of many rows, whose number of instructions counts, as multiply-adds, 100000 x 400 39.0, the other way 39.6.)
template <bool FEW>
__device__ __forceinline__ double sum_of(const rows8::Eight<uint16_t> &c)
{
    constexpr float EIGHTH = 0.125f;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = rows8::to_float(c.v[e]) * (FEW ? EIGHTH : 1.f);
    if (FEW) return 8.0 * (double)(((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])));
    float even = x[0] * EIGHTH, odd = x[1] * EIGHTH;
#pragma unroll
    for (int e = 2; e < 8; e += 2) {
        even = fmaf(x[e], EIGHTH, even);
        odd = fmaf(x[e + 1], EIGHTH, odd);
    }
    return 8.0 * (double)(even + odd);
}
template <bool FEW>
__device__ __forceinline__ double sum_of(const rows8::Eight<float> &c)
{
    return (((double)c.v[0] + (double)c.v[1]) + ((double)c.v[2] + (double)c.v[3])) + (((double)c.v[4] + (double)c.v[5]) + ((double)c.v[6] + (double)c.v[7]));
}
struct Mean { float mean, rest; };
// (The quotient is corrected by what it leaves over, so that it is rounded once: the mean of a row of one number is this number, and nothing is left over, which a large
// number's 2^-53 times rstd would make visible.)
__device__ __forceinline__ Mean mean_of(double sum, double inverse, double K)
{
    const double about = sum * inverse, mean = fma(fma(-K, about, sum), inverse, about);
    const float rounded = (float)about;
    return {rounded, (float)(mean - (double)rounded)};
}
// 0 where the squares' sum is infinite, which it is of finite rows alone (whose rest may have an infinite square too): rows with an infinity or a NaN have NaN among their squares.
__device__ __forceinline__ float rstd_of(float squares, float rest, float inverse, float eps)
{
    const float variance = squares * inverse - rest * rest;
    return squares == INFINITY ? 0.f : 1.0f / sqrtf((variance < 0.f ? 0.f : variance) + eps);           // (a NaN stays)
}
// What is taken off a row's numbers where they are multiplied by rstd: nothing where that is 0, so that differences beyond 32 bits are not infinite there. (Whole numbers are
// compared, which the scalar unit can do where a row has a wavefront.)
__device__ __forceinline__ float centre_of(float mean, float rstd) { return __float_as_uint(rstd) == 0 ? 0.f : mean; }
// v, which nothing is made of before c is there.
template <typename T>
__device__ __forceinline__ float after(rows8::Eight<T> &c, float v)
{
    uint32_t w;
    __builtin_memcpy(&w, &c, 4);
    asm volatile("" : "+v"(w), "+v"(v));
    __builtin_memcpy(&c, &w, 4);
    return v;
}

// Few rows, which should each be spread over many lanes: THREADS lanes hold a row, HELD times eight numbers each; a workgroup goes through rows, whose next one is
// loaded while the present one is worked on, and keeps its columns' gains and offsets. Bound by latency: 1 x 1025 4.4 us, 333 x 5121, float32, with the launch 8; of
// longer rows than norm_wave_kernel has registers for by memory (5000 x 16385, float32 148 us, 4.4 TB/s).
template <typename T, int THREADS, int HELD, bool DROP>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void norm_kernel(NormJob job)
{
    constexpr int ROWS = THREADS >= 256 ? 1 : 256 / THREADS, WAVES = THREADS > 64 ? THREADS / 64 : 1;
    __shared__ double part_sum[WAVES][1];
    __shared__ float part_squares[WAVES][1];
    const int lane = threadIdx.x % THREADS, K = (int)job.K;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const double inverse = 1.0 / (double)K;
    float gain[HELD][8], shift[HELD][8];
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
        load_or(job.gain, 8 * (lane + u * THREADS), K, 1.f, gain[u]);
        load_or(job.offset, 8 * (lane + u * THREADS), K, 0.f, shift[u]);
    }
    const uint64_t counter = DROP ? dropout::offset_of(job.dropout) : 0;
    const T *X = static_cast<const T *>(job.X);
    T *Y = static_cast<T *>(job.Y);
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    rows8::Eight<T> next[HELD], now[HELD];
#pragma unroll
    for (int u = 0; u < HELD; ++u) next[u] = rows8::load_raw(X + std::min(row, job.N - 1) * job.ldx, 8 * (lane + u * THREADS), K);
    // (all rows of a workgroup take as many turns, so that everybody meets at the barriers)
    for (int64_t turn = (int64_t)blockIdx.x * ROWS; turn < job.N; turn += step, row += step) {
        double sum[1] = {0.0};
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            now[u] = next[u];
            sum[0] += sum_of<true>(now[u]);
        }
        if (turn + step < job.N) {
#pragma unroll
            for (int u = 0; u < HELD; ++u) next[u] = rows8::load_raw(X + std::min(row + step, job.N - 1) * job.ldx, 8 * (lane + u * THREADS), K);
        }
        add_up<THREADS>(sum, part_sum);
        const Mean m = mean_of(sum[0], inverse, (double)K);
        float squares[1] = {0.f};
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * (lane + u * THREADS);
            if (k + 8 <= K) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = rows8::to_float(now[u].v[e]) - m.mean;
                    squares[0] = fmaf(d, d, squares[0]);
                }
            } else if (k < K) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = k + e < K ? rows8::to_float(now[u].v[e]) - m.mean : 0.f;
                    squares[0] = fmaf(d, d, squares[0]);
                }
            }
        }
        add_up<THREADS>(squares, part_squares);
        const float rstd = rstd_of(squares[0], m.rest, (float)inverse, job.eps);
        if (row >= job.N) continue;
        if (lane == 0) {
            if (job.mean) job.mean[row] = m.mean;
            if (job.rstd) job.rstd[row] = rstd;
        }
        const float centre = centre_of(m.mean, rstd);
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * (lane + u * THREADS);
            if (k >= K) continue;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf((rows8::to_float(now[u].v[e]) - centre - m.rest) * rstd, gain[u][e], shift[u][e]);
            if (DROP) dropout::apply(job.dropout, counter, job.dropout.first_row + (uint32_t)row, (uint32_t)k / 8, y);
            rows8::store(Y + row * job.ldy, k, K, y);
        }
    }
}

// The kernels for many rows take a row as eights of columns, up to HELD a lane, and what is left over, up to seven columns (features have 1 + M*D), as one number more for
// each of the first lanes: an eight of its own would take as long as a whole one (200003 x 65, bfloat16, backward 29 -> 24 us).

// Many rows: LANES of a wavefront have a row to themselves, and nobody waits for anybody; gains and offsets lie in LDS, once for all wavefronts of a CU. Of a lane's
// eights the first FULL are there for every lane. Bound by memory, with dropout on bfloat16 by the vector units as much (busy 71 % of the cycles, most of that the
// generator): 30000 x 10241, bfloat16 265 us (4.6 TB/s), with dropout 288; float32 513 (4.8 TB/s), 516; 200003 x 65, bfloat16 13.4. A workgroup to a row
// (norm_kernel) took 565 us of the second, gains and offsets from the L2 for every row or in registers of few wavefronts, everyone waiting for the row's slowest.
constexpr int wave_threads(size_t held_bytes) { return held_bytes <= 28 ? 1024 : held_bytes <= 42 ? 768 : 512; }
template <typename T, int LANES, int FULL, int HELD, bool DROP>
__global__ __launch_bounds__(wave_threads(HELD * sizeof(T))) void norm_wave_kernel(NormJob job)
{
    constexpr int THREADS = wave_threads(HELD * sizeof(T)), STEP = 8 * LANES, ROWS = THREADS / LANES;
    extern __shared__ __attribute__((aligned(16))) float columns[];          // gains, then offsets, each of HELD * STEP and eight
    constexpr int ROOM = STEP * HELD + 8;
    const int lane = threadIdx.x % LANES, K = (int)job.K, whole = K / 8 * 8, last = whole + lane;
    for (int k = threadIdx.x; k < ROOM; k += THREADS) {
        columns[k] = k < K && job.gain ? job.gain[k] : 1.f;
        columns[ROOM + k] = k < K && job.offset ? job.offset[k] : 0.f;
    }
    __syncthreads();
    const double inverse = 1.0 / (double)K;
    const uint64_t counter = DROP ? dropout::offset_of(job.dropout) : 0;
    int64_t row = (int64_t)blockIdx.x * ROWS + (LANES == 64 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / LANES)) : threadIdx.x / LANES);
    for (; row < job.N; row += (int64_t)gridDim.x * ROWS) {
        const T *x = static_cast<const T *>(job.X) + row * job.ldx;
        T *y_row = static_cast<T *>(job.Y) + row * job.ldy;
        rows8::Eight<T> held[HELD];
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * lane + STEP * u;
            if (u < FULL || k < whole) held[u] = *reinterpret_cast<const rows8::Eight<T> *>(x + k);
            else held[u] = {};
        }
        const float x_last = last < K ? rows8::to_float(x[last]) : 0.f;
        double sum[1] = {(double)x_last};
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            rows8::in_turn(held[u]);
            sum[0] += sum_of<false>(held[u]);
        }
        add_up<LANES>(sum, static_cast<double (*)[1]>(nullptr));
        const Mean m = mean_of(sum[0], inverse, (double)K);
        const float d_last = last < K ? x_last - m.mean : 0.f;
        float squares[1] = {d_last * d_last};
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            if (u >= FULL && 8 * lane + STEP * u >= whole) continue;
            rows8::in_turn(held[u]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = rows8::to_float(held[u].v[e]) - m.mean;
                squares[0] = fmaf(d, d, squares[0]);
            }
        }
        add_up<LANES>(squares, static_cast<float (*)[1]>(nullptr));
        const float rstd = rstd_of(squares[0], m.rest, (float)inverse, job.eps);
        if (lane == 0) {
            if (job.mean) job.mean[row] = m.mean;
            if (job.rstd) job.rstd[row] = rstd;
        }
        const float centre = centre_of(m.mean, rstd);
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * lane + STEP * u;
            if (u >= FULL && k >= whole) continue;
            rows8::in_turn(held[u]);
            float y[8], gain[8], shift[8];
            __builtin_memcpy(gain, columns + k, 32);
            __builtin_memcpy(shift, columns + ROOM + k, 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf((rows8::to_float(held[u].v[e]) - centre - m.rest) * rstd, gain[e], shift[e]);
            if (DROP) {
                uint32_t group = (uint32_t)k / 8;
                asm volatile("" : "+v"(group));            // (the first rounds' products, which are the same for all rows, would be kept for every u)
                dropout::apply(job.dropout, counter, job.dropout.first_row + (uint32_t)row, group, y);
            }
            rows8::store(y_row, k, k + 8, y);
        }
        if (last < K) {
            float y = fmaf((x_last - centre - m.rest) * rstd, columns[last], columns[ROOM + last]);
            if (DROP) y = dropout::keeps(job.dropout, counter, job.dropout.first_row + (uint32_t)row, (uint32_t)last) ? y * job.dropout.factor : 0.f;
            rows8::from_float(y, y_row + last);
        }
    }
}

// Rows of any length: a workgroup reads a row three times, of which the caches give the last two.
constexpr int kLongThreads = 1024;
template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(NormJob job, bool drop)
{
    __shared__ double part_sum[kLongThreads / 64][1];
    __shared__ float part_squares[kLongThreads / 64][1];
    const int64_t K = job.K, row = blockIdx.x;
    const double inverse = 1.0 / (double)K;
    const T *x_row = static_cast<const T *>(job.X) + row * job.ldx;
    float x[8];
    double sum[1] = {0.0};
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * kLongThreads) {
        rows8::load(x_row, k, K, x);
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (double)x[e];
        sum[0] += s;
    }
    add_up<kLongThreads>(sum, part_sum);
    const Mean m = mean_of(sum[0], inverse, (double)K);
    float squares[1] = {0.f};
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * kLongThreads) {
        rows8::load(x_row, k, K, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = k + e < K ? x[e] - m.mean : 0.f;
            squares[0] = fmaf(d, d, squares[0]);
        }
    }
    add_up<kLongThreads>(squares, part_squares);
    const float rstd = rstd_of(squares[0], m.rest, (float)inverse, job.eps);
    if (threadIdx.x == 0) {
        if (job.mean) job.mean[row] = m.mean;
        if (job.rstd) job.rstd[row] = rstd;
    }
    const float centre = centre_of(m.mean, rstd);
    const uint64_t counter = drop ? dropout::offset_of(job.dropout) : 0;
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * kLongThreads) {
        float gain[8], shift[8];
        rows8::load(x_row, k, K, x);
        load_or(job.gain, k, K, 1.f, gain);
        load_or(job.offset, k, K, 0.f, shift);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf((x[e] - centre - m.rest) * rstd, gain[e], shift[e]);
        if (drop) dropout::apply(job.dropout, counter, job.dropout.first_row + (uint32_t)row, (uint32_t)(k / 8), x);
        rows8::store(static_cast<T *>(job.Y) + row * job.ldy, k, K, x);
    }
}

__host__ __device__ __forceinline__ int64_t room_of(int64_t K) { return (K + 7) / 8 * 8; }
// Where part number `part` of the sums goes.
struct Sums { float *gain, *offset; };
__device__ __forceinline__ Sums sums_of(const BackJob &job, int64_t part, int64_t parts)
{
    if (parts == 1) return {job.dgain, job.doffset};
    const int64_t room = room_of(job.K);
    return {job.sums + part * 2 * room, job.sums + (part * 2 + 1) * room};
}

// The backward pass of rows that are held in registers, THREADS lanes a row, HELD eights each, of which all but the last are there for every lane; gains lie in LDS.
// Dropout's factor is taken out of all sums: it multiplies what comes of them. GAINS: a lane adds its columns' h z and h up over the rows of the workgroup, whose
// sums are then one of the parts that add_parts_kernel adds up: no atomics, so that equal calls give equal bits. KEEP: z and g stay in registers until dX is written, where
// there are some (200003 x 65, bfloat16, with dropout, all launches 28.7 -> 27.0 us; 30000 x 5121 without dropout 180 -> 197). Bound by memory: 10000 x 10241, float32,
// with dropout 247 us and 7.5 for the parts (4.8 TB/s), dX alone 242 (with registers for four wavefronts a SIMD, which spill, 313); narrow rows by the vector units
// (200003 x 65, bfloat16 19 us and 4).
template <typename T>
constexpr int back_waves(int held, bool gains) { return held == 1 || (!gains && (held == 2 || (held == 3 && sizeof(T) == 2))) ? 4 : held == 2 ? 3 : 2; }
template <typename T, int THREADS, int HELD, bool DROP, bool GAINS>
__global__ __launch_bounds__((THREADS > 256 ? THREADS : 256), back_waves<T>(HELD, GAINS)) void back_kernel(BackJob job)
{
    constexpr int GROUP = THREADS > 256 ? THREADS : 256, ROWS = GROUP / THREADS, WAVES = THREADS > 64 ? THREADS / 64 : 1, STEP = 8 * THREADS;
    constexpr bool AHEAD = HELD <= (sizeof(T) == 2 ? 4 : 3);          // registers for the next row
    constexpr bool KEEP = HELD <= 2 || (HELD == 3 && sizeof(T) == 2 && (DROP || THREADS <= 64));         // and for z and g from the sums to dX
    constexpr bool LATE = DROP && !AHEAD;               // the generator's work on the first eight does not wait for mean and rstd (10000 x 10241, bfloat16, dX alone 146 us if it does, 143)
    static_assert(AHEAD || HELD > 1, "a lane's first eight is always there");
    __shared__ float part[2][WAVES][2];
    __shared__ __attribute__((aligned(16))) float gains[STEP * HELD + 8];
    const int lane = threadIdx.x % THREADS, K = (int)job.K, whole = K / 8 * 8, last = whole + lane;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inverse = 1.0f / (float)K, factor = DROP ? job.dropout.factor : 1.f;
    for (int k = threadIdx.x; k < STEP * HELD + 8; k += GROUP) gains[k] = k < K && job.gain ? job.gain[k] : 1.f;
    __syncthreads();
    float of_gain[HELD][8], of_offset[HELD][8], of_gain_last = 0.f, of_offset_last = 0.f;
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) of_gain[u][e] = of_offset[u][e] = 0.f;
    const uint64_t counter = DROP ? dropout::offset_of(job.dropout) : 0;
    const T *X = static_cast<const T *>(job.X), *dY = static_cast<const T *>(job.dY);
    T *dX = static_cast<T *>(job.dX);
    int64_t row = (int64_t)blockIdx.x * ROWS + (THREADS >= 64 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / THREADS)) : threadIdx.x / THREADS);
    rows8::Eight<T> x[HELD], h[HELD], next_x[HELD], next_h[HELD];
    float mean, rstd, next_mean, next_rstd, x_last, h_last, next_x_last, next_h_last;
    auto load = [&](int64_t r) {
        r = r < job.N ? r : job.N - 1;
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * lane + STEP * u;
            if (u < HELD - 1 || k < whole) {
                next_x[u] = *reinterpret_cast<const rows8::Eight<T> *>(X + r * job.ldx + k);
                next_h[u] = *reinterpret_cast<const rows8::Eight<T> *>(dY + r * job.ldy + k);
            }
        }
        next_x_last = last < K ? rows8::to_float(X[r * job.ldx + last]) : 0.f;
        next_h_last = last < K ? rows8::to_float(dY[r * job.ldy + last]) : 0.f;
        next_mean = job.mean[r];
        next_rstd = job.rstd[r];
    };
    if (AHEAD) load(row);
    int which = 0;
    // (all rows of a workgroup take as many turns, so that everybody meets at the barriers)
    for (int64_t turn = (int64_t)blockIdx.x * ROWS; turn < job.N; turn += step, row += step) {
        if (!AHEAD) load(row);
        mean = next_mean;
        rstd = next_rstd;
        x_last = next_x_last;
        h_last = next_h_last;
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            x[u] = next_x[u];
            h[u] = next_h[u];
        }
        if (AHEAD && turn + step < job.N) load(row + step);
        const bool there = ROWS == 1 || row < job.N;
        float centre = LATE ? 0.f : centre_of(mean, rstd);
        float sums[2] = {0.f, 0.f};             // of g, of g z
        float kept_z[KEEP ? HELD : 1][8], kept_g[KEEP ? HELD : 1][8];
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * lane + STEP * u;
            if (u == HELD - 1 && k >= whole) continue;
            if (!KEEP) rows8::in_turn(x[u]);
            if (DROP) {
                uint32_t group = (uint32_t)k / 8;
                asm volatile("" : "+v"(group));            // (the first rounds' products, which are the same for all rows, would be kept for every u)
                dropout::choose(job.dropout, counter, job.dropout.first_row + (uint32_t)row, group, h[u]);
            }
            if (LATE && u == 0) centre = centre_of(mean, after(h[u], rstd));
            float gain[8];
            __builtin_memcpy(gain, gains + k, 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = there ? (rows8::to_float(x[u].v[e]) - centre) * rstd : 0.f, d = there ? rows8::to_float(h[u].v[e]) : 0.f, g = d * gain[e];
                if (KEEP) {
                    kept_z[u][e] = z;
                    kept_g[u][e] = g;
                }
                if (GAINS) {
                    of_gain[u][e] = fmaf(d, z, of_gain[u][e]);
                    of_offset[u][e] += d;
                }
                sums[0] += g;
                sums[1] = fmaf(g, z, sums[1]);
            }
        }
        float z_last = 0.f;
        if (last < K) {
            if (DROP) h_last = dropout::keeps(job.dropout, counter, job.dropout.first_row + (uint32_t)row, (uint32_t)last) ? h_last : 0.f;
            h_last = there ? h_last : 0.f;
            z_last = there ? (x_last - centre) * rstd : 0.f;
            const float g = h_last * gains[last];
            of_gain_last = fmaf(h_last, z_last, of_gain_last);
            of_offset_last += h_last;
            sums[0] += g;
            sums[1] = fmaf(g, z_last, sums[1]);
        }
        add_up<THREADS>(sums, part[which]);
        which ^= 1;
        if (!there) continue;
        sums[0] *= inverse;
        sums[1] *= inverse;
        const float scale = rstd * factor;
        T *to = dX + row * job.ldd;
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int k = 8 * lane + STEP * u;
            if (u == HELD - 1 && k >= whole) continue;
            float d[8];
            if constexpr (KEEP) {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = (kept_g[u][e] - fmaf(kept_z[u][e], sums[1], sums[0])) * scale;
            } else {
                rows8::in_turn(x[u]);
                rows8::in_turn(h[u]);
                float gain[8];
                __builtin_memcpy(gain, gains + k, 32);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = (rows8::to_float(x[u].v[e]) - centre) * rstd;
                    d[e] = (rows8::to_float(h[u].v[e]) * gain[e] - fmaf(z, sums[1], sums[0])) * scale;
                }
            }
            rows8::store(to, k, k + 8, d);
        }
        if (last < K) rows8::from_float((h_last * gains[last] - fmaf(z_last, sums[1], sums[0])) * scale, to + last);
    }
    if constexpr (GAINS) {
        const Sums mine = sums_of(job, blockIdx.x, gridDim.x);
        if constexpr (ROWS > 1) {                       // over the workgroup's rows
            __shared__ float all[ROWS][THREADS][9];
#pragma unroll
            for (int u = 0; u < HELD; ++u)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    __syncthreads();
#pragma unroll
                    for (int e = 0; e < 8; ++e) all[threadIdx.x / THREADS][lane][e] = w ? of_offset[u][e] : of_gain[u][e];
                    __syncthreads();
                    for (int at = threadIdx.x; at < THREADS * 8; at += GROUP) {
                        float s = 0.f;
#pragma unroll
                        for (int r = 0; r < ROWS; ++r) s += all[r][at / 8][at % 8];
                        const int k = STEP * u + at;
                        if (k < whole) (w ? mine.offset : mine.gain)[k] = s * factor;
                    }
                }
            __syncthreads();
            all[threadIdx.x / THREADS][lane][0] = of_gain_last;
            all[threadIdx.x / THREADS][lane][1] = of_offset_last;
            __syncthreads();
            if (threadIdx.x < THREADS && last < K) {
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    a += all[r][lane][0];
                    b += all[r][lane][1];
                }
                mine.gain[last] = a * factor;
                mine.offset[last] = b * factor;
            }
        } else {
#pragma unroll
            for (int u = 0; u < HELD; ++u) {
                const int k = 8 * lane + STEP * u;
                if (u == HELD - 1 && k >= whole) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    of_gain[u][e] *= factor;
                    of_offset[u][e] *= factor;
                }
                rows8::store(mine.gain, k, k + 8, of_gain[u]);
                rows8::store(mine.offset, k, k + 8, of_offset[u]);
            }
            if (last < K) {
                mine.gain[last] = of_gain_last * factor;
                mine.offset[last] = of_offset_last * factor;
            }
        }
    }
}

// dX of rows of any length: a workgroup reads a row twice.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void back_long_kernel(BackJob job, bool drop)
{
    __shared__ float part[kLongThreads / 64][2];
    const int64_t K = job.K, row = blockIdx.x;
    const float inverse = 1.0f / (float)K, rstd = job.rstd[row], mean = centre_of(job.mean[row], rstd);
    const uint64_t counter = drop ? dropout::offset_of(job.dropout) : 0;
    const T *X = static_cast<const T *>(job.X) + row * job.ldx, *dY = static_cast<const T *>(job.dY) + row * job.ldy;
    float z[8], g[8];
    auto load = [&](int64_t k) {
        float gain[8];
        rows8::load(X, k, K, z);
        rows8::load(dY, k, K, g);
        load_or(job.gain, k, K, 1.f, gain);
        if (drop) dropout::apply(job.dropout, counter, job.dropout.first_row + (uint32_t)row, (uint32_t)(k / 8), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            z[e] = (z[e] - mean) * rstd;
            g[e] *= gain[e];
        }
    };
    float sums[2] = {0.f, 0.f};
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * kLongThreads) {
        load(k);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < K) {
                sums[0] += g[e];
                sums[1] = fmaf(g[e], z[e], sums[1]);
            }
    }
    add_up<kLongThreads>(sums, part);
    sums[0] *= inverse;
    sums[1] *= inverse;
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * kLongThreads) {
        load(k);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = (g[e] - fmaf(z[e], sums[1], sums[0])) * rstd;
        rows8::store(static_cast<T *>(job.dX) + row * job.ldd, k, K, g);
    }
}

// dgain and doffset alone, which need no sums over rows' columns: a workgroup takes 8 * LANES columns of some rows, LANES lanes of it a row, four rows' loads ahead. Bound
// by memory: 10000 x 10241, float32 153 us (5.4 TB/s), 7494 x 1001 with dropout 14.6 and 3.7 for the parts (a wavefront has 512 columns; with 2048 a workgroup 36).
template <typename T>
__device__ __forceinline__ rows8::Eight<T> load_short(const T *row, int k, int K)
{
    rows8::Eight<T> c = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < K) c.v[e] = row[k + e];
    return c;
}
template <typename T, int LANES, bool DROP, bool SHORT>
__global__ __launch_bounds__(256, 4) void gains_kernel(BackJob job, uint32_t pieces)
{
    constexpr int ROWS = 256 / LANES, AHEAD = 4;
    __shared__ float all[ROWS][LANES][17];
    const int lane = threadIdx.x % LANES, sub = LANES == 64 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / LANES)) : threadIdx.x / LANES, K = (int)job.K;
    const int64_t part = blockIdx.x / pieces, step = (int64_t)(gridDim.x / pieces) * ROWS;
    const int k = 8 * ((int)(blockIdx.x % pieces) * LANES + lane);
    const uint64_t counter = DROP ? dropout::offset_of(job.dropout) : 0;
    const T *X = static_cast<const T *>(job.X), *dY = static_cast<const T *>(job.dY);
    float of_gain[8], of_offset[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) of_gain[e] = of_offset[e] = 0.f;
    for (int64_t row = part * ROWS + sub; row < job.N; row += AHEAD * step) {
        rows8::Eight<T> x[AHEAD], h[AHEAD];
        float mean[AHEAD], rstd[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t r = std::min(row + a * step, job.N - 1);
            x[a] = SHORT ? load_short(X + r * job.ldx, k, K) : rows8::load_raw(X + r * job.ldx, k, K);
            h[a] = SHORT ? load_short(dY + r * job.ldy, k, K) : rows8::load_raw(dY + r * job.ldy, k, K);
            mean[a] = job.mean[r];
            rstd[a] = job.rstd[r];
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t r = row + a * step;
            if (r >= job.N || k >= K) break;
            rows8::in_turn(x[a]);
            if (DROP) {
                uint32_t group = (uint32_t)k / 8;
                asm volatile("" : "+v"(group));
                dropout::choose(job.dropout, counter, job.dropout.first_row + (uint32_t)r, group, h[a]);
            }
            const float centre = centre_of(mean[a], rstd[a]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = rows8::to_float(h[a].v[e]);
                of_gain[e] = fmaf(d, (rows8::to_float(x[a].v[e]) - centre) * rstd[a], of_gain[e]);
                of_offset[e] += d;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        all[sub][lane][e] = of_gain[e];
        all[sub][lane][8 + e] = of_offset[e];
    }
    __syncthreads();
    const float factor = DROP ? job.dropout.factor : 1.f;
    const Sums mine = sums_of(job, part, gridDim.x / pieces);
    for (int at = threadIdx.x; at < 16 * LANES; at += 256) {
        const int w = at / (8 * LANES), c = at % (8 * LANES), column = 8 * LANES * (int)(blockIdx.x % pieces) + c;
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) s += all[r][c / 8][8 * w + c % 8];
        if (column < K) (w ? mine.offset : mine.gain)[column] = s * factor;
    }
}

// Adds the workgroups' sums up, in a fixed order: 32 columns a workgroup, 32 groups of lanes that share the parts, eight loads ahead.
constexpr int kAddColumns = 32, kAddThreads = 1024;
__global__ __launch_bounds__(kAddThreads) void add_parts_kernel(const float *sums, int64_t parts, int64_t K, float *dgain, float *doffset)
{
    constexpr int SLICES = kAddThreads / kAddColumns, AHEAD = 8;
    __shared__ float all[SLICES][kAddColumns + 1];
    const int lane = threadIdx.x % kAddColumns, slice = threadIdx.x / kAddColumns;
    const int64_t at = (int64_t)blockIdx.x * kAddColumns + lane, room = room_of(K);
    float s = 0.f;
    if (at < 2 * room)
        for (int64_t p = slice; p < parts; p += AHEAD * SLICES) {
            float v[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) v[a] = p + a * SLICES < parts ? sums[(p + a * SLICES) * 2 * room + at] : 0.f;
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) s += v[a];
        }
    all[slice][lane] = s;
    __syncthreads();
    const int64_t column = at < room ? at : at - room;
    if (slice != 0 || column >= K) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < SLICES; ++w) s += all[w][lane];
    (at < room ? dgain : doffset)[column] = s;
}

// f(lanes of a row, eights that each holds), of which all but the last are there for every lane.
template <int THREADS, int HELD> struct Shape {};
template <int THREADS, int HELD, typename... MORE, typename F>
auto with_first(int64_t eights, const F &f, Shape<THREADS, HELD>, MORE... more)
{
    if constexpr (sizeof...(MORE) > 0) {
        if (eights > THREADS * HELD) return with_first(eights, f, more...);
    }
    return f(std::integral_constant<int, THREADS>(), std::integral_constant<int, HELD>());
}
// (256 lanes with five eights of 32-bit numbers each have no registers for the next row: 10000 x 10241, backward 280 us, 512 with three 258; bfloat16 156 and 166. Less
// than a workgroup, where a row's next one is loaded later anyway, spill with five: 30000 x 2305 with dropout 236 us, more lanes with fewer 172; bfloat16 109 and 120.)
template <typename T, typename F>
auto with_shape(int64_t eights, const F &f)
{
    typedef std::conditional_t<sizeof(T) == 2, Shape<256, 5>, Shape<512, 3>> Wide;
    constexpr int most = sizeof(T) == 2 ? 5 : 4;
    return with_first(eights, f, Shape<8, 1>(), Shape<8, 2>(), Shape<8, 3>(), Shape<16, 2>(), Shape<16, 3>(), Shape<16, 4>(), Shape<16, most>(), Shape<64, 2>(), Shape<64, 3>(),
                      Shape<64, 4>(), Shape<64, most>(), Shape<256, 2>(), Shape<256, 3>(), Shape<256, 4>(), Wide(), Shape<512, 3>(), Shape<512, 4>(), Shape<512, 5>());
}
constexpr int group_threads(int threads) { return threads > 256 ? threads : 256; }
constexpr int group_rows(int threads) { return threads >= 256 ? 1 : 256 / threads; }
// Workgroups of a launch that goes through the rows: as many as the CUs hold at a time, of `waves` wavefronts a SIMD. With gains and offsets' gradients, of which each
// leaves a part: one for what it does in a few turns, which take less time than a second launch for adding parts up; and two turns rather than more than one workgroup
// a CU, where a part is as long as a row or two (333 x 5121, float32 23.5 -> 17.2 us).
constexpr int64_t kFewTurns = 4;
int64_t groups_of(int64_t N, int threads, int waves, bool gains)
{
    const int64_t groups = (N + group_rows(threads) - 1) / group_rows(threads);
    if (gains && groups <= kFewTurns) return 1;
    return std::min<int64_t>(gains && threads >= 256 && groups > kCus ? (groups + 1) / 2 : groups, kCus * (256 * waves / group_threads(threads)));
}
// Gradients of gains and offsets by a launch of their own, beside that of dX: where reading both matrices again takes fewer bytes than the parts
// (500 x 10241, bfloat16 33.0 -> 29.9 us; 333 x 5121 15.8 -> 14.2).
template <typename T>
bool apart(int64_t N, int64_t K)
{
    return with_shape<T>(K / 8, [&](auto threads, auto held) {
        if (threads < 256 || N <= kCus) return false;
        return 16 * groups_of(N, threads, back_waves<T>(held, true), true) > 2 * N * (int64_t)sizeof(T) + N / 2 * (int64_t)sizeof(T);
    });
}

// Parts of dgain and doffset. Fused with dX: one for each workgroup.
int gains_lanes(int64_t K) { return K <= 128 ? 16 : 64; }
int64_t gains_pieces(int64_t K) { return (K + 8 * gains_lanes(K) - 1) / (8 * gains_lanes(K)); }
template <typename T>
int64_t parts_of(int64_t N, int64_t K, bool with_dx)
{
    if (N == 0) return 0;
    if (with_dx && is_held(K) && !apart<T>(N, K)) return with_shape<T>(K / 8, [&](auto threads, auto held) { return groups_of(N, threads, back_waves<T>(held, true), true); });
    const int64_t rows = 256 / gains_lanes(K), groups = (N + rows - 1) / rows;
    return std::max<int64_t>(1, std::min<int64_t>(groups / 4, kCus * 4 / gains_pieces(K)));
}

// f(FULL, HELD): the eights that a lane holds, of a list, if `lanes` of them hold a row's.
template <int FULL, int HELD, int... MORE, typename F>
bool with_held(int64_t K, int lanes, const F &f)
{
    if (K / 8 <= lanes * HELD) {
        f(std::integral_constant<int, FULL>(), std::integral_constant<int, HELD>());
        return true;
    }
    if constexpr (sizeof...(MORE) > 0) return with_held<HELD, MORE...>(K, lanes, f);
    return false;
}
template <typename T, int LANES, int FULL, int HELD>
hipError_t launch_wave(const NormJob &job, bool drop, hipStream_t stream)
{
    constexpr int threads = wave_threads(HELD * sizeof(T)), rows = threads / LANES;
    constexpr size_t lds = 2 * (8 * LANES * HELD + 8) * sizeof(float);
    constexpr int64_t per_cu = std::min<int64_t>(2048 / threads, kLdsPerCu / lds);
    const dim3 grid((unsigned)std::min<int64_t>((job.N + rows - 1) / rows, kCus * per_cu));
    auto launch = [&](LdsLimit &limit, auto kernel) {
        const hipError_t e = allow_lds(limit, reinterpret_cast<const void *>(kernel), lds);
        if (e != hipSuccess) return e;
        kernel<<<grid, threads, lds, stream>>>(job);
        return hipGetLastError();
    };
    static LdsLimit limits[2];
    return drop ? launch(limits[1], norm_wave_kernel<T, LANES, FULL, HELD, true>) : launch(limits[0], norm_wave_kernel<T, LANES, FULL, HELD, false>);
}

template <typename T>
hipError_t norm(const NormJob &job, bool drop, hipStream_t stream)
{
    if (job.N >= kManyRows || job.K < kLeastHeld) {
        hipError_t e = hipSuccess;
        auto wave = [&](auto lanes) { return [&, lanes](auto full, auto held) { e = launch_wave<T, lanes, full, held>(job, drop, stream); }; };
        typedef std::integral_constant<int, 8> l8;
        typedef std::integral_constant<int, 16> l16;
        typedef std::integral_constant<int, 64> l64;
        if (with_held<0, 1, 2, 3>(job.K, 8, wave(l8())) || with_held<1, 2, 3, 4, 5>(job.K, 16, wave(l16())) ||
            with_held<1, 2, 3, 4, 5, 7, 8, 10, 12, 16, 20>(job.K, 64, wave(l64())))
            return e;
        // (32-bit numbers of longer rows have no room in a wavefront's registers. Each eight that not every lane has takes some more: with 24, 32 instead of all four, which
        // spills, 20000 x 16385 with dropout 417 us instead of 322)
        if constexpr (sizeof(T) == 2) {
            if (with_held<20, 24, 28, 30, 32>(job.K, 64, wave(l64()))) return e;
        }
    }
    if (is_held(job.K)) {
        with_shape<T>((job.K + 7) / 8, [&](auto threads, auto held) {
            const dim3 grid((unsigned)groups_of(job.N, threads, 4, false));
            if (drop) norm_kernel<T, threads, held, true><<<grid, group_threads(threads), 0, stream>>>(job);
            else norm_kernel<T, threads, held, false><<<grid, group_threads(threads), 0, stream>>>(job);
        });
        return hipGetLastError();
    }
    constexpr int64_t kMost = 1 << 21;          // workgroups of a launch
    for (int64_t n0 = 0; n0 < job.N; n0 += kMost) {
        NormJob part = job;
        part.X = static_cast<const T *>(job.X) + n0 * job.ldx;
        part.Y = static_cast<T *>(job.Y) + n0 * job.ldy;
        if (job.mean) part.mean = job.mean + n0;
        if (job.rstd) part.rstd = job.rstd + n0;
        part.dropout.first_row += (uint32_t)n0;
        norm_long_kernel<T><<<dim3((unsigned)std::min(kMost, job.N - n0)), kLongThreads, 0, stream>>>(part, drop);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t back_held(const BackJob &job, bool drop, bool gains, hipStream_t stream)
{
    with_shape<T>(job.K / 8, [&](auto threads, auto held) {
        const dim3 grid((unsigned)groups_of(job.N, threads, back_waves<T>(held, gains), gains));
        auto launch = [&](auto kernel) { kernel<<<grid, group_threads(threads), 0, stream>>>(job); };
        if (drop && gains) launch(back_kernel<T, threads, held, true, true>);
        else if (drop) launch(back_kernel<T, threads, held, true, false>);
        else if (gains) launch(back_kernel<T, threads, held, false, true>);
        else launch(back_kernel<T, threads, held, false, false>);
    });
    return hipGetLastError();
}
template <typename T>
hipError_t back_long(const BackJob &job, bool drop, hipStream_t stream)
{
    constexpr int64_t kMost = 1 << 21;          // workgroups of a launch
    for (int64_t n0 = 0; n0 < job.N; n0 += kMost) {
        BackJob part = job;
        part.X = static_cast<const T *>(job.X) + n0 * job.ldx;
        part.dY = static_cast<const T *>(job.dY) + n0 * job.ldy;
        part.dX = static_cast<T *>(job.dX) + n0 * job.ldd;
        part.mean = job.mean + n0;
        part.rstd = job.rstd + n0;
        part.dropout.first_row += (uint32_t)n0;
        back_long_kernel<T><<<dim3((unsigned)std::min(kMost, job.N - n0)), kLongThreads, 0, stream>>>(part, drop);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T>
hipError_t back(const BackJob &job, bool drop, hipStream_t stream)
{
    const bool gains = job.dgain != nullptr, held = is_held(job.K);
    const bool fused = gains && job.dX && held && !apart<T>(job.N, job.K);
    const int64_t parts = gains ? parts_of<T>(job.N, job.K, job.dX != nullptr) : 0;
    hipError_t e = hipSuccess;
    if (gains && !fused) {          // (first: dX may lie where dY is)
        const int64_t pieces = gains_pieces(job.K);
        const dim3 grid((unsigned)(parts * pieces));
        auto launch = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(job, (uint32_t)pieces); };
        if (job.K < kLeastHeld) drop ? launch(gains_kernel<T, 16, true, true>) : launch(gains_kernel<T, 16, false, true>);
        else if (gains_lanes(job.K) == 16) drop ? launch(gains_kernel<T, 16, true, false>) : launch(gains_kernel<T, 16, false, false>);
        else drop ? launch(gains_kernel<T, 64, true, false>) : launch(gains_kernel<T, 64, false, false>);
        e = hipGetLastError();
    }
    if (e == hipSuccess && job.dX) e = held ? back_held<T>(job, drop, fused, stream) : back_long<T>(job, drop, stream);
    if (e == hipSuccess && gains && parts > 1) {
        add_parts_kernel<<<dim3((unsigned)((2 * room_of(job.K) + kAddColumns - 1) / kAddColumns)), kAddThreads, 0, stream>>>(job.sums, parts, job.K, job.dgain, job.doffset);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t layer_norm_backward_bytes(const rfsf_layer_norm_shape &s, bool with_dx)
{
    const int64_t parts = s.bf16 ? parts_of<uint16_t>(s.N, s.K, with_dx) : parts_of<float>(s.N, s.K, with_dx);
    return (size_t)std::max<int64_t>(1, parts) * 2 * (size_t)room_of(s.K) * sizeof(float) + 256;
}

hipError_t launch_layer_norm(const rfsf_layer_norm_shape &s, const void *X, const float *gain, const float *offset, float eps, const rfsf_dropout_mask *mask, void *Y,
                             float *mean, float *rstd, hipStream_t stream)
{
    const NormJob job = {X, Y, gain, offset, mean, rstd, s.N, s.K, s.ld_x, s.ld_y, eps, dropout_job(mask)};
    return s.bf16 ? norm<uint16_t>(job, mask != nullptr, stream) : norm<float>(job, mask != nullptr, stream);
}

hipError_t launch_layer_norm_backward(const rfsf_layer_norm_shape &s, const void *X, const float *mean, const float *rstd, const float *gain, const void *dY,
                                      const rfsf_dropout_mask *mask, void *dX, float *dgain, float *doffset, void *workspace, hipStream_t stream)
{
    const size_t mis = (size_t)(reinterpret_cast<uintptr_t>(workspace) % 256);
    float *sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + (mis ? 256 - mis : 0));
    const BackJob job = {X, dY, dX, mean, rstd, gain, sums, dgain, doffset, s.N, s.K, s.ld_x, s.ld_y, s.ld_dx, dropout_job(mask)};
    return s.bf16 ? back<uint16_t>(job, mask != nullptr, stream) : back<float>(job, mask != nullptr, stream);
}

}  // namespace rfsf
