// The largest magnitudes of matrices' rows, and the packing of matrices and their transposes (plane_pack.h). Both are bound by
// memory: a matrix is read twice, each operand written once; by rows alone, once. 8192 x 2049 and 32768 x 2049, bfloat16, by rows and transposed: largest 48 us
// (3.5 TB/s), packing 102 us (4.9 TB/s).
#include "plane_pack.h"

#include <algorithm>

namespace rfsf {
namespace {

constexpr int kEdge = 64;                 // of a tile that is packed
constexpr int kRowsPerGroup = 4;          // rows of a workgroup that searches, one a wavefront

// Eight numbers of a row from k on.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };
template <typename T>
__device__ __forceinline__ void load8(const T *row, int64_t k, int64_t K, float (&x)[8])
{
    if (k + 8 <= K) {
        const Eight<T> c = *reinterpret_cast<const Eight<T> *>(row + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = plane::number(c.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < K ? plane::number(row[k + e]) : 0.f;
    }
}

__device__ __forceinline__ int64_t source_row(const PackJob &job, int64_t row) { return job.order ? job.order[row] : row; }

// A wavefront takes a row, eight numbers of it a lane and load, two loads at a time.
template <typename T>
__global__ __launch_bounds__(64 * kRowsPerGroup) void largest_kernel(PackPair pair, unsigned groups_of_first)
{
    const bool second = blockIdx.x >= groups_of_first;
    const PackJob &job = pair.job[second ? 1 : 0];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (pair.stats && blockIdx.x == 0 && threadIdx.x == 0) *pair.stats = {0, 0};
    const int64_t row = (int64_t)(blockIdx.x - (second ? groups_of_first : 0)) * kRowsPerGroup + wave;
    if (row >= job.R) return;
    uint32_t largest = 0;
    if (!(job.labels && job.labels[row] < 0)) {
        const T *src = static_cast<const T *>(job.src) + source_row(job, row) * job.ld;
        for (int64_t k = 8 * lane; k < job.K; k += 1024) {
            float x[2][8];
            load8(src, k, job.K, x[0]);
            load8(src, k + 512, job.K, x[1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = max(largest, max(__float_as_uint(x[0][e]) & 0x7fffffffu, __float_as_uint(x[1][e]) & 0x7fffffffu));
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
    }
    if (lane == 0) job.largest[row] = largest;
}

template <typename T, bool TWO>
__global__ __launch_bounds__(256) void pack_kernel(PackPair pair, unsigned tiles_of_first)
{
    __shared__ float tile[kEdge][kEdge + 1];
    const bool second = blockIdx.x >= tiles_of_first;
    const PackJob &job = pair.job[second ? 1 : 0];
    const unsigned id = blockIdx.x - (second ? tiles_of_first : 0), across = (unsigned)((job.K + kEdge - 1) / kEdge);
    const int64_t r0 = (int64_t)(id / across) * kEdge, c0 = (int64_t)(id % across) * kEdge;
    const T *src = static_cast<const T *>(job.src);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int at = threadIdx.x >> 3, group = threadIdx.x & 7;       // a row (column) of the tile and eight numbers of it
    float x[kEdge / 32][8];
    int shift[kEdge / 32];
#pragma unroll
    for (int u = 0; u < kEdge / 32; ++u) {
        const int64_t row = r0 + at + 32 * u;
        const bool there = row < job.R && !(job.labels && job.labels[row] < 0);
        shift[u] = there ? shift_of(job.largest[row]) : 0;
        if (there) {
            load8(src + source_row(job, row) * job.ld, c0 + 8 * group, job.K, x[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < kEdge / 32; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = ldexpf(x[u][e], shift[u]);
        const int64_t row = r0 + at + 32 * u;
        if (row < job.R) plane::store_terms<TWO>(job.rows + row * job.pitch_rows, c0 + 8 * group, plane::terms_of<TWO>(x[u]));
        if (job.columns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[at + 32 * u][8 * group + e] = x[u][e];
        }
    }
    if (job.columns) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kEdge; u += 32) {
            if (c0 + at + u >= job.K) break;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = tile[8 * group + e][at + u];
            plane::store_terms<TWO>(job.columns + (c0 + at + u) * job.pitch_columns, r0 + 8 * group, plane::terms_of<TWO>(y));
        }
    }
    if (second && pair.stats && c0 == 0 && wave == 0) {             // the rows of this tile
        const int64_t row = r0 + lane;
        const bool counts = row < job.R && job.labels[row] >= 0;
        uint32_t top = 0;
        if (counts) {
            const int e = exponent_of(job.largest[row]) + (pair.weight ? exponent_of(__float_as_uint(pair.weight[row])) : 0);
            top = (uint32_t)(e + kTopBias);
        }
        const uint32_t count = (uint32_t)__popcll(__ballot(counts));
#pragma unroll
        for (int o = 32; o > 0; o /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (lane == 0 && count != 0) {
            atomicAdd(&pair.stats->count, count);
            atomicMax(&pair.stats->top, top);
        }
    }
}

// Packing by rows alone (no transposes, no statistics): a workgroup, or a wavefront for up to kNarrowRow columns, holds a row in registers, so that it
// is read once and in one launch. 10000 x 5121 and 5003 x 5121, float32 96 us (6.4 TB/s), with two launches 54 and 112; a call without gradients 1.10 times
// as fast over 13 shapes (2000 x 9000, 2000 classes, bfloat16 133 us and 111; 1000 x 1025, 1000, float32 31.0 and 29.6).
constexpr int kRowThreads = 512;
constexpr int64_t kNarrowRow = 1024;
template <typename T, bool TWO, int HELD, int THREADS>
__global__ __launch_bounds__(kRowThreads) void pack_rows_kernel(PackPair pair, unsigned groups_of_first)
{
    constexpr int ROWS = kRowThreads / THREADS, STEP = 8 * THREADS;
    static_assert(THREADS == 64 || ROWS == 1, "");
    const bool second = blockIdx.x >= groups_of_first;
    const PackJob &job = pair.job[second ? 1 : 0];
    const int thread = ROWS == 1 ? threadIdx.x : threadIdx.x % THREADS;
    const int64_t group = blockIdx.x - (second ? groups_of_first : 0);
    const int64_t row = ROWS == 1 ? group : group * ROWS + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / THREADS));
    if (ROWS > 1 && row >= job.R) return;
    const bool there = !(job.labels && job.labels[row] < 0);
    const T *src = static_cast<const T *>(job.src) + source_row(job, row) * job.ld;
    float x[HELD][8];
    uint32_t largest = 0;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
        if (there) {
            load8(src, (int64_t)8 * thread + u * STEP, job.K, x[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(x[u][e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
    if constexpr (ROWS == 1) {
        __shared__ uint32_t part[kRowThreads / 64];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kRowThreads / 64; ++w) largest = max(largest, part[w]);
    }
    if (thread == 0) job.largest[row] = largest;
    const int shift = shift_of(largest);
    const int64_t end = (job.K + 63) / 64 * 64;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
        const int64_t k = (int64_t)8 * thread + u * STEP;
        if (k >= end) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = ldexpf(x[u][e], shift);
        plane::store_terms<TWO>(job.rows + row * job.pitch_rows, k, plane::terms_of<TWO>(x[u]));
    }
}
template <typename T, bool TWO>
void launch_rows(const PackPair &pair, hipStream_t stream)
{
    const int64_t K = pair.job[0].K, per = K <= kNarrowRow ? kRowThreads / 64 : 1;
    const unsigned first = (unsigned)((pair.job[0].R + per - 1) / per), all = first + (unsigned)((pair.job[1].R + per - 1) / per);
    if (per > 1) pack_rows_kernel<T, TWO, 2, 64><<<dim3(all), kRowThreads, 0, stream>>>(pair, first);
    else if (K <= 8 * kRowThreads) pack_rows_kernel<T, TWO, 1, kRowThreads><<<dim3(all), kRowThreads, 0, stream>>>(pair, first);
    else pack_rows_kernel<T, TWO, 3, kRowThreads><<<dim3(all), kRowThreads, 0, stream>>>(pair, first);
}

unsigned groups(const PackJob &job) { return (unsigned)((job.R + kRowsPerGroup - 1) / kRowsPerGroup); }
unsigned tiles(const PackJob &job) { return (unsigned)(((job.R + kEdge - 1) / kEdge) * ((job.K + kEdge - 1) / kEdge)); }

}  // namespace

hipError_t launch_largest(const PackPair &pair, bool bf16, hipStream_t stream)
{
    const unsigned first = groups(pair.job[0]), all = first + groups(pair.job[1]);
    if (bf16) largest_kernel<uint16_t><<<dim3(all), 64 * kRowsPerGroup, 0, stream>>>(pair, first);
    else largest_kernel<float><<<dim3(all), 64 * kRowsPerGroup, 0, stream>>>(pair, first);
    return hipGetLastError();
}

hipError_t launch_pack(const PackPair &pair, bool bf16, hipStream_t stream)
{
    const unsigned first = tiles(pair.job[0]), all = first + tiles(pair.job[1]);
    if (bf16) pack_kernel<uint16_t, false><<<dim3(all), 256, 0, stream>>>(pair, first);
    else pack_kernel<float, true><<<dim3(all), 256, 0, stream>>>(pair, first);
    return hipGetLastError();
}

hipError_t launch_pack_rows(const PackPair &pair, bool bf16, hipStream_t stream)
{
    static_assert(kPackRowsColumns == 3 * 8 * kRowThreads && kNarrowRow == 2 * 8 * 64, "");
    if (bf16) launch_rows<uint16_t, false>(pair, stream);
    else launch_rows<float, true>(pair, stream);
    return hipGetLastError();
}

}  // namespace rfsf
