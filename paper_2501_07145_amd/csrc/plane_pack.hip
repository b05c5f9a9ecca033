// The largest magnitudes of matrices' rows, and the packing of matrices and their transposes (plane_pack.h). Both are bound by
// memory: a matrix is read twice, each operand written once. 10000 x 5121 and 5003 x 5121, float32, by rows alone: largest 54 us (5.7 TB/s), packing 112 us
// (5.5 TB/s); 8192 x 2049 and 32768 x 2049, bfloat16, by rows and transposed: 48 us (3.5 TB/s) and 102 us (4.9 TB/s).
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
        const T *src = static_cast<const T *>(job.src) + row * job.ld;
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
            load8(src + row * job.ld, c0 + 8 * group, job.K, x[u]);
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

}  // namespace rfsf
