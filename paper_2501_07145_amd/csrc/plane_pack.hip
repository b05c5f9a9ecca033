// The largest magnitudes of matrices' rows, and the packing of matrices and their transposes (plane_pack.h). Both are bound by
// memory: a matrix is read twice, each operand written once.
#include "plane_pack.h"

#include <algorithm>

namespace rfsf {
namespace {

constexpr int kEdge = 64;                 // of a tile that is packed
constexpr int kRowsPerGroup = 4;          // rows of a workgroup that searches, one a wavefront

// A wavefront takes a row, four numbers of it a lane and step.
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
        for (int64_t k = lane; k < job.K; k += 256) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k + 64 * u < job.K) largest = max(largest, __float_as_uint(plane::number(src[k + 64 * u])) & 0x7fffffffu);
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
    const int64_t c = c0 + lane;
#pragma unroll 4
    for (int r = wave; r < kEdge; r += 4) {
        const int64_t row = r0 + r;
        const bool there = row < job.R && c < job.K && !(job.labels && job.labels[row] < 0);
        tile[r][lane] = there ? ldexpf(plane::number(src[row * job.ld + c]), shift_of(job.largest[row])) : 0.f;
    }
    __syncthreads();
    const int at = threadIdx.x >> 3, group = threadIdx.x & 7;       // a row (column) of the tile and eight numbers of it
#pragma unroll
    for (int u = 0; u < kEdge; u += 32) {
        float x[8];
        if (r0 + at + u < job.R) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = tile[at + u][8 * group + e];
            plane::store_terms<TWO>(job.rows + (r0 + at + u) * job.pitch_rows, c0 + 8 * group, plane::terms_of<TWO>(x));
        }
        if (job.columns && c0 + at + u < job.K) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = tile[8 * group + e][at + u];
            plane::store_terms<TWO>(job.columns + (c0 + at + u) * job.pitch_columns, r0 + 8 * group, plane::terms_of<TWO>(x));
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
