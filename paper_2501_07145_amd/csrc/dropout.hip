// Dropout of a matrix (dropout.h): one pass, the mask computed on the way.
#include <algorithm>

#include "../../include/rfsf_ts.h"
#include "dropout.h"
#include "rows8.h"

namespace rfsf {
namespace {

constexpr int kThreads = 512, kCus = 256;

// n / divisor for n < 2^31, as (n multiplier) >> shift: with 2^(shift - 31) >= divisor the product is too large by less than n / 2^31 of the divisor's part.
struct Division { uint32_t multiplier; int shift; };
Division division_by(uint32_t divisor)
{
    int shift = 31;
    while ((uint64_t)1 << (shift - 31) < divisor) ++shift;
    return {(uint32_t)((((uint64_t)1 << shift) + divisor - 1) / divisor), shift};
}

// A lane takes eight columns, counted through all rows, so that no lane is idle whatever the number of columns. Bound by memory (vector units busy 57 % of the cycles for
// bfloat16): 30000 x 5121, bfloat16 118 us (5.2 TB/s), 30000 x 10241, float32 447 to 460 (5.3 to 5.5 TB/s), 200003 x 65, bfloat16 15, 1000000 x 5, float32 22. (Two
// eights a lane 123 of the first, four 134; lanes that share a row, pieces of long ones, 127 of the first, 71 of the last.) Few eights go to workgroups of one wave, so
// that more CUs have some: 100 x 1025, float32 2.8 us, 3.1 with eight waves each.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutJob job, const T *X, int64_t ldx, int64_t K, T *Y, int64_t ldy, uint32_t eights, uint32_t total, Division division)
{
    const uint32_t at = blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= total) return;
    const uint32_t row = (uint32_t)((uint64_t)at * division.multiplier >> division.shift), group = at - row * eights;
    float x[8];
    rows8::load(X + row * ldx, (int64_t)group * 8, K, x);
    dropout::apply(job, dropout::offset_of(job), job.first_row + row, group, x);
    rows8::store(Y + row * ldy, (int64_t)group * 8, K, x);
}

template <typename T>
hipError_t launch(const DropoutJob &whole, const T *X, int64_t N, int64_t ldx, int64_t K, T *Y, int64_t ldy, hipStream_t stream)
{
    const int64_t eights = (K + 7) / 8, most = std::max<int64_t>(((int64_t)1 << 30) / eights, 1);        // rows of a launch
    const Division division = division_by((uint32_t)eights);
    DropoutJob job = whole;
    for (int64_t n0 = 0; n0 < N; n0 += most) {
        const int64_t total = std::min(N - n0, most) * eights;
        job.first_row = whole.first_row + (uint32_t)n0;
        const int threads = total < kCus * kThreads ? 64 : kThreads;
        dropout_kernel<T><<<dim3((unsigned)((total + threads - 1) / threads)), threads, 0, stream>>>(job, X + n0 * ldx, ldx, K, Y + n0 * ldy, ldy, (uint32_t)eights, (uint32_t)total, division);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_dropout(const rfsf_dropout_mask &mask, const void *X, bool bf16, int64_t N, int64_t ldx, int64_t K, void *Y, int64_t ldy, hipStream_t stream)
{
    const DropoutJob job = dropout_job(&mask);
    if (bf16) return launch(job, static_cast<const uint16_t *>(X), N, ldx, K, static_cast<uint16_t *>(Y), ldy, stream);
    return launch(job, static_cast<const float *>(X), N, ldx, K, static_cast<float *>(Y), ldy, stream);
}

}  // namespace rfsf
