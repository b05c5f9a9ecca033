// Dropout of a matrix (dropout.h): one pass, the mask computed on the way.
#include <algorithm>

#include "../../include/rfsf_ts.h"
#include "dropout.h"
#include "rows8.h"

namespace rfsf {
namespace {

constexpr int kThreads = 256, kUnroll = 2;
constexpr int64_t kMostGroups = 1 << 23;        // a launch has fewer than 2^32 threads

// THREADS of a workgroup share a row, kUnroll times eight numbers each; longer rows are worked on in pieces of that many. Bound by memory, at its rate with the
// vector units busy 77 % of the cycles: 30000 x 5121, bfloat16 127 us (4.8 TB/s); 30000 x 10241, float32 445 us (5.5 TB/s); 100 x 1025 2.8 us.
template <typename T, int THREADS>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutJob job, const T *X, int64_t N, int64_t ldx, int64_t K, T *Y, int64_t ldy, uint32_t pieces)
{
    constexpr int ROWS = kThreads / THREADS;
    const uint32_t piece = blockIdx.x % pieces;
    const int64_t row = (int64_t)(blockIdx.x / pieces) * ROWS + threadIdx.x / THREADS;
    if (row >= N) return;
    const uint64_t offset = dropout::offset_of(job);
    const int64_t first = ((int64_t)piece * kUnroll * THREADS + threadIdx.x % THREADS) * 8;
    float x[kUnroll][8];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) rows8::load(X + row * ldx, first + 8 * u * THREADS, K, x[u]);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t k = first + 8 * u * THREADS;
        if (k >= K) break;
        dropout::apply(job, offset, job.first_row + (uint32_t)row, (uint32_t)(k / 8), x[u]);
        rows8::store(Y + row * ldy, k, K, x[u]);
    }
}

template <typename T, int THREADS>
hipError_t launch(const DropoutJob &whole, const T *X, int64_t N, int64_t ldx, int64_t K, T *Y, int64_t ldy, hipStream_t stream)
{
    constexpr int ROWS = kThreads / THREADS;
    const int64_t pieces = (K + 8 * kUnroll * THREADS - 1) / (8 * kUnroll * THREADS), most = std::max<int64_t>(kMostGroups / pieces, 1) * ROWS;
    DropoutJob job = whole;
    for (int64_t n0 = 0; n0 < N; n0 += most) {
        const int64_t rows = std::min(N - n0, most);
        job.first_row = whole.first_row + (uint32_t)n0;
        dropout_kernel<T, THREADS><<<dim3((unsigned)((rows + ROWS - 1) / ROWS * pieces)), kThreads, 0, stream>>>(job, X + n0 * ldx, rows, ldx, K, Y + n0 * ldy,
                                                                                                            ldy, (uint32_t)pieces);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T>
hipError_t launch_of(const DropoutJob &job, const T *X, int64_t N, int64_t ldx, int64_t K, T *Y, int64_t ldy, hipStream_t stream)
{
    const int64_t eights = (K + 7) / 8;
    if (eights <= 16 * kUnroll) return launch<T, 16>(job, X, N, ldx, K, Y, ldy, stream);
    if (eights <= 64 * kUnroll) return launch<T, 64>(job, X, N, ldx, K, Y, ldy, stream);
    return launch<T, 256>(job, X, N, ldx, K, Y, ldy, stream);
}

}  // namespace

hipError_t launch_dropout(const rfsf_dropout_mask &mask, const void *X, bool bf16, int64_t N, int64_t ldx, int64_t K, void *Y, int64_t ldy, hipStream_t stream)
{
    const DropoutJob job = dropout_job(&mask);
    if (bf16) return launch_of(job, static_cast<const uint16_t *>(X), N, ldx, K, static_cast<uint16_t *>(Y), ldy, stream);
    return launch_of(job, static_cast<const float *>(X), N, ldx, K, static_cast<float *>(Y), ldy, stream);
}

}  // namespace rfsf
