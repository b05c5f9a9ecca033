// Gram of feature rows against rows held in 8-bit integers (rfsf_int8_gram): K[i, j] = sx_i sy_j sum_k qx[i, k] qy[j, k], with
// q = round(x (127 (1 / largest of the row))), ties to even, each operation rounded to 32 bits, and s = largest (1 / 127). The sums are exact integers (K < 133000 columns); what is rounded is
// x to its code, and the result to 32 bits.
#include "plane_product.h"

#include <algorithm>

#include "../../include/rfsf_ts.h"
#include "plane_pack.h"

namespace rfsf {
namespace {

constexpr float kLeast = 1.504632769052528e-36f;            // 2^-119: rows with nothing larger count as zero (127 / largest stays finite)

// A workgroup per row, which it reads twice (the second time from a cache): the largest magnitude, then the codes, 16 of them a lane,
// zeros up to the end of the last step. A row with an infinity or a NaN has the scale NaN.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(const T *X, int64_t K, int64_t ld, int8_t *codes, int64_t ld_codes, float *scales)
{
    __shared__ uint32_t part[4];
    const T *x = X + (int64_t)blockIdx.x * ld;
    uint32_t largest = 0;
    for (int64_t k = threadIdx.x; k < K; k += 256) largest = max(largest, __float_as_uint(plane::number(x[k])) & 0x7fffffffu);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = largest;
    __syncthreads();
    largest = max(max(part[0], part[1]), max(part[2], part[3]));
    const float top = __uint_as_float(largest);
    const bool finite = largest < 0x7f800000u;
    const float inverse = top < kLeast || !finite ? 0.f : (1.0f / top) * 127.0f;
    if (threadIdx.x == 0) scales[blockIdx.x] = finite ? top * (1.0f / 127.0f) : NAN;
    int8_t *q = codes + (int64_t)blockIdx.x * ld_codes;
    const int64_t end = (K + kStepBytes - 1) / kStepBytes * kStepBytes;
    for (int64_t k = 4 * (int64_t)threadIdx.x; k < end; k += 1024) {
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = k + e < K && inverse != 0.f ? rintf(plane::number(x[k + e]) * inverse) : 0.f;
            word |= ((uint32_t)(int)v & 0xffu) << (8 * e);
        }
        *reinterpret_cast<uint32_t *>(q + k) = word;
    }
}

// Rows of the tile: stored rows (contiguous in the result).
struct Scaled {
    float *out;
    int64_t ld, rows_i, cols_j;
    const float *scale_i, *scale_j;

    template <typename T>
    __device__ __forceinline__ void operator()(T &t) const
    {
        struct __attribute__((packed, aligned(4))) Float4u { float x, y, z, w; };
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        t.each_block([&](const auto &acc, int64_t first, int b) __attribute__((always_inline)) {
            const int64_t j = t.j0 + 32 * b + col;
            if (j >= cols_j) return;
            const float sj = scale_j[j];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t i = first + 8 * q + 4 * half;
                float *dst = out + j * ld + i;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)acc[4 * q + e] * (sj * (i + e < rows_i ? scale_i[i + e] : 0.f));
                if (i + 3 < rows_i) {
                    *reinterpret_cast<Float4u *>(dst) = {v[0], v[1], v[2], v[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < rows_i) dst[e] = v[e];
                }
            }
        });
    }
};

size_t up(size_t v) { return (v + 255) / 256 * 256; }
int64_t code_pitch(int64_t K) { return odd_steps(K); }
size_t row_bytes(int64_t rows, int64_t K) { return up((size_t)rows * code_pitch(K)) + up(4 * (size_t)rows); }
constexpr int64_t kMostRows = 1 << 20;      // quantised at a time

}  // namespace

hipError_t launch_int8_quantize(const void *X, bool bf16, int64_t N, int64_t ld, int64_t K, int8_t *codes, int64_t ld_codes, float *scales,
                                hipStream_t stream)
{
    if (bf16) quantize_kernel<uint16_t><<<dim3((unsigned)N), 256, 0, stream>>>(static_cast<const uint16_t *>(X), K, ld, codes, ld_codes, scales);
    else quantize_kernel<float><<<dim3((unsigned)N), 256, 0, stream>>>(static_cast<const float *>(X), K, ld, codes, ld_codes, scales);
    return hipGetLastError();
}

void int8_gram_bytes(int64_t Nx, int64_t K, size_t *recommended, size_t *minimum)
{
    *recommended = row_bytes(std::min(std::max<int64_t>(Nx, 1), kMostRows), K) + 256;
    *minimum = row_bytes(1, K) + 256;
}

hipError_t launch_int8_gram(const void *X, bool bf16, int64_t Nx, int64_t ldx, const int8_t *codes, const float *scales, int64_t Ny, int64_t ldy,
                            int64_t K, float *out, int64_t ldk, void *workspace, size_t bytes, hipStream_t stream)
{
    const size_t mis = (size_t)(reinterpret_cast<uintptr_t>(workspace) % 256), room = bytes - 256;
    int64_t most = std::min<int64_t>(Nx, kMostRows);
    while (most > 1 && row_bytes(most, K) > room) most = (most + 1) / 2;
    char *ws = static_cast<char *>(workspace) + (mis ? 256 - mis : 0);
    int8_t *qx = reinterpret_cast<int8_t *>(ws);
    float *sx = reinterpret_cast<float *>(ws + up((size_t)most * code_pitch(K)));
    const size_t element = bf16 ? 2 : 4;
    for (int64_t n0 = 0; n0 < Nx; n0 += most) {
        const int64_t rows = std::min(most, Nx - n0);
        hipError_t e = launch_int8_quantize(static_cast<const char *>(X) + (size_t)n0 * ldx * element, bf16, rows, ldx, K, qx, code_pitch(K), sx, stream);
        if (e != hipSuccess) return e;
        const Scaled epilogue = {out + n0 * ldk, ldk, Ny, rows, scales, sx};
        e = launch_plane_product<kInt8>(Planes{reinterpret_cast<const char *>(codes), ldy, Ny}, Planes{reinterpret_cast<const char *>(qx), code_pitch(K), rows},
                                        (K + kStepBytes - 1) / kStepBytes, plane_tile(Ny, rows), epilogue, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rfsf
