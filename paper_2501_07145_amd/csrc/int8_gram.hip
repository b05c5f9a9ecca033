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

// What brings a row whose largest magnitude has these bits to its codes, and the scale.
__device__ __forceinline__ float inverse_of(uint32_t largest, float *scale)
{
    const float top = __uint_as_float(largest);
    const bool finite = largest < 0x7f800000u;
    *scale = finite ? top * (1.0f / 127.0f) : NAN;
    return top < kLeast || !finite ? 0.f : (1.0f / top) * 127.0f;
}
// A sum of products of codes times both scales, the smaller scale first: nothing on the way is beyond what 32 bits hold unless the result is. (The product of
// the scales may be: two scales of 2^95 made a sum of zero NaN, two of 2^-75 lost everything.) Scales that are NaN stay.
__device__ __forceinline__ float scaled(int sum, float a, float b)
{
    const bool less = a < b;
    return ((float)sum * (less ? a : b)) * (less ? b : a);
}
template <int PER>
__device__ __forceinline__ void store_codes(int8_t *q, const float (&v)[PER], float inverse)
{
    uint32_t word[PER / 4];
#pragma unroll
    for (int w = 0; w < PER / 4; ++w) {
        word[w] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) word[w] |= ((uint32_t)(int)(inverse != 0.f ? rintf(v[4 * w + e] * inverse) : 0.f) & 0xffu) << (8 * e);
    }
    if constexpr (PER == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(word[0], word[1]);
    else *reinterpret_cast<uint32_t *>(q) = word[0];
}

// A workgroup per row, or a wavefront for many rows of up to kNarrow columns: the largest magnitude, then the codes, zeros up to the end of the last step. Rows of up to
// HELD loads a lane are read once, 16 bytes a lane and load, and stay in registers; of longer ones what lies beyond is read again. A row with an infinity or a
// NaN has the scale NaN. Bound by reading X: 5000 x 10241, float32, 47 us (5.4 TB/s).
constexpr int kQuantizeThreads = 512;
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Chunk { T v[16 / sizeof(T)]; };
// (us, a workgroup and a wavefront: 1000 x 193, bfloat16 5.1 and 6.1; 1000 x 513, float32 5.4 and 5.8; 20000 x 1024, float32 34 and 18; 200000 x 300, float32
// 302 and 73; 1000000 x 65, bfloat16 1447 and 292.)
constexpr int64_t kNarrow = 1024, kManyNarrow = 4096;
template <typename T, int HELD, int THREADS>
__global__ __launch_bounds__(kQuantizeThreads) void quantize_kernel(const T *X, int64_t N, int64_t K, int64_t ld, int8_t *codes, int64_t ld_codes, float *scales)
{
    constexpr int PER = 16 / sizeof(T), STEP = PER * THREADS, ROWS = kQuantizeThreads / THREADS;
    static_assert(THREADS == 64 || ROWS == 1, "");
    const int thread = ROWS == 1 ? threadIdx.x : threadIdx.x % THREADS;
    const int64_t row = ROWS == 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / THREADS));
    if (ROWS > 1 && row >= N) return;
    const T *x = X + row * ld;
    auto load = [&](int64_t k, float (&v)[PER]) {
        if (k + PER <= K) {
            const Chunk<T> c = *reinterpret_cast<const Chunk<T> *>(x + k);
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = plane::number(c.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = k + e < K ? plane::number(x[k + e]) : 0.f;
        }
    };
    float held[HELD][PER];
    uint32_t largest = 0;
    const int64_t first = (int64_t)thread * PER;
#pragma unroll
    for (int u = 0; u < HELD; ++u) load(first + u * STEP, held[u]);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < PER; ++e) largest = max(largest, __float_as_uint(held[u][e]) & 0x7fffffffu);
    for (int64_t k = first + HELD * STEP; k < K; k += STEP) {
        float v[PER];
        load(k, v);
#pragma unroll
        for (int e = 0; e < PER; ++e) largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
    if constexpr (ROWS == 1) {
        __shared__ uint32_t part[kQuantizeThreads / 64];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantizeThreads / 64; ++w) largest = max(largest, part[w]);
    }
    float scale;
    const float inverse = inverse_of(largest, &scale);
    if (thread == 0) scales[row] = scale;
    int8_t *q = codes + row * ld_codes;
    const int64_t end = (K + kStepBytes - 1) / kStepBytes * kStepBytes;
    auto store = [&](int64_t k, const float (&v)[PER]) {
        if (k < end) store_codes<PER>(q + k, v, inverse);
    };
#pragma unroll
    for (int u = 0; u < HELD; ++u) store(first + u * STEP, held[u]);
    for (int64_t k = first + HELD * STEP; k < end; k += STEP) {
        float v[PER];
        load(k, v);
        store(k, v);
    }
}

// Up to 16 rows of X against 16 BM stored rows a workgroup (blocks of 16 x 16, v_mfma_i32_16x16x64_i8: lane l holds 16 columns, a
// quarter of 64, of row l % 16), straight from memory to registers. The wavefronts share out the columns, AHEAD steps of 128 bytes, a cache line
// of each row, at a time, and add their sums up in LDS. What bounds it is reading the stored rows once, and with more rows of X
// the cache lines of these, which every workgroup reads again.
// 50000 x 10241 codes, us: 4 rows 91 (5.65 TB/s), 9 rows 98, 16 rows 112; four wavefronts a workgroup instead of two, one step each, 103 with 7
// rows, wavefronts with stored rows of their own 118 and more. 1000 x 1025 codes 2.9, with two wavefronts 3.4; 1000 x 10241 7.7 and 12.5.
typedef int intx4 __attribute__((ext_vector_type(4)));
constexpr int kFewRows = 16;
template <int BM, int AHEAD, int NW>
__global__ __launch_bounds__(64 * NW) void few_rows_kernel(const int8_t *qx, int64_t pitch_x, const float *sx, int64_t Nx, const int8_t *codes, int64_t ld,
                                                          const float *scales, int64_t Ny, int64_t steps, float *out, int64_t ld_out)
{
    static_assert(BM <= NW, "a wavefront for every block");
    __shared__ int shared[BM * NW * 4 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
    const int64_t j0 = (int64_t)blockIdx.x * (16 * BM);
    const int8_t *x = qx + (col < Nx ? col : Nx - 1) * pitch_x + 16 * quarter;           // rows that do not exist are the last one, and not stored
    const int8_t *y[BM];
#pragma unroll
    for (int a = 0; a < BM; ++a) y[a] = codes + std::min(j0 + 16 * a + col, Ny - 1) * ld + 16 * quarter;
    intx4 acc[BM];
#pragma unroll
    for (int a = 0; a < BM; ++a) acc[a] = intx4{0, 0, 0, 0};
    for (int64_t s = AHEAD * wave; s < steps; s += AHEAD * NW) {
        intx4 fx[AHEAD][2], fy[AHEAD][BM][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t at = std::min(s + u, steps - 1) * kStepBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int a = 0; a < BM; ++a) fy[u][a][h] = *reinterpret_cast<const intx4 *>(y[a] + at + 64 * h);
                fx[u][h] = *reinterpret_cast<const intx4 *>(x + at + 64 * h);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (s + u >= steps) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int a = 0; a < BM; ++a) acc[a] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fy[u][a][h], fx[u][h], acc[a], 0, 0, 0);
        }
    }
#pragma unroll
    for (int a = 0; a < BM; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) shared[((a * NW + wave) * 4 + e) * 64 + lane] = acc[a][e];
    __syncthreads();
    if (wave >= BM || col >= Nx) return;
    const float s = sx[col];
    const int64_t first = j0 + 16 * wave + 4 * quarter;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += shared[((wave * NW + w) * 4 + e) * 64 + lane];
        if (first + e < Ny) out[col * ld_out + first + e] = scaled(sum, s, scales[first + e]);
    }
}
template <int BM, int AHEAD, int NW>
void launch_few_rows(const int8_t *qx, int64_t pitch_x, const float *sx, int64_t Nx, const int8_t *codes, int64_t ld, const float *scales, int64_t Ny,
                     int64_t steps, float *out, int64_t ld_out, hipStream_t stream)
{
    few_rows_kernel<BM, AHEAD, NW><<<dim3((unsigned)((Ny + 16 * BM - 1) / (16 * BM))), 64 * NW, 0, stream>>>(qx, pitch_x, sx, Nx, codes, ld, scales, Ny, steps,
                                                                                                         out, ld_out);
}

// The same for rows of X of kHeldCodes columns altogether, quantised by every workgroup for itself into LDS: one launch instead of two, where there
// are few workgroups and the second launch is what counts (1 x 1025 against 1000: 5.5 us for the kernel, 7.6 for the call; 6.0 for the two kernels).
constexpr int kHeldCodes = 8192, kHeldPad = 16;          // (rows 16 bytes apart in their banks)
template <typename T>
__global__ __launch_bounds__(256) void few_small_kernel(const T *X, int64_t ldx, int Nx, int K, const int8_t *codes, int64_t ld, const float *scales,
                                                        int64_t Ny, float *out, int64_t ld_out)
{
    constexpr int PER = 16 / sizeof(T), NW = 4;
    __shared__ __attribute__((aligned(16))) int8_t held[kHeldCodes + kFewRows * (kStepBytes + kHeldPad)];
    __shared__ int shared[NW * 4 * 64];
    __shared__ float sx[kFewRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
    const int steps = (K + kStepBytes - 1) / kStepBytes, pitch = steps * kStepBytes + kHeldPad;
    const int64_t j0 = (int64_t)blockIdx.x * 16;
    const int8_t *y = codes + std::min(j0 + col, Ny - 1) * ld + 16 * quarter;
    auto load = [&](const T *x, int k, float (&v)[PER]) {
        if (k + PER <= K) {
            const Chunk<T> c = *reinterpret_cast<const Chunk<T> *>(x + k);
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = plane::number(c.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = k + e < K ? plane::number(x[k + e]) : 0.f;
        }
    };
    for (int n = wave; n < Nx; n += NW) {
        const T *x = X + n * ldx;
        uint32_t largest = 0;
        for (int k = PER * lane; k < K; k += PER * 64) {
            float v[PER];
            load(x, k, v);
#pragma unroll
            for (int e = 0; e < PER; ++e) largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o));
        float scale;
        const float inverse = inverse_of(largest, &scale);
        if (lane == 0) sx[n] = scale;
        for (int k = PER * lane; k < steps * kStepBytes; k += PER * 64) {
            float v[PER];
            load(x, k, v);
            store_codes<PER>(held + n * pitch + k, v, inverse);
        }
    }
    __syncthreads();
    const int8_t *x = held + (col < Nx ? col : Nx - 1) * pitch + 16 * quarter;
    intx4 acc = {0, 0, 0, 0};
    for (int s = wave; s < steps; s += NW) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const intx4 *>(y + s * kStepBytes + 64 * h),
                                                        *reinterpret_cast<const intx4 *>(x + s * kStepBytes + 64 * h), acc, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) shared[(wave * 4 + e) * 64 + lane] = acc[e];
    __syncthreads();
    if (wave >= 1 || col >= Nx) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += shared[(w * 4 + e) * 64 + lane];
        const int64_t j = j0 + 4 * quarter + e;
        if (j < Ny) out[col * ld_out + j] = scaled(sum, sx[col], scales[j]);
    }
}

// More rows: the product of packed operands. Rows of the tile: stored rows (contiguous in the result). 333 x 10000 x 5121 36 us (940 TOP/s, 237 tiles of 128:
// one round that does not fill the CUs), 5000 x 50000 x 10241 2.43 to 2.56 ms (2000 to 2110 TOP/s).
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
                for (int e = 0; e < 4; ++e) v[e] = scaled(acc[4 * q + e], sj, i + e < rows_i ? scale_i[i + e] : 0.f);
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
constexpr int64_t kMostQuantized = 1 << 22; // rows of a launch
constexpr int64_t kManyStored = 16384;      // stored rows that make workgroups enough of two wavefronts

}  // namespace

hipError_t launch_int8_quantize(const void *X, bool bf16, int64_t N, int64_t ld, int64_t K, int8_t *codes, int64_t ld_codes, float *scales,
                                hipStream_t stream)
{
    // registers for the columns that there are; a launch has fewer than 2^32 threads
    const bool narrow = K <= kNarrow && N >= kManyNarrow;
    for (int64_t n0 = 0; n0 < N; n0 += kMostQuantized) {
        const int64_t rows = std::min(N - n0, kMostQuantized);
        auto launch = [&](auto kernel, const auto *x, int64_t rows_of_group) {
            kernel<<<dim3((unsigned)((rows + rows_of_group - 1) / rows_of_group)), kQuantizeThreads, 0, stream>>>(x + n0 * ld, rows, K, ld, codes + n0 * ld_codes, ld_codes,
                                                                                                                 scales + n0);
        };
        if (bf16) {
            const uint16_t *x = static_cast<const uint16_t *>(X);
            if (narrow) launch(quantize_kernel<uint16_t, kNarrow / 512, 64>, x, kQuantizeThreads / 64);
            else if (K <= 8 * kQuantizeThreads) launch(quantize_kernel<uint16_t, 1, kQuantizeThreads>, x, 1);
            else launch(quantize_kernel<uint16_t, 3, kQuantizeThreads>, x, 1);
        } else {
            const float *x = static_cast<const float *>(X);
            if (narrow) launch(quantize_kernel<float, kNarrow / 256, 64>, x, kQuantizeThreads / 64);
            else if (K <= 8 * kQuantizeThreads) launch(quantize_kernel<float, 2, kQuantizeThreads>, x, 1);
            else launch(quantize_kernel<float, 6, kQuantizeThreads>, x, 1);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

void int8_gram_bytes(int64_t Nx, int64_t K, size_t *recommended, size_t *minimum)
{
    *recommended = row_bytes(std::min(std::max<int64_t>(Nx, 1), kMostRows), K) + 256;
    *minimum = row_bytes(1, K) + 256;
}

hipError_t launch_int8_gram(const void *X, bool bf16, int64_t Nx, int64_t ldx, const int8_t *codes, const float *scales, int64_t Ny, int64_t ldy,
                            int64_t K, float *out, int64_t ldk, void *workspace, size_t bytes, hipStream_t stream)
{
    if (Nx <= kFewRows && Nx * K <= kHeldCodes && Ny < kManyStored) {
        const dim3 grid((unsigned)((Ny + 15) / 16));
        if (bf16) few_small_kernel<uint16_t><<<grid, 256, 0, stream>>>(static_cast<const uint16_t *>(X), ldx, (int)Nx, (int)K, codes, ldy, scales, Ny, out, ldk);
        else few_small_kernel<float><<<grid, 256, 0, stream>>>(static_cast<const float *>(X), ldx, (int)Nx, (int)K, codes, ldy, scales, Ny, out, ldk);
        return hipGetLastError();
    }
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
        const int64_t steps = (K + kStepBytes - 1) / kStepBytes;
        if (rows <= kFewRows) {
            auto launch = Ny < kManyStored ? launch_few_rows<1, 1, 4> : rows <= 9 ? launch_few_rows<1, 2, 2> : launch_few_rows<2, 1, 2>;
            launch(qx, code_pitch(K), sx, rows, codes, ldy, scales, Ny, steps, out + n0 * ldk, ldk, stream);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            continue;
        }
        const Scaled epilogue = {out + n0 * ldk, ldk, Ny, rows, scales, sx};
        e = launch_plane_product<kInt8>(Planes{reinterpret_cast<const char *>(codes), ldy, Ny}, Planes{reinterpret_cast<const char *>(qx), code_pitch(K), rows},
                                        steps, plane_tile(Ny, rows), epilogue, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rfsf
