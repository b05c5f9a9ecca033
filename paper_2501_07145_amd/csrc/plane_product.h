// Products C[j, i] = sum_k A[i, k] B[j, k] on the 16-bit and 8-bit matrix instructions, for operands that lie packed in memory.
//
// A packed operand has rows of `pitch` bytes, a row being a series of steps of 128 bytes, which hold
//   kHalf     64 columns of 16-bit floating point;
//   kHalfTwo  32 columns of two terms: 64 bytes of the rounded numbers, then 64 bytes of what rounding left over. The product
//             of a pair of numbers is lo*hi + hi*lo + hi*hi, accumulated in 32 bits in this order (lo*lo is below 2^-22 of it);
//   kInt8     128 columns of 8-bit integers, accumulated exactly in 32 bits.
// Columns beyond the operands' are zero in one of the two at least (kInt8) or in both. All three ways move the same bytes from
// memory through LDS into registers and differ in the matrix instructions alone: a lane's 16 bytes are 8 or 16 consecutive columns of one row.
//
// Tile TM x TN, WM x WN wavefronts, blocks of 32 x 32. A step of the tile goes from memory straight into LDS (16 bytes a
// lane), into the buffer that the step before last used, while the step that arrived before is multiplied: one barrier a
// step. LDS: row r's 128 bytes are 8 chunks of 16, chunk c at place c ^ (r & 7), so that 8 lanes that read the same chunk of 8
// rows meet all banks once (and the permutation is made by the loads' addresses, at no cost).
#pragma once

#include "rfsf_internal.h"

namespace rfsf {

enum PlaneMode { kHalf = 0, kHalfTwo = 1, kInt8 = 2 };
constexpr int kStepBytes = 128;

struct Planes {
    const char *data;
    int64_t pitch;          // bytes from row to row
    int64_t rows;           // >= 1; rows beyond are read as the last one, and what they give is not stored
};

namespace plane {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

template <PlaneMode MODE> struct Acc { typedef floatx16 type; };
template <> struct Acc<kInt8> { typedef intx16 type; };

__device__ __forceinline__ floatx16 mfma(const intx4 &a, const intx4 &b, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}
__device__ __forceinline__ intx16 mfma(const intx4 &a, const intx4 &b, const intx16 &c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

// 16 bytes a lane from base + off to LDS at dst + 16 * lane. Written out because the compiler, which cannot tell the buffers
// apart, would wait for the loads in flight before every read of LDS; the caller waits (m0 is the compiler's own register,
// that it is written has to be said, and is warned about).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void direct_load16(const char *base, uint32_t off, uint32_t dst)
{
    const uint32_t to = __builtin_amdgcn_readfirstlane(dst);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Tiles in the order that the XCDs' L2s see them: eight contiguous pieces of an order that goes through strips of kStrip tiles of A.
constexpr int kStrip = 8;
__device__ __forceinline__ bool tile_of_block(int64_t tiles_i, int64_t tiles_j, int64_t *ti, int64_t *tj)
{
    const int64_t tiles = tiles_i * tiles_j, per = (tiles + 7) / 8;
    const int64_t rank = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
    if ((int64_t)(blockIdx.x / 8) >= per || rank >= tiles) return false;
    const int64_t strip = rank / (kStrip * tiles_j), at = rank - strip * kStrip * tiles_j;
    const int64_t left = tiles_i - strip * kStrip, width = left < kStrip ? left : kStrip;
    *tj = at / width;
    *ti = strip * kStrip + (at - *tj * width);
    return true;
}
inline unsigned blocks_of(int64_t tiles) { return (unsigned)((tiles + 7) / 8 * 8); }

// What an epilogue is given: the wavefront's accumulators and where they belong. Element e of acc[a][b] of a lane is row
// i0 + 32 a + 8 (e / 4) + 4 (lane / 32) + e % 4 and column j0 + 32 b + lane % 32.
template <PlaneMode MODE, int TM, int TN, int WM, int WN>
struct Tile {
    static constexpr int BM = TM / WM / 32, BN = TN / WN / 32, COLUMNS = TN, WAVES_I = WM;
    typename Acc<MODE>::type acc[BM][BN];
    int64_t i0, j0, tile_i, tile_j;
    int wave_i, wave_j;
    char *lds;                  // free for the epilogue after a barrier
};

template <PlaneMode MODE, int TM, int TN, int WM, int WN, typename Epilogue>
__global__ __launch_bounds__(64 * WM * WN, 2)
void plane_product(Planes A, Planes B, int64_t steps, int64_t tiles_i, int64_t tiles_j, Epilogue epilogue)
{
    extern __shared__ __attribute__((aligned(1024))) char buffers[];
    typedef Tile<MODE, TM, TN, WM, WN> T;
    constexpr int BM = T::BM, BN = T::BN, kBuffer = (TM + TN) * kStepBytes, NL = (TM + TN) / 8 / (WM * WN);
    static_assert((TM + TN) % (8 * WM * WN) == 0 && TM % 8 == 0, "every wavefront loads whole groups of eight rows");
    T t;
    if (!tile_of_block(tiles_i, tiles_j, &t.tile_i, &t.tile_j)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int half = lane >> 5, col = lane & 31;
    const int64_t first_i = t.tile_i * TM, first_j = t.tile_j * TN;
    t.wave_i = wave / WN;
    t.wave_j = wave % WN;
    t.i0 = first_i + t.wave_i * (TM / WM);
    t.j0 = first_j + t.wave_j * (TN / WN);
    t.lds = buffers;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)buffers;

    const char *base_a = A.data + first_i * A.pitch, *base_b = B.data + first_j * B.pitch;
    uint32_t off[NL];           // from the tile's first row: at most 255 rows on, checked by the launcher to stay below 2^32
#pragma unroll
    for (int l = 0; l < NL; ++l) {
        const int row0 = 8 * (wave * NL + l), row = row0 + (lane >> 3);
        const bool is_b = row0 >= TM;
        const int64_t last = is_b ? B.rows - 1 - first_j : A.rows - 1 - first_i, r = is_b ? row - TM : row;
        off[l] = (uint32_t)((r < last ? r : last) * (is_b ? B.pitch : A.pitch)) + 16u * (uint32_t)((lane & 7) ^ (lane >> 3));
    }
    auto load = [&](int64_t step, int buffer) {
#pragma unroll
        for (int l = 0; l < NL; ++l) {
            const int row0 = 8 * (wave * NL + l);
            direct_load16((row0 >= TM ? base_b : base_a) + step * kStepBytes, off[l], lds + (uint32_t)(buffer * kBuffer + row0 * kStepBytes));
        }
    };
#pragma unroll
    for (int a = 0; a < BM; ++a)
#pragma unroll
        for (int b = 0; b < BN; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) t.acc[a][b][e] = 0;

    const int row_a = t.wave_i * (TM / WM) + col, row_b = TM + t.wave_j * (TN / WN) + col;
    load(0, 0);
    for (int64_t s = 0; s < steps; ++s) {
        // this wavefront's loads of the step have landed and its reads of the step before are done; then everybody's
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < steps) load(s + 1, (int)((s + 1) & 1));
        const char *buf = buffers + (int)(s & 1) * kBuffer;
        auto chunk = [&](int row, int c) {
            return *reinterpret_cast<const intx4 *>(buf + row * kStepBytes + 16 * ((c + half) ^ (col & 7)));
        };
        if constexpr (MODE == kHalfTwo) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                intx4 bh[BN], bl[BN];
#pragma unroll
                for (int b = 0; b < BN; ++b) {
                    bh[b] = chunk(row_b + 32 * b, 2 * ks);
                    bl[b] = chunk(row_b + 32 * b, 4 + 2 * ks);
                }
#pragma unroll
                for (int a = 0; a < BM; ++a) {
                    const intx4 ah = chunk(row_a + 32 * a, 2 * ks), al = chunk(row_a + 32 * a, 4 + 2 * ks);
#pragma unroll
                    for (int b = 0; b < BN; ++b) t.acc[a][b] = mfma(al, bh[b], t.acc[a][b]);
#pragma unroll
                    for (int b = 0; b < BN; ++b) t.acc[a][b] = mfma(ah, bl[b], t.acc[a][b]);
#pragma unroll
                    for (int b = 0; b < BN; ++b) t.acc[a][b] = mfma(ah, bh[b], t.acc[a][b]);
                }
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                intx4 fb[BN];
#pragma unroll
                for (int b = 0; b < BN; ++b) fb[b] = chunk(row_b + 32 * b, 2 * ks);
#pragma unroll
                for (int a = 0; a < BM; ++a) {
                    const intx4 fa = chunk(row_a + 32 * a, 2 * ks);
#pragma unroll
                    for (int b = 0; b < BN; ++b) t.acc[a][b] = mfma(fa, fb[b], t.acc[a][b]);
                }
            }
        }
    }
    epilogue(t);
}

template <PlaneMode MODE, int TM, int TN, int WM, int WN, typename Epilogue>
hipError_t launch_tiles(const Planes &A, const Planes &B, int64_t steps, const Epilogue &epilogue, hipStream_t stream)
{
    constexpr size_t lds = 2 * (size_t)(TM + TN) * kStepBytes;
    static LdsLimit limit;
    auto kernel = plane_product<MODE, TM, TN, WM, WN, Epilogue>;
    const hipError_t e = allow_lds(limit, reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    const int64_t tiles_i = (A.rows + TM - 1) / TM, tiles_j = (B.rows + TN - 1) / TN;
    kernel<<<dim3(blocks_of(tiles_i * tiles_j)), dim3(64 * WM * WN), lds, stream>>>(A, B, steps, tiles_i, tiles_j, epilogue);
    return hipGetLastError();
}

}  // namespace plane

// The edge of the tiles that a product of this size is cut into. 256: eight wavefronts, one workgroup a CU; the smaller ones where
// the larger would leave CUs without work.
inline int plane_tile(int64_t rows_a, int64_t rows_b)
{
    auto tiles = [&](int64_t edge) { return ((rows_a + edge - 1) / edge) * ((rows_b + edge - 1) / edge); };
    if (tiles(256) >= 192) return 256;
    if (tiles(128) >= 192) return 128;
    return 64;
}

template <PlaneMode MODE, typename Epilogue>
hipError_t launch_plane_product(const Planes &A, const Planes &B, int64_t steps, int tile, const Epilogue &epilogue, hipStream_t stream)
{
    if (tile == 256) return plane::launch_tiles<MODE, 256, 256, 2, 4>(A, B, steps, epilogue, stream);
    if (tile == 128) return plane::launch_tiles<MODE, 128, 128, 2, 2>(A, B, steps, epilogue, stream);
    return plane::launch_tiles<MODE, 64, 64, 2, 2>(A, B, steps, epilogue, stream);
}

}  // namespace rfsf
