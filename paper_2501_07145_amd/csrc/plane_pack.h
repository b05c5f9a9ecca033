// Packing of row-major matrices into the operands of plane_product.h, and the 16-bit numbers they hold.
//
// 32-bit numbers enter as two terms of 16-bit floating point, hi + lo, of the number times a power of two that brings the
// largest of its row into [2^14, 2^15): 22 significand bits for numbers down to 2^-17 of that largest one, an
// error of 2^-39 of it or less below. bfloat16 numbers enter as one such term, without any error down to 2^-30 of the
// row's largest. Products are scaled back by exact powers of two. A row with an infinity or a NaN gives NaN (or infinities).
//
// The transposed operand holds the same 16-bit numbers. Where it is multiplied, a row's power of two belongs to an index that is
// summed over, and is taken back in the other factor: (G[n, c] 2^e_c) (W[c, k] 2^-e_c). A class whose weights are far larger than the
// others' (an offset of -1e30 that shuts it off) then costs the others nothing, as long as its G is zero.
//
// That other factor, G, always enters as two terms, whatever the operands' type: differences of almost equal numbers of G are gradients like any others.
#pragma once

#include "rfsf_internal.h"
#include "plane_product.h"

namespace rfsf {

// The power of two for a row whose largest magnitude has these bits (0: all zero, any will do).
constexpr int kTopBit = 14;
__host__ __device__ __forceinline__ int shift_of(uint32_t largest)
{
    return largest == 0 ? 0 : kTopBit - ((int)(largest >> 23) - 127);
}

// Bytes from row to row of an operand of `columns` columns: whole groups of 64, and an odd number of steps, so that a step of
// many rows lies in all channels of the L2 (a product of 32768 x 2048 x 8192 with rows of 16384 bytes 1057 us, of 16512 878).
inline int64_t odd_steps(int64_t bytes) { return ((bytes + kStepBytes - 1) / kStepBytes | 1) * kStepBytes; }
inline int64_t plane_pitch(int64_t columns, bool two) { return odd_steps((columns + 63) / 64 * 64 * (two ? 4 : 2)); }
inline int64_t plane_steps(int64_t columns, bool two) { return two ? (columns + 31) / 32 : (columns + 63) / 64; }

namespace plane {

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

struct Terms8 { uint32_t hi[4], lo[4]; };
// Eight numbers, already scaled, as terms (without TWO the second one is left out).
template <bool TWO>
__device__ __forceinline__ Terms8 terms_of(const float (&x)[8])
{
    Terms8 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const floatx2 v = {x[2 * i], x[2 * i + 1]};
        const halfx2 hi = __builtin_convertvector(v, halfx2);
        t.hi[i] = __builtin_bit_cast(uint32_t, hi);
        if (TWO) {
            const floatx2 rest = {v[0] - (float)hi[0], v[1] - (float)hi[1]};
            t.lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, halfx2));
        }
    }
    return t;
}
// Writes eight consecutive columns from `column` (a multiple of 8) on.
template <bool TWO>
__device__ __forceinline__ void store_terms(char *row, int64_t column, const Terms8 &t)
{
    char *at = TWO ? row + (column >> 5) * kStepBytes + 2 * (column & 31) : row + 2 * column;
    *reinterpret_cast<uint4 *>(at) = make_uint4(t.hi[0], t.hi[1], t.hi[2], t.hi[3]);
    if (TWO) *reinterpret_cast<uint4 *>(at + 64) = make_uint4(t.lo[0], t.lo[1], t.lo[2], t.lo[3]);
}
__device__ __forceinline__ float number(float x) { return x; }
__device__ __forceinline__ float number(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

}  // namespace plane

// What the rows of Phi come to that gradients need to know: how many count, and the exponent of the largest |weight| * 2^exponent(row).
struct RowStats {
    uint32_t count;
    uint32_t top;               // biased by kTopBias, so that 0 is below all
};
constexpr int kTopBias = 1024;
__host__ __device__ __forceinline__ int exponent_of(uint32_t bits) { return (int)((bits & 0x7fffffffu) >> 23) - 127; }

// A matrix to pack: R rows of K numbers (float, or uint16_t for the bits of bfloat16), ld numbers apart. Rows whose label is
// negative (labels may be null) count as zero whatever they hold.
// largest: bits of the magnitude of each row's largest number, written by launch_largest and read by launch_pack.
// rows: the matrix as operand; columns (may be null): the transpose of the same numbers, scaled by rows of the matrix as they are. Columns
// of the operands beyond K and R, up to a multiple of 64, are written as zero.
struct PackJob {
    const void *src;
    int64_t R, K, ld;
    const int64_t *labels;
    uint32_t *largest;
    char *rows, *columns;
    int64_t pitch_rows, pitch_columns;
    const int32_t *order = nullptr;     // the matrix' row that a packed row is (columns null); null: the same one
};
// Two matrices in a launch (the second one may have no rows). stats (may be null): launch_largest clears it, launch_pack brings it
// up to the second matrix' rows, of these weights (null: all one).
struct PackPair {
    PackJob job[2];
    RowStats *stats;
    const float *weight;
};
hipError_t launch_largest(const PackPair &pair, bool bf16, hipStream_t stream);
hipError_t launch_pack(const PackPair &pair, bool bf16, hipStream_t stream);
// Both in one, for matrices of up to kPackRowsColumns columns that are packed by rows alone, without stats.
constexpr int64_t kPackRowsColumns = 12288;
hipError_t launch_pack_rows(const PackPair &pair, bool bf16, hipStream_t stream);

}  // namespace rfsf
