// Eight numbers of a row of a matrix at a time, float or bfloat16 (as uint16_t), at any alignment of the type: one load or store of 16 bytes,
// or two of them, and single numbers at the end of a row.
#pragma once

#include "rfsf_internal.h"

namespace rfsf {
namespace rows8 {

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void from_float(float x, float *out) { *out = x; }
// the nearest bfloat16, ties to even; a NaN stays one
__device__ __forceinline__ void from_float(float x, uint16_t *out) { *out = __builtin_bit_cast(uint16_t, (__bf16)x); }

// Columns k .. k + 7 of a row of K; 0 beyond.
template <typename T>
__device__ __forceinline__ void load(const T *row, int64_t k, int64_t K, float (&x)[8])
{
    if (k + 8 <= K) {
        const Eight<T> c = *reinterpret_cast<const Eight<T> *>(row + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_float(c.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < K ? to_float(row[k + e]) : 0.f;
    }
}
// The same of a row of at least eight columns, as they lie in memory and without a load for each number at its end: there the row's last eight numbers are loaded and
// moved down.
__device__ __forceinline__ void move_down(Eight<float> &c, int by)
{
#pragma unroll
    for (int step = 4; step > 0; step /= 2) {
        const bool now = (by & step) != 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) c.v[e] = now ? (e + step < 8 ? c.v[e + step] : 0.f) : c.v[e];
    }
}
__device__ __forceinline__ void move_down(Eight<uint16_t> &c, int by)
{
    uint32_t w[4];
    __builtin_memcpy(w, &c, 16);
#pragma unroll
    for (int step = 2; step > 0; step /= 2) {
        const bool now = (by & (2 * step)) != 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = now ? (i + step < 4 ? w[i + step] : 0u) : w[i];
    }
    if (by & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = w[i] >> 16 | (i < 3 ? w[i + 1] << 16 : 0u);
    }
    __builtin_memcpy(&c, w, 16);
}
template <typename T>
__device__ __forceinline__ Eight<T> load_raw(const T *row, int k, int K)
{
    Eight<T> c = {};
    if (k < K) {
        const int start = k + 8 <= K ? k : K - 8;
        c = *reinterpret_cast<const Eight<T> *>(row + start);
        if (start < k) move_down(c, k - start);
    }
    return c;
}
template <typename T>
__device__ __forceinline__ void store(T *row, int64_t k, int64_t K, const float (&x)[8])
{
    if (k + 8 <= K) {
        Eight<T> c;
#pragma unroll
        for (int e = 0; e < 8; ++e) from_float(x[e], &c.v[e]);
        *reinterpret_cast<Eight<T> *>(row + k) = c;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < K) from_float(x[e], row + k + e);
    }
}

// Numbers that are held from pass to pass as they came, so that what one pass made of them (32 bits of each) is not kept for the next one; and what is done
// with a lane's eight numbers is done before the next eight's turn. (Without both the compiler holds all of it at once, and spills: 30000 x 10241, bfloat16 1170 us.)
template <typename T>
__device__ __forceinline__ void in_turn(Eight<T> &c)
{
    uint32_t w[2 * sizeof(T)];
    __builtin_memcpy(w, &c, sizeof(c));
#pragma unroll
    for (size_t i = 0; i < 2 * sizeof(T); i += 4) asm volatile("" : "+v"(w[i]), "+v"(w[i + 1]), "+v"(w[i + 2]), "+v"(w[i + 3]));
    __builtin_memcpy(&c, w, sizeof(c));
    __builtin_amdgcn_sched_barrier(0);
}

}  // namespace rows8
}  // namespace rfsf
