// Dropout's random numbers, which are computed where they are needed and never stored.
//
// A number of 16 bits belongs to every place (row, column) of a matrix: Philox 4x32 of 10 rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011) under the key `seed` makes four words of 32 bits of the counter (column / 8, row, offset's two words), which
// serve eight columns: word (column % 8) / 2, its lower half for even columns. A place is kept if its number is not below the threshold
// round(65536 p), so that the factor 65536 / (65536 - threshold) of the kept ones makes the mean exact for the probability that is really used.
// 16 bits and not 32: ten rounds are 20 products of 32 x 32 bits at a quarter of the rate of others, which must not take longer than the memory does.
#pragma once

#include "rfsf_internal.h"
#include "rows8.h"

namespace rfsf {

struct DropoutJob {
    uint32_t key[2];
    uint32_t first_row, threshold;
    uint64_t offset;
    const uint64_t *offset_on_device;   // NULL, or a number in device memory that is added to offset when the kernel runs
    float factor;
};
inline DropoutJob dropout_job(const rfsf_dropout_mask *m)
{
    DropoutJob job = {};
    if (!m) return job;
    job.key[0] = (uint32_t)m->seed;
    job.key[1] = (uint32_t)(m->seed >> 32);
    job.first_row = (uint32_t)m->first_row;
    job.threshold = dropout_threshold(m->p);
    job.offset = m->offset;
    job.offset_on_device = m->offset_on_device;
    job.factor = job.threshold < 65536 ? (float)(65536.0 / (65536 - job.threshold)) : 0.f;
    return job;
}

namespace dropout {

__device__ __forceinline__ uint64_t offset_of(const DropoutJob &job) { return job.offset + (job.offset_on_device ? *job.offset_on_device : 0); }

// The numbers of eight columns from 8 * group on.
__device__ __forceinline__ void numbers(const DropoutJob &job, uint64_t offset, uint32_t row, uint32_t group, uint32_t (&word)[4])
{
    uint32_t c0 = group, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = job.key[0], k1 = job.key[1];
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t first = (uint64_t)0xD2511F53u * c0, second = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(second >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)second;
        c2 = (uint32_t)(first >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)first;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    word[0] = c0;
    word[1] = c1;
    word[2] = c2;
    word[3] = c3;
}
__device__ __forceinline__ bool kept(const DropoutJob &job, const uint32_t (&word)[4], int e)
{
    return (e & 1 ? word[e / 2] >> 16 : word[e / 2] & 0xffffu) >= job.threshold;
}
__device__ __forceinline__ bool keeps(const DropoutJob &job, uint64_t offset, uint32_t row, uint32_t column)
{
    uint32_t word[4];
    numbers(job, offset, row, column / 8, word);
    bool keep = false;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (column % 8 == e) keep = kept(job, word, e);
    return keep;
}
// Eight numbers of a row: those that are kept times the factor, 0 (also of infinities and NaN) for the others.
__device__ __forceinline__ void apply(const DropoutJob &job, uint64_t offset, uint32_t row, uint32_t group, float (&x)[8])
{
    uint32_t word[4];
    numbers(job, offset, row, group, word);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = kept(job, word, e) ? x[e] * job.factor : 0.f;
}

// The same of numbers as they lie in memory, without the factor, for sums that it can multiply afterwards.
__device__ __forceinline__ void choose(const DropoutJob &job, uint64_t offset, uint32_t row, uint32_t group, rows8::Eight<float> &c)
{
    uint32_t word[4];
    numbers(job, offset, row, group, word);
#pragma unroll
    for (int e = 0; e < 8; ++e) c.v[e] = kept(job, word, e) ? c.v[e] : 0.f;
}
__device__ __forceinline__ void choose(const DropoutJob &job, uint64_t offset, uint32_t row, uint32_t group, rows8::Eight<uint16_t> &c)
{
    uint32_t word[4], two[4];
    numbers(job, offset, row, group, word);
    __builtin_memcpy(two, &c, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) two[i] = (kept(job, word, 2 * i) ? two[i] & 0xffffu : 0u) | (kept(job, word, 2 * i + 1) ? two[i] & 0xffff0000u : 0u);
    __builtin_memcpy(&c, two, 16);
}

}  // namespace dropout
}  // namespace rfsf
