// AdamW step over many tensors in one launch (rfsf_adamw_step), states of 32 bits or of 8:
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + ((1 - b2) g) g;
//   p = p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// Every operation is rounded by itself (no fused multiply-adds), so that the states' codes do not depend on how the compiler
// arranges the formula. Bound by memory: 28 bytes a number with 32-bit states and gradients, 16 with 8-bit states. 67e6 numbers, 32-bit states, bfloat16
// gradients and a bfloat16 copy 376 us (5.0 TB/s). 19e6 numbers in 61 tensors, 8-bit states: 82 us (3.7 TB/s), where the roots and the quotient, correctly
// rounded, count as well, and 36 for reading the states (5.3 TB/s).
//
// 8-bit states: 256 numbers share a scale, their largest magnitude. m = scale * u |u| with u = code / 127, code -127 .. 127: the grid is
// finer near zero, where most of a block lies. v = scale * u^4 with u = code / 255, code 0 .. 255, covers 2^32 : 1 with steps of 4 / code;
// a v above zero never becomes zero, which would leave m without its divisor: its code is at least the first one that does not stand for
// zero in 32 bits, 1 for scales from 2^-116 on and up to 255 for the smallest. An m of a block with nothing above 2^-119 becomes zero.
#include "rfsf_internal.h"

#include <algorithm>

#include "../../include/rfsf_ts.h"

#pragma clang fp contract(off)

namespace rfsf {
namespace {

constexpr int kShare = 256;                     // numbers of a scale
constexpr int kChunk = 4096;                    // numbers of a workgroup
constexpr int kTensors = 40;                    // of a launch: their descriptions are its arguments
constexpr float kLeast = 1.504632769052528e-36f;        // 2^-119: scales of m below count as zero; shares of v below are taken of 2^64 times it and its scale
constexpr float kLift = 18446744073709551616.0f;        // 2^64
constexpr float kSmall = 1.2037062152420224e-35f;       // 2^-116: scales from there on have code 1 stand for more than zero
constexpr float kInv127 = 1.0f / 127.0f, kInv255 = 1.0f / 255.0f;

struct Job {
    rfsf_adamw_tensor tensor[kTensors];
    int32_t first_chunk[kTensors + 1];          // workgroups of the tensors before
    int32_t aligned[kTensors];                  // all addresses allow loads of four numbers
    int32_t count;
};
struct Numbers {
    float beta1, rest1, beta2, rest2, decay, step, root_scale, eps, grad_scale;
};

__device__ __forceinline__ int tensor_of(const Job &job, int chunk)
{
    int low = 0, high = job.count - 1;
    while (low < high) {
        const int mid = (low + high + 1) / 2;
        if (job.first_chunk[mid] <= chunk) low = mid;
        else high = mid - 1;
    }
    return low;
}
struct Four { float x[4]; };
template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

template <typename T>
__device__ __forceinline__ void load4(const T *p, int64_t left, bool aligned, float (&x)[4])
{
    struct __attribute__((aligned(4 * sizeof(T)))) V { T v[4]; };
    if (aligned && left >= 4) {
        const V v = *reinterpret_cast<const V *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = to_float<T>(v.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < left ? to_float<T>(p[e]) : 0.f;
    }
}
__device__ __forceinline__ void store4(float *p, int64_t left, bool aligned, const float (&x)[4])
{
    if (aligned && left >= 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = x[e];
    }
}
__device__ __forceinline__ void store4_bf16(void *p, int64_t left, bool aligned, const float (&x)[4])
{
    struct __attribute__((aligned(8))) V { __bf16 v[4]; };
    __bf16 *q = static_cast<__bf16 *>(p);
    const V v = {{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]}};
    if (aligned && left >= 4) {
        *reinterpret_cast<V *>(q) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) q[e] = v.v[e];
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int64_t left, bool aligned)
{
    if (aligned && left >= 4) return *reinterpret_cast<const uint32_t *>(p);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) w |= (uint32_t)p[e] << (8 * e);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t *p, int64_t left, bool aligned, uint32_t w)
{
    if (aligned && left >= 4) {
        *reinterpret_cast<uint32_t *>(p) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (uint8_t)(w >> (8 * e));
    }
}
__device__ __forceinline__ float decode_m(uint32_t w, int e, float scale)
{
    const float u = (float)(int8_t)(w >> (8 * e)) * kInv127;
    return (u * fabsf(u)) * scale;
}
__device__ __forceinline__ float decode_v(uint32_t w, int e, float scale)
{
    float u = (float)((w >> (8 * e)) & 0xffu) * kInv255;
    u = u * u;
    return (u * u) * scale;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int o = 32; o > 0; o /= 2) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}
// Scale of a block whose largest magnitude has these bits, and what brings its numbers to shares of it. An infinity or a NaN in a block
// makes its scale NaN: the step shows it rather than hide it behind a code.
__device__ __forceinline__ void scale_and_inverse(uint32_t largest, float *scale, float *inverse)
{
    const float top = __uint_as_float(largest);
    *scale = largest < 0x7f800000u ? top : NAN;
    *inverse = largest < 0x7f800000u && top >= kLeast ? 1.0f / top : 0.f;
}
// The same for v, of v * lift, and the least code of a v above zero: (least code / 255)^4 scale is about 2^-149, the smallest number above zero, or more.
__device__ __forceinline__ void scale_and_inverse_v(uint32_t largest, float *scale, float *inverse, float *lift, float *least)
{
    const float top = __uint_as_float(largest);
    const bool finite = largest < 0x7f800000u;
    *scale = finite ? top : NAN;
    *lift = top < kLeast ? kLift : 1.0f;
    *inverse = finite && top > 0.f ? 1.0f / (top * *lift) : 0.f;
    *least = 1.0f;
    if (top > 0.f && top < kSmall) *least = fminf(ceilf(sqrtf(sqrtf(2.5849394142282115e-26f / (top * kLift))) * 255.0f), 255.0f);          // (2^-85: 2^-149 lifted)
}

// A wavefront takes 256 numbers at a time, four a lane: a block of 8-bit states is a wavefront's own.
template <typename G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(Job job, Numbers c)
{
    const int k = tensor_of(job, (int)blockIdx.x);
    const rfsf_adamw_tensor &t = job.tensor[k];
    const bool aligned = job.aligned[k] != 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t start = (int64_t)((int)blockIdx.x - job.first_chunk[k]) * kChunk;
    float *param = static_cast<float *>(t.param);
    const G *grad = static_cast<const G *>(t.grad);
#pragma unroll 2
    for (int u = 0; u < kChunk / 1024; ++u) {
        const int64_t base = start + 1024 * u + 256 * wave;        // the wavefront's
        if (base >= t.n) break;
        const int64_t i = base + 4 * lane, left = t.n - i;
        float p[4], g[4], m[4], v[4];
        load4(param + i, left, aligned, p);
        load4(grad + i, left, aligned, g);
        if constexpr (EIGHT) {
            const float ms = t.m_scale[base / kShare], vs = t.v_scale[base / kShare];
            const uint32_t mw = load_codes(static_cast<const uint8_t *>(t.m) + i, left, aligned), vw = load_codes(static_cast<const uint8_t *>(t.v) + i, left, aligned);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = decode_m(mw, e, ms);
                v[e] = decode_v(vw, e, vs);
            }
        } else {
            load4(static_cast<const float *>(t.m) + i, left, aligned, m);
            load4(static_cast<const float *>(t.v) + i, left, aligned, v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = g[e] * c.grad_scale;
            m[e] = m[e] * c.beta1 + x * c.rest1;
            v[e] = v[e] * c.beta2 + (x * c.rest2) * x;
            p[e] = p[e] * c.decay - (m[e] * c.step) / (sqrtf(v[e]) * c.root_scale + c.eps);
        }
        store4(param + i, left, aligned, p);
        if (t.copy) store4_bf16(static_cast<uint16_t *>(t.copy) + i, left, aligned, p);
        if constexpr (EIGHT) {
            uint32_t mt = 0, vt = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e < left) {
                    mt = max(mt, __float_as_uint(m[e]) & 0x7fffffffu);
                    vt = max(vt, __float_as_uint(v[e]) & 0x7fffffffu);
                }
            }
            float ms, mi, vs, vi, lift, least;
            scale_and_inverse(wave_max(mt), &ms, &mi);
            scale_and_inverse_v(wave_max(vt), &vs, &vi, &lift, &least);
            uint32_t mw = 0, vw = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mc = mi == 0.f ? 0.f : fminf(rintf(sqrtf(fabsf(m[e]) * mi) * 127.0f), 127.0f);
                const float share = vi == 0.f ? 0.f : (v[e] * lift) * vi;
                float vc = fminf(rintf(sqrtf(sqrtf(share)) * 255.0f), 255.0f);
                if (vi != 0.f && v[e] > 0.f) vc = fmaxf(vc, least);
                mw |= ((uint32_t)(int)(m[e] < 0.f ? -mc : mc) & 0xffu) << (8 * e);
                vw |= (uint32_t)(int)vc << (8 * e);
            }
            store_codes(static_cast<uint8_t *>(t.m) + i, left, aligned, mw);
            store_codes(static_cast<uint8_t *>(t.v) + i, left, aligned, vw);
            if (lane == 0) {
                t.m_scale[base / kShare] = ms;
                t.v_scale[base / kShare] = vs;
            }
        } else {
            store4(static_cast<float *>(t.m) + i, left, aligned, m);
            store4(static_cast<float *>(t.v) + i, left, aligned, v);
        }
    }
}

// The numbers that 8-bit states stand for: param takes m, copy takes v (as floats), the other fields as above.
__global__ __launch_bounds__(256) void moments_kernel(Job job)
{
    const int k = tensor_of(job, (int)blockIdx.x);
    const rfsf_adamw_tensor &t = job.tensor[k];
    const bool aligned = job.aligned[k] != 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t start = (int64_t)((int)blockIdx.x - job.first_chunk[k]) * kChunk;
#pragma unroll 2
    for (int u = 0; u < kChunk / 1024; ++u) {
        const int64_t base = start + 1024 * u + 256 * wave;
        if (base >= t.n) break;
        const int64_t i = base + 4 * lane, left = t.n - i;
        const float ms = t.m_scale[base / kShare], vs = t.v_scale[base / kShare];
        const uint32_t mw = load_codes(static_cast<const uint8_t *>(t.m) + i, left, aligned), vw = load_codes(static_cast<const uint8_t *>(t.v) + i, left, aligned);
        float m[4], v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = decode_m(mw, e, ms);
            v[e] = decode_v(vw, e, vs);
        }
        store4(static_cast<float *>(t.param) + i, left, aligned, m);
        store4(static_cast<float *>(t.copy) + i, left, aligned, v);
    }
}

bool four(const void *p, size_t element) { return reinterpret_cast<uintptr_t>(p) % (4 * element) == 0; }

// Goes through the tensors, at most kTensors a launch, and not more than 2^32 threads; tensors without numbers take no part.
template <typename Tensor, typename Launch>
hipError_t for_each_launch(const Tensor &tensor, int64_t count, size_t grad_size, size_t state_size, size_t copy_size, const Launch &launch)
{
    Job job;
    job.count = 0;
    int64_t chunks = 0;
    for (int64_t k = 0; k <= count; ++k) {
        const int64_t more = k < count ? (tensor(k).n + kChunk - 1) / kChunk : 0;
        if (job.count > 0 && (k == count || job.count == kTensors || chunks + more > (1 << 23))) {
            job.first_chunk[job.count] = (int32_t)chunks;
            launch(job, (unsigned)chunks);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            job.count = 0;
            chunks = 0;
        }
        if (k == count || more == 0) continue;
        const rfsf_adamw_tensor t = tensor(k);
        job.tensor[job.count] = t;
        job.first_chunk[job.count] = (int32_t)chunks;
        job.aligned[job.count] = four(t.param, 4) && four(t.grad, grad_size) && four(t.m, state_size) && four(t.v, state_size) &&
                                 (!t.copy || four(t.copy, copy_size));
        ++job.count;
        chunks += more;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adamw(const rfsf_adamw_tensor *tensors, int64_t count, const rfsf_adamw_config &c, double correction1, double correction2,
                        hipStream_t stream)
{
    const Numbers numbers = {(float)c.beta1, (float)(1.0 - c.beta1), (float)c.beta2, (float)(1.0 - c.beta2), (float)(1.0 - c.lr * c.weight_decay),
                             (float)(c.lr / correction1), (float)(1.0 / correction2), (float)c.eps, (float)c.grad_scale};
    const bool eight = c.state_bits == 8, bf16 = c.grad_bf16 != 0;
    auto tensor = [&](int64_t k) { return tensors[k]; };
    return for_each_launch(tensor, count, bf16 ? 2 : 4, eight ? 1 : 4, 2, [&](const Job &job, unsigned chunks) {
        if (eight && bf16) adamw_kernel<uint16_t, true><<<dim3(chunks), 256, 0, stream>>>(job, numbers);
        else if (eight) adamw_kernel<float, true><<<dim3(chunks), 256, 0, stream>>>(job, numbers);
        else if (bf16) adamw_kernel<uint16_t, false><<<dim3(chunks), 256, 0, stream>>>(job, numbers);
        else adamw_kernel<float, false><<<dim3(chunks), 256, 0, stream>>>(job, numbers);
    });
}

hipError_t launch_adamw_moments(const rfsf_adamw_tensor *tensors, int64_t count, float *const *m_out, float *const *v_out, hipStream_t stream)
{
    auto tensor = [&](int64_t k) {
        rfsf_adamw_tensor t = tensors[k];
        t.param = m_out[k];
        t.copy = v_out[k];
        t.grad = nullptr;
        return t;
    };
    return for_each_launch(tensor, count, 4, 1, 4, [&](const Job &job, unsigned chunks) { moments_kernel<<<dim3(chunks), 256, 0, stream>>>(job); });
}

}  // namespace rfsf
