// C entry points of the operators of linear models on features: argument checks, then the launches.
#include "rfsf_internal.h"

#include <cmath>

namespace {

constexpr int64_t kMostColumns = 3500000;       // 287 packed rows of a tile stay below 2^32 bytes; grids
constexpr int64_t kMostRows = 0x7fffffffLL;
constexpr int64_t kMostCodes = 131072;          // 127 * 128 times that stays below 2^31
constexpr int64_t kMostStored = 100000000;
constexpr int64_t kMostNumbers = (int64_t)1 << 35;          // 2^23 workgroups of 256 threads: a launch has fewer than 2^32 threads

int check(const rfsf_xent_shape *s)
{
    if (!s) return RFSF_E_NULLPTR;
    if (s->N < 0 || s->K < 1 || s->C < 1 || (s->gradients & ~(RFSF_XENT_DPHI | RFSF_XENT_DW)) != 0) return RFSF_E_BAD_SHAPE;
    if (s->ld_phi < s->K || s->ld_w < s->K) return RFSF_E_BAD_STRIDE;
    if ((s->gradients & RFSF_XENT_DPHI) && s->ld_dphi < s->K) return RFSF_E_BAD_STRIDE;
    if ((s->gradients & RFSF_XENT_DW) && s->ld_dw < s->K) return RFSF_E_BAD_STRIDE;
    if (s->N > kMostRows || s->K > kMostColumns || s->C > kMostColumns) return RFSF_E_UNSUPPORTED;
    return RFSF_OK;
}
int64_t code_room(int64_t K) { return (K + 127) / 128 * 128; }
bool misplaced(const void *codes, int64_t ld) { return reinterpret_cast<uintptr_t>(codes) % 16 != 0 || ld % 16 != 0; }

int check_tensors(const rfsf_adamw_tensor *tensors, int64_t count)
{
    if (count < 0) return RFSF_E_BAD_SHAPE;
    if (count > 0 && !tensors) return RFSF_E_NULLPTR;
    for (int64_t k = 0; k < count; ++k) {
        if (tensors[k].n < 0) return RFSF_E_BAD_SHAPE;
        if (tensors[k].n > kMostNumbers) return RFSF_E_UNSUPPORTED;
    }
    return RFSF_OK;
}

}  // namespace

extern "C" int rfsf_softmax_xent_workspace_bytes(const rfsf_xent_shape *shape, size_t *recommended_bytes, size_t *minimum_bytes)
{
    const int rc = check(shape);
    if (rc != RFSF_OK) return rc;
    size_t recommended, minimum;
    rfsf::softmax_xent_bytes(*shape, &recommended, &minimum);
    if (recommended_bytes) *recommended_bytes = recommended;
    if (minimum_bytes) *minimum_bytes = minimum;
    return RFSF_OK;
}

extern "C" int rfsf_softmax_xent(const rfsf_xent_shape *shape, const void *Phi, const void *W, const int64_t *labels, const float *weight,
                                 float *loss, void *dPhi, void *dW, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = check(shape);
    if (rc != RFSF_OK) return rc;
    const bool d_phi = (shape->gradients & RFSF_XENT_DPHI) != 0, d_w = (shape->gradients & RFSF_XENT_DW) != 0;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (shape->N == 0) {
        if (!d_w) return RFSF_OK;
        if (!dW) return RFSF_E_NULLPTR;
        return rfsf::launch_clear_rows(dW, shape->C, shape->K, shape->ld_dw, shape->bf16 != 0, stream) == hipSuccess ? RFSF_OK : RFSF_E_HIP;
    }
    if (!Phi || !W || !labels || !loss || !workspace || (d_phi && !dPhi) || (d_w && !dW)) return RFSF_E_NULLPTR;
    size_t recommended, minimum;
    rfsf::softmax_xent_bytes(*shape, &recommended, &minimum);
    if (workspace_bytes < minimum) return RFSF_E_WORKSPACE_TOO_SMALL;
    return rfsf::launch_softmax_xent(*shape, Phi, W, labels, weight, loss, dPhi, dW, workspace, workspace_bytes, stream) == hipSuccess
               ? RFSF_OK : RFSF_E_HIP;
}

extern "C" int rfsf_adamw_step(const rfsf_adamw_tensor *tensors, int64_t count, const rfsf_adamw_config *c, void *hip_stream)
{
    if (!c) return RFSF_E_NULLPTR;
    const int rc = check_tensors(tensors, count);
    if (rc != RFSF_OK) return rc;
    if (c->state_bits != 8 && c->state_bits != 32) return RFSF_E_UNSUPPORTED;
    const double correction1 = 1.0 - std::pow(c->beta1, (double)c->step), correction2 = std::sqrt(1.0 - std::pow(c->beta2, (double)c->step));
    // what the step uses of the settings is held in 32 bits
    for (double v : {c->lr, c->beta1, c->beta2, c->eps, c->weight_decay, c->grad_scale, c->lr * c->weight_decay, c->lr / correction1})
        if (!std::isfinite((float)v)) return RFSF_E_BAD_SETTING;
    if (c->lr < 0 || c->eps < 0 || c->weight_decay < 0 || c->beta1 < 0 || c->beta1 >= 1 || c->beta2 < 0 || c->beta2 >= 1 ||
        c->step < 1)
        return RFSF_E_BAD_SETTING;
    for (int64_t k = 0; k < count; ++k) {
        const rfsf_adamw_tensor &t = tensors[k];
        if (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (c->state_bits == 8 && (!t.m_scale || !t.v_scale)))) return RFSF_E_NULLPTR;
    }
    return rfsf::launch_adamw(tensors, count, *c, correction1, correction2, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RFSF_OK : RFSF_E_HIP;
}

extern "C" int rfsf_adamw_moments(const rfsf_adamw_tensor *tensors, int64_t count, float *const *m_out, float *const *v_out, void *hip_stream)
{
    const int rc = check_tensors(tensors, count);
    if (rc != RFSF_OK) return rc;
    if (count > 0 && (!m_out || !v_out)) return RFSF_E_NULLPTR;
    for (int64_t k = 0; k < count; ++k) {
        const rfsf_adamw_tensor &t = tensors[k];
        if (t.n > 0 && (!t.m || !t.v || !t.m_scale || !t.v_scale || !m_out[k] || !v_out[k])) return RFSF_E_NULLPTR;
    }
    return rfsf::launch_adamw_moments(tensors, count, m_out, v_out, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RFSF_OK : RFSF_E_HIP;
}

extern "C" int rfsf_int8_quantize(const void *X, int32_t bf16, int64_t N, int64_t ldx, int64_t K, int8_t *codes, int64_t ld_codes, float *scales,
                                  void *hip_stream)
{
    if (N < 0 || K < 1) return RFSF_E_BAD_SHAPE;
    if (ldx < K || ld_codes < code_room(K)) return RFSF_E_BAD_STRIDE;
    if (N > kMostRows || K > kMostCodes) return RFSF_E_UNSUPPORTED;
    if (N == 0) return RFSF_OK;
    if (!X || !codes || !scales) return RFSF_E_NULLPTR;
    if (misplaced(codes, ld_codes)) return RFSF_E_BAD_STRIDE;
    return rfsf::launch_int8_quantize(X, bf16 != 0, N, ldx, K, codes, ld_codes, scales, static_cast<hipStream_t>(hip_stream)) == hipSuccess
               ? RFSF_OK : RFSF_E_HIP;
}

extern "C" int rfsf_int8_gram_workspace_bytes(int64_t Nx, int64_t Ny, int64_t K, size_t *recommended_bytes, size_t *minimum_bytes)
{
    if (Nx < 0 || Ny < 0 || K < 1) return RFSF_E_BAD_SHAPE;
    if (Nx > kMostRows || Ny > kMostStored || K > kMostCodes) return RFSF_E_UNSUPPORTED;
    size_t recommended, minimum;
    rfsf::int8_gram_bytes(Nx, K, &recommended, &minimum);
    if (recommended_bytes) *recommended_bytes = recommended;
    if (minimum_bytes) *minimum_bytes = minimum;
    return RFSF_OK;
}

extern "C" int rfsf_int8_gram(const void *X, int32_t bf16, int64_t Nx, int64_t ldx, const int8_t *codes, const float *scales, int64_t Ny,
                              int64_t ld_codes, int64_t K, float *out, int64_t ld_out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    size_t minimum;
    const int rc = rfsf_int8_gram_workspace_bytes(Nx, Ny, K, nullptr, &minimum);
    if (rc != RFSF_OK) return rc;
    if (ldx < K || ld_codes < code_room(K) || ld_out < Ny) return RFSF_E_BAD_STRIDE;
    if (Nx == 0 || Ny == 0) return RFSF_OK;
    if (!X || !codes || !scales || !out || !workspace) return RFSF_E_NULLPTR;
    if (misplaced(codes, ld_codes) || ld_codes > (1 << 23)) return RFSF_E_BAD_STRIDE;     // 287 rows of a tile stay below 2^32 bytes
    if (workspace_bytes < minimum) return RFSF_E_WORKSPACE_TOO_SMALL;
    return rfsf::launch_int8_gram(X, bf16 != 0, Nx, ldx, codes, scales, Ny, ld_codes, K, out, ld_out, workspace, workspace_bytes,
                                  static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RFSF_OK : RFSF_E_HIP;
}
