// C ABI of the operators of a layer: checks of arguments, then the launches (see include/sig.h for the contracts).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "layer.hpp"

namespace {

constexpr int64_t kMost = (int64_t)1 << 38;       // bound of sizes and of their products: more than the memory holds, and no overflow below
constexpr int64_t kMostStride = kMost;

int hip_code(hipError_t e) { return e == hipSuccess ? SIG_OK : e == sig::kTooManyThreads ? SIG_ETOOLARGE : sig::record_hip_error(e); }

bool bad_type(int64_t t) { return t != SIG_F32 && t != SIG_BF16; }

int check_sizes(std::initializer_list<int64_t> sizes)
{
    int64_t p = 1;
    for (int64_t v : sizes)
        if (v < 0) return SIG_EINVAL;
    for (int64_t v : sizes) {
        if (v > kMost || (v && p > kMost / v)) return SIG_ETOOLARGE;
        p *= std::max<int64_t>(v, 1);
    }
    return SIG_OK;
}
int check_strides(std::initializer_list<int64_t> strides)
{
    for (int64_t s : strides)
        if (s < 0 || s > kMostStride) return s < 0 ? SIG_EINVAL : SIG_ETOOLARGE;
    return SIG_OK;
}

int check_norm(const sig_norm_args* a)
{
    if (!a || bad_type(a->dtype) || a->C < 1 || !(a->eps >= 0.0) || std::isinf(a->eps)) return SIG_EINVAL;
    int rc = check_sizes({a->rows, a->C});
    return rc != SIG_OK ? rc : check_strides({a->x_stride, a->residual_stride});
}

int check_linear(const sig_linear_args* a, bool gradient)
{
    if (!a || a->N < 1 || a->K < 1 || a->act < SIG_ACT_NONE || a->act > SIG_ACT_GELU) return SIG_EINVAL;
    if (gradient ? bad_type(a->dtype) : bad_type(a->out_dtype) || (a->dtype != SIG_E4M3 && a->dtype != a->out_dtype)) return SIG_EINVAL;
    if (a->dtype != SIG_E4M3 && !gradient && (a->x_scale || a->weight_scale)) return SIG_EINVAL;
    for (int rc : {check_sizes({a->M, a->K}), check_sizes({a->M, a->N}), check_sizes({a->N, a->K}), check_strides({a->x_stride, gradient ? 0 : a->residual_stride})})
        if (rc != SIG_OK) return rc;
    for (int64_t v : {a->M, a->N, a->K})
        if (v >= (1ll << 31) - 256) return SIG_ETOOLARGE;
    return SIG_OK;
}

int check_gated(const sig_gated_args* a, bool prompt = true)
{
    if (!a || bad_type(a->dtype) || a->D < 1) return SIG_EINVAL;
    int rc = check_sizes({a->B, prompt ? a->L : 1, a->D});
    if (rc != SIG_OK) return rc;
    if ((a->B > 0 && a->D > INT32_MAX / a->B) || a->D >= (1 << 22)) return SIG_ETOOLARGE;      // a round's tokens are reached by 32-bit offsets
    if (prompt && a->L >= (1 << 30)) return SIG_ETOOLARGE;        // tokens are counted in 32 bits, up to the end of a round
    rc = check_strides({a->x_stride_b, a->decay_stride_b, a->input_stride_b});
    if (rc != SIG_OK || !prompt) return rc;
    for (int64_t s : {a->x_stride_t, a->decay_stride_t, a->input_stride_t})
        if (s < 0 || s >= (1 << 22)) return s < 0 ? SIG_EINVAL : SIG_ETOOLARGE;
    return SIG_OK;
}

size_t ckpt_bytes(const sig_gated_args& a) { return (size_t)(a.B * ((a.L + sig::kGatedTile - 1) / sig::kGatedTile) * a.D * 4); }

}  // namespace

extern "C" {

int sig_norm_forward(const sig_norm_args* a, void* y, float* scale, void* total, void* stream)
{
    int rc = check_norm(a);
    if (rc != SIG_OK || a->rows == 0) return rc;
    if (!a->x || !a->weight || !y || (total && !a->residual)) return SIG_EINVAL;
    return hip_code(sig::norm_forward(*a, y, scale, total, (hipStream_t)stream));
}

size_t sig_norm_backward_workspace_bytes(const sig_norm_args* a) { return check_norm(a) == SIG_OK ? sig::norm_backward_workspace(*a) : 0; }

int sig_norm_backward(const sig_norm_args* a, const void* grad_y, int64_t gy_stride, const void* grad_total, int64_t gt_stride, void* grad_x,
                      float* grad_weight, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_norm(a);
    if (rc == SIG_OK) rc = check_strides({gy_stride, gt_stride});
    if (rc != SIG_OK) return rc;
    if (!a->weight || !grad_weight || (a->rows && (!a->x || !grad_y || !grad_x))) return SIG_EINVAL;
    const size_t need = sig::norm_backward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    sig::NormGrads g{grad_y, gy_stride, grad_total, gt_stride, grad_x, grad_weight};
    return hip_code(sig::norm_backward(*a, g, (float*)workspace, (hipStream_t)stream));
}

int sig_quantize(int64_t dtype, int64_t rows, int64_t C, int64_t x_stride, const void* x, void* q, float* scale, void* stream)
{
    sig_norm_args a{dtype, rows, C, x_stride, 0, 0.0, x, nullptr, nullptr};
    int rc = check_norm(&a);
    if (rc != SIG_OK || rows == 0) return rc;
    if (!x || !q || !scale) return SIG_EINVAL;
    return hip_code(sig::norm_forward(a, q, scale, nullptr, (hipStream_t)stream));
}

size_t sig_linear_forward_workspace_bytes(const sig_linear_args* a) { return check_linear(a, false) == SIG_OK ? sig::linear_forward_workspace(*a) : 0; }

int sig_linear_forward(const sig_linear_args* a, void* y, void* pre, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_linear(a, false);
    if (rc != SIG_OK || a->M == 0) return rc;
    if (!a->x || !a->weight || !y) return SIG_EINVAL;
    const size_t need = sig::linear_forward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::linear_forward(*a, y, pre, workspace, (hipStream_t)stream));
}

size_t sig_linear_backward_workspace_bytes(const sig_linear_args* a) { return check_linear(a, true) == SIG_OK ? sig::linear_backward_workspace(*a) : 0; }

int sig_linear_backward(const sig_linear_args* a, const void* grad_y, int64_t gy_stride, const void* pre, void* grad_x, void* grad_weight, void* grad_bias,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_linear(a, true);
    if (rc == SIG_OK) rc = check_strides({gy_stride});
    if (rc != SIG_OK) return rc;
    if (a->M && (!grad_y || (grad_weight && !a->x) || (grad_x && !a->weight) || (a->act != SIG_ACT_NONE && !pre))) return SIG_EINVAL;
    const size_t need = sig::linear_backward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::linear_backward(*a, grad_y, gy_stride, pre, grad_x, grad_weight, grad_bias, workspace, (hipStream_t)stream));
}

size_t sig_gated_scan_checkpoint_bytes(const sig_gated_args* a) { return check_gated(a) == SIG_OK ? ckpt_bytes(*a) : 0; }
size_t sig_gated_scan_forward_workspace_bytes(const sig_gated_args* a) { return check_gated(a) == SIG_OK ? sig::gated_forward_workspace(*a) : 0; }
size_t sig_gated_scan_backward_workspace_bytes(const sig_gated_args* a) { return check_gated(a) == SIG_OK ? sig::gated_backward_workspace(*a) : 0; }

int sig_gated_scan_forward(const sig_gated_args* a, void* y, float* final_state, void* checkpoint, size_t checkpoint_bytes, void* workspace,
                           size_t workspace_bytes, void* stream)
{
    int rc = check_gated(a);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!a->log_rate || (a->L && (!a->x || !a->decay_gate || !a->input_gate || !y))) return SIG_EINVAL;
    if (checkpoint && checkpoint_bytes < ckpt_bytes(*a)) return SIG_EWORKSPACE;
    const size_t need = sig::gated_forward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::gated_forward(*a, y, final_state, (float*)checkpoint, (float*)workspace, (hipStream_t)stream));
}

int sig_gated_scan_backward(const sig_gated_args* a, const sig_gated_grads* g, const void* checkpoint, size_t checkpoint_bytes, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    int rc = check_gated(a);
    if (rc != SIG_OK) return rc;
    const bool tokens = a->B > 0 && a->L > 0;
    if (!g || !g->grad_log_rate || !a->log_rate) return SIG_EINVAL;
    if (tokens) {
        if (!a->x || !a->decay_gate || !a->input_gate || !g->grad_y || !g->grad_x || !g->grad_decay_gate || !g->grad_input_gate) return SIG_EINVAL;
        rc = check_strides({g->gy_stride_b});
        if (rc != SIG_OK) return rc;
        if (g->gy_stride_t < 0) return SIG_EINVAL;
        if (g->gy_stride_t >= (1 << 22)) return SIG_ETOOLARGE;
        if (!checkpoint) return SIG_EWORKSPACE;
    }
    if (checkpoint_bytes < ckpt_bytes(*a)) return SIG_EWORKSPACE;
    const size_t need = sig::gated_backward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::gated_backward(*a, *g, (const float*)checkpoint, (float*)workspace, (hipStream_t)stream));
}

int sig_gated_scan_step(const sig_gated_args* a, float* state, void* y, void* stream)
{
    int rc = check_gated(a, false);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!a->log_rate || !a->x || !a->decay_gate || !a->input_gate || !state || !y) return SIG_EINVAL;
    return hip_code(sig::gated_step(*a, state, y, (hipStream_t)stream));
}

}  // extern "C"
