// C ABI of the sequence operators: checks of arguments, then the launches (see include/sig.h for the contracts).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "seq.hpp"

namespace {

constexpr int64_t kMost = (int64_t)1 << 38;       // bound of sizes and of their products: more than the memory holds, and no overflow below

int hip_code(hipError_t e) { return e == hipSuccess ? SIG_OK : e == sig::kTooManyThreads ? SIG_ETOOLARGE : sig::record_hip_error(e); }

bool bad_type(int64_t t) { return t != SIG_F32 && t != SIG_BF16; }

// SIG_EINVAL for a negative size, SIG_ETOOLARGE where the product of the (non-negative) sizes passes kMost
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

// prompt = false: a call of one token, which does not look at L and at what is there for several
int check_conv(const sig_conv_args* a, bool prompt = true)
{
    if (!a || bad_type(a->dtype) || a->D < 1 || a->W < 1) return SIG_EINVAL;
    if (a->W > SIG_MAX_CONV_WIDTH) return SIG_EUNSUPPORTED;
    if (a->silu != 0 && a->silu != 1) return SIG_EINVAL;
    return check_sizes({a->B, prompt ? a->L : 1, a->D});
}

int check_scan(const sig_scan_args* a, bool prompt = true)
{
    if (!a || bad_type(a->dtype) || a->D < 1 || a->G < 1 || a->N < 1 || a->D % a->G != 0) return SIG_EINVAL;
    if (a->N > SIG_MAX_SCAN_STATES) return SIG_EUNSUPPORTED;
    if (a->softplus != 0 && a->softplus != 1) return SIG_EINVAL;
    // a launch numbers at least the streams' channels; the kernels count tokens in 32 bits and reach those of a tile by 32-bit offsets
    if (a->B > 0 && a->D > INT32_MAX / a->B) return SIG_ETOOLARGE;
    if (prompt && a->L >= (1 << 30)) return SIG_ETOOLARGE;        // a chunk's end is at most L rounded up to tiles, times two at the most
    for (int64_t s : {prompt ? a->x_stride_t : 0, prompt ? a->dt_stride_t : 0, prompt ? a->gate_stride_t : 0, a->b_stride_t, a->c_stride_t, a->D})
        if (s < 0 || s >= (1 << 24)) return s < 0 ? SIG_EINVAL : SIG_ETOOLARGE;
    for (int64_t s : {a->b_stride_t, a->c_stride_t})           // the kernels tell tokens that count from others by where their rows end
        if (prompt && a->L > 1 && s > 0 && s < a->N) return SIG_EINVAL;
    return check_sizes({a->B, prompt ? a->L : 1, a->D, a->N});
}

bool scan_inputs_there(const sig_scan_args& a, bool tokens)
{
    return a.A && (!tokens || (a.x && a.dt && a.b && a.c));
}

// Elements of a workgroup of the clipping kernels: 4,096 until the chip is full, then twice as many as often as it takes to keep the sums that
// one workgroup adds up in the end few.
int64_t clip_block(int64_t total)
{
    int64_t block = sig::kClipBlock;
    while (total / block > sig::kClipBlocks && block < (1 << 30)) block *= 2;
    return block;
}

// Products beyond the size of the cache before the memory (256 MB) would not be there for whoever reads them next; they are stored past it: 166e6
// elements, 340 MB into 662 MB, call after call on the same tensors 243 us, 275 through the cache.  Smaller ones stay in it: 128 MB and the next kernel's pass over them 91 us, 110 past it.
constexpr int64_t kCacheBytes = 256 << 20;

size_t ckpt_bytes(const sig_scan_args& a) { return (size_t)(a.B * ((a.L + sig::kScanTile - 1) / sig::kScanTile) * a.D * a.N * 4); }

}  // namespace

extern "C" {

int sig_conv_forward(const sig_conv_args* a, void* y, void* final_state, void* stream)
{
    int rc = check_conv(a);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!a->weight || (a->L && (!a->x || !y))) return SIG_EINVAL;
    return hip_code(sig::conv_forward(*a, y, final_state, (hipStream_t)stream));
}

size_t sig_conv_backward_workspace_bytes(const sig_conv_args* a) { return check_conv(a) == SIG_OK ? sig::conv_backward_workspace(*a) : 0; }

int sig_conv_backward(const sig_conv_args* a, const void* grad_y, int64_t gy_stride_b, int64_t gy_stride_t, const void* grad_final_state,
                      void* grad_x, float* grad_weight, float* grad_bias, void* grad_initial_state, void* workspace, size_t workspace_bytes,
                      void* stream)
{
    int rc = check_conv(a);
    if (rc != SIG_OK) return rc;
    if (!a->weight || !grad_weight || (a->B && a->L && (!a->x || !grad_y || !grad_x))) return SIG_EINVAL;
    if (workspace_bytes < sig::conv_backward_workspace(*a) || (!workspace && sig::conv_backward_workspace(*a))) return SIG_EWORKSPACE;
    sig::ConvGrads g{grad_y, gy_stride_b, gy_stride_t, grad_final_state, grad_x, grad_weight, grad_bias, grad_initial_state};
    return hip_code(sig::conv_backward(*a, g, (float*)workspace, (hipStream_t)stream));
}

int sig_conv_step(const sig_conv_args* a, void* state, void* y, void* stream)
{
    int rc = check_conv(a, false);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!a->weight || !a->x || !y || (a->W > 1 && !state)) return SIG_EINVAL;
    return hip_code(sig::conv_step(*a, state, y, (hipStream_t)stream));
}

size_t sig_scan_checkpoint_bytes(const sig_scan_args* a) { return check_scan(a) == SIG_OK ? ckpt_bytes(*a) : 0; }
size_t sig_scan_forward_workspace_bytes(const sig_scan_args* a) { return check_scan(a) == SIG_OK ? sig::scan_forward_workspace(*a) : 0; }
size_t sig_scan_backward_workspace_bytes(const sig_scan_args* a) { return check_scan(a) == SIG_OK ? sig::scan_backward_workspace(*a) : 0; }

int sig_scan_forward(const sig_scan_args* a, void* y, float* final_state, void* checkpoint, size_t checkpoint_bytes, void* workspace,
                     size_t workspace_bytes, void* stream)
{
    int rc = check_scan(a);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!scan_inputs_there(*a, a->L > 0) || (a->L && !y)) return SIG_EINVAL;
    if (checkpoint && checkpoint_bytes < ckpt_bytes(*a)) return SIG_EWORKSPACE;
    size_t need = sig::scan_forward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::scan_forward(*a, y, final_state, (float*)checkpoint, (float*)workspace, (hipStream_t)stream));
}

int sig_scan_backward(const sig_scan_args* a, const sig_scan_grads* g, const void* checkpoint, size_t checkpoint_bytes, void* workspace,
                      size_t workspace_bytes, void* stream)
{
    int rc = check_scan(a);
    if (rc != SIG_OK) return rc;
    bool tokens = a->B > 0 && a->L > 0;
    if (!g || !g->grad_A || !scan_inputs_there(*a, tokens)) return SIG_EINVAL;
    if (tokens && g->gy_stride_t < 0) return SIG_EINVAL;
    if (tokens && g->gy_stride_t >= (1 << 24)) return SIG_ETOOLARGE;
    if ((a->skip && !g->grad_skip) || (a->dt_bias && !g->grad_dt_bias)) return SIG_EINVAL;
    if (tokens && (!g->grad_y || !g->grad_x || !g->grad_dt || !g->grad_b || !g->grad_c || (a->gate && !g->grad_gate))) return SIG_EINVAL;
    if (checkpoint_bytes < ckpt_bytes(*a) || (tokens && !checkpoint)) return SIG_EWORKSPACE;
    size_t need = sig::scan_backward_workspace(*a);
    if (workspace_bytes < need || (need && !workspace)) return SIG_EWORKSPACE;
    return hip_code(sig::scan_backward(*a, *g, (const float*)checkpoint, (float*)workspace, (hipStream_t)stream));
}

int sig_scan_step(const sig_scan_args* a, float* state, void* y, void* stream)
{
    int rc = check_scan(a, false);
    if (rc != SIG_OK || a->B == 0) return rc;
    if (!scan_inputs_there(*a, true) || !state || !y) return SIG_EINVAL;
    return hip_code(sig::scan_step(*a, state, y, (hipStream_t)stream));
}

size_t sig_grad_clip_workspace_bytes(int64_t n_tensors, const int64_t* sizes)
{
    if (n_tensors <= 0 || !sizes) return 0;
    int64_t total = 0, blocks = 0;
    for (int64_t i = 0; i < n_tensors; i++) {
        if (sizes[i] < 0 || sizes[i] > kMost || (total += sizes[i]) > kMost) return 0;
    }
    const int64_t block = clip_block(total);
    for (int64_t i = 0; i < n_tensors; i++) blocks += (sizes[i] + block - 1) / block;
    return (size_t)blocks * sizeof(double);
}

int sig_grad_clip(int64_t n_tensors, const void* const* in, void* const* out, const int64_t* sizes, const int64_t* in_dtypes,
                  const int64_t* out_dtypes, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (n_tensors < 0 || !norm || !(max_norm >= 0.0f)) return SIG_EINVAL;
    if (n_tensors && (!in || !out || !sizes || !in_dtypes || !out_dtypes)) return SIG_EINVAL;
    int64_t total = 0, blocks = 0, written = 0;
    for (int64_t i = 0; i < n_tensors; i++) {
        if (sizes[i] < 0 || bad_type(in_dtypes[i]) || bad_type(out_dtypes[i])) return SIG_EINVAL;
        if (sizes[i] && (!in[i] || !out[i] || (in[i] == out[i] && in_dtypes[i] != out_dtypes[i]))) return SIG_EINVAL;
        if (sizes[i] > kMost || (total += sizes[i]) > kMost) return SIG_ETOOLARGE;
        written += sizes[i] * (out_dtypes[i] == SIG_BF16 ? 2 : 4);
    }
    const int64_t block = clip_block(total);
    for (int64_t i = 0; i < n_tensors; i++) blocks += (sizes[i] + block - 1) / block;
    if (workspace_bytes < (size_t)blocks * sizeof(double) || (blocks && !workspace)) return SIG_EWORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    // all tables of the norm first, then its square root, then the tables of the products in the opposite order, whose kernel goes
    // backwards too: it begins with what the cache still holds
    const int64_t per = sig::kClipTensors, tables = (n_tensors + per - 1) / per;
    double* part = (double*)workspace;
    for (int64_t k = 0; k < 2 * tables; k++) {
        if (k == tables) {
            hipError_t e = sig::norm_total((const double*)workspace, blocks, norm, s);
            if (e != hipSuccess) return sig::record_hip_error(e);
        }
        const int64_t first = per * (k < tables ? k : 2 * tables - 1 - k), last = std::min(n_tensors, first + per);
        sig::ClipTable tab;
        tab.n = 0;
        tab.block = (uint32_t)block;
        for (int64_t i = first; i < last; i++) {
            if (!sizes[i]) continue;
            const int j = tab.n++;
            tab.in[j] = in[i];
            tab.out[j] = out[i];
            tab.size[j] = sizes[i];
            tab.kind[j] = (uint8_t)(in_dtypes[i] | out_dtypes[i] << 1);
            tab.end[j] = (j ? tab.end[j - 1] : 0) + (uint32_t)((sizes[i] + block - 1) / block);
        }
        if (tab.n == 0) continue;
        hipError_t e = k < tables ? sig::norm_parts(tab, part, s) : sig::clip_scaled(tab, norm, max_norm, written > kCacheBytes, s);
        if (e != hipSuccess) return sig::record_hip_error(e);
        part += k < tables ? tab.end[tab.n - 1] : 0;
    }
    if (tables == 0) {
        hipError_t e = sig::norm_total((const double*)workspace, 0, norm, s);
        if (e != hipSuccess) return sig::record_hip_error(e);
    }
    return SIG_OK;
}

}  // extern "C"
