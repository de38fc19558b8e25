// Sequence operators over tokens [batch, time, channels]: launch interface between the C ABI (api_seq.cpp) and the HIP kernels, and the
// device functions that these kernels share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/sig.h"

namespace sig {

int record_hip_error(hipError_t e);     // keeps it for sig_last_hip_error and returns SIG_EHIP (api.cpp)

// The hardware numbers the threads of a launch in 32 bits.  Where a call would need more in one of its launches, the functions below return
// kTooManyThreads and enqueue nothing; the calls then return SIG_ETOOLARGE.
constexpr hipError_t kTooManyThreads = hipErrorInvalidConfiguration;
inline bool launchable(int64_t workgroups, int64_t threads) { return workgroups <= 0xffffffffll / threads; }

// ---- convolution (kernels_conv.hip)
struct ConvGrads {
    const void* grad_y;                 // [B, L, D] with its own strides
    int64_t gy_stride_b, gy_stride_t;
    const void* grad_final;             // [B, W - 1, D] or null
    void* grad_x;                       // [B, L, D]
    float* grad_weight;                 // [D, W]
    float* grad_bias;                   // [D] or null
    void* grad_initial;                 // [B, W - 1, D] or null
};
hipError_t conv_forward(const sig_conv_args& a, void* y, void* final_state, hipStream_t stream);
size_t conv_backward_workspace(const sig_conv_args& a);
hipError_t conv_backward(const sig_conv_args& a, const ConvGrads& g, float* workspace, hipStream_t stream);
hipError_t conv_step(const sig_conv_args& a, void* state, void* y, hipStream_t stream);

// ---- selective scan (kernels_scan.hip)
constexpr int kScanTile = 16;           // tokens between two states of a checkpoint
size_t scan_forward_workspace(const sig_scan_args& a);
size_t scan_backward_workspace(const sig_scan_args& a);
hipError_t scan_forward(const sig_scan_args& a, void* y, float* final_state, float* checkpoint, float* workspace, hipStream_t stream);
hipError_t scan_backward(const sig_scan_args& a, const sig_scan_grads& g, const float* checkpoint, float* workspace, hipStream_t stream);
hipError_t scan_step(const sig_scan_args& a, float* state, void* y, hipStream_t stream);

// ---- gradient norm and clipping (kernels_clip.hip)
constexpr int kClipTensors = 128;       // tensors that one launch takes: their table is a kernel argument (of at most 4 KB)
constexpr int kClipBlock = 4096;        // elements of a workgroup, at least
constexpr int kClipBlocks = 16384;      // workgroups that all tensors are spread over at most, about (166e6 elements: 8 % less time than with 4,096)
struct ClipTable {
    const void* in[kClipTensors];
    void* out[kClipTensors];
    int64_t size[kClipTensors];         // elements of the tensor
    uint32_t end[kClipTensors];         // workgroups up to and with this tensor
    uint8_t kind[kClipTensors];         // bit 0: in is bf16, bit 1: out is bf16
    int n;
    uint32_t block;                     // elements of a workgroup
};
hipError_t norm_parts(const ClipTable& tab, double* part, hipStream_t stream);     // part: one sum of squares for each workgroup
hipError_t norm_total(const double* part, int64_t n, float* norm, hipStream_t stream);
hipError_t clip_scaled(const ClipTable& tab, const float* norm, float max_norm, bool past_cache, hipStream_t stream);

#ifdef __HIPCC__
// ---- device side
struct bf16 { uint16_t bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v)     // to nearest, ties to even (a conversion of the hardware)
{
    __bf16 h = (__bf16)v;
    bf16 r;
    __builtin_memcpy(&r, &h, 2);
    return r;
}

// V consecutive elements, one access of V * sizeof(T) bytes: the address is a multiple of that
template <class T, int V> struct alignas(V * sizeof(T)) Pack { T v[V]; };

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float fast_exp(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
// The exponent v log2(e) is rounded, so exp is off by up to |v| 2^-24 of itself and a few units in the last place besides; so are sigmoid where v is
// far below zero, a value of the size of exp(v), and a decay exp(D A), which that far down has little left to be off by.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + fast_exp(-v)); }

// log(1 + exp(v)) = max(v, 0) + log(1 + e) with e = exp(-|v|) <= 1, and log(1 + e) = 2 artanh(s) with s = e / (2 + e) <= 1/3: the
// power series 2 s (1 + s^2/3 + s^4/5 + ..) keeps its relative precision where e is small (step sizes of 1e-3), which the logarithm of a
// rounded 1 + e does not.  The first omitted term is s^14 / 15 < 2e-8.
__device__ __forceinline__ float softplus(float v)
{
    float e = fast_exp(-fabsf(v));
    float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float p = fmaf(q, 1.0f / 13.0f, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 1.0f / 5.0f);
    p = fmaf(p, q, 1.0f / 3.0f);
    p = fmaf(p, q, 1.0f);
    return fmaxf(v, 0.0f) + 2.0f * s * p;
}

// The sum over rows of a column, p[r step], by a workgroup of sixteen wavefronts whose lanes have a column each: wavefront w adds up rows
// w, w + 16, .., the first one their sums in order.  Returned to the first wavefront.
__device__ __forceinline__ float sum_rows(const float* p, int64_t rows, int64_t step)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x / 64;
    float v[4] = {};
    int64_t r = w;
    for (; r + 112 < rows; r += 128) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; i++) q[i] = p[(r + 16 * i) * step];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i % 4] += q[i];
    }
    for (; r < rows; r += 16) v[0] += p[r * step];
    part[w][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    float s = 0.0f;
    if (w == 0)
#pragma unroll
        for (int i = 0; i < 16; i++) s += part[i][lane];
    return s;
}

__device__ __forceinline__ int64_t live_length(const int32_t* lengths, int64_t b, int64_t L)
{
    if (!lengths) return L;
    int64_t n = lengths[b];
    return n < 0 ? 0 : (n > L ? L : n);
}
#endif

}  // namespace sig
