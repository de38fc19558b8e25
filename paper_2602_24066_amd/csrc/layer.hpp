// Operators of a layer (norm, matrix product, gated recurrence): launch interface between the C ABI (api_layer.cpp) and the HIP kernels.
#pragma once
#include "seq.hpp"

namespace sig {

// ---- norm (kernels_norm.hip)
struct NormGrads {
    const void* grad_y;
    int64_t gy_stride;
    const void* grad_total;             // or null
    int64_t gt_stride;
    void* grad_x;
    float* grad_weight;
};
hipError_t norm_forward(const sig_norm_args& a, void* y, float* scale, void* total, hipStream_t stream);     // weight null: rows to 8 bits as they are
size_t norm_backward_workspace(const sig_norm_args& a);
hipError_t norm_backward(const sig_norm_args& a, const NormGrads& g, float* workspace, hipStream_t stream);

// ---- matrix product (kernels_linear.hip)
size_t linear_forward_workspace(const sig_linear_args& a);
hipError_t linear_forward(const sig_linear_args& a, void* y, void* pre, void* workspace, hipStream_t stream);
size_t linear_backward_workspace(const sig_linear_args& a);
hipError_t linear_backward(const sig_linear_args& a, const void* grad_y, int64_t gy_stride, const void* pre, void* grad_x, void* grad_weight,
                           void* grad_bias, void* workspace, hipStream_t stream);

// ---- gated recurrence (kernels_gated.hip)
constexpr int kGatedTile = 16;          // tokens between two states of a checkpoint
size_t gated_forward_workspace(const sig_gated_args& a);
size_t gated_backward_workspace(const sig_gated_args& a);
hipError_t gated_forward(const sig_gated_args& a, void* y, float* final_state, float* checkpoint, float* workspace, hipStream_t stream);
hipError_t gated_backward(const sig_gated_args& a, const sig_gated_grads& g, const float* checkpoint, float* workspace, hipStream_t stream);
hipError_t gated_step(const sig_gated_args& a, float* state, void* y, hipStream_t stream);

#ifdef __HIPCC__
struct e4m3 { uint8_t bits; };
// to nearest, ties to even, values a little beyond 448 to 448, a NaN stays one (conversion of the hardware)
template <> __device__ __forceinline__ e4m3 from_float<e4m3>(float v) { return {(uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xff)}; }

// V values of float32 or bfloat16 in words, as they lie in memory (elements of their own would take a register each)
template <class T, int V, bool kWhole = V * sizeof(T) % 4 == 0> struct Words {
    typedef uint32_t Vector __attribute__((ext_vector_type(V * sizeof(T) / 4)));
    Vector w;
    __device__ __forceinline__ void load(const T* p) { w = *(const Vector*)p; }
    __device__ __forceinline__ float value(int j) const { return sizeof(T) == 4 ? __uint_as_float(w[j]) : __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); }
};
template <> struct Words<bf16, 1, false> {
    uint16_t w;
    __device__ __forceinline__ void load(const bf16* p) { w = p->bits; }
    __device__ __forceinline__ float value(int) const { return __uint_as_float((uint32_t)w << 16); }
};

// Neighbouring values as they lie in memory, converted two (bfloat16, e4m3) an instruction; V a multiple of the values of a word
__device__ __forceinline__ uint32_t word_of(const float* v, bf16*)
{
    typedef float F2 __attribute__((ext_vector_type(2)));
    typedef __bf16 B2 __attribute__((ext_vector_type(2)));
    const B2 h = __builtin_convertvector(F2{v[0], v[1]}, B2);
    uint32_t w;
    __builtin_memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ uint32_t word_of(const float* v, float*) { return __float_as_uint(v[0]); }
__device__ __forceinline__ uint32_t word_of(const float* v, e4m3*)
{
    return __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), true);
}
template <class T, int V> __device__ __forceinline__ void store_words(T* p, const float* v)
{
    constexpr int kEach = 4 / sizeof(T), kWords = V / kEach;
    typedef uint32_t Vector __attribute__((ext_vector_type(kWords)));
    Vector w;
#pragma unroll
    for (int i = 0; i < kWords; i++) w[i] = word_of(v + i * kEach, (T*)nullptr);
    *(Vector*)p = w;
}
#endif

}  // namespace sig
