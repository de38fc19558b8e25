// Global norm over many tensors, n = sqrt(sum g^2), and the clipped tensors min(1, max_norm / (n + 1e-6)) g.
// Bound by memory: everything is read for the norm and once more for the product, whose input the cache between the chip and its memory
// (256 MB) still holds in part.  Squares are summed in float64: no overflow for any finite float32, and sums whose order is fixed.
#include "seq.hpp"

namespace sig {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = kClipBlock;

struct Piece { int t; int64_t first, count; };
__device__ __forceinline__ Piece piece_of(const ClipTable& tab, uint32_t block)
{
    int lo = 0, hi = tab.n - 1;
    while (lo < hi) {
        int mid = (lo + hi) / 2;
        if (block < tab.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    int64_t first = (int64_t)(block - (lo ? tab.end[lo - 1] : 0)) * kBlock;
    return {lo, first, min((int64_t)kBlock, tab.size[lo] - first)};
}

__device__ __forceinline__ double sum_block(double v)
{
    __shared__ double part[kThreads / 64];
#pragma unroll
    for (int m = 32; m; m /= 2) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; i++) v += part[i];
    return v;
}

template <class T> __device__ __forceinline__ double squares(const T* p, int64_t n)
{
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
        double g = to_float(p[i]);
        v = fma(g, g, v);
    }
    return v;
}

__global__ __launch_bounds__(kThreads) void norm_part_kernel(ClipTable tab, double* part)
{
    Piece p = piece_of(tab, blockIdx.x);
    double v = tab.kind[p.t] & 1 ? squares((const bf16*)tab.in[p.t] + p.first, p.count) : squares((const float*)tab.in[p.t] + p.first, p.count);
    v = sum_block(v);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* part, int64_t n, float* norm)
{
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) v += part[i];
    v = sum_block(v);
    if (threadIdx.x == 0) *norm = (float)sqrt(v);
}

template <class I, class O> __device__ __forceinline__ void scaled(const I* in, O* out, int64_t n, float scale)
{
    for (int64_t i = threadIdx.x; i < n; i += kThreads) out[i] = from_float<O>(to_float(in[i]) * scale);
}

__global__ __launch_bounds__(kThreads) void clip_kernel(ClipTable tab, const float* norm, float max_norm)
{
    Piece p = piece_of(tab, blockIdx.x);
    float q = max_norm / (*norm + 1e-6f), scale = q > 1.0f ? 1.0f : q;      // a NaN stays one
    const void* in = tab.in[p.t];
    void* out = tab.out[p.t];
    switch (tab.kind[p.t]) {
        case 0: scaled((const float*)in + p.first, (float*)out + p.first, p.count, scale); break;
        case 1: scaled((const bf16*)in + p.first, (float*)out + p.first, p.count, scale); break;
        case 2: scaled((const float*)in + p.first, (bf16*)out + p.first, p.count, scale); break;
        default: scaled((const bf16*)in + p.first, (bf16*)out + p.first, p.count, scale); break;
    }
}

}  // namespace

hipError_t norm_parts(const ClipTable& tab, double* part, hipStream_t stream)
{
    norm_part_kernel<<<tab.end[tab.n - 1], kThreads, 0, stream>>>(tab, part);
    return hipGetLastError();
}
hipError_t norm_total(const double* part, int64_t n, float* norm, hipStream_t stream)
{
    norm_kernel<<<1, kThreads, 0, stream>>>(part, n, norm);
    return hipGetLastError();
}
hipError_t clip_scaled(const ClipTable& tab, const float* norm, float max_norm, hipStream_t stream)
{
    clip_kernel<<<tab.end[tab.n - 1], kThreads, 0, stream>>>(tab, norm, max_norm);
    return hipGetLastError();
}

}  // namespace sig
