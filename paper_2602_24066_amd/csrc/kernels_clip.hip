// Global norm over many tensors, n = sqrt(sum g^2), and the clipped tensors min(1, max_norm / (n + 1e-6)) g.
// Bound by memory: everything is read for the norm and once more for the product, whose input the cache between the chip and its memory
// (256 MB) still holds in part.  166e6 elements, 340 MB (bfloat16, the small ones float32) into 662 MB of float32, call after call: 58 us for the
// norm, 169 us for the product (5.9 TB/s each, above a large copy's 5.1 by the cache's part), 5 us for the sum of the parts between them.
// Squares are summed in float64, in a fixed order: none overflows.  A norm beyond what float32 holds is infinite, and the finite products are 0 then.
#include "seq.hpp"

namespace sig {
namespace {

constexpr int kThreads = 256;

struct Piece { int t; int64_t first, count; };
__device__ __forceinline__ Piece piece_of(const ClipTable& tab, uint32_t block)
{
    int lo = 0, hi = tab.n - 1;
    while (lo < hi) {
        int mid = (lo + hi) / 2;
        if (block < tab.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    int64_t first = (int64_t)(block - (lo ? tab.end[lo - 1] : 0)) * tab.block;
    return {lo, first, min((int64_t)tab.block, tab.size[lo] - first)};
}

template <int N> __device__ __forceinline__ double sum_block(double v)      // over N threads
{
    __shared__ double part[N / 64];
#pragma unroll
    for (int m = 32; m; m /= 2) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < N / 64; i++) v += part[i];
    return v;
}

template <class T> __device__ __forceinline__ double squares(const T* p, int64_t n)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    const int64_t head = min(n, (int64_t)((-(uintptr_t)p & 15) / sizeof(T))), vecs = (n - head) / V, tail = head + vecs * V;
    double v = 0.0;
    auto add = [&](T x) {
        double g = to_float(x);
        v = fma(g, g, v);
    };
    if (threadIdx.x < head) add(p[threadIdx.x]);
    if (tail + threadIdx.x < n) add(p[tail + threadIdx.x]);
    const Pack<T, V>* q = (const Pack<T, V>*)(p + head);
    int64_t i = threadIdx.x;
    for (; i + (U - 1) * kThreads < vecs; i += U * kThreads) {
        Pack<T, V> r[U];
#pragma unroll
        for (int u = 0; u < U; u++) r[u] = q[i + u * kThreads];
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int k = 0; k < V; k++) add(r[u].v[k]);
    }
    for (; i < vecs; i += kThreads)
#pragma unroll
        for (int k = 0; k < V; k++) add(q[i].v[k]);
    return v;
}

__global__ __launch_bounds__(kThreads) void norm_part_kernel(ClipTable tab, double* part)
{
    Piece p = piece_of(tab, blockIdx.x);
    double v = tab.kind[p.t] & 1 ? squares((const bf16*)tab.in[p.t] + p.first, p.count) : squares((const float*)tab.in[p.t] + p.first, p.count);
    v = sum_block<kThreads>(v);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

__global__ __launch_bounds__(1024) void norm_kernel(const double* part, int64_t n, float* norm)
{
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) v += part[i];
    v = sum_block<1024>(v);
    if (threadIdx.x == 0) *norm = (float)sqrt(v);
}

template <class P> __device__ __forceinline__ void store_past_cache(P* to, const P& v)
{
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(P) / 4)));
    Words w;
    __builtin_memcpy(&w, &v, sizeof(P));
    __builtin_nontemporal_store(w, (Words*)to);
}

// Accesses of 16 bytes of the narrower side where both sides allow it, of single elements otherwise (views at odd offsets)
template <bool kPast, class I, class O> __device__ __forceinline__ void scaled(const I* in, O* out, int64_t n, float scale)
{
    constexpr int V = 16 / (sizeof(I) > sizeof(O) ? sizeof(I) : sizeof(O)), U = 4;
    const uintptr_t pi = (uintptr_t)in, po = (uintptr_t)out;
    int64_t head = min(n, (int64_t)((-po & (V * sizeof(O) - 1)) / sizeof(O)));
    if (((pi + head * sizeof(I)) & (V * sizeof(I) - 1)) != 0) head = n;
    const int64_t vecs = (n - head) / V, tail = head + vecs * V;
    const Pack<I, V>* q = (const Pack<I, V>*)(in + head);
    Pack<O, V>* to = (Pack<O, V>*)(out + head);
    auto one = [&](const Pack<I, V>& r) {
        Pack<O, V> w;
#pragma unroll
        for (int k = 0; k < V; k++) w.v[k] = from_float<O>(to_float(r.v[k]) * scale);
        return w;
    };
    int64_t i = threadIdx.x;
    for (; i + (U - 1) * kThreads < vecs; i += U * kThreads) {
        Pack<I, V> r[U];
#pragma unroll
        for (int u = 0; u < U; u++) r[u] = q[i + u * kThreads];
#pragma unroll
        for (int u = 0; u < U; u++) {
            if constexpr (kPast) store_past_cache(to + i + u * kThreads, one(r[u]));
            else to[i + u * kThreads] = one(r[u]);
        }
    }
    for (; i < vecs; i += kThreads) to[i] = one(q[i]);
    for (i = threadIdx.x; i < head; i += kThreads) out[i] = from_float<O>(to_float(in[i]) * scale);
    for (i = tail + threadIdx.x; i < n; i += kThreads) out[i] = from_float<O>(to_float(in[i]) * scale);
}

// kPast: the products go past the cache, which keeps what it holds of the tensors that are still to be read
template <bool kPast> __global__ __launch_bounds__(kThreads) void clip_kernel(ClipTable tab, const float* norm, float max_norm)
{
    // from the last workgroup to the first: what the norm read last is still in the cache
    Piece p = piece_of(tab, gridDim.x - 1 - blockIdx.x);
    float q = max_norm / (*norm + 1e-6f), scale = q > 1.0f ? 1.0f : q;      // a NaN stays one
    const void* in = tab.in[p.t];
    void* out = tab.out[p.t];
    switch (tab.kind[p.t]) {
        case 0: scaled<kPast>((const float*)in + p.first, (float*)out + p.first, p.count, scale); break;
        case 1: scaled<kPast>((const bf16*)in + p.first, (float*)out + p.first, p.count, scale); break;
        case 2: scaled<kPast>((const float*)in + p.first, (bf16*)out + p.first, p.count, scale); break;
        default: scaled<kPast>((const bf16*)in + p.first, (bf16*)out + p.first, p.count, scale); break;
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
    norm_kernel<<<1, 1024, 0, stream>>>(part, n, norm);
    return hipGetLastError();
}
hipError_t clip_scaled(const ClipTable& tab, const float* norm, float max_norm, bool past_cache, hipStream_t stream)
{
    if (past_cache) clip_kernel<true><<<tab.end[tab.n - 1], kThreads, 0, stream>>>(tab, norm, max_norm);
    else clip_kernel<false><<<tab.end[tab.n - 1], kThreads, 0, stream>>>(tab, norm, max_norm);
    return hipGetLastError();
}

}  // namespace sig
