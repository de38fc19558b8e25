// Root-mean-square norm of rows with the residual's addition, rows to 8 bits, and the norm's gradient.
//
//   r = x + residual (rounded to the tokens' type: the stream as it is kept),  s = rsqrt(mean r^2 + eps),  y = r s weight,
//   8 bits: y / scale in e4m3 with scale = max |y| / 448
//   gradient: h = weight grad_y, n = r s:  grad_x = s (h - n mean(h n)) + grad_r,  grad_weight = sum over rows of grad_y n
//
// Bound by memory: a row is held in the registers of 64, 256 or 1,024 threads, so that everything is read once and written once.  Rows longer than
// that are read again for each pass.  32,768 rows of 2,048 bfloat16 values with a residual to 8 bits: 96 us, 4.9 TB/s (a copy: 5.1).  The gradient's workgroups keep the same columns for all their rows, so the weight's sums stay in
// registers too; a second kernel adds them up over workgroups in a fixed order.  11,137 rows of 333 float32 values, single accesses: forward 14.6 us,
// gradient 16.9 and 3.8, bound by the latency of a row's loads.
#include <algorithm>
#include <type_traits>

#include "layer.hpp"

namespace sig {
namespace {

// Sum (or largest magnitude, kMax; a NaN wins) over the threads of a row: all lanes get it.  The workgroup is the row, or every wavefront is one.
template <int kThreads, bool kMax> __device__ __forceinline__ float over_row(float v)
{
    auto join = [](float a, float b) { return kMax ? (a > b || a != a ? a : b) : a + b; };
#pragma unroll
    for (int m = 32; m; m /= 2) v = join(v, __shfl_xor(v, m));
    if constexpr (kThreads > 64) {
        __shared__ float part[kThreads / 64];
        __syncthreads();                                                       // the last call's readers are done
        if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int i = 1; i < kThreads / 64; i++) v = join(v, part[i]);
    }
    return v;
}

template <class T, int V> __device__ __forceinline__ void load(const T* p, float* v)
{
    const Pack<T, V> r = *(const Pack<T, V>*)p;
#pragma unroll
    for (int j = 0; j < V; j++) v[j] = to_float(r.v[j]);
}
template <class T, int V> __device__ __forceinline__ void store(T* p, const float* v)
{
    if constexpr (V * sizeof(T) >= 4) store_words<T, V>(p, v);
    else
#pragma unroll
        for (int j = 0; j < V; j++) p[j] = from_float<T>(v[j]);
}

// A row's scale, and its values over it: v 448 / top.  The quotient is corrected once, so that one that float32 holds is met: quotients of bfloat16 values
// lie on the borders between two values of e4m3 now and then, and ties go to even.
struct Scaled {
    float scale, up, times, top;
    __device__ __forceinline__ float of(float v) const
    {
        const float t = v * times;
        return fmaf(fmaf(-t, top, v * up), times * (1.0f / 448.0f), t);
    }
};
__device__ __forceinline__ Scaled scale_of(float top)
{
    // 448 / top would overflow where top is tiny; 2^126 takes such values to at most 128.  Products with 448 stay finite below 2^100.
    if (top == 0.0f) return {0.0f, 1.0f, 1.0f, 1.0f};
    if (top < 0x1p-100f) return top < 0x1p-119f ? Scaled{0x1p-126f, 0.0f, 0x1p126f, 0.0f} : Scaled{top / 448.0f, 0.0f, 448.0f / top, 0.0f};
    if (!(top < 0x1p100f)) return {top / 448.0f, 0.0f, 448.0f / top, 0.0f};
    return {top / 448.0f, 448.0f, 448.0f / top, top};
}

// T: type of x, residual and total; O: of y.  V elements an access, N accesses of a thread, kThreads threads a row (64: four rows a workgroup).
template <class T, class O, bool kNorm, int V, int N, int kThreads>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) void norm_kernel(sig_norm_args a, O* y, float* scale, T* total)
{
    constexpr bool kEight = sizeof(O) == 1;
    const int64_t row = kThreads == 64 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x;
    const int lane = kThreads == 64 ? threadIdx.x & 63 : threadIdx.x, C = (int)a.C;
    if (row >= a.rows) return;
    const T *x = (const T*)a.x + row * a.x_stride, *res = (const T*)a.residual + row * a.residual_stride;
    float v[N][V], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int c = (i * kThreads + lane) * V;
        if (c < C) load<T, V>(x + c, v[i]);
        else
#pragma unroll
            for (int j = 0; j < V; j++) v[i][j] = 0.0f;
    }
    if (kNorm && a.residual) {
        float w[N][V];
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c < C) load<T, V>(res + c, w[i]);
        }
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c < C) {
#pragma unroll
                for (int j = 0; j < V; j++) v[i][j] = to_float(from_float<T>(v[i][j] + w[i][j]));
                if (total) store<T, V>(total + row * C + c, v[i]);
            }
        }
    }
    float top = 0.0f, s = 1.0f;
    if constexpr (kNorm) {
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int j = 0; j < V; j++) sum = fmaf(v[i][j], v[i][j], sum);
        s = rsqrtf(over_row<kThreads, false>(sum) / (float)C + (float)a.eps);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c >= C) continue;
            float w[V];
            load<float, V>(a.weight + c, w);
#pragma unroll
            for (int j = 0; j < V; j++) v[i][j] = kEight ? v[i][j] * w[j] : v[i][j] * s * w[j];     // in 8 bits the row's factor goes into its scale
        }
    }
    if constexpr (kEight) {
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int j = 0; j < V; j++) top = top > fabsf(v[i][j]) || top != top ? top : fabsf(v[i][j]);
        const Scaled q = scale_of(over_row<kThreads, true>(top));
        if (lane == 0) scale[row] = q.scale * s;
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int j = 0; j < V; j++) v[i][j] = q.of(v[i][j]);
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int c = (i * kThreads + lane) * V;
        if (c < C) store<O, V>(y + row * C + c, v[i]);
    }
}

// Rows that no thread count holds: read once for the sum, once for the largest magnitude (8 bits), once for the output
template <class T, class O, bool kNorm> __global__ __launch_bounds__(1024) void norm_long_kernel(sig_norm_args a, O* y, float* scale, T* total)
{
    constexpr bool kEight = sizeof(O) == 1;
    const int64_t row = blockIdx.x, C = a.C;
    const T *x = (const T*)a.x + row * a.x_stride, *res = (const T*)a.residual + row * a.residual_stride;
    auto at = [&](int64_t c) {
        const float v = to_float(x[c]);
        return kNorm && a.residual ? to_float(from_float<T>(v + to_float(res[c]))) : v;
    };
    float s = 1.0f;
    if constexpr (kNorm) {
        float sum = 0.0f;
        for (int64_t c = threadIdx.x; c < C; c += 1024) {
            const float v = at(c);
            sum = fmaf(v, v, sum);
            if (a.residual && total) total[row * C + c] = from_float<T>(v);
        }
        s = rsqrtf(over_row<1024, false>(sum) / (float)C + (float)a.eps);
    }
    auto out = [&](int64_t c) { return !kNorm ? at(c) : kEight ? at(c) * a.weight[c] : at(c) * s * a.weight[c]; };
    Scaled q{};
    if constexpr (kEight) {
        float top = 0.0f;
        for (int64_t c = threadIdx.x; c < C; c += 1024) {
            const float v = fabsf(out(c));
            top = top > v || top != top ? top : v;
        }
        q = scale_of(over_row<1024, true>(top));
        if (threadIdx.x == 0) scale[row] = q.scale * s;
    }
    for (int64_t c = threadIdx.x; c < C; c += 1024) y[row * C + c] = from_float<O>(kEight ? q.of(out(c)) : out(c));
}

template <class T, int V, int N, int kThreads>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) void norm_grad_kernel(sig_norm_args a, NormGrads g, float* parts)
{
    constexpr int kRows = kThreads == 64 ? 4 : 1;
    const int lane = kThreads == 64 ? threadIdx.x & 63 : threadIdx.x, C = (int)a.C;
    float sums[N][V] = {};
    // a row's values are under way while the row before is worked on, where the registers hold both.  Every wavefront (or workgroup) walks its own rows: barriers inside over_row only
    // where the workgroup is the row.
    struct { Words<T, V> r[N], gy[N], gt[N]; } now, next;
    auto load_row = [&](int64_t row, auto& to) {
        const T *r = (const T*)a.x + row * a.x_stride, *gy = (const T*)g.grad_y + row * g.gy_stride, *gt = (const T*)g.grad_total + row * g.gt_stride;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c >= C) continue;
            to.r[i].load(r + c);
            to.gy[i].load(gy + c);
            if (g.grad_total) to.gt[i].load(gt + c);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kRows + (kThreads == 64 ? threadIdx.x / 64 : 0);
    constexpr bool kAhead = kThreads < 1024 && N * V * (6 * (int)sizeof(T) / 4 + 1) <= 160;
    if (kAhead && row < a.rows) load_row(row, next);
    for (; row < a.rows; row += (int64_t)gridDim.x * kRows) {
        if constexpr (kAhead) {
            now = next;
            if (row + (int64_t)gridDim.x * kRows < a.rows) load_row(row + (int64_t)gridDim.x * kRows, next);
        } else load_row(row, now);
        float square = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c >= C) continue;
            float w[V];
            load<float, V>(a.weight + c, w);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float v = now.r[i].value(j);
                square = fmaf(v, v, square);
                dot = fmaf(v * w[j], now.gy[i].value(j), dot);
            }
        }
        const float s = rsqrtf(over_row<kThreads, false>(square) / (float)C + (float)a.eps);
        const float m = over_row<kThreads, false>(dot) / (float)C * s * s;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c >= C) continue;
            float w[V], o[V];
            load<float, V>(a.weight + c, w);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float v = now.r[i].value(j), h = now.gy[i].value(j);
                o[j] = s * (h * w[j] - v * m);
                if (g.grad_total) o[j] += now.gt[i].value(j);
                sums[i][j] = fmaf(h, v * s, sums[i][j]);
            }
            store<T, V>((T*)g.grad_x + row * C + c, o);
        }
    }
    float* to = parts + (int64_t)blockIdx.x * C;
    if constexpr (kThreads == 64) {                                            // the four rows' sums
        __shared__ float join[4][64 * V];
#pragma unroll
        for (int i = 0; i < N; i++) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; j++) join[threadIdx.x / 64][lane * V + j] = sums[i][j];
            __syncthreads();
            for (int k = threadIdx.x; k < 64 * V; k += 256)
                if (i * 64 * V + k < C) to[i * 64 * V + k] = (join[0][k] + join[1][k]) + (join[2][k] + join[3][k]);
        }
    } else
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int c = (i * kThreads + lane) * V;
            if (c < C) store<float, V>(to + c, sums[i]);
        }
}

// Long rows: the tokens' gradient and the row's factor s, then the weight's sums by columns
template <class T> __global__ __launch_bounds__(1024) void norm_grad_long_kernel(sig_norm_args a, NormGrads g, float* factors)
{
    const int64_t row = blockIdx.x, C = a.C;
    const T *r = (const T*)a.x + row * a.x_stride, *gy = (const T*)g.grad_y + row * g.gy_stride, *gt = (const T*)g.grad_total + row * g.gt_stride;
    float square = 0.0f, dot = 0.0f;
    for (int64_t c = threadIdx.x; c < C; c += 1024) {
        const float v = to_float(r[c]);
        square = fmaf(v, v, square);
        dot = fmaf(v * a.weight[c], to_float(gy[c]), dot);
    }
    const float s = rsqrtf(over_row<1024, false>(square) / (float)C + (float)a.eps);
    const float m = over_row<1024, false>(dot) / (float)C * s * s;
    for (int64_t c = threadIdx.x; c < C; c += 1024)
        ((T*)g.grad_x)[row * C + c] = from_float<T>(s * (to_float(gy[c]) * a.weight[c] - to_float(r[c]) * m) + (g.grad_total ? to_float(gt[c]) : 0.0f));
    if (threadIdx.x == 0) factors[row] = s;
}
template <class T> __global__ __launch_bounds__(256) void norm_grad_columns_kernel(sig_norm_args a, NormGrads g, const float* factors, float* parts, int groups, int64_t span)
{
    const int64_t c = (int64_t)(blockIdx.x % groups) * 256 + threadIdx.x, part = blockIdx.x / groups;
    if (c >= a.C) return;
    const T *r = (const T*)a.x + c, *gy = (const T*)g.grad_y + c;
    float v = 0.0f;
    for (int64_t row = part * span; row < min((part + 1) * span, a.rows); row++) v = fmaf(to_float(gy[row * g.gy_stride]), to_float(r[row * a.x_stride]) * factors[row], v);
    parts[part * a.C + c] = v;
}

// The partial sums' rows added up: sixteen columns a workgroup, a sixty-fourth of the rows each thread, then in order.  (Sixty-four columns leave a few
// workgroups: 1,024 rows of 333 columns took 5.2 us.)
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float* parts, int64_t rows, int64_t C, float* grad_weight)
{
    __shared__ float part[64][16];
    const int col = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + col;
    const float* p = parts + min(c, C - 1);
    float v[8] = {};
    int64_t r = r0;
    for (; r + 7 * 64 < rows; r += 8 * 64)
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += p[(r + i * 64) * C];
    for (; r < rows; r += 64) v[0] += p[r * C];
    part[r0][col] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    __syncthreads();
    if (threadIdx.x < 16 && c < C) {
        float s[4] = {};
#pragma unroll
        for (int i = 0; i < 64; i += 4)
#pragma unroll
            for (int k = 0; k < 4; k++) s[k] += part[i + k][col];
        grad_weight[c] = (s[0] + s[1]) + (s[2] + s[3]);
    }
}

constexpr int64_t kLongParts = 64;

// Threads of a row, and accesses of a thread, for rows of `vecs` accesses of V elements: the first that holds them (a wavefront for as long as it can: it
// needs no barrier)
template <int V, class F> bool held(int64_t vecs, F&& f)
{
    auto pick = [&](auto n, auto t) { f(n, t); return true; };
    using std::integral_constant;
    if (vecs <= 64) return pick(integral_constant<int, 1>(), integral_constant<int, 64>());
    if (vecs <= 128) return pick(integral_constant<int, 2>(), integral_constant<int, 64>());
    if (vecs <= 256) return pick(integral_constant<int, 4>(), integral_constant<int, 64>());
    if constexpr (V < 8)
        if (vecs <= 512) return pick(integral_constant<int, 8>(), integral_constant<int, 64>());
    if (vecs <= 1024) return pick(integral_constant<int, 4>(), integral_constant<int, 256>());
    if constexpr (V < 8)
        if (vecs <= 2048) return pick(integral_constant<int, 8>(), integral_constant<int, 256>());
    if (vecs <= 4096) return pick(integral_constant<int, 4>(), integral_constant<int, 1024>());
    return false;
}

bool wide(const void* p, int64_t stride, int bytes, int e) { return !p || ((uintptr_t)p % bytes == 0 && stride * e % bytes == 0); }

template <class T, class O, bool kNorm> hipError_t forward_of(const sig_norm_args& a, O* y, float* scale, T* total, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T), e = sizeof(T);
    auto fits = [&](int v) {
        return a.C % v == 0 && wide(a.x, a.x_stride, v * e, e) && wide(a.residual, a.residual_stride, v * e, e) && wide(total, 0, v * e, e) && wide(a.weight, 0, v * 4, 4) &&
               wide(y, 0, v * (int)sizeof(O), 1);
    };
    hipError_t err = hipSuccess;
    auto run = [&](auto v) {
        constexpr int kV = decltype(v)::value;
        return held<kV>((a.C + kV - 1) / kV, [&](auto n, auto t) {
            constexpr int kN = decltype(n)::value, kThreads = decltype(t)::value;
            const int64_t blocks = kThreads == 64 ? (a.rows + 3) / 4 : a.rows, threads = kThreads == 64 ? 256 : kThreads;
            if (!launchable(blocks, threads)) err = kTooManyThreads;
            else norm_kernel<T, O, kNorm, kV, kN, kThreads><<<(uint32_t)blocks, threads, 0, stream>>>(a, y, scale, total);
        });
    };
    const bool done = fits(V) ? run(std::integral_constant<int, V>()) : V > 4 && fits(2) ? run(std::integral_constant<int, V / 4 < 1 ? 1 : V / 4>()) : run(std::integral_constant<int, 1>());
    if (!done) {
        if (!launchable(a.rows, 1024)) return kTooManyThreads;
        norm_long_kernel<T, O, kNorm><<<(uint32_t)a.rows, 1024, 0, stream>>>(a, y, scale, total);
    }
    return err == hipSuccess ? hipGetLastError() : err;
}

struct GradPlan { bool registers; int64_t blocks, parts; };            // parts: rows of partial sums of the weight's gradient, one a workgroup
template <int V> GradPlan grad_plan(const sig_norm_args& a)
{
    GradPlan p{false, 0, 0};
    p.registers = held<V>((a.C + V - 1) / V, [&](auto, auto t) {
        constexpr int kThreads = decltype(t)::value, kRows = kThreads == 64 ? 4 : 1;
        p.blocks = p.parts = std::min<int64_t>((a.rows + kRows - 1) / kRows, kThreads == 1024 ? 512 : 1024);
    });
    if (!p.registers) p.parts = std::min<int64_t>(kLongParts, a.rows);
    return p;
}

template <class T, int V> hipError_t backward_by(const sig_norm_args& a, const NormGrads& g, float* ws, hipStream_t stream)
{
    const GradPlan p = grad_plan<V>(a);
    const int64_t groups = (a.C + 15) / 16;
    if (!launchable(groups, 1024)) return kTooManyThreads;
    if (a.rows && p.registers) {
        held<V>((a.C + V - 1) / V, [&](auto n, auto t) {
            constexpr int kN = decltype(n)::value, kThreads = decltype(t)::value;
            norm_grad_kernel<T, V, kN, kThreads><<<(uint32_t)p.blocks, kThreads == 64 ? 256 : kThreads, 0, stream>>>(a, g, ws);
        });
    } else if (a.rows) {
        const int64_t wide_groups = (a.C + 255) / 256, span = (a.rows + p.parts - 1) / p.parts;
        if (!launchable(a.rows, 1024) || !launchable(wide_groups * p.parts, 256)) return kTooManyThreads;
        float* factors = ws + p.parts * a.C;
        norm_grad_long_kernel<T><<<(uint32_t)a.rows, 1024, 0, stream>>>(a, g, factors);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        norm_grad_columns_kernel<T><<<(uint32_t)(wide_groups * p.parts), 256, 0, stream>>>(a, g, factors, ws, (int)wide_groups, span);
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    norm_weight_kernel<<<(uint32_t)groups, 1024, 0, stream>>>(ws, p.parts, a.C, g.grad_weight);
    return hipGetLastError();
}

// 16 bytes an access where everything allows it, else pairs of bfloat16 values, else single values
template <class T> hipError_t backward_of(const sig_norm_args& a, const NormGrads& g, float* ws, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T), e = sizeof(T);
    auto fits = [&](int v) {
        return a.C % v == 0 && wide(a.x, a.x_stride, v * e, e) && wide(g.grad_y, g.gy_stride, v * e, e) && wide(g.grad_total, g.gt_stride, v * e, e) && wide(g.grad_x, 0, v * e, e) &&
               wide(a.weight, 0, v * 4, 4) && wide(ws, 0, 16, 4);
    };
    if (fits(V)) return backward_by<T, V>(a, g, ws, stream);
    if constexpr (V > 4)
        if (fits(2)) return backward_by<T, 2>(a, g, ws, stream);
    return backward_by<T, 1>(a, g, ws, stream);
}

}  // namespace

hipError_t norm_forward(const sig_norm_args& a, void* y, float* scale, void* total, hipStream_t stream)
{
    const bool b = a.dtype == SIG_BF16;
    if (!a.weight) return b ? forward_of<bf16, e4m3, false>(a, (e4m3*)y, scale, nullptr, stream) : forward_of<float, e4m3, false>(a, (e4m3*)y, scale, nullptr, stream);
    if (scale) return b ? forward_of<bf16, e4m3, true>(a, (e4m3*)y, scale, (bf16*)total, stream) : forward_of<float, e4m3, true>(a, (e4m3*)y, scale, (float*)total, stream);
    return b ? forward_of<bf16, bf16, true>(a, (bf16*)y, nullptr, (bf16*)total, stream) : forward_of<float, float, true>(a, (float*)y, nullptr, (float*)total, stream);
}
// the larger of what aligned and other addresses take (they are not known yet)
size_t norm_backward_workspace(const sig_norm_args& a)
{
    size_t most = 0;
    for (const GradPlan& p : {grad_plan<1>(a), grad_plan<2>(a), a.dtype == SIG_BF16 ? grad_plan<8>(a) : grad_plan<4>(a)})
        most = std::max(most, (size_t)(p.parts * a.C + (p.registers ? 0 : a.rows)) * 4);
    return most;
}
hipError_t norm_backward(const sig_norm_args& a, const NormGrads& g, float* workspace, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? backward_of<bf16>(a, g, workspace, stream) : backward_of<float>(a, g, workspace, stream);
}

}  // namespace sig
