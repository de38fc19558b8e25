// Short causal convolution over time, a filter for each channel (depthwise), with an optional SiLU:
//   s_t = bias + sum_k w[k] x_{t - W + 1 + k},   y_t = s_t sigmoid(s_t)  or  s_t,   k = 0 .. W - 1
// and its gradient: g_t = dL/ds_t,  dL/dx_p = sum_k w[k] g_{p + W - 1 - k},  dL/dw[k] = sum_t g_t x_{t - W + 1 + k}.
// Both directions are bound by memory: 2 W multiply-adds stand against 4 bytes (bf16) a token and channel.
#include <algorithm>

#include "seq.hpp"

namespace sig {
namespace {

constexpr int kThreads = 256;

// A thread walks one time chunk of V neighbouring channels with the last W tokens in registers, so a token is read once and (at
// chunk starts) W - 1 tokens twice.  Threads of a wavefront are neighbours in the channel axis: their accesses are contiguous.
struct Split {
    int64_t chunk;       // tokens of a chunk
    int64_t chunks;
    int64_t vecs;        // groups of V channels
    int64_t threads;
};
Split split_time(int64_t B, int64_t L, int64_t D, int V)
{
    Split s;
    s.vecs = (D + V - 1) / V;
    // four wavefronts on each SIMD (4,096 of 64 threads), each with two groups of loads under way, hide the memory's latency (8 x 2048 x 2048 in
    // bf16 with 2,048, 3,072, 4,096, 6,144 and 8,192: forward 35, 29, 30, 30, 30 us, gradient 56, 57, 52, 58, 62 us); chunks shorter
    // than 16 tokens would read a fifth and more of their input twice
    int64_t want = (int64_t)4096 * 64 / std::max<int64_t>(1, B * s.vecs) + 1;
    s.chunk = std::min<int64_t>(1 << 30, std::max<int64_t>(16, (L + want - 1) / want));      // the kernels count a chunk's tokens in 32 bits
    s.chunks = std::max<int64_t>(1, (L + s.chunk - 1) / s.chunk);
    s.threads = B * s.chunks * s.vecs;
    return s;
}

template <class T, int V> __device__ __forceinline__ void load(float (&r)[V], const T* p)
{
    Pack<T, V> q = *(const Pack<T, V>*)p;
#pragma unroll
    for (int i = 0; i < V; i++) r[i] = to_float(q.v[i]);
}
template <class T, int V> __device__ __forceinline__ void store(T* p, const float (&r)[V])
{
    Pack<T, V> q;
#pragma unroll
    for (int i = 0; i < V; i++) q.v[i] = from_float<T>(r[i]);
    *(Pack<T, V>*)p = q;
}

// token p of the sequence that starts W - 1 tokens before the first: the initial state, then x
template <class T, int V, int W> __device__ __forceinline__ void load_token(float (&r)[V], const T* x, int64_t stride_t, const T* initial, int64_t D, int64_t p)
{
    if (p >= 0) {
        load<T, V>(r, x + p * stride_t);
    } else if (initial) {
        load<T, V>(r, initial + (W - 1 + p) * D);
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) r[i] = 0.0f;
    }
}

template <int V, int W> __device__ __forceinline__ void load_filter(float (&w)[W][V], float (&bias)[V], const sig_conv_args& a, int64_t d)
{
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int k = 0; k < W; k++) w[k][i] = a.weight[(d + i) * W + k];
        bias[i] = a.bias ? a.bias[d + i] : 0.0f;
    }
}

// The W - 1 tokens before token t0 >= 0 of a stream, of which x holds token t0: no branches, so that nothing waits for the loads here.
template <class T, int V, int W>
__device__ __forceinline__ void load_window(float (&r)[W][V], const T* x, int64_t stride_t, const T* initial, int64_t D, int64_t t0)
{
#pragma unroll
    for (int k = 0; k < W - 1; k++) {
        const int64_t p = t0 - W + 1 + k;
        const T* q = p >= 0 || !initial ? x + (p >= 0 ? p : t0) * stride_t : initial + (W - 1 + p) * D;
        load<T, V>(r[k + 1], q);
#pragma unroll
        for (int i = 0; i < V; i++) r[k + 1][i] = p >= 0 || initial ? r[k + 1][i] : 0.0f;
    }
}

// V elements as whole words: the compiler takes a load of an array of halves apart
template <int kBytes> struct Words { typedef uint32_t type __attribute__((ext_vector_type(kBytes / 4))); };
template <> struct Words<4> { typedef uint32_t type; };
template <> struct Words<2> { typedef uint16_t type; };
template <class T, int V> using Raw = typename Words<sizeof(T) * V>::type;
template <class T, int V> __device__ __forceinline__ float element(const Raw<T, V>& r, int i)
{
    if constexpr (sizeof(T) * V == 2) return to_float(bf16{r});
    else if constexpr (sizeof(T) * V == 4) return sizeof(T) == 4 ? __uint_as_float(r) : __uint_as_float(i ? r & 0xffff0000u : r << 16);
    else if constexpr (sizeof(T) == 4) return __uint_as_float(r[i]);
    else return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
}

// keeps the compiler from unpacking a group as soon as its loads are made, which would wait for them and take twice the registers
template <class R> __device__ __forceinline__ R here(R r)
{
    asm volatile("" : "+v"(r));
    return r;
}

// U tokens from p on, of which there are `left` (at least one, at first): after the last one it is read again.  A load that is always made
// lets the compiler count how many are under way; behind a condition it waits for all of them and for the stores among them.
template <class T, int V, int U> __device__ __forceinline__ void load_group(Raw<T, V> (&to)[U], const T*& p, int64_t stride, int& left)
{
#pragma unroll
    for (int u = 0; u < U; u++, left--) {
        to[u] = *(const Raw<T, V>*)p;
        p += left > 1 ? stride : 0;
    }
}

__device__ __forceinline__ float either(uint32_t mask, float v, float other) { return __uint_as_float((__float_as_uint(v) & mask) | (__float_as_uint(other) & ~mask)); }

// 8 x 2048 x 2048: 30 us in bf16, 4.5 TB/s of the 5.1 TB/s that a copy of 1 GB reaches, 45 us in float32, 6.0 TB/s (what the cache before the memory
// holds counts too).  A limit of 128 registers (a wavefront more on each SIMD) made it 32 us.
template <class T, int V, int W>
__global__ __launch_bounds__(kThreads) void conv_fwd_kernel(sig_conv_args a, T* y, T* final_state, Split s)
{
    int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= s.threads) return;
    int64_t d = id % s.vecs * V, row = id / s.vecs, c = row % s.chunks, b = row / s.chunks;
    const T* x = (const T*)a.x + b * a.x_stride_b + d;
    const T* initial = a.initial_state ? (const T*)a.initial_state + b * (W - 1) * a.D + d : nullptr;
    const int64_t t0 = c * s.chunk, len = live_length(a.lengths, b, a.L);
    const int n = (int)(min(t0 + s.chunk, a.L) - t0), live = (int)max((int64_t)0, min((int64_t)n, len - t0));
    const uint32_t silu = a.silu ? ~0u : 0u;
    y += (b * a.L + t0) * a.D + d;
    int t = 0;
    if (live > 0) {
        float w[W][V], bias[V], r[W][V];
        load_filter<V, W>(w, bias, a, d);
        load_window<T, V, W>(r, x, a.x_stride_t, initial, a.D, t0);
        auto token = [&](const Raw<T, V>& packed) {
            const Raw<T, V> in = here(packed);
            float o[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
                o[i] = bias[i];
#pragma unroll
                for (int k = 0; k < W - 1; k++) r[k][i] = r[k + 1][i], o[i] = fmaf(w[k][i], r[k][i], o[i]);
                r[W - 1][i] = element<T, V>(in, i);
                o[i] = fmaf(w[W - 1][i], r[W - 1][i], o[i]);
                o[i] *= either(silu, sigmoid(o[i]), 1.0f);
            }
            store<T, V>(y, o);
            y += a.D;
        };
        // groups of U tokens, the next one's loads under way while one is worked on
        constexpr int U = V >= 4 ? 4 : 8;
        Raw<T, V> now[U], next[U];
        const T* p = x + t0 * a.x_stride_t;
        int left = live;
        load_group<T, V, U>(now, p, a.x_stride_t, left);
        for (; t + U <= live; t += U) {
            load_group<T, V, U>(next, p, a.x_stride_t, left);
#pragma unroll
            for (int u = 0; u < U; u++) token(now[u]);
#pragma unroll
            for (int u = 0; u < U; u++) now[u] = next[u];
        }
#pragma unroll
        for (int u = 0; u < U - 1; u++) {
            if (t >= live) break;
            token(now[u]);
            t++;
        }
    }
    float zero[V] = {};
    for (; t < n; t++, y += a.D) store<T, V>(y, zero);
    if (final_state && c == 0) {
        final_state += b * (W - 1) * a.D + d;
#pragma unroll
        for (int k = 0; k < W - 1; k++) {
            float v[V];
            load_token<T, V, W>(v, x, a.x_stride_t, initial, a.D, len - W + 1 + k);
            store<T, V>(final_state + k * a.D, v);
        }
    }
}

// The gradient walks forward as well: at token t it has s_t from the window of x, g_t from it and the upstream gradient, and with the
// last W of them the gradient of token t - W + 1.  A chunk goes W - 1 tokens past its end for the gradients of its last tokens.
// 8 x 2048 x 2048: 53 us in bf16, 3.8 TB/s, where s_t, the slope and three products of W taps make the vector instructions count, and 89 us in
// float32, 4.5 TB/s.  Loads of the next group behind a condition: 15 % more time (waits for all that is under way, stores among it).
template <class T, int V, int W>
__global__ __launch_bounds__(kThreads) void conv_bwd_kernel(sig_conv_args a, ConvGrads g, float* part, Split s)
{
    const bool there = (int64_t)blockIdx.x * kThreads + threadIdx.x < s.threads;
    const int64_t id = there ? (int64_t)blockIdx.x * kThreads + threadIdx.x : 0;
    const int64_t d = id % s.vecs * V, row = id / s.vecs, c = row % s.chunks, b = row / s.chunks;
    T* gi = g.grad_initial && c == 0 ? (T*)g.grad_initial + b * (W - 1) * a.D + d : nullptr;
    const T* gf = g.grad_final ? (const T*)g.grad_final + b * (W - 1) * a.D + d : nullptr;
    const int64_t t0 = c * s.chunk, len = live_length(a.lengths, b, a.L);
    const int n = (int)(min(t0 + s.chunk, a.L) - t0);
    T* gx = (T*)g.grad_x + (b * a.L + t0) * a.D + d;
    float gw[W + 1][V] = {};
    if (there && t0 < len) {
        const T* x = (const T*)a.x + b * a.x_stride_b + d;
        const T* initial = a.initial_state ? (const T*)a.initial_state + b * (W - 1) * a.D + d : nullptr;
        const int live = (int)min((int64_t)n + W - 1, len - t0), lowest = gi ? 1 - W : 0;      // tokens that count, from t0 on
        const uint32_t silu = a.silu ? ~0u : 0u;
        float w[W][V], bias[V], r[W][V], h[W][V] = {};
        load_filter<V, W>(w, bias, a, d);
        load_window<T, V, W>(r, x, a.x_stride_t, initial, a.D, t0);
        // takes token t0 + t (x and upstream gradient) and stores the gradient of token t0 + t - W + 1; kWhole: it counts and is of the chunk
        auto token = [&](auto whole, int t, const Raw<T, V>& packed_in, const Raw<T, V>& packed_up) {
            const Raw<T, V> in = here(packed_in), up = here(packed_up);
            constexpr bool kWhole = decltype(whole)::value;
            const bool counts = kWhole || t < live, ours = kWhole || t < min(n, live);
#pragma unroll
            for (int i = 0; i < V; i++) {
#pragma unroll
                for (int k = 0; k < W - 1; k++) r[k][i] = r[k + 1][i], h[k][i] = h[k + 1][i];
                r[W - 1][i] = counts ? element<T, V>(in, i) : 0.0f;
                float o = bias[i];
#pragma unroll
                for (int k = 0; k < W; k++) o = fmaf(w[k][i], r[k][i], o);
                const float p = sigmoid(o), q = element<T, V>(up, i) * either(silu, p * fmaf(o, 1.0f - p, 1.0f), 1.0f);
                h[W - 1][i] = counts ? q : 0.0f;
                if (ours) {
#pragma unroll
                    for (int k = 0; k < W; k++) gw[k][i] = fmaf(q, r[k][i], gw[k][i]);
                    gw[W][i] += q;
                }
            }
            const int p = t - W + 1;
            if (p < (kWhole ? 0 : lowest)) return;      // whole groups begin after the initial state's tokens
            float o[V] = {};
#pragma unroll
            for (int k = 0; k < W; k++) {
                // tokens that are not there or do not count add nothing, whatever their weight is
                const bool adds = kWhole || (t >= k && t - k < live);
#pragma unroll
                for (int i = 0; i < V; i++) o[i] = adds ? fmaf(w[k][i], h[W - 1 - k][i], o[i]) : o[i];
            }
            if (!kWhole && gf && t0 + p < len && t0 + p >= len - (W - 1)) {
                float v[V];
                load<T, V>(v, gf + (t0 + p - len + W - 1) * a.D);
#pragma unroll
                for (int i = 0; i < V; i++) o[i] += v[i];
            }
            store<T, V>(kWhole || p >= 0 ? gx + p * a.D : gi + (W - 1 + p) * a.D, o);
        };
        // groups of U tokens, the next one's loads under way while one is worked on
        constexpr int U = V >= 4 ? 4 : 8;
        Raw<T, V> nx[U], ng[U], mx[U], mg[U];
        const T *qx = x + t0 * a.x_stride_t, *qg = (const T*)g.grad_y + b * g.gy_stride_b + t0 * g.gy_stride_t + d;
        int left_x = live, left_g = live, t = 0;
        load_group<T, V, U>(nx, qx, a.x_stride_t, left_x), load_group<T, V, U>(ng, qg, g.gy_stride_t, left_g);
        // incomplete groups, tokens before the first, after the chunk and such as do not count among them
        auto guarded = [&](auto last, int until) {
            while (t < until) {
                load_group<T, V, U>(mx, qx, a.x_stride_t, left_x), load_group<T, V, U>(mg, qg, g.gy_stride_t, left_g);
#pragma unroll
                for (int u = 0; u < U; u++) {
                    if (t + u >= n + W - 1) break;
                    token(std::false_type(), t + u, nx[u], ng[u]);
                }
                t += U;
                if (decltype(last)::value && t >= until) break;         // nothing waits for loads that nobody needs
#pragma unroll
                for (int u = 0; u < U; u++) nx[u] = mx[u], ng[u] = mg[u];
            }
        };
        if (__any(gi != nullptr)) guarded(std::false_type(), W - 1);       // the whole wavefront, whose threads keep step
        for (const int whole = min(n, live); t + U <= whole; t += U) {
            load_group<T, V, U>(mx, qx, a.x_stride_t, left_x), load_group<T, V, U>(mg, qg, g.gy_stride_t, left_g);
#pragma unroll
            for (int u = 0; u < U; u++) token(std::true_type(), t + u, nx[u], ng[u]);
#pragma unroll
            for (int u = 0; u < U; u++) nx[u] = mx[u], ng[u] = mg[u];
        }
        guarded(std::true_type(), n + W - 1);
    } else if (there) {
        float zero[V] = {};
        for (int t = 0; t < n; t++) store<T, V>(gx + t * a.D, zero);
        for (int k = 0; gi && k < W - 1; k++) {      // no tokens: the final state is the initial one
            float v[V] = {};
            if (gf) load<T, V>(v, gf + k * a.D);
            store<T, V>(gi + k * a.D, v);
        }
    }
    // The sums of channels that several threads of the workgroup share are added up here, in their order: otherwise the second kernel would
    // add up a row for every 16 tokens where channels are few (gradient of 64 x 4096 x 64 in bf16: a third of the time with the sums here, now 32 us).
    if (s.vecs >= kThreads) {
        if (!there) return;
        part += row * (W + 1) * a.D + d;
#pragma unroll
        for (int k = 0; k <= W; k++)
#pragma unroll
            for (int i = 0; i < V; i++) part[k * a.D + i] = gw[k][i];
        return;
    }
    __shared__ float sums[(W + 1) * V][kThreads];
#pragma unroll
    for (int k = 0; k <= W; k++)
#pragma unroll
        for (int i = 0; i < V; i++) sums[k * V + i][threadIdx.x] = gw[k][i];
    __syncthreads();
    const int vecs = (int)s.vecs, first = (int)((int64_t)blockIdx.x * kThreads % vecs);
    part += (int64_t)blockIdx.x * (W + 1) * a.D;
    for (int j = threadIdx.x; j < vecs * (W + 1) * V; j += kThreads) {
        const int v = j % vecs, q = j / vecs;
        float sum = 0.0f;
        for (int t = (v - first + vecs) % vecs; t < kThreads; t += vecs) sum += sums[q][t];
        part[(int64_t)(q / V) * a.D + v * V + q % V] = sum;
    }
}

// sums the filter gradients part[rows][W + 1][D] in a fixed order, 64 sums a workgroup
template <int W> __global__ __launch_bounds__(1024) void conv_bwd_sum_kernel(const float* part, int64_t rows, int64_t D, float* gw, float* gb)
{
    const int64_t id = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63), n = (W + 1) * D;
    const float v = sum_rows(part + id, id < n ? rows : 0, n);
    if (threadIdx.x >= 64 || id >= n) return;
    const int64_t k = id / D, d = id % D;
    if (k < W) gw[d * W + k] = v;
    else if (gb) gb[d] = v;
}

// One token: a thread for every 4 bytes of it, so that few streams still give many threads.  64 x 2048 in bf16: 2.7 us, a launch's own time
// (the 2 MB would take 0.4 us).
template <class T, int V, int W> __global__ __launch_bounds__(kThreads) void conv_step_kernel(sig_conv_args a, T* state, T* y, int64_t vecs)
{
    int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= a.B * vecs) return;
    int64_t d = id % vecs * V, b = id / vecs;
    state += b * (W - 1) * a.D + d;
    float w[W][V], bias[V], r[W][V], o[V];
    load_filter<V, W>(w, bias, a, d);
#pragma unroll
    for (int k = 0; k < W - 1; k++) load<T, V>(r[k], state + k * a.D);
    load<T, V>(r[W - 1], (const T*)a.x + b * a.x_stride_b + d);
#pragma unroll
    for (int k = 0; k < W - 1; k++) store<T, V>(state + k * a.D, r[k + 1]);
#pragma unroll
    for (int i = 0; i < V; i++) {
        o[i] = bias[i];
#pragma unroll
        for (int k = 0; k < W; k++) o[i] = fmaf(w[k][i], r[k][i], o[i]);
        if (a.silu) o[i] *= sigmoid(o[i]);
    }
    store<T, V>(y + b * a.D + d, o);
}

// V channels in one access need rows that start at multiples of its size
bool aligned_rows(const void* p, int64_t stride_b, int64_t stride_t, int64_t D, int V, int bytes)
{
    return ((uintptr_t)p % (V * bytes)) == 0 && stride_b % V == 0 && stride_t % V == 0 && D % V == 0;
}

// rows of filter gradients that the gradient's main kernel leaves
int64_t part_rows(int64_t B, const Split& s) { return s.vecs >= kThreads ? B * s.chunks : (s.threads + kThreads - 1) / kThreads; }

int64_t blocks_for(int64_t threads) { return (threads + kThreads - 1) / kThreads; }

template <class F> hipError_t with_width(int64_t W, F f)
{
    switch (W) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 4: return f(std::integral_constant<int, 4>());
        case 5: return f(std::integral_constant<int, 5>());
        case 6: return f(std::integral_constant<int, 6>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, 8>());
    }
}

constexpr int wide(const float*) { return 4; }
constexpr int wide(const bf16*) { return 8; }

template <class T> hipError_t forward(const sig_conv_args& a, T* y, T* fin, hipStream_t stream)
{
    constexpr int V = wide((T*)nullptr);
    bool vec = aligned_rows(a.x, a.x_stride_b, a.x_stride_t, a.D, V, sizeof(T)) && aligned_rows(y, 0, 0, a.D, V, sizeof(T)) &&
               aligned_rows(a.initial_state, 0, 0, a.D, V, sizeof(T)) && aligned_rows(fin, 0, 0, a.D, V, sizeof(T));
    Split s = split_time(a.B, a.L, a.D, vec ? V : 1);
    const int64_t blocks = blocks_for(s.threads);
    if (!launchable(blocks, kThreads)) return kTooManyThreads;
    return with_width(a.W, [&](auto w) {
        constexpr int W = decltype(w)::value;
        if (vec) conv_fwd_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, y, fin, s);
        else conv_fwd_kernel<T, 1, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, y, fin, s);
        return hipGetLastError();
    });
}

template <class T> hipError_t backward(const sig_conv_args& a, const ConvGrads& g, float* part, hipStream_t stream)
{
    constexpr int V = wide((T*)nullptr) / 2;     // 8 bytes: the two windows and the filter's sums of more channels would not fit the registers
    bool vec = aligned_rows(a.x, a.x_stride_b, a.x_stride_t, a.D, V, sizeof(T)) && aligned_rows(g.grad_y, g.gy_stride_b, g.gy_stride_t, a.D, V, sizeof(T)) &&
               aligned_rows(g.grad_x, 0, 0, a.D, V, sizeof(T)) && aligned_rows(a.initial_state, 0, 0, a.D, V, sizeof(T)) &&
               aligned_rows(g.grad_final, 0, 0, a.D, V, sizeof(T)) && aligned_rows(g.grad_initial, 0, 0, a.D, V, sizeof(T));
    Split s = split_time(a.B, a.L, a.D, vec ? V : 1);
    const int64_t blocks = blocks_for(s.threads), sums = ((a.W + 1) * a.D + 63) / 64;
    if (!launchable(blocks, kThreads) || !launchable(sums, 1024)) return kTooManyThreads;
    return with_width(a.W, [&](auto w) {
        constexpr int W = decltype(w)::value;
        if (a.B == 0) {}     // the sums below are zero
        else if (vec) conv_bwd_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, g, part, s);
        else conv_bwd_kernel<T, 1, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, g, part, s);
        conv_bwd_sum_kernel<W><<<(unsigned)sums, 1024, 0, stream>>>(part, part_rows(a.B, s), a.D, g.grad_weight, g.grad_bias);
        return hipGetLastError();
    });
}

template <class T> hipError_t step(const sig_conv_args& a, T* state, T* y, hipStream_t stream)
{
    constexpr int V = wide((T*)nullptr) / 4;
    bool vec = aligned_rows(a.x, a.x_stride_b, 0, a.D, V, sizeof(T)) && aligned_rows(state, 0, 0, a.D, V, sizeof(T)) && aligned_rows(y, 0, 0, a.D, V, sizeof(T));
    const int64_t vecs = vec ? a.D / V : a.D, blocks = blocks_for(a.B * vecs);
    if (!launchable(blocks, kThreads)) return kTooManyThreads;
    return with_width(a.W, [&](auto w) {
        constexpr int W = decltype(w)::value;
        if (vec) conv_step_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, state, y, vecs);
        else conv_step_kernel<T, 1, W><<<(unsigned)blocks, kThreads, 0, stream>>>(a, state, y, vecs);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t conv_forward(const sig_conv_args& a, void* y, void* final_state, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? forward<bf16>(a, (bf16*)y, (bf16*)final_state, stream) : forward<float>(a, (float*)y, (float*)final_state, stream);
}

size_t conv_backward_workspace(const sig_conv_args& a)
{
    // either split of the channels into accesses may be taken, the addresses decide
    int V = a.dtype == SIG_BF16 ? 4 : 2;
    int64_t rows = std::max(part_rows(a.B, split_time(a.B, a.L, a.D, V)), part_rows(a.B, split_time(a.B, a.L, a.D, 1)));
    return (size_t)(rows * (a.W + 1) * a.D * 4);
}

hipError_t conv_backward(const sig_conv_args& a, const ConvGrads& g, float* workspace, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? backward<bf16>(a, g, workspace, stream) : backward<float>(a, g, workspace, stream);
}

hipError_t conv_step(const sig_conv_args& a, void* state, void* y, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? step<bf16>(a, (bf16*)state, (bf16*)y, stream) : step<float>(a, (float*)state, (float*)y, stream);
}

}  // namespace sig
