// Gated linear recurrence over tokens [batch, time, channels] and its gradient.
//
//   u_t = exp(log_rate) sigmoid(p_t),  a_t = exp(-u_t),  b_t = sqrt(1 - a_t^2),  i_t = sigmoid(q_t),   h_t = a_t h_(t-1) + b_t i_t x_t = y_t
//
// A stretch of tokens maps the state before it to the state after it by h -> A h + H, and two stretches join to (A2 A1, A2 H1 + H2).  A workgroup
// has 64 channels and walks time in rounds of 128 tokens: eight wavefronts of 16 tokens, of which each half wavefront has 8, a lane two
// neighbouring channels.  Every half computes its stretch in registers, halves join by a lane swap, wavefronts through LDS (one barrier a round); then the
// states follow from what is in registers.  So everything is read once, and the next round's loads are under way meanwhile.  Few streams get
// time chunks: a first pass over the inputs leaves every chunk's (A, H).
//
// Gradient: with c_t what comes back from the tokens after t, l_t = grad_y_t + c_t and c_(t-1) = a_t l_t, the same structure from the end.  With U_t = u_t dL/du_t
//   grad x = l b i,  grad q = l b x i (1 - i),  U = l (u a^2 / b i x - u a h_(t-1)),  grad p = U (1 - sigmoid(p)),  grad log_rate = sum U:
// u / b goes to zero like sqrt(u / 2), so nothing here is infinite at u = 0.
#include "layer.hpp"

namespace sig {
namespace {

constexpr int kWaves = 8, kHalf = 8, kRound = kWaves * kGatedTile, kGroup = 64;

struct Two { float v[2]; };

template <class T, bool kPairs> __device__ __forceinline__ Pack<T, 2> load_two(const T* p, int c, int D)
{
    if constexpr (kPairs) return *(const Pack<T, 2>*)(p + c);                  // D is even: c < D has c + 1 < D
    Pack<T, 2> r;
    r.v[0] = p[c];
    r.v[1] = p[min(c + 1, D - 1)];
    return r;
}
template <class T, bool kPairs> __device__ __forceinline__ void store_two(T* p, int c, int D, float v0, float v1)
{
    Pack<T, 2> r{{from_float<T>(v0), from_float<T>(v1)}};
    if constexpr (kPairs) *(Pack<T, 2>*)(p + c) = r;
    else {
        p[c] = r.v[0];
        if (c + 1 < D) p[c + 1] = r.v[1];
    }
}

// sigmoid(v) and 1 - sigmoid(v) = sigmoid(-v), which keeps its relative precision where it is small
struct Gate { float s, rest; };
__device__ __forceinline__ Gate gate(float v)
{
    const float e = fast_exp(-v), s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, v > 0.0f ? e * s : 1.0f - s};
}

// exp(-u) and 1 - exp(-2 u) for u >= 0.  Small u: -expm1(-v) = v (1 - v/2 (1 - v/3 (1 - ...))) with v = 2u < 1/2, whose first omitted term is
// v^7 / 8! < 2e-7 of the value; from there on 1 - a^2 >= 0.39 loses a bit and a half at most.  u is bounded, as 0 times infinity would follow.
struct Decay { float u, a, w; };
__device__ __forceinline__ Decay decay(float rate, float open)
{
    float u = rate * open;
    u = u > 128.0f ? 128.0f : u;                                               // exp(-128) is 0 in float32's normal range; a NaN stays one
    float a = fast_exp(-u), v = 2.0f * u;
    float p = fmaf(v, -1.0f / 8.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 7.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 6.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 5.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 4.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 3.0f, 1.0f);
    p = fmaf(p * v, -1.0f / 2.0f, 1.0f);
    return {u, a, v < 0.5f ? p * v : fmaf(-a, a, 1.0f)};
}

// exp(log_rate), log_rate taken as 64 beyond that: a product with a shut gate's zero stays one.  A NaN stays one.
__device__ __forceinline__ float rate_of(float log_rate) { return fast_exp(log_rate > 64.0f ? 64.0f : log_rate); }

struct Where {                       // of a workgroup: stream, channels, tokens of its chunk, and how many of them count
    int64_t b;
    int chunk, c, first, last, live;
    bool on;
};
__device__ __forceinline__ Where where(const sig_gated_args& a, int groups, int chunks, int rounds)
{
    Where w;
    const uint32_t id = blockIdx.x;
    w.chunk = id % chunks;
    const uint32_t row = id / chunks;
    w.b = row / groups;
    w.c = (row % groups) * kGroup + (threadIdx.x & 31) * 2;
    w.on = w.c < a.D;
    w.c = min(w.c, (int)a.D - 1);
    const int64_t span = (int64_t)rounds * kRound;
    w.first = (int)min((int64_t)w.chunk * span, a.L);
    w.last = (int)min((w.chunk + 1) * span, a.L);
    w.live = (int)live_length(a.lengths, w.b, a.L);
    return w;
}

template <class T> struct Raw { Pack<T, 2> x[kHalf], p[kHalf], q[kHalf]; };

// kSummary: only (A, H) of the chunk from a state of zero
template <class T, bool kPairs, bool kSummary>
__global__ __launch_bounds__(kWaves * 64) void gated_forward_kernel(sig_gated_args a, T* y, float* final_state, float* ckpt, float* sums, int groups, int chunks,
                                                                     int rounds)
{
    __shared__ float4 joined[2][kWaves][32];
    const Where w = where(a, groups, chunks, rounds);
    const int wave = threadIdx.x / 64, half = (threadIdx.x >> 5) & 1, li = threadIdx.x & 31, D = (int)a.D;
    const bool even = kPairs || w.c + 1 < D;
    const T *x = (const T*)a.x + w.b * a.x_stride_b, *p = (const T*)a.decay_gate + w.b * a.decay_stride_b, *q = (const T*)a.input_gate + w.b * a.input_stride_b;
    const int c1 = even ? w.c + 1 : w.c;
    const float rate[2] = {rate_of(a.log_rate[w.c]), rate_of(a.log_rate[c1])};
    float state[2] = {}, decayed[2] = {1.0f, 1.0f};
    if constexpr (!kSummary) {
        if (a.initial_state) {
            state[0] = a.initial_state[w.b * D + w.c];
            state[1] = a.initial_state[w.b * D + c1];
        }
        for (int j = 0; j < w.chunk; j++) {                                    // the chunks before this one
            const float* s = sums + ((w.b * chunks + j) * 2) * D;
            state[0] = fmaf(s[w.c], state[0], s[D + w.c]);
            state[1] = fmaf(s[c1], state[1], s[D + c1]);
        }
    }
    const int end = min(w.last, w.live);
    const int64_t tiles = (a.L + kGatedTile - 1) / kGatedTile;
    auto load = [&](int t0, Raw<T>& r) {
#pragma unroll
        for (int k = 0; k < kHalf; k++) {
            const int64_t t = min(t0 + k, end - 1);
            r.x[k] = load_two<T, kPairs>(x + t * a.x_stride_t, w.c, D);
            r.p[k] = load_two<T, kPairs>(p + t * a.decay_stride_t, w.c, D);
            r.q[k] = load_two<T, kPairs>(q + t * a.input_stride_t, w.c, D);
        }
    };
    const int mine = wave * kGatedTile + half * kHalf;
    Raw<T> next;
    if (w.first < end) load(w.first + mine, next);
    int buf = 0;
    for (int r = w.first; r < end; r += kRound, buf ^= 1) {
        const Raw<T> now = next;
        if (r + kRound < end) load(r + kRound + mine, next);
        const int t0 = r + mine;
        float f[kHalf][2], d[kHalf][2], A[2] = {1.0f, 1.0f}, H[2] = {};
#pragma unroll
        for (int k = 0; k < kHalf; k++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const Decay e = decay(rate[j], sigmoid(to_float(now.p[k].v[j])));
                const bool live = t0 + k < end;
                d[k][j] = live ? e.a : 1.0f;
                f[k][j] = live ? __builtin_amdgcn_sqrtf(e.w) * sigmoid(to_float(now.q[k].v[j])) * to_float(now.x[k].v[j]) : 0.0f;
                A[j] *= d[k][j];
                H[j] = fmaf(d[k][j], H[j], f[k][j]);
            }
        float preA[2], preH[2], bothA[2], bothH[2];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const float oA = __shfl_xor(A[j], 32), oH = __shfl_xor(H[j], 32);
            preA[j] = half ? oA : 1.0f;
            preH[j] = half ? oH : 0.0f;
            bothA[j] = oA * A[j];
            bothH[j] = half ? fmaf(A[j], oH, H[j]) : fmaf(oA, H[j], oH);
        }
        if (!half) joined[buf][wave][li] = float4{bothA[0], bothA[1], bothH[0], bothH[1]};
        __syncthreads();
        float start[2];
#pragma unroll
        for (int j = 0; j < kWaves; j++) {
            const float4 v = joined[buf][j][li];
            if (j == wave) {
                start[0] = state[0];
                start[1] = state[1];
            }
            state[0] = fmaf(v.x, state[0], v.z);
            state[1] = fmaf(v.y, state[1], v.w);
            if constexpr (kSummary) {
                decayed[0] *= v.x;
                decayed[1] *= v.y;
            }
        }
        if constexpr (!kSummary) {
            if (ckpt && !half && w.on && t0 < end) {
                float* to = ckpt + (w.b * tiles + t0 / kGatedTile) * D;
                to[w.c] = start[0];
                if (even) to[w.c + 1] = start[1];
            }
            float h[2] = {fmaf(preA[0], start[0], preH[0]), fmaf(preA[1], start[1], preH[1])};
#pragma unroll
            for (int k = 0; k < kHalf; k++) {
                h[0] = fmaf(d[k][0], h[0], f[k][0]);
                h[1] = fmaf(d[k][1], h[1], f[k][1]);
                const bool live = t0 + k < end;
                if (w.on && t0 + k < w.last) store_two<T, kPairs>(y + (w.b * a.L + t0 + k) * D, w.c, D, live ? h[0] : 0.0f, live ? h[1] : 0.0f);
            }
        }
    }
    if constexpr (kSummary) {
        if (threadIdx.x < 32 && w.on) {
            float* s = sums + ((w.b * chunks + w.chunk) * 2) * D;
            s[w.c] = decayed[0];
            s[D + w.c] = state[0];
            if (even) {
                s[w.c + 1] = decayed[1];
                s[D + w.c + 1] = state[1];
            }
        }
    } else {
        // what no round has reached
        const int done = w.first + (max(end - w.first, 0) + kRound - 1) / kRound * kRound;
        for (int t = done + (threadIdx.x >> 5); t < w.last; t += kWaves * 2)
            if (w.on) store_two<T, kPairs>(y + (w.b * a.L + t) * D, w.c, D, 0.0f, 0.0f);
        if (final_state && w.chunk == chunks - 1 && threadIdx.x < 32 && w.on) {
            final_state[w.b * D + w.c] = state[0];
            if (even) final_state[w.b * D + w.c + 1] = state[1];
        }
    }
}

template <class T> struct RawBack { Pack<T, 2> x[kHalf], p[kHalf], q[kHalf], g[kHalf]; };

template <class T, bool kPairs, bool kSummary>
__global__ __launch_bounds__(kWaves * 64) void gated_backward_kernel(sig_gated_args a, sig_gated_grads g, const float* ckpt, float* sums, float* rates, int groups,
                                                                      int chunks, int rounds)
{
    __shared__ float4 joined[2][kWaves][32];
    const Where w = where(a, groups, chunks, rounds);
    const int wave = threadIdx.x / 64, half = (threadIdx.x >> 5) & 1, li = threadIdx.x & 31, D = (int)a.D;
    const bool even = kPairs || w.c + 1 < D;
    const T *x = (const T*)a.x + w.b * a.x_stride_b, *p = (const T*)a.decay_gate + w.b * a.decay_stride_b, *q = (const T*)a.input_gate + w.b * a.input_stride_b;
    const T* gy = (const T*)g.grad_y + w.b * g.gy_stride_b;
    T *gx = (T*)g.grad_x + w.b * a.L * D, *gp = (T*)g.grad_decay_gate + w.b * a.L * D, *gq = (T*)g.grad_input_gate + w.b * a.L * D;
    const int c1 = even ? w.c + 1 : w.c;
    const float rate[2] = {rate_of(a.log_rate[w.c]), rate_of(a.log_rate[c1])};
    float back[2] = {}, decayed[2] = {1.0f, 1.0f}, total[2] = {};
    if constexpr (!kSummary) {
        if (g.grad_final_state) {
            back[0] = g.grad_final_state[w.b * D + w.c];
            back[1] = g.grad_final_state[w.b * D + c1];
        }
        for (int j = chunks - 1; j > w.chunk; j--) {
            const float* s = sums + ((w.b * chunks + j) * 2) * D;
            back[0] = fmaf(s[w.c], back[0], s[D + w.c]);
            back[1] = fmaf(s[c1], back[1], s[D + c1]);
        }
    }
    const int end = min(w.last, w.live);
    const int64_t tiles = (a.L + kGatedTile - 1) / kGatedTile;
    auto load = [&](int t0, RawBack<T>& r) {
#pragma unroll
        for (int k = 0; k < kHalf; k++) {
            const int64_t t = min(t0 + k, end - 1);
            r.p[k] = load_two<T, kPairs>(p + t * a.decay_stride_t, w.c, D);
            r.g[k] = load_two<T, kPairs>(gy + t * g.gy_stride_t, w.c, D);
            if constexpr (!kSummary) {
                r.x[k] = load_two<T, kPairs>(x + t * a.x_stride_t, w.c, D);
                r.q[k] = load_two<T, kPairs>(q + t * a.input_stride_t, w.c, D);
            }
        }
    };
    const int mine = wave * kGatedTile + half * kHalf;
    const int many = (max(end - w.first, 0) + kRound - 1) / kRound;
    if constexpr (!kSummary) {
        for (int t = w.first + many * kRound + (threadIdx.x >> 5); t < w.last; t += kWaves * 2)
            if (w.on) {
                store_two<T, kPairs>(gx + (int64_t)t * D, w.c, D, 0.0f, 0.0f);
                store_two<T, kPairs>(gp + (int64_t)t * D, w.c, D, 0.0f, 0.0f);
                store_two<T, kPairs>(gq + (int64_t)t * D, w.c, D, 0.0f, 0.0f);
            }
    }
    RawBack<T> next;
    if (many) load(w.first + (many - 1) * kRound + mine, next);
    int buf = 0;
    for (int r = w.first + (many - 1) * kRound; r >= w.first; r -= kRound, buf ^= 1) {
        const RawBack<T> now = next;
        if (r > w.first) load(r - kRound + mine, next);
        const int t0 = r + mine;
        float at[2] = {};
        if constexpr (!kSummary) {
            if (t0 - half * kHalf < end) {
                const float* from = ckpt + (w.b * tiles + t0 / kGatedTile) * D;
                at[0] = from[w.c];
                at[1] = from[c1];
            }
        }
        Decay e[kHalf][2];
        float A[2] = {1.0f, 1.0f}, H[2] = {}, C[2] = {}, fx[kHalf][2];
#pragma unroll
        for (int k = 0; k < kHalf; k++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                e[k][j] = decay(rate[j], sigmoid(to_float(now.p[k].v[j])));
                const bool live = t0 + k < end;
                if (!live) e[k][j] = {0.0f, 1.0f, 0.0f};
                A[j] *= e[k][j].a;
                if constexpr (!kSummary) {
                    fx[k][j] = live ? sigmoid(to_float(now.q[k].v[j])) * to_float(now.x[k].v[j]) : 0.0f;
                    H[j] = fmaf(e[k][j].a, H[j], __builtin_amdgcn_sqrtf(e[k][j].w) * fx[k][j]);
                }
            }
#pragma unroll
        for (int k = kHalf - 1; k >= 0; k--)
#pragma unroll
            for (int j = 0; j < 2; j++) C[j] = e[k][j].a * ((t0 + k < end ? to_float(now.g[k].v[j]) : 0.0f) + C[j]);
        float preA[2], preC[2], bothA[2], bothC[2], h[2];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const float oA = __shfl_xor(A[j], 32), oC = __shfl_xor(C[j], 32);
            preA[j] = half ? 1.0f : oA;
            preC[j] = half ? 0.0f : oC;
            bothA[j] = oA * A[j];
            bothC[j] = half ? fmaf(oA, C[j], oC) : fmaf(A[j], oC, C[j]);
            if constexpr (!kSummary) {
                const float oH = __shfl_xor(H[j], 32);
                h[j] = half ? fmaf(oA, at[j], oH) : at[j];
            }
        }
        if (!half) joined[buf][wave][li] = float4{bothA[0], bothA[1], bothC[0], bothC[1]};
        __syncthreads();
        float start[2];
#pragma unroll
        for (int j = kWaves - 1; j >= 0; j--) {
            const float4 v = joined[buf][j][li];
            if (j == wave) {
                start[0] = back[0];
                start[1] = back[1];
            }
            back[0] = fmaf(v.x, back[0], v.z);
            back[1] = fmaf(v.y, back[1], v.w);
            if constexpr (kSummary) {
                decayed[0] *= v.x;
                decayed[1] *= v.y;
            }
        }
        if constexpr (!kSummary) {
            float before[kHalf][2], sum[2] = {};
#pragma unroll
            for (int k = 0; k < kHalf; k++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    before[k][j] = h[j];
                    h[j] = fmaf(e[k][j].a, h[j], __builtin_amdgcn_sqrtf(e[k][j].w) * fx[k][j]);
                }
            float c[2] = {fmaf(preA[0], start[0], preC[0]), fmaf(preA[1], start[1], preC[1])};
#pragma unroll
            for (int k = kHalf - 1; k >= 0; k--) {
                float ox[2], op[2], oq[2];
                const bool live = t0 + k < end;
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const Decay& v = e[k][j];
                    const float l = to_float(now.g[k].v[j]) + c[j];
                    const Gate i = gate(to_float(now.q[k].v[j])), s = gate(to_float(now.p[k].v[j]));
                    const float rb = __builtin_amdgcn_rsqf(fmaxf(v.w, 1.1754944e-38f)), lb = l * (v.w * rb);      // 1 / b, and b l
                    const float U = l * v.a * (v.u * rb * v.a * fx[k][j] - v.u * before[k][j]);
                    ox[j] = live ? lb * i.s : 0.0f;
                    oq[j] = live ? lb * fx[k][j] * i.rest : 0.0f;
                    op[j] = live ? U * s.rest : 0.0f;
                    sum[j] += live ? U : 0.0f;
                    c[j] = live ? v.a * l : c[j];
                }
                if (w.on && t0 + k < w.last) {
                    store_two<T, kPairs>(gx + (int64_t)(t0 + k) * D, w.c, D, ox[0], ox[1]);
                    store_two<T, kPairs>(gp + (int64_t)(t0 + k) * D, w.c, D, op[0], op[1]);
                    store_two<T, kPairs>(gq + (int64_t)(t0 + k) * D, w.c, D, oq[0], oq[1]);
                }
            }
            total[0] += sum[0];
            total[1] += sum[1];
        }
    }
    if constexpr (kSummary) {
        if (threadIdx.x < 32 && w.on) {
            float* s = sums + ((w.b * chunks + w.chunk) * 2) * D;
            s[w.c] = decayed[0];
            s[D + w.c] = back[0];
            if (even) {
                s[w.c + 1] = decayed[1];
                s[D + w.c + 1] = back[1];
            }
        }
    } else {
        if (g.grad_initial_state && w.chunk == 0 && threadIdx.x < 32 && w.on) {
            g.grad_initial_state[w.b * D + w.c] = back[0];
            if (even) g.grad_initial_state[w.b * D + w.c + 1] = back[1];
        }
        __syncthreads();
        float* parts = (float*)joined;                                         // [16 halves][64 channels]
        parts[(threadIdx.x >> 5) * 64 + li * 2] = total[0];
        parts[(threadIdx.x >> 5) * 64 + li * 2 + 1] = total[1];
        __syncthreads();
        if (threadIdx.x < 32 && w.on) {
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves * 2; k++) {
                s0 += parts[k * 64 + li * 2];
                s1 += parts[k * 64 + li * 2 + 1];
            }
            float* to = rates + (w.b * chunks + w.chunk) * D;
            to[w.c] = s0;
            if (even) to[w.c + 1] = s1;
        }
    }
}

__global__ __launch_bounds__(1024) void gated_rates_kernel(const float* rates, int64_t rows, int64_t D, float* grad_log_rate)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const float s = sum_rows(rates + min(c, D - 1), rows, D);
    if (threadIdx.x < 64 && c < D) grad_log_rate[c] = s;
}

template <class T> __global__ __launch_bounds__(256) void gated_step_kernel(sig_gated_args a, float* state, T* y)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.B * a.D) return;
    const int64_t b = id / a.D, c = id % a.D;
    const Decay e = decay(rate_of(a.log_rate[c]), sigmoid(to_float(((const T*)a.decay_gate)[b * a.decay_stride_b + c])));
    const float f = __builtin_amdgcn_sqrtf(e.w) * sigmoid(to_float(((const T*)a.input_gate)[b * a.input_stride_b + c])) * to_float(((const T*)a.x)[b * a.x_stride_b + c]);
    const float h = fmaf(e.a, state[id], f);
    state[id] = h;
    y[id] = from_float<T>(h);
}

struct Plan { int groups, chunks, rounds; };
Plan plan(const sig_gated_args& a)
{
    Plan p;
    p.groups = (int)((a.D + kGroup - 1) / kGroup);
    const int64_t all = (a.L + kRound - 1) / kRound, rows = a.B * p.groups;
    int64_t chunks = rows >= 256 ? 1 : (512 + rows - 1) / (rows > 0 ? rows : 1);
    chunks = chunks > all ? (all ? all : 1) : chunks;
    p.rounds = (int)((all + chunks - 1) / chunks);
    if (p.rounds < 1) p.rounds = 1;
    p.chunks = (int)((all + p.rounds - 1) / p.rounds);
    if (p.chunks < 1) p.chunks = 1;
    return p;
}

bool pairs_fit(const void* p, int64_t sb, int64_t st, int e) { return (uintptr_t)p % (2 * e) == 0 && sb % 2 == 0 && st % 2 == 0; }

template <class T> hipError_t forward_of(const sig_gated_args& a, T* y, float* final_state, float* ckpt, float* sums, hipStream_t stream)
{
    const Plan p = plan(a);
    const int64_t blocks = a.B * p.groups * p.chunks;
    if (!launchable(blocks, kWaves * 64)) return kTooManyThreads;
    const int e = sizeof(T);
    const bool pairs = a.D % 2 == 0 && pairs_fit(y, 0, 0, e) && pairs_fit(a.x, a.x_stride_b, a.x_stride_t, e) && pairs_fit(a.decay_gate, a.decay_stride_b, a.decay_stride_t, e) &&
                       pairs_fit(a.input_gate, a.input_stride_b, a.input_stride_t, e);
    auto go = [&](auto k) { k<<<(uint32_t)blocks, kWaves * 64, 0, stream>>>(a, y, final_state, ckpt, sums, p.groups, p.chunks, p.rounds); };
    if (p.chunks > 1) {
        pairs ? go(gated_forward_kernel<T, true, true>) : go(gated_forward_kernel<T, false, true>);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    pairs ? go(gated_forward_kernel<T, true, false>) : go(gated_forward_kernel<T, false, false>);
    return hipGetLastError();
}

template <class T> hipError_t backward_of(const sig_gated_args& a, const sig_gated_grads& g, const float* ckpt, float* ws, hipStream_t stream)
{
    const Plan p = plan(a);
    const int64_t blocks = a.B * p.groups * p.chunks, parts = a.B * p.chunks;
    if (!launchable(blocks, kWaves * 64) || !launchable(p.groups, 1024)) return kTooManyThreads;
    float *sums = ws, *rates = ws + (p.chunks > 1 ? parts * 2 * a.D : 0);
    if (blocks) {
        const int e = sizeof(T);
        const bool pairs = a.D % 2 == 0 && pairs_fit(g.grad_x, 0, 0, e) && pairs_fit(g.grad_decay_gate, 0, 0, e) && pairs_fit(g.grad_input_gate, 0, 0, e) &&
                           pairs_fit(g.grad_y, g.gy_stride_b, g.gy_stride_t, e) && pairs_fit(a.x, a.x_stride_b, a.x_stride_t, e) &&
                           pairs_fit(a.decay_gate, a.decay_stride_b, a.decay_stride_t, e) && pairs_fit(a.input_gate, a.input_stride_b, a.input_stride_t, e);
        auto go = [&](auto k) { k<<<(uint32_t)blocks, kWaves * 64, 0, stream>>>(a, g, ckpt, sums, rates, p.groups, p.chunks, p.rounds); };
        if (p.chunks > 1) {
            pairs ? go(gated_backward_kernel<T, true, true>) : go(gated_backward_kernel<T, false, true>);
            hipError_t err = hipGetLastError();
            if (err != hipSuccess) return err;
        }
        pairs ? go(gated_backward_kernel<T, true, false>) : go(gated_backward_kernel<T, false, false>);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    gated_rates_kernel<<<(uint32_t)p.groups, 1024, 0, stream>>>(rates, parts, a.D, g.grad_log_rate);
    return hipGetLastError();
}

}  // namespace

size_t gated_forward_workspace(const sig_gated_args& a)
{
    const Plan p = plan(a);
    return p.chunks > 1 ? (size_t)(a.B * p.chunks * 2 * a.D * 4) : 0;
}
size_t gated_backward_workspace(const sig_gated_args& a)
{
    const Plan p = plan(a);
    return (size_t)(a.B * p.chunks * (p.chunks > 1 ? 3 : 1) * a.D * 4);
}
hipError_t gated_forward(const sig_gated_args& a, void* y, float* final_state, float* checkpoint, float* workspace, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? forward_of(a, (bf16*)y, final_state, checkpoint, workspace, stream) : forward_of(a, (float*)y, final_state, checkpoint, workspace, stream);
}
hipError_t gated_backward(const sig_gated_args& a, const sig_gated_grads& g, const float* checkpoint, float* workspace, hipStream_t stream)
{
    return a.dtype == SIG_BF16 ? backward_of<bf16>(a, g, checkpoint, workspace, stream) : backward_of<float>(a, g, checkpoint, workspace, stream);
}
hipError_t gated_step(const sig_gated_args& a, float* state, void* y, hipStream_t stream)
{
    const int64_t blocks = (a.B * a.D + 255) / 256;
    if (!launchable(blocks, 256)) return kTooManyThreads;
    if (a.dtype == SIG_BF16) gated_step_kernel<<<(uint32_t)blocks, 256, 0, stream>>>(a, state, (bf16*)y);
    else gated_step_kernel<<<(uint32_t)blocks, 256, 0, stream>>>(a, state, (float*)y);
    return hipGetLastError();
}

}  // namespace sig
