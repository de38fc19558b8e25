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
// Bound by memory where there are many streams: 8 x 2048 x 2048 in bfloat16 takes 68 us forward (277 MB with the states that are kept, 4.1 TB/s) and 106
// backward (478 MB, 4.5 TB/s); the vector units have about 40 and 72 instructions a token and channel.  One stream reads its inputs twice: 1 x 16384 x 1024
// takes 23 us for the chunks' maps and 30 for the outputs.
//
// Gradient: with c_t what comes back from the tokens after t, l_t = grad_y_t + c_t and c_(t-1) = a_t l_t, the same structure from the end.  With U_t = u_t dL/du_t
//   grad x = l b i,  grad q = l b x i (1 - i),  U = l (u a^2 / b i x - u a h_(t-1)),  grad p = U (1 - sigmoid(p)),  grad log_rate = sum U:
// u / b goes to zero like sqrt(u / 2), so nothing here is infinite at u = 0.
#include <algorithm>
#include <type_traits>

#include "gated_lane.hpp"
#include "layer.hpp"

namespace sig {
namespace {

constexpr int kWaves = 8, kHalf = 8, kRound = kWaves * kGatedTile, kGroup = kGatedGroup;

struct Two { float v[2]; };

// Tokens first .. last - 1 of a stream's channels, as a buffer that begins with token `first` and ends with token last - 1: accesses behind it give
// zeros and write nothing.  A lane's place in it is 32 bits, which tokens of a round do not pass (time strides below 2^22 elements).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tokens(const void* stream, int64_t stride_t, int64_t first, int64_t last, int64_t D, int e)
{
    const int64_t n = min(last - first, (int64_t)kRound);
    const uint32_t bytes = n > 0 ? (uint32_t)(((n - 1) * stride_t + D) * e) : 0;
    return __builtin_amdgcn_make_buffer_rsrc((char*)stream + first * stride_t * e, 0, bytes, 0x27000);
}
// A lane's two channels of a token, in words as they lie in memory (elements of their own would take a register each)
template <class T> struct Both { uint32_t w[sizeof(T) / 2]; };
__device__ __forceinline__ float value(const Both<bf16>& v, int j) { return __uint_as_float(j ? v.w[0] & 0xffff0000u : v.w[0] << 16); }
__device__ __forceinline__ float value(const Both<float>& v, int j) { return __uint_as_float(v.w[j]); }

// kHalf tokens' channels, the first at `at` bytes, the others `step` bytes apart; not kPairs: `second` bytes lie between the two
template <class T, bool kPairs> __device__ __forceinline__ void load_two(__amdgpu_buffer_rsrc_t from, int at, int second, int step, Both<T>* to)
{
#pragma unroll
    for (int k = 0; k < kHalf; k++) {
        if constexpr (!kPairs && sizeof(T) == 2) {
            const uint32_t u = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, at, k * step, 0), v = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, at + second, k * step, 0);
            to[k].w[0] = u | v << 16;
        } else if constexpr (!kPairs) {
            to[k].w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, k * step, 0);
            to[k].w[1] = __builtin_amdgcn_raw_buffer_load_b32(from, at + second, k * step, 0);
        } else if constexpr (sizeof(T) == 2) {
            to[k].w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, k * step, 0);
        } else {
            typedef uint32_t Words __attribute__((ext_vector_type(2)));
            const Words u = __builtin_amdgcn_raw_buffer_load_b64(from, at, k * step, 0);
            to[k].w[0] = u[0];
            to[k].w[1] = u[1];
        }
    }
}
// All ones for a token that counts, else 0; masked() keeps v or makes it 0.  Selections by a condition the compiler turns into branches, and puts behind
// them the work that the selected value takes, with all that this work needs held in registers; hence a mask whose origin it does not see.
// kAll: every token of the round counts, and nothing is masked.
template <bool kAll> __device__ __forceinline__ uint32_t mask_of(bool counts)
{
    if constexpr (kAll) return ~0u;
    uint32_t m = counts ? ~0u : 0u;
    asm("" : "+v"(m));
    return m;
}
// v, computed here: the compiler moves what is used behind a barrier there, and holds all that it is made of instead
__device__ __forceinline__ float here(float v)
{
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ float masked(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }
template <class T> __device__ __forceinline__ Both<T> masked(Both<T> v, uint32_t mask)
{
#pragma unroll
    for (uint32_t& word : v.w) word &= mask;
    return v;
}
__device__ __forceinline__ void pack(Both<bf16>& r, float v0, float v1)
{
    const float v[2] = {v0, v1};
    r.w[0] = word_of(v, (bf16*)nullptr);
}
__device__ __forceinline__ void pack(Both<float>& r, float v0, float v1)
{
    r.w[0] = __float_as_uint(v0);
    r.w[1] = __float_as_uint(v1);
}
template <class T, bool kPairs> __device__ __forceinline__ void store_two(__amdgpu_buffer_rsrc_t to, int at, int second, int step, uint32_t mask, float v0, float v1)
{
    Both<T> r;
    pack(r, v0, v1);
    r = masked(r, mask);
    if constexpr (!kPairs && sizeof(T) == 2) {
        __builtin_amdgcn_raw_buffer_store_b16((uint16_t)r.w[0], to, at, step, 0);
        if (second) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(r.w[0] >> 16), to, at + second, step, 0);
    } else if constexpr (!kPairs) {
        __builtin_amdgcn_raw_buffer_store_b32(r.w[0], to, at, step, 0);
        if (second) __builtin_amdgcn_raw_buffer_store_b32(r.w[1], to, at + second, step, 0);
    } else if constexpr (sizeof(T) == 2) {
        __builtin_amdgcn_raw_buffer_store_b32(r.w[0], to, at, step, 0);
    } else {
        typedef uint32_t Words __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(Words{r.w[0], r.w[1]}, to, at, step, 0);
    }
}
constexpr int kNowhere = (int)0x80000000;      // a place behind every such buffer: its stores write nothing

// sigmoid(v) and 1 - sigmoid(v) = sigmoid(-v), which keeps its relative precision where it is small
struct Gate { float s, rest; };
__device__ __forceinline__ Gate gate(float v)
{
    const float e = fast_exp(-v), s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, v > 0.0f ? e * s : 1.0f - s};
}

// u log2(e) = x, a = 2^-x and w = 1 - a^2 for x >= 0.  Small x: the power series of 1 - exp(-v), v = 2 u < 1/2, up to v^7, whose first omitted term is
// v^8 / 8! < 2.5e-7 of the value; from there on 1 - a^2 >= 0.39 loses a bit and a half at most.
struct Decay { float x, a, w; };
__device__ __forceinline__ Decay decay(float rate, float open)                 // rate: exp(log_rate) log2(e)
{
    constexpr float v = 1.3862943611f;                                         // of an x of one
    constexpr float k1 = v, k2 = -k1 * v / 2, k3 = -k2 * v / 3, k4 = -k3 * v / 4, k5 = -k4 * v / 5, k6 = -k5 * v / 6, k7 = -k6 * v / 7;
    const float x = rate * open, a = __builtin_amdgcn_exp2f(-x);
    float p = fmaf(x, k7, k6);
    p = fmaf(p, x, k5);
    p = fmaf(p, x, k4);
    p = fmaf(p, x, k3);
    p = fmaf(p, x, k2);
    p = fmaf(p, x, k1);
    return {x, a, x < 0.5f / v ? p * x : fmaf(-a, a, 1.0f)};
}

// exp(log_rate) log2(e), log_rate taken as 64 beyond that: u is finite, and a product with a shut gate's zero stays one.  A NaN stays one.
constexpr float kMostLogRate = 64.0f;
__device__ __forceinline__ float rate_of(float log_rate) { return fast_exp(log_rate > kMostLogRate ? kMostLogRate : log_rate) * kLog2e; }

struct Where {                       // of a workgroup: stream, channels, tokens of its chunk, and how many of them count
    int64_t b;
    int chunk, c, c1, first, last, live;
    bool on, even;                   // see GatedLane
};
template <bool kPairs> __device__ __forceinline__ Where where(const sig_gated_args& a, int groups, int chunks, int rounds)
{
    Where w;
    const uint32_t id = blockIdx.x;
    w.chunk = id % chunks;
    const uint32_t row = id / chunks;
    w.b = row / groups;
    const GatedLane lane = gated_lane(row % groups, threadIdx.x & 31, (int)a.D, kPairs);
    w.c = lane.c;
    w.c1 = lane.c1;
    w.on = lane.on;
    w.even = lane.even;
    const int64_t span = (int64_t)rounds * kRound;
    w.first = (int)min((int64_t)w.chunk * span, a.L);
    w.last = (int)min((w.chunk + 1) * span, a.L);
    w.live = (int)live_length(a.lengths, w.b, a.L);
    return w;
}

template <class T> struct Raw { Both<T> x[kHalf], p[kHalf], q[kHalf], g[kHalf]; };

// Where a lane's channels are in buffers of tokens, in bytes
struct Lane { int second, x, p, q, g, out; };
template <class T, bool kPairs, bool kBack>
__device__ __forceinline__ void load_round(const sig_gated_args& a, const void* gy, int64_t gy_stride, const Where& w, const Lane& l, int64_t first, int64_t end, bool inputs, Raw<T>& r)
{
    constexpr int e = sizeof(T);
    load_two<T, kPairs>(tokens((const T*)a.decay_gate + w.b * a.decay_stride_b, a.decay_stride_t, first, end, a.D, e), l.p, l.second, (int)a.decay_stride_t * e, r.p);
    if (inputs) {
        load_two<T, kPairs>(tokens((const T*)a.x + w.b * a.x_stride_b, a.x_stride_t, first, end, a.D, e), l.x, l.second, (int)a.x_stride_t * e, r.x);
        load_two<T, kPairs>(tokens((const T*)a.input_gate + w.b * a.input_stride_b, a.input_stride_t, first, end, a.D, e), l.q, l.second, (int)a.input_stride_t * e, r.q);
    }
    if constexpr (kBack) load_two<T, kPairs>(tokens(gy, gy_stride, first, end, a.D, e), l.g, l.second, (int)gy_stride * e, r.g);
}

// The maps (A, H) of sixteen half wavefronts' stretches, in the order of time or (kBack) against it: `state`, the value before all of them, becomes the one
// behind them; `wave` is the value before this wavefront's stretch, `half` the one before this half's.  One barrier.
template <bool kBack> __device__ __forceinline__ void cross(float4 (*joined)[32], const float* A, const float* H, float* state, float* wave_start, float* start)
{
    const int w = threadIdx.x / 64, li = threadIdx.x & 31;
    const bool upper = threadIdx.x & 32, first = upper == kBack;
    float preA[2], preH[2], bothA[2], bothH[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const float oA = __shfl_xor(A[j], 32), oH = __shfl_xor(H[j], 32);
        preA[j] = first ? 1.0f : oA;
        preH[j] = first ? 0.0f : oH;
        bothA[j] = oA * A[j];
        bothH[j] = first ? fmaf(oA, H[j], oH) : fmaf(A[j], oH, H[j]);
    }
    if (!upper) joined[w][li] = float4{bothA[0], bothA[1], bothH[0], bothH[1]};
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; k++) {
        const int j = kBack ? kWaves - 1 - k : k;
        const float4 v = joined[j][li];
        if (j == w) {
            wave_start[0] = state[0];
            wave_start[1] = state[1];
        }
        state[0] = fmaf(v.x, state[0], v.z);
        state[1] = fmaf(v.y, state[1], v.w);
    }
#pragma unroll
    for (int j = 0; j < 2; j++) start[j] = fmaf(preA[j], wave_start[j], preH[j]);
}

// `state`, given for the stream's beginning (kBack: end), becomes the value before this workgroup's chunk: the maps of the chunks on the way, a sixteenth of
// them each half wavefront
template <bool kBack> __device__ __forceinline__ void enter(float4 (*joined)[32], const float* sums, int64_t D, int c, int c1, int chunk, int chunks, float* state)
{
    const int n = kBack ? chunks - 1 - chunk : chunk, base = kBack ? chunk + 1 : 0, part = threadIdx.x >> 5;
    const int from = part * n / (2 * kWaves), to = (part + 1) * n / (2 * kWaves);
    float A[2] = {1.0f, 1.0f}, H[2] = {}, wave_start[2], start[2];
#pragma unroll 4
    for (int k = from; k < to; k++) {
        const float* s = sums + (int64_t)(base + (kBack ? to - 1 - (k - from) : k)) * 2 * D;
        H[0] = fmaf(s[c], H[0], s[D + c]);
        H[1] = fmaf(s[c1], H[1], s[D + c1]);
        A[0] *= s[c];
        A[1] *= s[c1];
    }
    cross<kBack>(joined, A, H, state, wave_start, start);
}

// A chunk's map (A, H): a wavefront has a sixteenth of its tokens, in a row
template <class T, bool kPairs, bool kBack>
__global__ __launch_bounds__(kWaves * 64) void gated_sums_kernel(sig_gated_args a, sig_gated_grads g, float* sums, int groups, int chunks, int rounds)
{
    __shared__ float4 joined[kWaves][32];
    const Where w = where<kPairs>(a, groups, chunks, rounds);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = (threadIdx.x >> 5) & 1, D = (int)a.D, e = sizeof(T);
    const bool even = w.even;
    const int c1 = w.c1, mine = half * kHalf;
    const float rate[2] = {rate_of(a.log_rate[w.c]), rate_of(a.log_rate[c1])};
    const T* gy = kBack ? (const T*)g.grad_y + w.b * g.gy_stride_b : nullptr;
    const Lane l{(c1 - w.c) * e, (int)(mine * a.x_stride_t + w.c) * e, (int)(mine * a.decay_stride_t + w.c) * e, (int)(mine * a.input_stride_t + w.c) * e, (int)(mine * g.gy_stride_t + w.c) * e, 0};
    const int end = min(w.last, w.live), from = w.first + wave * rounds * kGatedTile, to = min(end, from + rounds * kGatedTile);
    const int many = (max(to - from, 0) + kGatedTile - 1) / kGatedTile;
    auto at = [&](int k) { return from + (kBack ? many - 1 - k : k) * kGatedTile; };
    float A[2] = {1.0f, 1.0f}, H[2] = {};                                      // of the tokens so far
    Raw<T> next;
    if (many) load_round<T, kPairs, kBack>(a, gy, g.gy_stride_t, w, l, at(0), to, !kBack, next);
    for (int n = 0; n < many; n++) {
        const Raw<T> now = next;
        if (n + 1 < many) load_round<T, kPairs, kBack>(a, gy, g.gy_stride_t, w, l, at(n + 1), to, !kBack, next);
        const int t0 = at(n) + mine;
        float B[2] = {1.0f, 1.0f}, G[2] = {};
        auto tile = [&](auto all) {
#pragma unroll
            for (int q = 0; q < kHalf; q++) {
                const int k = kBack ? kHalf - 1 - q : q;
                const uint32_t mask = mask_of<decltype(all)::value>(t0 + k < to);
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const Decay v = decay(rate[j], masked(sigmoid(value(now.p[k], j)), mask));
                    if constexpr (kBack) G[j] = v.a * (masked(value(now.g[k], j), mask) + G[j]);
                    else G[j] = fmaf(v.a, G[j], masked(__builtin_amdgcn_sqrtf(v.w) * sigmoid(value(now.q[k], j)) * value(now.x[k], j), mask));
                    B[j] *= v.a;
                }
            }
        };
        if (at(n) + kGatedTile <= to) tile(std::true_type());
        else tile(std::false_type());
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const float oB = __shfl_xor(B[j], 32), oG = __shfl_xor(G[j], 32);
            const float bothG = (half == 1) == kBack ? fmaf(oB, G[j], oG) : fmaf(B[j], oG, G[j]), bothB = oB * B[j];
            H[j] = fmaf(bothB, H[j], bothG);
            A[j] *= bothB;
        }
    }
    if (!half) joined[wave][threadIdx.x & 31] = float4{A[0], A[1], H[0], H[1]};
    __syncthreads();
    if (threadIdx.x < 32 && w.on) {
        float4 all = joined[kBack ? kWaves - 1 : 0][threadIdx.x];
#pragma unroll
        for (int k = 1; k < kWaves; k++) {
            const float4 v = joined[kBack ? kWaves - 1 - k : k][threadIdx.x];
            all = float4{all.x * v.x, all.y * v.y, fmaf(v.x, all.z, v.z), fmaf(v.y, all.w, v.w)};
        }
        float* s = sums + ((w.b * chunks + w.chunk) * 2) * D;
        s[w.c] = all.x;
        s[D + w.c] = all.z;
        if (even) {
            s[w.c + 1] = all.y;
            s[D + w.c + 1] = all.w;
        }
    }
}

template <class T, bool kPairs>
__global__ __launch_bounds__(kWaves * 64) void gated_forward_kernel(sig_gated_args a, T* y, float* final_state, float* ckpt, float* sums, int groups, int chunks,
                                                                     int rounds)
{
    __shared__ float4 joined[2][kWaves][32];
    const Where w = where<kPairs>(a, groups, chunks, rounds);
    const int wave = threadIdx.x / 64, half = (threadIdx.x >> 5) & 1, D = (int)a.D;
    const bool even = w.even;
    const int c1 = w.c1;
    const float rate[2] = {rate_of(a.log_rate[w.c]), rate_of(a.log_rate[c1])};
    float state[2] = {};
    if (a.initial_state) {
        state[0] = a.initial_state[w.b * D + w.c];
        state[1] = a.initial_state[w.b * D + c1];
    }
    if (chunks > 1) enter<false>(joined[1], sums + w.b * chunks * 2 * D, D, w.c, c1, w.chunk, chunks, state);
    const int end = min(w.last, w.live);
    const int64_t tiles = (a.L + kGatedTile - 1) / kGatedTile;
    const int mine = wave * kGatedTile + half * kHalf, e = sizeof(T);
    const Lane l{(c1 - w.c) * e, (int)(mine * a.x_stride_t + w.c) * e, (int)(mine * a.decay_stride_t + w.c) * e, (int)(mine * a.input_stride_t + w.c) * e, 0, w.on ? (mine * D + w.c) * e : kNowhere};
    T* out = y + w.b * a.L * D;
    Raw<T> next;
    if (w.first < end) load_round<T, kPairs, false>(a, nullptr, 0, w, l, w.first, end, true, next);
    int buf = 0;
    for (int r = w.first; r < end; r += kRound, buf ^= 1) {
        const Raw<T> now = next;
        if (r + kRound < end) load_round<T, kPairs, false>(a, nullptr, 0, w, l, r + kRound, end, true, next);
        auto round = [&](auto all) {
            const int t0 = r + mine;
            float f[kHalf][2], d[kHalf][2], A[2] = {1.0f, 1.0f}, H[2] = {};
#pragma unroll
            for (int k = 0; k < kHalf; k++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    // a token that does not count has u = 0: nothing decays, and b is 0
                    const uint32_t mask = mask_of<decltype(all)::value>(t0 + k < end);
                    const Decay v = decay(rate[j], masked(sigmoid(value(now.p[k], j)), mask));
                    d[k][j] = v.a;
                    f[k][j] = masked(__builtin_amdgcn_sqrtf(v.w) * sigmoid(value(now.q[k], j)) * value(now.x[k], j), mask);
                    A[j] *= d[k][j];
                    H[j] = fmaf(d[k][j], H[j], f[k][j]);
                }
            float wave_start[2], h[2];
            cross<false>(joined[buf], A, H, state, wave_start, h);
            if (ckpt && !half && w.on && t0 < end) {
                float* to = ckpt + (w.b * tiles + t0 / kGatedTile) * D;
                to[w.c] = wave_start[0];
                if (even) to[w.c + 1] = wave_start[1];
            }
            const __amdgpu_buffer_rsrc_t to = tokens(out, D, r, w.last, D, e);
#pragma unroll
            for (int k = 0; k < kHalf; k++) {
                h[0] = fmaf(d[k][0], h[0], f[k][0]);
                h[1] = fmaf(d[k][1], h[1], f[k][1]);
                store_two<T, kPairs>(to, l.out, l.second, k * D * e, mask_of<decltype(all)::value>(t0 + k < end), h[0], h[1]);
            }
        };
        if (r + kRound <= end) round(std::true_type());
        else round(std::false_type());
    }
    // what no round has reached
    const int done = w.first + (max(end - w.first, 0) + kRound - 1) / kRound * kRound;
    for (int t = done; t < w.last; t += kRound)
#pragma unroll
        for (int k = 0; k < kHalf; k++) store_two<T, kPairs>(tokens(out, D, t, w.last, D, e), l.out, l.second, k * D * e, 0, 0.0f, 0.0f);
    if (final_state && w.chunk == chunks - 1 && threadIdx.x < 32 && w.on) {
        final_state[w.b * D + w.c] = state[0];
        if (even) final_state[w.b * D + w.c + 1] = state[1];
    }
}

template <class T, bool kPairs>
__global__ __launch_bounds__(kWaves * 64) void gated_backward_kernel(sig_gated_args a, sig_gated_grads g, const float* ckpt, float* sums, float* rates, int groups,
                                                                      int chunks, int rounds)
{
    __shared__ float4 joined[2][kWaves][32];
    const Where w = where<kPairs>(a, groups, chunks, rounds);
    const int wave = threadIdx.x / 64, half = (threadIdx.x >> 5) & 1, li = threadIdx.x & 31, D = (int)a.D;
    const bool even = w.even;
    const T* gy = (const T*)g.grad_y + w.b * g.gy_stride_b;
    T *gx = (T*)g.grad_x + w.b * a.L * D, *gp = (T*)g.grad_decay_gate + w.b * a.L * D, *gq = (T*)g.grad_input_gate + w.b * a.L * D;
    const int c1 = w.c1;
    const float rate[2] = {rate_of(a.log_rate[w.c]), rate_of(a.log_rate[c1])};
    float back[2] = {}, total[2] = {};
    if (g.grad_final_state) {
        back[0] = g.grad_final_state[w.b * D + w.c];
        back[1] = g.grad_final_state[w.b * D + c1];
    }
    if (chunks > 1) enter<true>(joined[1], sums + w.b * chunks * 2 * D, D, w.c, c1, w.chunk, chunks, back);
    const int end = min(w.last, w.live);
    const int64_t tiles = (a.L + kGatedTile - 1) / kGatedTile;
    const int mine = wave * kGatedTile + half * kHalf, e = sizeof(T);
    const Lane l{(c1 - w.c) * e, (int)(mine * a.x_stride_t + w.c) * e, (int)(mine * a.decay_stride_t + w.c) * e, (int)(mine * a.input_stride_t + w.c) * e, (int)(mine * g.gy_stride_t + w.c) * e,
                 w.on ? (mine * D + w.c) * e : kNowhere};
    const int many = (max(end - w.first, 0) + kRound - 1) / kRound;
    for (int t = w.first + many * kRound; t < w.last; t += kRound)
#pragma unroll
        for (int k = 0; k < kHalf; k++) {
            store_two<T, kPairs>(tokens(gx, D, t, w.last, D, e), l.out, l.second, k * D * e, 0, 0.0f, 0.0f);
            store_two<T, kPairs>(tokens(gp, D, t, w.last, D, e), l.out, l.second, k * D * e, 0, 0.0f, 0.0f);
            store_two<T, kPairs>(tokens(gq, D, t, w.last, D, e), l.out, l.second, k * D * e, 0, 0.0f, 0.0f);
        }
    Raw<T> next;
    if (many) load_round<T, kPairs, true>(a, gy, g.gy_stride_t, w, l, w.first + (many - 1) * kRound, end, true, next);
    int buf = 0;
    for (int r = w.first + (many - 1) * kRound; r >= w.first; r -= kRound, buf ^= 1) {
        Raw<T> now = next;
        if (r > w.first) load_round<T, kPairs, true>(a, gy, g.gy_stride_t, w, l, r - kRound, end, true, next);
        const int t0 = r + mine;
        float at[2] = {};
        if (t0 - half * kHalf < end) {
            const float* from = ckpt + (w.b * tiles + t0 / kGatedTile) * D;
            at[0] = from[w.c];
            at[1] = from[c1];
        }
        // of every token: its decay a, and what l is multiplied by in the gradients of x, q (both with b) and p; U = l (own - from h)
        float d[kHalf][2], toward_x[kHalf][2], f[kHalf][2], toward_q[kHalf][2], shut[kHalf][2], own[kHalf][2], from[kHalf][2], A[2] = {1.0f, 1.0f}, H[2] = {}, C[2] = {};
#pragma unroll
        for (int k = 0; k < kHalf; k++) {
            __builtin_amdgcn_sched_barrier(0);      // a token's values are done before the next one's begin: all at once do not fit the registers
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const uint32_t mask = mask_of<false>(t0 + k < end);
                const Gate open = gate(value(now.p[k], j));
                const Decay v = decay(rate[j], masked(open.s, mask));
                d[k][j] = v.a;
                A[j] *= d[k][j];
                const Gate in = gate(value(now.q[k], j));
                const float rb = __builtin_amdgcn_rsqf(fmaxf(v.w, 1.1754944e-38f)), xi = masked(value(now.x[k], j) * in.s, mask);      // 1 / b
                toward_x[k][j] = here(v.w * rb * in.s);
                f[k][j] = here(v.w * rb * xi);
                toward_q[k][j] = here(in.rest);
                shut[k][j] = here(open.rest);
                own[k][j] = here(v.a * v.a * (v.x * 0.69314718f * rb) * xi);
                from[k][j] = here(v.a * (v.x * 0.69314718f));
                H[j] = fmaf(d[k][j], H[j], f[k][j]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kHalf; k++) now.g[k] = masked(now.g[k], mask_of<false>(t0 + k < end));
#pragma unroll
        for (int k = kHalf - 1; k >= 0; k--)
#pragma unroll
            for (int j = 0; j < 2; j++) C[j] = d[k][j] * (value(now.g[k], j) + C[j]);
        float wave_start[2], c[2], h[2];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const float oA = __shfl_xor(A[j], 32), oH = __shfl_xor(H[j], 32);
            h[j] = half ? fmaf(oA, at[j], oH) : at[j];
        }
        cross<true>(joined[buf], A, C, back, wave_start, c);
        float sum[2] = {};
#pragma unroll
        for (int k = 0; k < kHalf; k++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                own[k][j] = fmaf(-from[k][j], h[j], own[k][j]);
                h[j] = fmaf(d[k][j], h[j], f[k][j]);
            }
        const __amdgpu_buffer_rsrc_t tx = tokens(gx, D, r, w.last, D, e), tp = tokens(gp, D, r, w.last, D, e), tq = tokens(gq, D, r, w.last, D, e);
#pragma unroll
        for (int k = kHalf - 1; k >= 0; k--) {
            float ox[2], op[2], oq[2];
            const uint32_t mask = mask_of<false>(t0 + k < end);
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const float lam = value(now.g[k], j) + c[j], U = masked(lam * own[k][j], mask);
                ox[j] = lam * toward_x[k][j];
                oq[j] = lam * f[k][j] * toward_q[k][j];
                op[j] = U * shut[k][j];
                sum[j] += U;
                c[j] = d[k][j] * lam;
            }
            store_two<T, kPairs>(tx, l.out, l.second, k * D * e, mask, ox[0], ox[1]);
            store_two<T, kPairs>(tp, l.out, l.second, k * D * e, mask, op[0], op[1]);
            store_two<T, kPairs>(tq, l.out, l.second, k * D * e, mask, oq[0], oq[1]);
        }
        total[0] += sum[0];
        total[1] += sum[1];
    }
    if (g.grad_initial_state && w.chunk == 0 && threadIdx.x < 32 && w.on) {
        g.grad_initial_state[w.b * D + w.c] = back[0];
        if (even) g.grad_initial_state[w.b * D + w.c + 1] = back[1];
    }
    __syncthreads();
    float* parts = (float*)joined;                                             // [16 halves][64 channels]
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

// The sums of U over streams and chunks; zero where log_rate is beyond what it counts as
__global__ __launch_bounds__(1024) void gated_rates_kernel(const float* rates, int64_t rows, int64_t D, const float* log_rate, float* grad_log_rate)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const float s = sum_rows(rates + min(c, D - 1), rows, D);
    if (threadIdx.x < 64 && c < D) grad_log_rate[c] = log_rate[c] > kMostLogRate ? 0.0f : s;
}

// One token: bound by latency and the call (64 x 2048 in bfloat16: 3.0 us)
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

// Time chunks: as many as the compute units have room for with one workgroup each (1 x 16384 x 1024 in bfloat16, forward and backward: 256 workgroups 51 and
// 63 us, 128 83 and 102, 512 56 and 70; 1 x 8192 x 1536: 240 workgroups 43 and 54 us, 264 62 and 74).  None forward where the streams give half of that
// already: a first pass costs more than the idle half (4 x 8192 x 2048: 185 us without, 208 with one; backward 346 without, 269 with one).  Four rounds in a
// row are already worse than two passes over chunks of them (7 x 301 x 277 float32 training step: 53.6 us for 43).
struct Plan { int groups, chunks, rounds; };
Plan plan(const sig_gated_args& a, bool back)
{
    Plan p;
    p.groups = (int)((a.D + kGroup - 1) / kGroup);
    const int64_t all = (a.L + kRound - 1) / kRound, rows = a.B * p.groups;
    int64_t chunks = rows >= (back ? 256 : 128) ? 1 : 256 / std::max<int64_t>(rows, 1);
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
    const Plan p = plan(a, false);
    const int64_t blocks = a.B * p.groups * p.chunks;
    if (!launchable(blocks, kWaves * 64)) return kTooManyThreads;
    const int e = sizeof(T);
    const bool pairs = a.D % 2 == 0 && pairs_fit(y, 0, 0, e) && pairs_fit(a.x, a.x_stride_b, a.x_stride_t, e) && pairs_fit(a.decay_gate, a.decay_stride_b, a.decay_stride_t, e) &&
                       pairs_fit(a.input_gate, a.input_stride_b, a.input_stride_t, e);
    auto go = [&](auto k) { k<<<(uint32_t)blocks, kWaves * 64, 0, stream>>>(a, y, final_state, ckpt, sums, p.groups, p.chunks, p.rounds); };
    if (p.chunks > 1) {
        const sig_gated_grads none{};
        auto first = [&](auto k) { k<<<(uint32_t)blocks, kWaves * 64, 0, stream>>>(a, none, sums, p.groups, p.chunks, p.rounds); };
        pairs ? first(gated_sums_kernel<T, true, false>) : first(gated_sums_kernel<T, false, false>);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    pairs ? go(gated_forward_kernel<T, true>) : go(gated_forward_kernel<T, false>);
    return hipGetLastError();
}

template <class T> hipError_t backward_of(const sig_gated_args& a, const sig_gated_grads& g, const float* ckpt, float* ws, hipStream_t stream)
{
    const Plan p = plan(a, true);
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
            auto first = [&](auto k) { k<<<(uint32_t)blocks, kWaves * 64, 0, stream>>>(a, g, sums, p.groups, p.chunks, p.rounds); };
            pairs ? first(gated_sums_kernel<T, true, true>) : first(gated_sums_kernel<T, false, true>);
            hipError_t err = hipGetLastError();
            if (err != hipSuccess) return err;
        }
        pairs ? go(gated_backward_kernel<T, true>) : go(gated_backward_kernel<T, false>);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    gated_rates_kernel<<<(uint32_t)p.groups, 1024, 0, stream>>>(rates, parts, a.D, a.log_rate, g.grad_log_rate);
    return hipGetLastError();
}

}  // namespace

size_t gated_forward_workspace(const sig_gated_args& a)
{
    const Plan p = plan(a, false);
    return p.chunks > 1 ? (size_t)(a.B * p.chunks * 2 * a.D * 4) : 0;
}
size_t gated_backward_workspace(const sig_gated_args& a)
{
    const Plan p = plan(a, true);
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
