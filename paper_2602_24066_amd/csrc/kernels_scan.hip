// Selective state space scan over tokens t, for each stream b and channel d (group g = d / (D / G)) with N states n:
//   D_t = softplus(dt_t + dt_bias) or the sum itself,   a_t[n] = exp(D_t A[n]),   h_t[n] = a_t[n] h_{t-1}[n] + D_t x_t B_t[n],
//   s_t = sum_n C_t[n] h_t[n] + skip x_t,   y_t = s_t silu(gate_t) or s_t.
// Gradient, with S_t = dL/ds_t and l_t[n] = dL/dh_t[n]:
//   l_t = C_t S_t + a_{t+1} l_{t+1} (plus the final state's gradient at the last token),
//   dx_t = D_t sum_n l_t B_t + skip S_t,            dD_t = sum_n l_t (x_t B_t + A a_t h_{t-1}),   ddt_t = dD_t sigmoid(dt_t + dt_bias),
//   dB_t = sum_{d in g} l_t D_t x_t,                dC_t = sum_{d in g} S_t h_t,
//   dA = sum_{b,t} l_t a_t h_{t-1} D_t,             dgate_t = dL/dy_t s_t silu'(gate_t),          dh_0 = a_1 l_1.
// States, sums and gradients in registers are float32; y and the tokens' gradients are rounded once, when they are stored.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "kernels.hpp"
#include "seq.hpp"

namespace sig {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kScanTile;

// ---- forward
// A workgroup takes 64 neighbouring channels of one stream and group, a channel a lane; its W wavefronts share out the states, S each, so
// that loads and stores of tokens are whole lines and sums over states meet in LDS once a token.  Tiles of 16 tokens: the wavefronts
// prepare D_t and D_t x_t of the tile's tokens (LDS), all run the recurrence of their states over the tile, and each adds up and
// stores the outputs of the tokens that it prepared.  B and C of a tile lie across the 16 lanes of a row, 16 / S tokens in a
// register, and reach the products as row broadcasts of the instruction itself: no LDS, no unpacking a token.
// What bounds it: vector instructions, of which a state and token needs an exponential (3.5 ns on a SIMD) and four others (1.1 to 2.2 ns).
// 8 x 4096 x 2048 bf16, 16 states: 380 us, 2.8e12 states a second; the bytes alone would take 105 us.
template <int S_, int W_> struct Group { static constexpr int S = S_, W = W_; };

template <int I, int N, class F> __device__ __forceinline__ void unrolled(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        unrolled<I + 1, N>(f);
    }
}
// v times what lane K of each row of 16 lanes holds in r: one instruction
template <int K> __device__ __forceinline__ float times_broadcast(float r, float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(r), 0x150 + K, 0xf, 0xf, true)) * v;
}
// o[t] = sum_s r[K + S t + s] h[t][s] for four tokens t, r[k] the value of lane k of each row.  The compiler does not merge the broadcast into a
// multiply-add; s_nop keeps the two wait states between a write of r and its first use across lanes, which it does not look for in here.
#define SIG_FMAC(o, h, k) "v_fmac_f32_dpp %" #o ", %4, %" #h " row_newbcast:%" #k " row_mask:0xf bank_mask:0xf\n\t"
template <int K, int S, int s = 1> __device__ __forceinline__ void sum_broadcast(float (&o)[4], float r, const float (&h)[4][S])
{
    if constexpr (s == 1) {
        o[0] = times_broadcast<K>(r, h[0][0]), o[1] = times_broadcast<K + S>(r, h[1][0]);
        o[2] = times_broadcast<K + 2 * S>(r, h[2][0]), o[3] = times_broadcast<K + 3 * S>(r, h[3][0]);
    }
    if constexpr (s < S) {
        asm("s_nop 1\n\t" SIG_FMAC(0, 5, 9) SIG_FMAC(1, 6, 10) SIG_FMAC(2, 7, 11) SIG_FMAC(3, 8, 12)
            : "+&v"(o[0]), "+&v"(o[1]), "+&v"(o[2]), "+&v"(o[3])
            : "v"(r), "v"(h[0][s]), "v"(h[1][s]), "v"(h[2][s]), "v"(h[3][s]), "n"(K + s), "n"(K + S + s), "n"(K + 2 * S + s), "n"(K + 3 * S + s));
        sum_broadcast<K, S, s + 1>(o, r, h);
    }
}
#undef SIG_FMAC

// Loads and stores at a lane's byte offset from a row that is the same for the wavefront, and an offset between rows in bytes; an offset
// of kNowhere, or one past a buffer's bytes, makes a load give zero and a store do nothing: tokens that are not there need no branches around them.
using Buffer = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Buffer buffer_at(const void* p, unsigned bytes = 0xfffffff0u) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00020000); }
template <class T> __device__ __forceinline__ T buffer_load(Buffer r, unsigned at, unsigned row)
{
    T v;
    if constexpr (sizeof(T) == 2) {
        uint16_t q = __builtin_amdgcn_raw_buffer_load_b16(r, at, row, 0);
        __builtin_memcpy(&v, &q, 2);
    } else {
        uint32_t q = __builtin_amdgcn_raw_buffer_load_b32(r, at, row, 0);
        __builtin_memcpy(&v, &q, 4);
    }
    return v;
}
template <class T> __device__ __forceinline__ void buffer_store(Buffer r, unsigned at, unsigned row, T v)
{
    if constexpr (sizeof(T) == 2) {
        uint16_t q;
        __builtin_memcpy(&q, &v, 2);
        __builtin_amdgcn_raw_buffer_store_b16(q, r, at, row, 0);
    } else {
        uint32_t q;
        __builtin_memcpy(&q, &v, 4);
        __builtin_amdgcn_raw_buffer_store_b32(q, r, at, row, 0);
    }
}
// p some bytes on (32 bits: a tile's rows, see the limits of strides in api_seq.cpp; scalar registers are few)
template <class T> __device__ __forceinline__ void forth(T*& p, unsigned bytes) { p = (T*)((const char*)p + bytes); }
// Keeps a row pointer in its own two scalar registers from tile to tile: the compiler otherwise makes it the sum of a start and an offset shared with
// others, more values than there are registers, and moves them to and from vector registers.  The backward pass of 16 states takes an eighth
// less with it (a hundred other scalars are still moved); that of more than 16 spills more vector registers then, and the forward pass
// loses (large case 380 -> 403 us).
template <class T> __device__ __forceinline__ void held(T*& p) { asm volatile("" : "+s"(p)); }
constexpr unsigned kNowhere = 0xfffffffcu;
// v, an infinity as the largest number of its sign.  A log2(e) and a chunk's sum of step sizes are infinite where A and the steps need not be, and both
// are multiplied with zeros: steps of tokens that do not count, rates of states that are there to fill a register.
__device__ __forceinline__ float bounded(float v) { return fabsf(v) > 3.4028235e38f ? copysignf(3.4028235e38f, v) : v; }
// at, or kNowhere: a selection that the compiler does not turn into branches around two accesses (worth 1 % of the backward pass)
__device__ __forceinline__ unsigned offset_if(bool there, unsigned at)
{
    unsigned r = there ? at : kNowhere;
    asm("" : "+v"(r));
    return r;
}
// v where mask is all ones, 0 or `other` where it is zero; the masks are the same for the wavefront
__device__ __forceinline__ float only_if(uint32_t mask, float v) { return __uint_as_float(__float_as_uint(v) & mask); }
__device__ __forceinline__ float either(uint32_t mask, float v, float other) { return __uint_as_float((__float_as_uint(v) & mask) | (__float_as_uint(other) & ~mask)); }

// The workgroups of a launch: 64 channels of a group of one stream, one time chunk.
struct Blocks {
    int64_t per_group;   // channels of a group
    unsigned runs;       // workgroups for the channels of a group
    unsigned chunks;
    int chunk;           // tokens of a time chunk, a multiple of kTile
    int64_t total;
};

// Time chunks: where a launch has few workgroups, a first kernel runs every chunk from a state of zero and leaves its last state and the sum
// of its step sizes; exp(A sum D) is the chunk's decay, so the state before any chunk is a short recurrence over the chunks before it.
struct ChunkStates {
    float* last;         // [B, chunks, N, D]
    float* steps;        // [B, chunks, D]
};
// h over the chunks from `from` to `to` (without it, in either direction): h = exp2(A2 steps) h + last, eight chunks' loads under way at a
// time.  last, steps: the lane's channel and the wavefront's first state in the stream's first chunk; n: states there are.
// Where states grow, a chunk's factor may pass float32's range although h is zero or so small that the product does not.  What comes of it
// is no finite number any more, so all is done again then, the factor's exponent split into one of at most 127 and a power of two.
template <int S> __device__ __forceinline__ void join_chunks(float (&h)[S], const float (&A2)[S], int from, int to, const float* last, const float* steps, int64_t N, int64_t D, int n)
{
    constexpr int U = 8;
    const int way = to >= from ? 1 : -1, count = (to - from) * way;
    float first[S];
#pragma unroll
    for (int s = 0; s < S; s++) first[s] = h[s];
    for (int j0 = 0; j0 < count; j0 += U) {
        float sum[U], l[U][S];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const bool there = j0 + u < count;
            const int64_t row = there ? from + way * (j0 + u) : from;
            sum[u] = there ? steps[row * D] : 0.0f;
#pragma unroll
            for (int s = 0; s < S; s++) l[u][s] = there && s < n ? last[(row * N + s) * D] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int s = 0; s < S; s++) h[s] = fmaf(__builtin_amdgcn_exp2f(A2[s] * sum[u]), h[s], l[u][s]);
    }
    bool finite = true;
#pragma unroll
    for (int s = 0; s < S; s++) finite = finite && fabsf(h[s]) <= 3.4028235e38f;
    if (finite) return;
#pragma unroll
    for (int s = 0; s < S; s++) h[s] = first[s];
#pragma unroll 1
    for (int j = 0; j < count; j++) {
        const int64_t row = from + way * j;
#pragma unroll
        for (int s = 0; s < S; s++) {
            const float x = A2[s] * steps[row * D];
            const int k = x > 127.0f ? (int)fminf(x, 1000.0f) - 126 : 0;
            h[s] = fmaf(__builtin_amdgcn_exp2f(x > 1000.0f ? 127.0f : x - (float)k), __builtin_amdgcn_ldexpf(h[s], k), s < n ? last[(row * N + s) * D] : 0.0f);
        }
    }
}

// kOutputs = false: a time chunk's last state from zero and its sum of step sizes alone.  kStates: the states before every tile go to the checkpoint.
template <class T, class Gr, bool kOutputs, bool kStates>
__global__ __launch_bounds__(Gr::W * 64, Gr::S == 4 ? 4 : 2) void scan_fwd_kernel(sig_scan_args a, Blocks bl, ChunkStates cs, T* y, float* final_state, float* checkpoint)
{
    constexpr int S = Gr::S, W = Gr::W, PT = kTile / W, RT = 16 / S, KB = kTile / RT;
    extern __shared__ float lds[];
    // D_t and D_t x_t of two tokens for each lane, and the wavefronts' sums of four (where there are outputs), each twice
    float4(*steps)[64] = (float4(*)[64])lds;                                             // [2][kTile / 2][64]
    float4(*sums)[kTile / 4][64] = (float4(*)[kTile / 4][64])(lds + 4 * kTile * 64);     // [2][W][kTile / 4][64]
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned c = blockIdx.x % bl.chunks, rest = blockIdx.x / bl.chunks, run = rest % bl.runs, bg = rest / bl.runs;
    if (!kOutputs && c + 1 == bl.chunks) return;          // nothing comes after the last chunk's state
    const int64_t g = bg % (unsigned)a.G, b = bg / (unsigned)a.G;
    const int64_t d0 = g * bl.per_group + run * 64;       // the workgroup's first channel
    const bool on = run * 64 + lane < bl.per_group;
    const unsigned e = on ? lane : 0;                     // lanes without a channel read the first one's and store nothing
    const int64_t d = d0 + e;
    const int len = (int)live_length(a.lengths, b, a.L), t_first = (int)c * bl.chunk, t_end = min(t_first + bl.chunk, (int)a.L);
    int left = min(t_end, len) - t_first;                 // tokens from the tile's first to the last of the chunk that counts
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
    const uint32_t soft = a.softplus ? ~0u : 0u, gated = a.gate ? ~0u : 0u;
    const int n0 = w * S;                                 // first state of the wavefront
    float A[S], h[S];
#pragma unroll
    for (int s = 0; s < S; s++) {
        A[s] = n0 + s < a.N ? bounded(a.A[d * a.N + n0 + s] * kLog2e) : 0.0f;
        h[s] = kOutputs && a.initial_state && n0 + s < a.N ? a.initial_state[(b * a.D + d) * a.N + n0 + s] : 0.0f;
    }
    if constexpr (kOutputs) {
        const int before = len > 0 ? min((int)c, (len - 1) / bl.chunk + 1) : 0;          // chunks with tokens before this one
        join_chunks(h, A, 0, before, cs.last + (b * bl.chunks * a.N + n0) * a.D + d, cs.steps + b * bl.chunks * a.D + d, a.N, a.D, (int)a.N - n0);
    }
    // rows of the wavefront's first token of the chunk, and of its first token's B and C
    const int64_t t1 = t_first + w * PT;
    const T *px = (const T*)a.x + b * a.x_stride_b + t1 * a.x_stride_t + d0, *pdt = (const T*)a.dt + b * a.dt_stride_b + t1 * a.dt_stride_t + d0;
    const T *pz = a.gate ? (const T*)a.gate + b * a.gate_stride_b + t1 * a.gate_stride_t + d0 : px;
    const T *pb = (const T*)a.b + b * a.b_stride_b + g * a.b_stride_g + t_first * a.b_stride_t + n0;
    const T *pc = (const T*)a.c + b * a.c_stride_b + g * a.c_stride_g + t_first * a.c_stride_t + n0;
    T* py = kOutputs ? y + (b * a.L + t1) * a.D + d0 : nullptr;
    float* pk = kStates ? checkpoint + ((b * ((a.L + kTile - 1) / kTile) + t_first / kTile) * a.N + n0) * a.D + d0 : nullptr;
    constexpr unsigned E = sizeof(T);
    const unsigned x_row = (unsigned)a.x_stride_t * E, dt_row = (unsigned)a.dt_stride_t * E, z_row = gated ? (unsigned)a.gate_stride_t * E : x_row;
    const unsigned y_row = (unsigned)a.D * E;
    // Where the lane's state and tokens of B and C lie in a tile.  The buffers end with the row of the last token that counts (rows do not overlap, or
    // are all the same): no selection a lane, which the compiler makes branches of.  A tile is one block of instructions then, with or without
    // states to keep (kStates): 7 % less time in the large case, 13 % less with states.
    unsigned b_at[KB], c_at[KB];
#pragma unroll
    for (int j = 0; j < KB; j++) {
        const int k = j * RT + lane % 16 / S;
        b_at[j] = n0 + lane % S < a.N ? (unsigned)(k * a.b_stride_t + lane % S) * E : kNowhere;
        c_at[j] = n0 + lane % S < a.N ? (unsigned)(k * a.c_stride_t + lane % S) * E : kNowhere;
    }
    const unsigned b_step = (unsigned)a.b_stride_t * E, c_step = (unsigned)a.c_stride_t * E, n_bytes = (unsigned)max(0, (int)a.N - n0) * E;
    unsigned k_at[S];
#pragma unroll
    for (int s = 0; s < S; s++) k_at[s] = n0 + s < a.N ? e * 4 : kNowhere;

    T x[PT], dt[PT], z[PT], bv[KB], cv[KB];
    float f[PT], keep[PT], f_next[PT], keep_next[PT], o[PT], B[KB], C[KB], total = 0.0f;
    // reads the tile at the row pointers, n tokens of it; the pointers go on to the next
    auto fetch = [&](int n) {
        const unsigned before = n < kTile ? n - 1 : kTile - 1;
        Buffer rx = buffer_at(px), rdt = buffer_at(pdt), rz = buffer_at(pz);
        Buffer rb = buffer_at(pb, __builtin_amdgcn_readfirstlane(n > 0 ? before * b_step + n_bytes : 0)), rc = buffer_at(pc, __builtin_amdgcn_readfirstlane(n > 0 ? before * c_step + n_bytes : 0));
#pragma unroll
        for (int i = 0; i < PT; i++) {
            unsigned at = w * PT + i < n ? e * E : kNowhere;
            x[i] = buffer_load<T>(rx, at, i * x_row);
            dt[i] = buffer_load<T>(rdt, at, i * dt_row);
            if (kOutputs) z[i] = buffer_load<T>(rz, at, i * z_row);
        }
#pragma unroll
        for (int j = 0; j < KB; j++) {
            bv[j] = buffer_load<T>(rb, b_at[j], 0);
            if (kOutputs) cv[j] = buffer_load<T>(rc, c_at[j], 0);
        }
        forth(px, kTile * x_row), forth(pdt, kTile * dt_row), forth(pz, kTile * z_row), forth(pb, kTile * b_step), forth(pc, kTile * c_step);
    };
    // D_t and D_t x_t of the wavefront's tokens of a tile with n tokens (zero beyond: states stay), and what its outputs need besides
    auto prepare = [&](float4 (*to)[64], int n, const float (&xf)[PT], const float (&df)[PT], const float (&zf)[PT]) {
        float2 step[PT];
#pragma unroll
        for (int i = 0; i < PT; i++) {
            float D = df[i] + bias;
            D = only_if(w * PT + i < n ? ~0u : 0u, either(soft, softplus(D), D));
            step[i] = make_float2(D, D * xf[i]);
            if (kOutputs) {
                keep_next[i] = skip * xf[i];
                f_next[i] = either(gated, zf[i] * sigmoid(zf[i]), 1.0f);
            }
        }
        if constexpr (PT == 1) {
            ((float2*)&to[w / 2][lane])[w % 2] = step[0];
        } else {
#pragma unroll
            for (int i = 0; i < PT; i += 2) to[(w * PT + i) / 2][lane] = make_float4(step[i].x, step[i].y, step[i + 1].x, step[i + 1].y);
        }
    };
    auto collect = [&](const float4 (*from)[kTile / 4][64]) {
        constexpr int P = PT < 4 ? PT : 4;                // tokens of an access
#pragma unroll
        for (int i = 0; i < PT; i += P) {
#pragma unroll
            for (int j = 0; j < P; j++) o[i + j] = keep[i + j];
#pragma unroll
            for (int v = 0; v < W; v++) {
                const Pack<float, P> q = *(const Pack<float, P>*)((const float*)&from[v][(w * PT + i) / 4][lane] + (w * PT + i) % 4);
#pragma unroll
                for (int j = 0; j < P; j++) o[i + j] += q.v[j];
            }
#pragma unroll
            for (int j = 0; j < P; j++) o[i + j] *= f[i + j];
        }
    };
    // Three tiles are in work at a time: while one runs, the step sizes of the next are prepared and the outputs of the one before are
    // added up, so that no wavefront waits for the latencies of either; one barrier a tile.
    float xf[PT], df[PT], zf[PT];
    fetch(left);
#pragma unroll
    for (int i = 0; i < PT; i++) xf[i] = to_float(x[i]), df[i] = to_float(dt[i]), zf[i] = kOutputs ? to_float(z[i]) : 0.0f;
    prepare(steps, left, xf, df, zf);
#pragma unroll
    for (int j = 0; j < KB; j++) B[j] = to_float(bv[j]), C[j] = kOutputs ? to_float(cv[j]) : 0.0f;
    fetch(left - kTile);
    __syncthreads();
    bool stores = false;                   // no outputs to store in the first turn
    auto tile = [&](auto parity) {         // which half of LDS: a constant, so that the compiler sees that reads and writes do not meet
        constexpr int turn = decltype(parity)::value;
        float4(*now)[64] = steps + turn * kTile / 2, (*next)[64] = steps + (turn ^ 1) * kTile / 2;
        float4(*sums_now)[kTile / 4][64] = sums + turn * W, (*sums_before)[kTile / 4][64] = sums + (turn ^ 1) * W;
        float b_next[KB], c_next[KB];
#pragma unroll
        for (int i = 0; i < PT; i++) xf[i] = to_float(x[i]), df[i] = to_float(dt[i]), zf[i] = kOutputs ? to_float(z[i]) : 0.0f;
#pragma unroll
        for (int j = 0; j < KB; j++) b_next[j] = to_float(bv[j]), c_next[j] = kOutputs ? to_float(cv[j]) : 0.0f;
        fetch(left - 2 * kTile);
        if (kStates) {
#pragma unroll
            for (int s = 0; s < S; s++) buffer_store(buffer_at(pk), k_at[s], (unsigned)(s * a.D) * 4, h[s]);
            pk += a.N * a.D;
        }
        if (kOutputs) {
            collect(sums_before);
#pragma unroll
            for (int i = 0; i < PT; i++) f[i] = f_next[i], keep[i] = keep_next[i];
        }
        prepare(next, left - kTile, xf, df, zf);
        unrolled<0, kTile / 4>([&](auto jt) {
            constexpr int i = decltype(jt)::value * 4, k = i % RT * S;
            float4 p = now[i / 2][lane], q = now[i / 2 + 1][lane];
            const float D[4] = {p.x, p.z, q.x, q.z}, u[4] = {p.y, p.w, q.y, q.w};
            float decay[4][S], ht[4][S];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (!kOutputs) total += D[j];
#pragma unroll
                for (int s = 0; s < S; s++) decay[j][s] = __builtin_amdgcn_exp2f(D[j] * A[s]);
            }
            unrolled<0, 4>([&](auto it) {
                constexpr int j = decltype(it)::value;
                unrolled<0, S>([&](auto is) {
                    constexpr int s = decltype(is)::value;
                    ht[j][s] = h[s] = fmaf(decay[j][s], h[s], times_broadcast<k + j * S + s>(B[i / RT], u[j]));
                });
            });
            if constexpr (kOutputs) {
                float y4[4];
                sum_broadcast<k>(y4, C[i / RT], ht);
                sums_now[w][i / 4][lane] = make_float4(y4[0], y4[1], y4[2], y4[3]);
            }
        });
        if (kOutputs) {                    // lanes without a channel repeat the first one's outputs
#pragma unroll
            for (int i = 0; i < PT; i++) buffer_store(buffer_at(py), stores ? e * E : kNowhere, i * y_row, from_float<T>(o[i]));
            py += stores ? kTile * a.D : 0;
            stores = true;
        }
#pragma unroll
        for (int j = 0; j < KB; j++) B[j] = b_next[j], C[j] = c_next[j];
        left -= kTile;
        __syncthreads();
    };
    unsigned turn = 0;
    while (left > 0) {
        tile(std::integral_constant<int, 0>());
        turn = 1;
        if (left <= 0) break;
        tile(std::integral_constant<int, 1>());
        turn = 0;
    }
    int room = t_end - t_first;            // tokens of the chunk from the first whose output is not stored yet
    if constexpr (kOutputs) {
        if (len > t_first) {               // the last tile, of left + kTile tokens
            room -= (min(t_end, len) - t_first - 1) / kTile * kTile;
            collect(sums + (turn ^ 1) * W);
#pragma unroll
            for (int i = 0; i < PT; i++)
                buffer_store(buffer_at(py), w * PT + i < room ? e * E : kNowhere, i * y_row, from_float<T>(w * PT + i < left + kTile ? o[i] : 0.0f));
            py += kTile * a.D, room -= kTile;
        }
        for (py -= w * (PT - 1) * a.D; room > 0; room -= W, py += W * a.D)
            if (w < room) py[e] = from_float<T>(0.0f);
        if (final_state && (int)c == (len > 0 ? (len - 1) / bl.chunk : 0))
#pragma unroll
            for (int s = 0; s < S; s++)
                if (n0 + s < a.N) final_state[(b * a.D + d) * a.N + n0 + s] = h[s];
    } else {
#pragma unroll
        for (int s = 0; s < S; s++)
            if (n0 + s < a.N) (cs.last + ((b * bl.chunks + c) * a.N + n0 + s) * a.D + d0)[e] = h[s];
        if (w == 0) cs.steps[(b * bl.chunks + c) * a.D + d] = bounded(total);
    }
}

// ---- backward
// The same workgroups, tiles from the last to the first.  The states of a tile are computed again from the checkpoint before it and stay in
// registers with their decays (with four states a wavefront the decays are computed twice instead: the registers hold one of the two);
// the adjoint states walk back over them.  Three sums over states a token (for dx, dD and, for the gate, y) meet in LDS by half tiles, two
// barriers a tile.  dB and dC are sums over channels, that is over lanes: a reduction that halves the number of values at each of its
// six steps leaves the 64 sums of 16 tokens (2 states, dB and dC) one to a lane in 129 instructions, where a sum to all lanes would take six for
// each; the workgroups' sums are added by a second kernel in their order, no atomics.
// What bounds it: vector instructions, 24 a state and token (two exponentials with four states a wavefront, else one), on SIMDs that are busy
// 76 % of the time with two wavefronts each.  8 x 2048 x 2048 bf16, 16 states: 491 us, 1.1e12 states a second; the bytes (seven tensors of
// tokens, the checkpoint, the workgroups' sums, 0.67 GB) alone 131 us.  More than 32 states: 260 of the registers that a lane wants go to
// memory, 5.5 ms where 32 states take 0.95.
template <int K, int S> __device__ __forceinline__ void add_broadcast(float (&o)[S], float r, float v)      // o[s] += r[K + s] v
{
    static_assert(S == 2 || S == 4, "states of a wavefront");
    if constexpr (S == 2)
        asm("s_nop 1\n\tv_fmac_f32_dpp %0, %2, %3 row_newbcast:%4 row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %1, %2, %3 row_newbcast:%5 row_mask:0xf bank_mask:0xf"
            : "+&v"(o[0]), "+&v"(o[1]) : "v"(r), "v"(v), "n"(K), "n"(K + 1));
    else
        asm("s_nop 1\n\tv_fmac_f32_dpp %0, %4, %5 row_newbcast:%6 row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %1, %4, %5 row_newbcast:%7 row_mask:0xf bank_mask:0xf\n\t"
            "v_fmac_f32_dpp %2, %4, %5 row_newbcast:%8 row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %3, %4, %5 row_newbcast:%9 row_mask:0xf bank_mask:0xf"
            : "+&v"(o[0]), "+&v"(o[1]), "+&v"(o[2]), "+&v"(o[3]) : "v"(r), "v"(v), "n"(K), "n"(K + 1), "n"(K + 2), "n"(K + 3));
}
// Steps of the reduction over lanes: from a and b one register that holds, where the lane's bit is clear, a's sum over the two lanes that
// differ in that bit, and b's where it is set.
__device__ __forceinline__ float fold5(float a, float b)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold4(float a, float b)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold3(float a, float b)       // banks of four lanes: 0, 1 take a, 2, 3 take b
{
    float r;
    asm("s_nop 1\n\tv_add_f32_dpp %0, %1, %1 row_ror:8 row_mask:0xf bank_mask:0x3\n\tv_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xc" : "=&v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float fold2(float a, float b)       // 0, 2 take a, 1, 3 take b
{
    float r;
    asm("s_nop 1\n\tv_add_f32_dpp %0, %1, %1 row_ror:12 row_mask:0xf bank_mask:0x5\n\tv_add_f32_dpp %0, %2, %2 row_ror:4 row_mask:0xf bank_mask:0xa" : "=&v"(r) : "v"(a), "v"(b));
    return r;
}
template <int Bit> __device__ __forceinline__ float fold_quad(float a, float b, int lane)      // bits 1 and 0, within four lanes
{
    float keep = lane & (1 << Bit) ? b : a, send = lane & (1 << Bit) ? a : b;
    return keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), Bit ? 0x4e : 0xb1, 0xf, 0xf, true));
}
// the token of a tile whose sums a lane has in the end: its four lower bits, reversed
__device__ __forceinline__ int token_of(int lane) { return (lane & 1) << 3 | (lane & 2) << 1 | (lane & 4) >> 1 | (lane & 8) >> 3; }

// float32 arrays of a backward launch
struct Parts {
    float* bc;           // [B, tiles, G, runs, W, S / 2, 64] sums of a workgroup's channels
    float* A;            // [B, chunks, N, D]
    float* rest;         // [B, chunks, 2, D] dskip, ddt_bias
};

// kFull = false: the adjoint states of a time chunk alone, from zero at its end (see ChunkStates).
template <class T, class Gr, bool kFull>
__global__ __launch_bounds__(Gr::W * 64, Gr::W > 8 ? 4 : 2) void scan_bwd_kernel(sig_scan_args a, sig_scan_grads g, Blocks bl, ChunkStates cs, const float* checkpoint, Parts parts)
{
    constexpr int S = Gr::S, W = Gr::W, PT = kTile / W, PH = PT > 1 ? PT / 2 : 1, RT = 16 / S, KB = kTile / RT, kHalf = kTile / 2, Q = S / 2;
    constexpr bool kDecays = S == 2, kHeld = S == 2, kTwice = W <= 8;      // decays stay in registers; row pointers are held; the sums' LDS is there for either half of a tile
    constexpr unsigned E = sizeof(T);
    extern __shared__ float lds[];
    float4(*in)[kTile / 4][64] = (float4(*)[kTile / 4][64])lds;                                          // [2][3: D, D x, dL/ds][kTile / 4][64]
    float(*sums)[3][kHalf][64] = (float(*)[3][kHalf][64])(lds + 2 * 3 * kTile * 64);                     // [2 or 1][W][3][kHalf][64]
    // dA of the tiles before, each lane's own: registers hold a tile's sum, as thousands of tokens one by one cost half a digit (1.0e-6 off, 0.57e-6 so)
    Pack<float, S>* gA_before = (Pack<float, S>*)(lds + 2 * 3 * kTile * 64 + (kTwice ? 2 : 1) * W * 3 * kHalf * 64) + threadIdx.x;
    if (kFull) *gA_before = {};
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned c = blockIdx.x % bl.chunks, rest = blockIdx.x / bl.chunks, run = rest % bl.runs, bg = rest / bl.runs;
    if (!kFull && c == 0) return;                          // nothing comes before the first chunk's adjoint state
    const int64_t grp = bg % (unsigned)a.G, b = bg / (unsigned)a.G;
    const int64_t d0 = grp * bl.per_group + run * 64;
    const bool on = run * 64 + lane < bl.per_group;
    const unsigned e = on ? lane : 0;                      // lanes without a channel read the first one's, add nothing and store nothing
    const int64_t d = d0 + e;
    const int len = (int)live_length(a.lengths, b, a.L), t_first = (int)c * bl.chunk, t_end = min(t_first + bl.chunk, (int)a.L), live = min(t_end, len) - t_first;
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
    const uint32_t soft = a.softplus ? ~0u : 0u, gated = a.gate ? ~0u : 0u;
    const int n0 = w * S;
    const int64_t tiles = (a.L + kTile - 1) / kTile;
    float A[S], A2[S], adj[S], gA[S] = {}, gskip = 0.0f, gbias = 0.0f, total = 0.0f;       // adj: a_{t+1} l_{t+1}
#pragma unroll
    for (int s = 0; s < S; s++) {
        A[s] = n0 + s < a.N ? a.A[d * a.N + n0 + s] : 0.0f;
        A2[s] = bounded(A[s] * kLog2e);
        adj[s] = kFull && g.grad_final_state && n0 + s < a.N ? g.grad_final_state[(b * a.D + d) * a.N + n0 + s] : 0.0f;
    }
    if constexpr (kFull) {
        const int after = len > 0 ? (len - 1) / bl.chunk : 0;      // the last chunk with tokens
        if (after > (int)c)
            join_chunks(adj, A2, after, (int)c, cs.last + (b * bl.chunks * a.N + n0) * a.D + d, cs.steps + b * bl.chunks * a.D + d, a.N, a.D, (int)a.N - n0);
    }
    // tiles with tokens that count, and the tokens of the last one: none for a chunk beyond the stream's length
    const int n_tiles = live > 0 ? (live + kTile - 1) / kTile : 0, n_last = n_tiles > 0 ? live - (n_tiles - 1) * kTile : 0;
    // rows of the last tile's first token; they go back a tile at a time
    const int64_t t1 = t_first + (int64_t)(n_tiles - 1) * kTile;
    const int64_t own1 = t1 + w * PH;                      // the wavefront's first token of it
    const T *px = (const T*)a.x + b * a.x_stride_b + own1 * a.x_stride_t + d0, *pdt = (const T*)a.dt + b * a.dt_stride_b + own1 * a.dt_stride_t + d0;
    const T *pz = a.gate ? (const T*)a.gate + b * a.gate_stride_b + own1 * a.gate_stride_t + d0 : px, *pg = (const T*)g.grad_y + b * g.gy_stride_b + own1 * g.gy_stride_t + d0;
    const T *pb = (const T*)a.b + b * a.b_stride_b + grp * a.b_stride_g + t1 * a.b_stride_t + n0, *pc = (const T*)a.c + b * a.c_stride_b + grp * a.c_stride_g + t1 * a.c_stride_t + n0;
    const float* ph = kFull ? checkpoint + ((b * tiles + t1 / kTile) * a.N + n0) * a.D + d0 : nullptr;
    const int64_t out = (b * a.L + own1 + kTile) * a.D + d0;       // one tile on: every turn begins with the lower half of the tile before
    T *qx = (T*)g.grad_x + out, *qdt = (T*)g.grad_dt + out, *qz = (T*)g.grad_gate + out;
    const unsigned x_row = (unsigned)a.x_stride_t * E, dt_row = (unsigned)a.dt_stride_t * E, z_row = gated ? (unsigned)a.gate_stride_t * E : x_row, g_row = (unsigned)g.gy_stride_t * E;
    const unsigned y_row = (unsigned)a.D * E, b_step = (unsigned)a.b_stride_t * E, c_step = (unsigned)a.c_stride_t * E;
    unsigned b_at[KB], c_at[KB];                            // as in the forward kernel
#pragma unroll
    for (int j = 0; j < KB; j++) {
        const int k = j * RT + lane % 16 / S;
        b_at[j] = n0 + lane % S < a.N ? (unsigned)(k * a.b_stride_t + lane % S) * E : kNowhere;
        c_at[j] = n0 + lane % S < a.N ? (unsigned)(k * a.c_stride_t + lane % S) * E : kNowhere;
    }
    const unsigned n_bytes = (unsigned)max(0, (int)a.N - n0) * E;
    auto from_own = [&](int half, int i) { return PT > 1 ? half * kHalf + i : 0; };        // the tokens that the wavefront prepares and stores, from its first
    auto own = [&](int half, int i) { return w * PH + from_own(half, i); };

    T x[PT], dt[PT], z[PT], up[PT], bv[KB], cv[KB];
    float hv[S];
    auto fetch = [&](int n) {              // the tile at the row pointers, n tokens of it
        Buffer rx = buffer_at(px), rdt = buffer_at(pdt), rz = buffer_at(pz), rg = buffer_at(pg), rh = buffer_at(ph);
        Buffer rb = buffer_at(pb, __builtin_amdgcn_readfirstlane(n > 0 ? (n - 1) * b_step + n_bytes : 0)), rc = buffer_at(pc, __builtin_amdgcn_readfirstlane(n > 0 ? (n - 1) * c_step + n_bytes : 0));
#pragma unroll
        for (int i = 0; i < PT; i++) {
            const int k = from_own(i / PH, i % PH);
            unsigned at = w * PH + k < n ? e * E : kNowhere;
            if (kFull) x[i] = buffer_load<T>(rx, at, k * x_row);
            dt[i] = buffer_load<T>(rdt, at, k * dt_row);
            z[i] = buffer_load<T>(rz, at, k * z_row);
            up[i] = buffer_load<T>(rg, at, k * g_row);
        }
#pragma unroll
        for (int j = 0; j < KB; j++) {
            if (kFull) bv[j] = buffer_load<T>(rb, b_at[j], 0);
            cv[j] = buffer_load<T>(rc, c_at[j], 0);
        }
        if (kFull)
#pragma unroll
            for (int s = 0; s < S; s++) hv[s] = buffer_load<float>(rh, n > 0 && n0 + s < a.N ? e * 4 : kNowhere, (unsigned)(s * a.D) * 4);
        px -= kTile * a.x_stride_t, pdt -= kTile * a.dt_stride_t, pz -= kTile * (gated ? a.gate_stride_t : a.x_stride_t), pg -= kTile * g.gy_stride_t;
        pb -= kTile * a.b_stride_t, pc -= kTile * a.c_stride_t, ph -= a.N * a.D;
        if constexpr (kHeld) held(px), held(pdt), held(pz), held(pg), held(pb), held(pc), held(ph);
    };
    // of each of the wavefront's tokens: x, D, dL/ds, dD/d(dt + bias), dL/dy times the gate's slope; of the tile at work and the one after it
    float xs[2][PT], Ds[2][PT], us[2][PT], sl[2][PT], gs[2][PT];
    int counts[2] = {0, 0}, rooms[2] = {0, 0};             // tokens of the tile that count, and that the chunk has
    auto prepare = [&](int slot, float4 (*to)[kTile / 4][64], int n, int room) {
        counts[slot] = n, rooms[slot] = room;
#pragma unroll
        for (int i = 0; i < PT; i++) {
            int k = own(i / PH, i % PH);
            uint32_t there = k < n ? ~0u : 0u;
            float raw = to_float(dt[i]) + bias, zf = to_float(z[i]), gy = to_float(up[i]), p = sigmoid(zf), v = kFull ? to_float(x[i]) : 0.0f;
            float D = only_if(there, either(soft, softplus(raw), raw)), u = gy * either(gated, zf * p, 1.0f);
            xs[slot][i] = v, Ds[slot][i] = D, us[slot][i] = u;
            sl[slot][i] = either(soft, sigmoid(raw), 1.0f);
            gs[slot][i] = gy * p * fmaf(zf, 1.0f - p, 1.0f);
            ((float*)&to[0][k / 4][lane])[k % 4] = D;
            if (kFull) ((float*)&to[1][k / 4][lane])[k % 4] = on ? D * v : 0.0f;
            ((float*)&to[2][k / 4][lane])[k % 4] = !kFull || on ? u : 0.0f;
        }
    };
    // the gradients of a half's tokens; from: the wavefronts' sums
    auto put = [&](int half, int slot, const float (*from)[3][kHalf][64]) {
        const int n = counts[slot], room = rooms[slot];
        Buffer rx = buffer_at(qx), rdt = buffer_at(qdt), rz = buffer_at(qz);
#pragma unroll
        for (int i = 0; i < PH; i++) {
            if (PT == 1 && w / kHalf != half) continue;
            const int k = own(half, i), kh = k % kHalf, m = PT > 1 ? half * PH + i : 0;
            float r[3] = {0.0f, 0.0f, skip * xs[slot][m]};
#pragma unroll
            for (int v = 0; v < W; v++)
#pragma unroll
                for (int q = 0; q < 3; q++) r[q] += from[v][q][kh][lane];
            const bool there = k < n;
            const float D = Ds[slot][m], u = us[slot][m], v = xs[slot][m];
            float dx = there ? fmaf(r[0], D, skip * u) : 0.0f, dD = there ? fmaf(r[0], v, r[1]) * sl[slot][m] : 0.0f, dz = there ? gs[slot][m] * r[2] : 0.0f;
            gskip += there ? u * v : 0.0f;
            gbias += dD;
            const unsigned at = offset_if(on && k < room, e * E);
            const unsigned row = from_own(half, i) * y_row;
            buffer_store(rx, at, row, from_float<T>(dx));
            buffer_store(rdt, at, row, from_float<T>(dD));
            buffer_store(rz, gated ? at : kNowhere, row, from_float<T>(dz));
        }
    };
    fetch(n_last);
    float B[KB], C[KB], h0[S];
    auto take = [&](float (&Bn)[KB], float (&Cn)[KB], float (&hn)[S]) {
#pragma unroll
        for (int j = 0; j < KB; j++) Bn[j] = kFull ? to_float(bv[j]) : 0.0f, Cn[j] = to_float(cv[j]);
#pragma unroll
        for (int s = 0; s < S; s++) hn[s] = kFull ? hv[s] : 0.0f;
    };
    take(B, C, h0);
    prepare(0, in, n_last, t_end - t_first - (n_tiles - 1) * kTile);
    fetch(n_tiles > 1 ? kTile : 0);
    __syncthreads();
    int tile = n_tiles - 1;
    // sums of the tile at work
    const int64_t bc_step = a.G * bl.runs * (W * Q * 64);
    float* bc = parts.bc + ((b * tiles + t_first / kTile + tile) * bc_step + ((grp * bl.runs + run) * W + w) * (Q * 64));
    auto work = [&](auto parity) {
        constexpr int slot = decltype(parity)::value;
        const float4(*now)[kTile / 4][64] = in + slot * 3;
        float(*upper)[3][kHalf][64] = sums, (*lower)[3][kHalf][64] = sums + (kTwice ? W : 0);
        float Bn[KB], Cn[KB], hn[S], group[4][Q];
        take(Bn, Cn, hn);
        if (kFull) {                       // what is left of the tile before (in the first turn nothing, whatever LDS holds)
            put(0, slot ^ 1, lower);
            qx -= kTile * a.D, qdt -= kTile * a.D, qz -= kTile * a.D;
            if constexpr (kHeld) held(qx), held(qdt), held(qz);
            if (!kTwice) __syncthreads();
        }
        prepare(slot ^ 1, in + (slot ^ 1) * 3, tile > 0 ? kTile : 0, kTile);
        fetch(tile > 1 ? kTile : 0);
        // D[t], D[t] x[t] and dL/ds[t] of four tokens from LDS
        auto four = [&](int q, int i, float (&v)[4]) {
            float4 r = now[q][i / 4][lane];
            v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
        };
        float h[kFull ? kTile + 1 : 1][S], decay[kDecays && kFull ? kTile : 1][S];       // h[t + 1]: after token t
        if constexpr (kFull) {
#pragma unroll
            for (int s = 0; s < S; s++) h[0][s] = h0[s];
            unrolled<0, kTile / 4>([&](auto jt) {
                constexpr int i = decltype(jt)::value * 4, k = i % RT * S;
                float D[4], u[4];
                four(0, i, D), four(1, i, u);
                unrolled<0, 4>([&](auto it) {
                    constexpr int j = decltype(it)::value;
                    unrolled<0, S>([&](auto is) {
                        constexpr int s = decltype(is)::value;
                        float f = __builtin_amdgcn_exp2f(D[j] * A2[s]);
                        if constexpr (kDecays) decay[i + j][s] = f;
                        h[i + j + 1][s] = fmaf(f, h[i + j][s], times_broadcast<k + j * S + s>(B[i / RT], u[j]));
                    });
                });
            });
        }
        auto half_back = [&](auto half_) {
            constexpr int half = decltype(half_)::value;
            unrolled<0, kHalf / 4>([&](auto jt) {
                constexpr int q = kHalf / 4 - 1 - decltype(jt)::value, i = half * kHalf + q * 4, k = i % RT * S;
                float D[4], u[4], v[4], lam[4][S], ht[4][S], dD[4] = {}, o[4], fold[4][Q];
                four(0, i, D), four(2, i, v);
                if (kFull) four(1, i, u);
                unrolled<0, 4>([&](auto it) {
                    constexpr int j = 3 - decltype(it)::value;
                    add_broadcast<k + j * S, S>(adj, C[i / RT], v[j]);
#pragma unroll
                    for (int s = 0; s < S; s++) {
                        lam[j][s] = adj[s];
                        float f;
                        if constexpr (kDecays && kFull) f = decay[i + j][s];
                        else f = __builtin_amdgcn_exp2f(D[j] * A2[s]);
                        adj[s] = lam[j][s] * f;
                        if constexpr (kFull) {
                            ht[j][s] = h[i + j + 1][s];
                            float keep = adj[s] * h[i + j][s];
                            gA[s] = fmaf(keep, D[j], gA[s]);
                            dD[j] = fmaf(keep, A[s], dD[j]);
                        }
                    }
                    if constexpr (kFull) {
#pragma unroll
                        for (int m = 0; m < Q; m++)
                            fold[j][m] = fold4(fold5(lam[j][2 * m] * u[j], v[j] * ht[j][2 * m]), fold5(lam[j][2 * m + 1] * u[j], v[j] * ht[j][2 * m + 1]));
                    } else {
                        total += D[j];
                    }
                });
                if constexpr (kFull) {
#pragma unroll
                    for (int m = 0; m < Q; m++) group[i / 4][m] = fold2(fold3(fold[0][m], fold[1][m]), fold3(fold[2][m], fold[3][m]));
                    float(*to)[3][kHalf][64] = half ? upper : lower;
                    sum_broadcast<k>(o, B[i / RT], lam);
#pragma unroll
                    for (int j = 0; j < 4; j++) to[w][0][q * 4 + j][lane] = o[j], to[w][1][q * 4 + j][lane] = dD[j];
                    sum_broadcast<k>(o, C[i / RT], ht);
#pragma unroll
                    for (int j = 0; j < 4; j++) to[w][2][q * 4 + j][lane] = o[j];
                }
            });
        };
        half_back(std::integral_constant<int, 1>());
        if constexpr (kFull) {
            __syncthreads();
            put(1, slot, upper);
            if (!kTwice) __syncthreads();
        }
        half_back(std::integral_constant<int, 0>());
        if constexpr (kFull) {
#pragma unroll
            for (int m = 0; m < Q; m++)
                (bc + m * 64)[lane] = fold_quad<0>(fold_quad<1>(group[0][m], group[1][m], lane), fold_quad<1>(group[2][m], group[3][m], lane), lane);
            bc -= bc_step;
        }
#pragma unroll
        for (int j = 0; j < KB; j++) B[j] = Bn[j], C[j] = Cn[j];
#pragma unroll
        for (int s = 0; s < S; s++) h0[s] = hn[s];
        if constexpr (kFull) {
            Pack<float, S> r = *gA_before;
#pragma unroll
            for (int s = 0; s < S; s++) r.v[s] += gA[s], gA[s] = 0.0f;
            *gA_before = r;
        }
        tile--;
        __syncthreads();
    };
    unsigned turn = 0;
    while (tile >= 0) {
        work(std::integral_constant<int, 0>());
        turn = 0;
        if (tile < 0) break;
        work(std::integral_constant<int, 1>());
        turn = 1;
    }
    if constexpr (kFull) {
        if (n_tiles > 0) {
            float(*lower)[3][kHalf][64] = sums + (kTwice ? W : 0);
            if (turn) put(0, 1, lower);
            else put(0, 0, lower);
        }
        // tokens that do not count
        T *rx = (T*)g.grad_x + (b * a.L + t_first) * a.D + d0, *rdt = (T*)g.grad_dt + (b * a.L + t_first) * a.D + d0, *rz = (T*)g.grad_gate + (b * a.L + t_first) * a.D + d0;
        for (int64_t t = n_tiles * kTile + w; t < t_end - t_first; t += W)
            if (on) {
                rx[t * a.D + e] = rdt[t * a.D + e] = from_float<T>(0.0f);
                if (gated) rz[t * a.D + e] = from_float<T>(0.0f);
            }
        __syncthreads();
        lds[(w * 2 + 0) * 64 + lane] = gskip, lds[(w * 2 + 1) * 64 + lane] = gbias;
        __syncthreads();
        if (!on) return;
        const int64_t row = b * bl.chunks + c;
#pragma unroll
        for (int s = 0; s < S; s++)
            if (n0 + s < a.N) {
                parts.A[(row * a.N + n0 + s) * a.D + d] = gA_before->v[s];
                if (g.grad_initial_state && c == 0) g.grad_initial_state[(b * a.D + d) * a.N + n0 + s] = adj[s];
            }
        if (w == 0) {
            float r[2] = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < W; v++) r[0] += lds[(v * 2 + 0) * 64 + lane], r[1] += lds[(v * 2 + 1) * 64 + lane];
            parts.rest[(row * 2 + 0) * a.D + d] = r[0];
            parts.rest[(row * 2 + 1) * a.D + d] = r[1];
        }
    } else {
        if (!on) return;
        const int64_t row = b * bl.chunks + c;
#pragma unroll
        for (int s = 0; s < S; s++)
            if (n0 + s < a.N) cs.last[(row * a.N + n0 + s) * a.D + d] = adj[s];
        if (w == 0) cs.steps[row * a.D + d] = bounded(total);
    }
}

// The sums over workgroups of a backward launch, in a fixed order; the two parts in one launch (7 x 301 x 278 in float32: 4.3 us, 4.9 and 4.0 in
// two).  Bound by memory: 8 x 2048 x 2048 in bf16 14.2 us for 70 MB, 21.7 with one load a time instead of eight.  Sixteen wavefronts a workgroup.
// Workgroups up to `params`: dA, dskip and ddt_bias, the sums over streams and time chunks.  64 sums a workgroup; each of its
// wavefronts takes every sixteenth row, so that few columns with many rows wait for memory a sixteenth as often.
// The others: dB and dC, the sums over the workgroups of a group's channels, a tile and two states a wavefront.
constexpr int kSumThreads = 1024;
template <class T, class Gr>
__global__ __launch_bounds__(kSumThreads) void scan_bwd_sums_kernel(sig_scan_args a, Blocks bl, Parts parts, int64_t rows, unsigned params, T* gB, T* gC, float* gA, float* gskip, float* gbias)
{
    const int lane = threadIdx.x & 63;
    if (blockIdx.x < params) {
        const int64_t id = (int64_t)blockIdx.x * 64 + lane, DN = a.D * a.N;
        const bool of_A = id < DN, of_rest = !of_A && id < DN + 2 * a.D;
        const float* from = of_A ? parts.A + id : parts.rest + (id - DN);
        const int64_t step = of_A ? DN : 2 * a.D;
        const float v = sum_rows(from, of_A || of_rest ? rows : 0, step);
        if (threadIdx.x >= 64) return;
        if (of_A) gA[id % a.D * a.N + id / a.D] = v;
        if (of_rest) {
            float* to = id - DN < a.D ? gskip : gbias;
            if (to) to[(id - DN) % a.D] = v;
        }
        return;
    }
    constexpr int Q = Gr::S / 2, R = Gr::W * Q, kWaves = kSumThreads / 64;
    const int64_t tiles = (a.L + kTile - 1) / kTile, all = a.B * tiles * a.G * R;
    for (int64_t id = (int64_t)(blockIdx.x - params) * kWaves + threadIdx.x / 64; id < all; id += (int64_t)(gridDim.x - params) * kWaves) {
        const int r = (int)(id % R);
        const int64_t grp = id / R % a.G, tile = id / R / a.G % tiles, b = id / R / a.G / tiles, t = tile * kTile + token_of(lane);
        const int n = r / Q * Gr::S + r % Q * 2 + (lane >> 4 & 1);
        const int64_t len = live_length(a.lengths, b, a.L);
        float v = 0.0f;
        if (tile * kTile < len) {
            const float* p = parts.bc + (((b * tiles + tile) * a.G + grp) * bl.runs * R + r) * 64 + lane;
#pragma unroll 8
            for (unsigned j = 0; j < bl.runs; j++) v += p[(int64_t)j * R * 64];
        }
        if (t < a.L && n < a.N) (lane & 32 ? gC : gB)[((b * a.L + t) * a.G + grp) * a.N + n] = from_float<T>(t < len ? v : 0.0f);
    }
}

// ---- one token
// Q lanes hold the states of a channel, S each (state n = lane * S + s; N <= Q S, the rest are zero): reads and writes of the states, which are
// nearly all there is, are contiguous over the wavefront, 16 bytes a lane where they are aligned (kWide).  Bound by memory: 64 x 2048 with 16
// states 7.4 us for 18 MB (3.5 us at a large copy's rate, a launch's own time on top), less than the call's time on the host.
template <int Q_, int S_> struct Shape { static constexpr int Q = Q_, S = S_, channels = 64 / Q_; };

template <class T, int S, bool kWide> __device__ __forceinline__ void load_states(float (&h)[S], const T* p, int n)
{
    if constexpr (kWide) {
        Pack<T, S> r = *(const Pack<T, S>*)p;
#pragma unroll
        for (int s = 0; s < S; s++) h[s] = to_float(r.v[s]);
    } else {
#pragma unroll
        for (int s = 0; s < S; s++) h[s] = s < n ? to_float(p[s]) : 0.0f;
    }
}

template <class T, class Sh, bool kWide> __global__ __launch_bounds__(kThreads) void scan_step_kernel(sig_scan_args a, float* state, T* y)
{
    constexpr int S = Sh::S, Q = Sh::Q;
    const unsigned D = (unsigned)a.D, id = blockIdx.x * (kThreads / Q) + threadIdx.x / Q, q = threadIdx.x % Q;      // the channel, over all streams
    const bool on = id < (unsigned)a.B * D;
    const unsigned at = on ? id : 0, b = at / D, d = at % D, g = d / (D / (unsigned)a.G);
    const int n = min(S, (int)a.N - (int)q * S);
    float A[S], h[S], B[S], C[S];
    float* to = state + (int64_t)at * a.N + q * S;
    load_states<float, S, kWide>(h, to, n);
    load_states<float, S, kWide>(A, a.A + (int64_t)d * a.N + q * S, n);
    load_states<T, S, false>(B, (const T*)a.b + b * a.b_stride_b + g * a.b_stride_g + q * S, n);
    load_states<T, S, false>(C, (const T*)a.c + b * a.c_stride_b + g * a.c_stride_g + q * S, n);
    const float x = to_float(((const T*)a.x)[b * a.x_stride_b + d]), z = a.gate ? to_float(((const T*)a.gate)[b * a.gate_stride_b + d]) : 0.0f;
    float step = to_float(((const T*)a.dt)[b * a.dt_stride_b + d]) + (a.dt_bias ? a.dt_bias[d] : 0.0f), o = 0.0f;
    if (a.softplus) step = softplus(step);
#pragma unroll
    for (int s = 0; s < S; s++) {
        h[s] = fmaf(fast_exp(step * A[s]), h[s], step * x * B[s]);
        o = fmaf(C[s], h[s], o);
    }
#pragma unroll
    for (int m = 1; m < Q; m *= 2) o += __shfl_xor(o, m);
    if (a.skip) o = fmaf(a.skip[d], x, o);
    if (a.gate) o *= z * sigmoid(z);
    if (!on) return;
    if constexpr (kWide) {
        Pack<float, S> r;
#pragma unroll
        for (int s = 0; s < S; s++) r.v[s] = h[s];
        *(Pack<float, S>*)to = r;
    } else {
#pragma unroll
        for (int s = 0; s < S; s++)
            if (s < n) to[s] = h[s];
    }
    if (q == 0) y[at] = from_float<T>(o);
}

int64_t tiles_of(const sig_scan_args& a) { return (a.L + kTile - 1) / kTile; }

// four lanes a channel up to 16 states, four states a lane beyond
template <class F> auto with_shape(int64_t N, F f)
{
    if (N <= 4) return f(Shape<4, 1>());
    if (N <= 8) return f(Shape<4, 2>());
    if (N <= 16) return f(Shape<4, 4>());
    if (N <= 32) return f(Shape<8, 4>());
    return f(Shape<16, 4>());
}
template <class F> auto with_type(int64_t dtype, F f) { return dtype == SIG_BF16 ? f(bf16()) : f(float()); }

// States of a wavefront and wavefronts of a workgroup, by the number of states.  Measured at 8 x 4096 x 2048 with 16 states: two states on
// eight wavefronts take 30 % less than four on four (a wavefront alone on its SIMD) and 36 % less than one on sixteen (their sums fill the
// LDS pipe).
template <class F> auto with_group(int64_t N, F f)
{
    if (N <= 8) return f(Group<2, 4>());
    if (N <= 16) return f(Group<2, 8>());
    if (N <= 32) return f(Group<4, 8>());
    return f(Group<4, 16>());
}

// Time chunks give a launch of few workgroups more of them, for a second pass over a part of the work (`second` of the first one's time).  The chunks are those
// with the least time by a model: a compute unit runs `resident` workgroups at once (what LDS allows; the registers allow as many), W wavefronts each, whose SIMDs
// issue at kRate of their rate with one to four wavefronts; workgroups beyond what the chip holds wait for a round of their own.
// Unit: a wavefront's work on a token, 104 of them a microsecond; with four states a wavefront it is more, which weighs a launch and the joining
// less than it should.  Measured in bf16 with 1, 2, 4 .. 64 chunks, us: the counts taken, their neighbours behind them.
//                                    forward                                    gradient
//   8 x 4096 x 2048, 16 states     1: 379 (2: 503)                            1: 1003 (2: 1227)
//   1 x 16384 x 1024, 16 states   32: 146 (16: 166, 64: 170)                 16: 336 (8: 644, 32: 335)
//   1 x 16384 x 1024, 8 states    47: 104 (32: 108, 64: 113)                 32: 214 (16: 304, 64: 220)
//   1 x 16384 x 1024, 32 states   32: 230 (16: 254, 64: 254)                 16: 587 (8: 1135, 32: 610)
//   4 x 2048 x 1024, 32 states     8: 125 (4: 138, 16: 129)                   4: 302 (2: 576, 8: 314)
//   1 x 4096 x 1024, 64 states    16: 125 (8: 220, 32: 160)                  16: 788 (8: 1262, 32: 853)
//   2 x 2048 x 2048, 64 states     4: 222 (2: 420, 8: 240)                    4: 1535 (2: 2577, 8: 1568)
constexpr double kRate[] = {0.45, 0.8, 0.93, 1.0};
constexpr int kUnits = 256;
double launch_time(int64_t workgroups, int W, int resident, double tokens)
{
    auto round = [&](int64_t n) {        // n workgroups on a compute unit
        const int waves = std::min<int64_t>(4, (n * W + 3) / 4);
        return n ? (double)(n * W) / kRate[waves - 1] : 0.0;
    };
    const int64_t most = (int64_t)kUnits * resident, left = workgroups % most;
    return tokens * ((double)(workgroups / most) * round(resident) + round((left + kUnits - 1) / kUnits));
}

Blocks blocks_of(const sig_scan_args& a, int resident, double second)
{
    Blocks bl;
    bl.per_group = a.D / a.G;
    bl.runs = (unsigned)((bl.per_group + 63) / 64);
    const int64_t rows = a.B * a.G * bl.runs, tiles = std::max<int64_t>(1, tiles_of(a));
    const int W = with_group(a.N, [](auto gr) { return decltype(gr)::W; });
    int64_t best = tiles;
    double least = launch_time(rows, W, resident, (double)tiles * kTile);
    for (int64_t c = 2; c <= 64 && 2 * c <= tiles; c++) {
        const int64_t per = (tiles + c - 1) / c, chunks = (tiles + per - 1) / per;
        // a launch more and, for every chunk before a workgroup's own, an eighth of a memory access' latency
        const double t = launch_time(rows * chunks, W, resident, (double)per * kTile) * (1.0 + second * (double)(chunks - 1) / (double)chunks) + 800.0 + 20.0 * (double)chunks;
        if (t < least) least = t, best = per;
    }
    bl.chunk = (int)(best * kTile);
    bl.chunks = (unsigned)((tiles + best - 1) / best);
    bl.total = rows * bl.chunks;
    return bl;
}

// dynamic LDS of the kernels in bytes, and the workgroups of a compute unit that it leaves room for
constexpr int kLds = 160 * 1024;
constexpr int forward_lds(int W) { return 2 * kTile * 64 * 8 + 2 * W * kTile * 64 * 4; }
constexpr int backward_lds(int W, int S) { return 2 * 3 * kTile * 64 * 4 + (W <= 8 ? 2 : 1) * W * 3 * kTile / 2 * 64 * 4 + W * S * 64 * 4; }
Blocks forward_blocks(const sig_scan_args& a)
{
    return blocks_of(a, with_group(a.N, [](auto gr) { return kLds / forward_lds(decltype(gr)::W); }), 0.7);
}
Blocks backward_blocks(const sig_scan_args& a)
{
    return blocks_of(a, with_group(a.N, [](auto gr) { return kLds / backward_lds(decltype(gr)::W, decltype(gr)::S); }), 0.25);
}

// floats of the chunks' states, and of a backward launch's sums
size_t chunk_floats(const sig_scan_args& a, const Blocks& bl) { return bl.chunks > 1 ? (size_t)(a.B * bl.chunks * a.D * (a.N + 1)) : 0; }
struct PartFloats { size_t bc, A, rest; };
PartFloats part_floats(const sig_scan_args& a, const Blocks& bl)
{
    int64_t W = 0, Q = 0;
    with_group(a.N, [&](auto gr) { W = decltype(gr)::W, Q = decltype(gr)::S / 2; return 0; });
    return {(size_t)(a.B * tiles_of(a) * a.G * bl.runs * W * Q * 64), (size_t)(a.B * bl.chunks * a.N * a.D), (size_t)(a.B * bl.chunks * 2 * a.D)};
}

}  // namespace

size_t scan_forward_workspace(const sig_scan_args& a) { return chunk_floats(a, forward_blocks(a)) * 4; }
size_t scan_backward_workspace(const sig_scan_args& a)
{
    Blocks bl = backward_blocks(a);
    PartFloats p = part_floats(a, bl);
    return (p.bc + p.A + p.rest + chunk_floats(a, bl)) * 4;
}

hipError_t scan_forward(const sig_scan_args& a, void* y, float* final_state, float* checkpoint, float* workspace, hipStream_t stream)
{
    Blocks bl = forward_blocks(a);
    ChunkStates cs{workspace, workspace ? workspace + a.B * bl.chunks * a.N * a.D : nullptr};
    return with_type(a.dtype, [&](auto t) {
        return with_group(a.N, [&](auto gr) {
            using T = decltype(t);
            using Gr = decltype(gr);
            constexpr int lds = forward_lds(Gr::W);
            if (!launchable(bl.total, Gr::W * 64)) return kTooManyThreads;
            if (bl.chunks > 1) scan_fwd_kernel<T, Gr, false, false><<<(unsigned)bl.total, Gr::W * 64, forward_lds(0), stream>>>(a, bl, cs, nullptr, nullptr, nullptr);
            auto launch = [&](auto kernel) {
                if (lds > 65536) {
                    hipError_t e = ensure_dynamic_lds((const void*)kernel, lds);
                    if (e != hipSuccess) return e;
                }
                kernel<<<(unsigned)bl.total, Gr::W * 64, lds, stream>>>(a, bl, cs, (T*)y, final_state, checkpoint);
                return hipGetLastError();
            };
            return checkpoint ? launch(scan_fwd_kernel<T, Gr, true, true>) : launch(scan_fwd_kernel<T, Gr, true, false>);
        });
    });
}

hipError_t scan_backward(const sig_scan_args& a, const sig_scan_grads& g, const float* checkpoint, float* workspace, hipStream_t stream)
{
    Blocks bl = backward_blocks(a);
    PartFloats p = part_floats(a, bl);
    Parts parts{workspace, workspace + p.bc, workspace + p.bc + p.A};
    float* states = parts.rest + p.rest;
    ChunkStates cs{states, states + a.B * bl.chunks * a.N * a.D};
    return with_type(a.dtype, [&](auto t) {
        return with_group(a.N, [&](auto gr) {
            using T = decltype(t);
            using Gr = decltype(gr);
            constexpr int lds = backward_lds(Gr::W, Gr::S);
            const unsigned params = (unsigned)((a.D * (a.N + 2) + 63) / 64);
            const int64_t sums = a.B * tiles_of(a) * a.G * Gr::W * (Gr::S / 2);        // wavefronts
            const unsigned others = (unsigned)std::min<int64_t>(1 << 20, (sums + kSumThreads / 64 - 1) / (kSumThreads / 64));
            if (!launchable(bl.total, Gr::W * 64) || !launchable((int64_t)params + others, kSumThreads)) return kTooManyThreads;
            if (lds > 65536) {
                hipError_t e = ensure_dynamic_lds((const void*)scan_bwd_kernel<T, Gr, true>, lds);
                if (e != hipSuccess) return e;
            }
            if (a.B > 0) {
                if (bl.chunks > 1) scan_bwd_kernel<T, Gr, false><<<(unsigned)bl.total, Gr::W * 64, backward_lds(0, 0), stream>>>(a, g, bl, cs, nullptr, parts);
                scan_bwd_kernel<T, Gr, true><<<(unsigned)bl.total, Gr::W * 64, lds, stream>>>(a, g, bl, cs, checkpoint, parts);
            }
            scan_bwd_sums_kernel<T, Gr><<<params + others, kSumThreads, 0, stream>>>(a, bl, parts, a.B * bl.chunks, params, (T*)g.grad_b, (T*)g.grad_c, g.grad_A, g.grad_skip, g.grad_dt_bias);
            return hipGetLastError();
        });
    });
}

hipError_t scan_step(const sig_scan_args& a, float* state, void* y, hipStream_t stream)
{
    return with_type(a.dtype, [&](auto t) {
        return with_shape(a.N, [&](auto sh) {
            using T = decltype(t);
            using Sh = decltype(sh);
            const bool wide = a.N == Sh::Q * Sh::S && (((uintptr_t)state | (uintptr_t)a.A) & (Sh::S * 4 - 1)) == 0;
            const int64_t blocks = (a.B * a.D * Sh::Q + kThreads - 1) / kThreads;
            if (!launchable(blocks, kThreads)) return kTooManyThreads;
            if (wide) scan_step_kernel<T, Sh, true><<<(unsigned)blocks, kThreads, 0, stream>>>(a, state, (T*)y);
            else scan_step_kernel<T, Sh, false><<<(unsigned)blocks, kThreads, 0, stream>>>(a, state, (T*)y);
            return hipGetLastError();
        });
    });
}

}  // namespace sig
