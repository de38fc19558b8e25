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
#include <climits>
#include <type_traits>
#include <utility>

#include "seq.hpp"

namespace sig {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kScanTile;

// Q lanes hold the states of a channel, S each (state n = lane * S + s; N <= Q S, the rest are zero): a wavefront has 64 / Q channels.
template <int Q_, int S_> struct Shape { static constexpr int Q = Q_, S = S_, channels = 64 / Q_; };

// The waves of a launch, one for each stream, group and run of channels of that group.
struct Rows {
    int64_t per_group;   // channels of a group
    int64_t runs;        // wavefronts for the channels of a group
    int64_t total;
};
template <class Sh> Rows rows_of(const sig_scan_args& a)
{
    Rows r;
    r.per_group = a.D / a.G;
    r.runs = (r.per_group + Sh::channels - 1) / Sh::channels;
    r.total = a.B * a.G * r.runs;
    return r;
}

template <int Q> __device__ __forceinline__ float sum_states(float v)     // over the Q lanes of a channel
{
#pragma unroll
    for (int m = 1; m < Q; m *= 2) v += __shfl_xor(v, m);
    return v;
}
template <int Q> __device__ __forceinline__ float sum_channels(float v)   // over the channels of the wavefront
{
#pragma unroll
    for (int m = Q; m < 64; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// what a lane knows of its channel
template <class T, class Sh> struct Lane {
    int64_t b, g, d, len;
    int q;
    bool on;             // the channel exists
    float A[Sh::S], skip, bias;
    const T *x, *dt, *gate, *B, *C;
    __device__ __forceinline__ Lane(const sig_scan_args& a, const Rows& r, int64_t row)
    {
        int lane = threadIdx.x & 63;
        int64_t run = row % r.runs, bg = row / r.runs;
        g = bg % a.G, b = bg / a.G;
        int64_t c = run * Sh::channels + lane / Sh::Q;
        q = lane % Sh::Q;
        on = c < r.per_group;
        d = g * r.per_group + (on ? c : 0);
        len = live_length(a.lengths, b, a.L);
#pragma unroll
        for (int s = 0; s < Sh::S; s++) A[s] = q * Sh::S + s < a.N ? a.A[d * a.N + q * Sh::S + s] : 0.0f;
        skip = a.skip ? a.skip[d] : 0.0f;
        bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
        x = (const T*)a.x + b * a.x_stride_b + d;
        dt = (const T*)a.dt + b * a.dt_stride_b + d;
        gate = a.gate ? (const T*)a.gate + b * a.gate_stride_b + d : nullptr;
        B = (const T*)a.b + b * a.b_stride_b + g * a.b_stride_g + q * Sh::S;
        C = (const T*)a.c + b * a.c_stride_b + g * a.c_stride_g + q * Sh::S;
    }
    __device__ __forceinline__ int64_t state(const sig_scan_args& a) const { return (b * a.D + d) * a.N + q * Sh::S; }
};

template <int S> __device__ __forceinline__ void load_states(float (&h)[S], const float* p, int n)
{
#pragma unroll
    for (int s = 0; s < S; s++) h[s] = p && s < n ? p[s] : 0.0f;
}
template <class T, int S> __device__ __forceinline__ void load_row(float (&h)[S], const T* p, int n)
{
#pragma unroll
    for (int s = 0; s < S; s++) h[s] = s < n ? to_float(p[s]) : 0.0f;
}

// ---- forward
// A workgroup takes 64 neighbouring channels of one stream and group, a channel a lane; its W wavefronts share out the states, S each, so
// that sums over states meet in LDS once a token while loads and stores of tokens are whole lines.  Tiles of 16 tokens: the wavefronts
// prepare D_t and D_t x_t of the tile's tokens in turn (LDS), all run the recurrence of their states over the tile, and each adds
// up and stores the outputs of the tokens that it prepared.  B and C of a tile lie across the 16 lanes of a row, 16 / S tokens in a
// register, and reach the multiply-adds as row broadcasts of the instruction itself.
// What bounds it: the exponentials (3.9 ns for 64 states on a SIMD) and the four other vector instructions a state and token.
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
// o + sum_s r[K + s] h[s], r[k] the value of lane k of each row.  The compiler does not merge the broadcast into a multiply-add; s_nop
// keeps the two wait states between a write of r and its first use across lanes, which it does not look for in here.
template <int K, int S> __device__ __forceinline__ float add_broadcast(float o, float r, const float (&h)[S])
{
    static_assert(S % 2 == 0, "states come in pairs");
#pragma unroll
    for (int s = 0; s < S; s += 2)
        asm("s_nop 1\n\tv_fmac_f32_dpp %0, %1, %2 row_newbcast:%4 row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %0, %1, %3 row_newbcast:%5 row_mask:0xf bank_mask:0xf"
            : "+v"(o) : "v"(r), "v"(h[s]), "v"(h[s + 1]), "n"(K + s), "n"(K + s + 1));
    return o;
}

// Element at a lane's byte offset from a row that is the same for the wavefront: the row stays in scalar registers.
template <class T> __device__ __forceinline__ T& lane_at(T* row, unsigned bytes) { return *(T*)((char*)row + bytes); }
template <class T> __device__ __forceinline__ const T& lane_at(const T* row, unsigned bytes) { return *(const T*)((const char*)row + bytes); }

// The workgroups of a launch: 64 channels of a group of one stream, one time chunk.
struct Blocks {
    int64_t per_group;   // channels of a group
    unsigned runs;       // workgroups for the channels of a group
    unsigned chunks;
    int64_t chunk;       // tokens of a time chunk, a multiple of kTile
    unsigned total;
};

// Time chunks: where a launch has few workgroups, a first kernel runs every chunk from a state of zero and leaves its last state and the sum
// of its step sizes; exp(A sum D) is the chunk's decay, so the state before any chunk is a short recurrence over the chunks before it.
struct ChunkStates {
    float* last;         // [B, chunks, N, D]
    float* steps;        // [B, chunks, D]
};

template <class T, class Gr, bool kOutputs>
__global__ __launch_bounds__(Gr::W * 64, Gr::W > 2 && Gr::S == 4 ? 4 : 2) void scan_fwd_kernel(sig_scan_args a, Blocks bl, ChunkStates cs, T* y, float* final_state, float* checkpoint)
{
    constexpr int S = Gr::S, W = Gr::W, PT = kTile / W, RT = 16 / S, KB = kTile / RT;
    __shared__ float2 steps[kTile][64];
    __shared__ float sums[kOutputs ? W : 1][kTile][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned c = blockIdx.x % bl.chunks, rest = blockIdx.x / bl.chunks, run = rest % bl.runs, bg = rest / bl.runs;
    const int64_t g = bg % (unsigned)a.G, b = bg / (unsigned)a.G;
    const int64_t d0 = g * bl.per_group + run * 64;       // the workgroup's first channel
    const bool on = run * 64 + lane < bl.per_group;
    const unsigned e = on ? lane : 0;                     // lanes without a channel read the first one's and store nothing
    const int64_t d = d0 + e;
    const int64_t len = live_length(a.lengths, b, a.L), t_first = c * bl.chunk, t_end = min(t_first + bl.chunk, a.L);
    int64_t left = min(t_end, len) - t_first;             // tokens from the tile's first to the last of the chunk that counts
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
    // rows of the wavefront's first token in the tile
    const int64_t t1 = t_first + w;
    const T *px = (const T*)a.x + b * a.x_stride_b + t1 * a.x_stride_t + d0, *pdt = (const T*)a.dt + b * a.dt_stride_b + t1 * a.dt_stride_t + d0;
    const T* pz = a.gate ? (const T*)a.gate + b * a.gate_stride_b + t1 * a.gate_stride_t + d0 : nullptr;
    T* py = kOutputs ? y + (b * a.L + t1) * a.D + d0 : nullptr;
    const int n0 = w * S, nb = n0 + lane % S;             // first state of the wavefront; the state whose B and C this lane loads
    const int tb = nb < a.N ? lane % 16 / S : INT_MAX / 2;    // and the first of their tokens in the tile
    const int64_t tbc = t_first + lane % 16 / S;
    const T *pb = (const T*)a.b + b * a.b_stride_b + g * a.b_stride_g + tbc * a.b_stride_t + nb;
    const T *pc = (const T*)a.c + b * a.c_stride_b + g * a.c_stride_g + tbc * a.c_stride_t + nb;
    if (checkpoint) checkpoint += ((b * ((a.L + kTile - 1) / kTile) + t_first / kTile) * a.N + n0) * a.D + d0;
    float A[S], h[S];
#pragma unroll
    for (int s = 0; s < S; s++) {
        A[s] = n0 + s < a.N ? a.A[d * a.N + n0 + s] * kLog2e : 0.0f;
        h[s] = kOutputs && a.initial_state && n0 + s < a.N ? a.initial_state[(b * a.D + d) * a.N + n0 + s] : 0.0f;
    }
    if constexpr (kOutputs) {
        const float *last = cs.last + (b * bl.chunks * a.N + n0) * a.D + d0, *sums_of = cs.steps + b * bl.chunks * a.D + d0;
        for (unsigned j = 0; j < c && j * bl.chunk < len; j++, last += a.N * a.D, sums_of += a.D) {
            float sum = sums_of[e];
#pragma unroll
            for (int s = 0; s < S; s++)
                if (n0 + s < a.N) h[s] = fmaf(__builtin_amdgcn_exp2f(A[s] * sum), h[s], (last + s * a.D)[e]);
        }
    }
    T x[PT], dt[PT], z[PT], bv[KB], cv[KB];
    float total = 0.0f;
    auto fetch = [&](int64_t left) {       // the tile at the pointers; they go on to the next
        unsigned et = e * sizeof(T);
        asm("" : "+v"(et));                // or the compiler carries a vector address for every row
#pragma unroll
        for (int i = 0; i < PT; i++) {
            if (i * W + w < left) {
                x[i] = lane_at(px, et);
                dt[i] = lane_at(pdt, et);
                if (kOutputs && pz) z[i] = lane_at(pz, et);
            }
            px += W * a.x_stride_t, pdt += W * a.dt_stride_t;
            if (kOutputs && pz) pz += W * a.gate_stride_t;
        }
#pragma unroll
        for (int j = 0; j < KB; j++) {
            bv[j] = cv[j] = from_float<T>(0.0f);
            if (j * RT + tb < left) {
                bv[j] = *pb;
                if (kOutputs) cv[j] = *pc;
            }
            pb += RT * a.b_stride_t;
            if (kOutputs) pc += RT * a.c_stride_t;
        }
    };
    fetch(left);
    int64_t room = t_end - t_first;        // tokens of the chunk from the tile's first
    for (; left > 0; left -= kTile, room -= kTile) {
        float keep[PT], f[PT], B[KB], C[KB];
        const int m = (int)min((int64_t)kTile, left), m_out = (int)min((int64_t)kTile, room);
#pragma unroll
        for (int i = 0; i < PT; i++) {
            int k = i * W + w;
            float D = 0.0f, u = 0.0f;
            f[i] = 0.0f, keep[i] = 0.0f;
            if (k < m) {
                float v = to_float(x[i]);
                D = to_float(dt[i]) + bias;
                if (a.softplus) D = softplus(D);
                u = D * v;
                keep[i] = skip * v;
                f[i] = 1.0f;
                if (kOutputs && pz) {
                    f[i] = to_float(z[i]);
                    f[i] *= sigmoid(f[i]);
                }
            }
            steps[k][lane] = make_float2(D, u);
        }
#pragma unroll
        for (int j = 0; j < KB; j++) B[j] = to_float(bv[j]), C[j] = to_float(cv[j]);
        if (kOutputs && checkpoint) {
            unsigned ef = e * 4;
            asm("" : "+v"(ef));
#pragma unroll
            for (int s = 0; s < S; s++)
                if (on && n0 + s < a.N) lane_at(checkpoint + s * a.D, ef) = h[s];
            checkpoint += a.N * a.D;
        }
        fetch(left - kTile);
        __syncthreads();
        unrolled<0, kTile>([&](auto it) {
            constexpr int i = decltype(it)::value, k = i % RT * S;
            float2 q = steps[i][lane];
            if (!kOutputs) total += q.x;
            unrolled<0, S>([&](auto is) {
                constexpr int s = decltype(is)::value;
                h[s] = fmaf(__builtin_amdgcn_exp2f(q.x * A[s]), h[s], times_broadcast<k + s>(B[i / RT], q.y));
            });
            if constexpr (kOutputs) sums[w][i][lane] = add_broadcast<k>(0.0f, C[i / RT], h);
        });
        __syncthreads();
        if constexpr (kOutputs) {
#pragma unroll
            for (int i = 0; i < PT; i++, py += W * a.D) {
                unsigned et = e * sizeof(T);
                asm("" : "+v"(et));
                int k = i * W + w;
                float o = keep[i];
#pragma unroll
                for (int v = 0; v < W; v++) o += sums[v][k][lane];
                if (on && k < m_out) lane_at(py, et) = from_float<T>(k < m ? o * f[i] : 0.0f);
            }
        }
    }
    if (!on) return;
    if constexpr (kOutputs) {
        for (int64_t k = w; k < room; k += W, py += W * a.D) py[e] = from_float<T>(0.0f);
        if (final_state && c == (unsigned)(len > 0 ? (len - 1) / bl.chunk : 0))
#pragma unroll
            for (int s = 0; s < S; s++)
                if (n0 + s < a.N) final_state[(b * a.D + d) * a.N + n0 + s] = h[s];
    } else {
#pragma unroll
        for (int s = 0; s < S; s++)
            if (n0 + s < a.N) (cs.last + ((b * bl.chunks + c) * a.N + n0 + s) * a.D + d0)[e] = h[s];
        if (w == 0) cs.steps[(b * bl.chunks + c) * a.D + d] = total;
    }
}

// Tiles of kTile tokens from the last to the first: the states inside a tile are computed again from the checkpoint before it and stay
// in registers with their decays; the adjoint states walk back over them.
template <class T, class Sh>
__global__ __launch_bounds__(kThreads) void scan_bwd_kernel(sig_scan_args a, sig_scan_grads g, Rows r, const float* checkpoint, int64_t tiles,
                                                            float* part_bc, float* part_a, float* part_d)
{
    constexpr int S = Sh::S;
    int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (row >= r.total) return;
    Lane<T, Sh> l(a, r, row);
    int n = (int)min((int64_t)S, a.N - l.q * S);
    float adj[S], gA[S] = {}, gskip = 0.0f, gbias = 0.0f;     // adj: a_{t+1} l_{t+1}
    load_states(adj, g.grad_final_state ? g.grad_final_state + l.state(a) : nullptr, n);
    const T* gy = (const T*)g.grad_y + l.b * g.gy_stride_b + l.d;
    int64_t out = l.b * a.L * a.D + l.d;
    T *gx = (T*)g.grad_x + out, *gdt = (T*)g.grad_dt + out, *gz = l.gate ? (T*)g.grad_gate + out : nullptr;
    if (l.on && l.q == 0)
        for (int64_t t = l.len; t < a.L; t++) {
            gx[t * a.D] = gdt[t * a.D] = from_float<T>(0.0f);
            if (gz) gz[t * a.D] = from_float<T>(0.0f);
        }
    for (int64_t tile = (l.len + kTile - 1) / kTile - 1; tile >= 0; tile--) {
        int64_t t0 = tile * kTile;
        int m = (int)min((int64_t)kTile, l.len - t0);
        float h0[S], h[kTile][S], e[kTile][S], x[kTile], D[kTile], raw[kTile];
#pragma unroll
        for (int s = 0; s < S; s++) h0[s] = s < n ? checkpoint[((l.b * tiles + tile) * a.N + l.q * S + s) * a.D + l.d] : 0.0f;
#pragma unroll
        for (int i = 0; i < kTile; i++) {
            int64_t t = t0 + (i < m ? i : 0);
            float B[S];
            x[i] = to_float(l.x[t * a.x_stride_t]);
            raw[i] = to_float(l.dt[t * a.dt_stride_t]) + l.bias;
            D[i] = a.softplus ? softplus(raw[i]) : raw[i];
            load_row(B, l.B + t * a.b_stride_t, n);
#pragma unroll
            for (int s = 0; s < S; s++) {
                e[i][s] = fast_exp(D[i] * l.A[s]);
                h[i][s] = fmaf(e[i][s], i ? h[i - 1][s] : h0[s], D[i] * x[i] * B[s]);
            }
        }
#pragma unroll
        for (int i = kTile - 1; i >= 0; i--) {
            if (i >= m) continue;
            int64_t t = t0 + i;
            float B[S], C[S], up = to_float(gy[t * g.gy_stride_t]), o = 0.0f, gB[S], gC[S], dx = 0.0f, dD = 0.0f;
            load_row(B, l.B + t * a.b_stride_t, n);
            load_row(C, l.C + t * a.c_stride_t, n);
            if (l.gate) {
                float z = to_float(l.gate[t * a.gate_stride_t]), p = sigmoid(z);
#pragma unroll
                for (int s = 0; s < S; s++) o = fmaf(C[s], h[i][s], o);
                o = fmaf(l.skip, x[i], sum_states<Sh::Q>(o));
                if (l.on && l.q == 0) gz[t * a.D] = from_float<T>(up * o * p * fmaf(z, 1.0f - p, 1.0f));
                up *= z * p;
            }
#pragma unroll
            for (int s = 0; s < S; s++) {
                float lam = fmaf(C[s], up, adj[s]), keep;
                adj[s] = lam * e[i][s];
                keep = adj[s] * (i ? h[i - 1][s] : h0[s]);
                gC[s] = sum_channels<Sh::Q>(l.on ? up * h[i][s] : 0.0f);
                gB[s] = sum_channels<Sh::Q>(l.on ? lam * D[i] * x[i] : 0.0f);
                gA[s] = fmaf(keep, D[i], gA[s]);
                dx = fmaf(lam, B[s], dx);
                dD = fmaf(keep, l.A[s], dD);
            }
            dx = sum_states<Sh::Q>(dx), dD = sum_states<Sh::Q>(dD);
            dD = fmaf(dx, x[i], dD);
            if (a.softplus) dD *= sigmoid(raw[i]);
            gskip = fmaf(up, x[i], gskip);
            gbias += dD;
            if (l.on && l.q == 0) {
                gx[t * a.D] = from_float<T>(fmaf(dx, D[i], l.skip * up));
                gdt[t * a.D] = from_float<T>(dD);
            }
            if ((threadIdx.x & 63) < Sh::Q) {
                int64_t at = (((l.b * a.L + t) * a.G + l.g) * r.runs + row % r.runs) * 2 * a.N + l.q * S;
                for (int s = 0; s < n; s++) part_bc[at + s] = gB[s], part_bc[at + a.N + s] = gC[s];
            }
        }
    }
    if (!l.on) return;
    for (int s = 0; s < n; s++) {
        part_a[l.state(a) + s] = gA[s];
        if (g.grad_initial_state) g.grad_initial_state[l.state(a) + s] = adj[s];
    }
    if (l.q == 0) {
        part_d[(l.b * 2 + 0) * a.D + l.d] = gskip;
        part_d[(l.b * 2 + 1) * a.D + l.d] = gbias;
    }
}

// dB and dC of a token: the sums over the runs of its group's channels, in their order
template <class T> __global__ __launch_bounds__(kThreads) void scan_bwd_bc_kernel(sig_scan_args a, Rows r, const float* part, T* gB, T* gC)
{
    int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, N2 = 2 * a.N;
    if (id >= a.B * a.L * a.G * N2) return;
    int64_t k = id % N2, tok = id / N2, t = tok / a.G % a.L, b = tok / a.G / a.L;
    float v = 0.0f;
    if (t < live_length(a.lengths, b, a.L))
        for (int64_t j = 0; j < r.runs; j++) v += part[(tok * r.runs + j) * N2 + k];
    (k < a.N ? gB : gC)[tok * a.N + k % a.N] = from_float<T>(v);
}

// dA, dskip and ddt_bias: the sums over the streams, in their order
__global__ __launch_bounds__(kThreads) void scan_bwd_params_kernel(sig_scan_args a, const float* part_a, const float* part_d, float* gA, float* gskip, float* gbias)
{
    int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, DN = a.D * a.N;
    float v = 0.0f;
    if (id < DN) {
        for (int64_t b = 0; b < a.B; b++) v += part_a[b * DN + id];
        gA[id] = v;
    } else if (id < DN + 2 * a.D) {
        int64_t k = (id - DN) / a.D, d = (id - DN) % a.D;
        float* to = k ? gbias : gskip;
        if (!to) return;
        for (int64_t b = 0; b < a.B; b++) v += part_d[(b * 2 + k) * a.D + d];
        to[d] = v;
    }
}

template <class T, class Sh> __global__ __launch_bounds__(kThreads) void scan_step_kernel(sig_scan_args a, Rows r, float* state, T* y)
{
    int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (row >= r.total) return;
    Lane<T, Sh> l(a, r, row);
    int n = (int)min((int64_t)Sh::S, a.N - l.q * Sh::S);
    float h[Sh::S], B[Sh::S], C[Sh::S];
    load_states(h, state + l.state(a), n);
    float x = to_float(l.x[0]), D = to_float(l.dt[0]) + l.bias, o = 0.0f;
    if (a.softplus) D = softplus(D);
    load_row(B, l.B, n);
    load_row(C, l.C, n);
#pragma unroll
    for (int s = 0; s < Sh::S; s++) {
        h[s] = fmaf(fast_exp(D * l.A[s]), h[s], D * x * B[s]);
        o = fmaf(C[s], h[s], o);
    }
    o = fmaf(l.skip, x, sum_states<Sh::Q>(o));
    if (l.gate) {
        float z = to_float(l.gate[0]);
        o *= z * sigmoid(z);
    }
    if (!l.on) return;
    for (int s = 0; s < n; s++) state[l.state(a) + s] = h[s];
    if (l.q == 0) y[l.b * a.D + l.d] = from_float<T>(o);
}

unsigned blocks_for(int64_t threads) { return (unsigned)((threads + kThreads - 1) / kThreads); }
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

// wavefronts of a workgroup by the number of states, four states each, eight beyond 32 (the sums of sixteen would not fit 64 KB of LDS)
template <class F> auto with_group(int64_t N, F f)
{
    if (N <= 4) return f(Group<4, 1>());
    if (N <= 8) return f(Group<4, 2>());
    if (N <= 16) return f(Group<4, 4>());
    if (N <= 32) return f(Group<4, 8>());
    return f(Group<8, 8>());
}

Blocks forward_blocks(const sig_scan_args& a)
{
    Blocks bl;
    bl.per_group = a.D / a.G;
    bl.runs = (unsigned)((bl.per_group + 63) / 64);
    int64_t rows = a.B * a.G * bl.runs, waves = rows * with_group(a.N, [](auto gr) { return decltype(gr)::W; });
    int64_t want = std::max<int64_t>(1, std::min<int64_t>(64, 2048 / std::max<int64_t>(1, waves)));
    int64_t tiles = std::max<int64_t>(1, tiles_of(a)), per = std::max<int64_t>(2, (tiles + want - 1) / want);
    bl.chunk = per * kTile;
    bl.chunks = (unsigned)((tiles + per - 1) / per);
    bl.total = (unsigned)(rows * bl.chunks);
    return bl;
}

struct BackwardParts { size_t bc, a, d; };
BackwardParts backward_parts(const sig_scan_args& a)
{
    int64_t runs = with_shape(a.N, [&](auto sh) { return rows_of<decltype(sh)>(a).runs; });
    return {(size_t)(a.B * a.L * a.G * runs * 2 * a.N), (size_t)(a.B * a.D * a.N), (size_t)(a.B * 2 * a.D)};
}

}  // namespace

size_t scan_forward_workspace(const sig_scan_args& a)
{
    Blocks bl = forward_blocks(a);
    return bl.chunks > 1 ? (size_t)(a.B * bl.chunks * a.D * (a.N + 1) * 4) : 0;
}
size_t scan_backward_workspace(const sig_scan_args& a)
{
    BackwardParts p = backward_parts(a);
    return (p.bc + p.a + p.d) * 4;
}

hipError_t scan_forward(const sig_scan_args& a, void* y, float* final_state, float* checkpoint, float* workspace, hipStream_t stream)
{
    Blocks bl = forward_blocks(a);
    ChunkStates cs{workspace, workspace ? workspace + a.B * bl.chunks * a.N * a.D : nullptr};
    return with_type(a.dtype, [&](auto t) {
        return with_group(a.N, [&](auto gr) {
            using T = decltype(t);
            using Gr = decltype(gr);
            if (bl.chunks > 1) scan_fwd_kernel<T, Gr, false><<<(unsigned)bl.total, Gr::W * 64, 0, stream>>>(a, bl, cs, nullptr, nullptr, nullptr);
            scan_fwd_kernel<T, Gr, true><<<(unsigned)bl.total, Gr::W * 64, 0, stream>>>(a, bl, cs, (T*)y, final_state, checkpoint);
            return hipGetLastError();
        });
    });
}

hipError_t scan_backward(const sig_scan_args& a, const sig_scan_grads& g, const float* checkpoint, float* workspace, hipStream_t stream)
{
    BackwardParts p = backward_parts(a);
    float *bc = workspace, *pa = bc + p.bc, *pd = pa + p.a;
    return with_type(a.dtype, [&](auto t) {
        return with_shape(a.N, [&](auto sh) {
            using T = decltype(t);
            using Sh = decltype(sh);
            Rows r = rows_of<Sh>(a);
            if (a.B > 0) scan_bwd_kernel<T, Sh><<<blocks_for(r.total * 64), kThreads, 0, stream>>>(a, g, r, checkpoint, tiles_of(a), bc, pa, pd);
            if (a.B > 0 && a.L > 0)
                scan_bwd_bc_kernel<T><<<blocks_for(a.B * a.L * a.G * 2 * a.N), kThreads, 0, stream>>>(a, r, bc, (T*)g.grad_b, (T*)g.grad_c);
            scan_bwd_params_kernel<<<blocks_for(a.D * (a.N + 2)), kThreads, 0, stream>>>(a, pa, pd, g.grad_A, g.grad_skip, g.grad_dt_bias);
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
            Rows r = rows_of<Sh>(a);
            scan_step_kernel<T, Sh><<<blocks_for(r.total * 64), kThreads, 0, stream>>>(a, r, state, (T*)y);
            return hipGetLastError();
        });
    });
}

}  // namespace sig
