// Matrix products y = f(x weight^T + bias) + residual over rows of tokens, and their gradient.
//
// One kernel shape for all types: a tile of outputs, both operands row by row along the contraction, 128 bytes of it (a slab) a step, 16 bytes (a
// chunk) an access.  A chunk of 16 rows is what a lane feeds to the matrix instructions: 8 bfloat16 (16x16x32), 4 float32 (four 16x16x4, whose
// order along the contraction is the same for both operands and so does not matter), or, two chunks together, 32 e4m3 (16x16x128).  The weight's rows are
// the instruction's first operand: a lane then holds four neighbouring outputs of one token.
// LDS: row r keeps chunk c at place c ^ (r & 7), so that eight rows' chunks lie in different banks.
// Few tiles and a long contraction: the contraction is split over workgroups, whose float32 sums a second kernel adds up in order.
// The gradient's operands lie the other way, a row for every place of the contraction: rows of whole chunks are turned by the LDS reads
// (see Side).  Operands whose rows are not whole chunks are copied first where that pays, for the gradient always.
//
// Bound by the matrix units where the contraction is long: bfloat16 8192^3 in 840 us (1,308 TFLOP/s), e4m3 in 476 (2,310), float32 4096^3 in 1,000 (137).
// Where it is short, by the outputs: 16384 x 1024 to 4096 in bfloat16 with SiLU 158 us, of which the product alone takes 105 at the rate above; a
// tile of 256 ends with 10 us of sums through LDS, activations and stores that the next one's loads do not overlap.  Few tokens are bound by
// the weight's way from memory and by latency (64 x 2048 to 1024 in bfloat16 7.0 us, float32 11.5, e4m3 5.3; 64 x 8192 to 8192 36, 90 and 27).
#include <algorithm>
#include <type_traits>

#include "layer.hpp"
#include "linear_tiles.hpp"

namespace sig {
namespace {

typedef float Acc __attribute__((ext_vector_type(4)));
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef int Int8 __attribute__((ext_vector_type(8)));

struct Out {                            // what becomes of a sum
    const void *bias, *residual;
    int64_t residual_stride;
    const float *x_scale, *weight_scale;
    void *y, *pre;
    int act;
    bool vec;                           // 16 bytes of neighbouring outputs are one access everywhere
};

// The normal distribution's Phi and its density.  exp(x^2) erfc(x) = t P(t) with t = 1 / (1 + c x), P fitted to the smallest relative error over x in
// [0, 14], and the exponential is the density's.  For float32 of degree 8, c = 0.3 (5e-8; with float32's roundings 5e-7 next to zero); for values
// rounded to bfloat16, whose half step is 4e-3, of degree 5, c = 0.45 (1e-5): the epilogue of a product is bound by this.  The tails keep their relative
// precision but for the exponential's, whose rounded exponent adds up to 1.13 z^2 2^-24 (in all 9e-7 down to -4, 2e-6 to -6, 7.5e-6 to -12.5).
struct Normal { float below, density; };
template <class O> __device__ __forceinline__ Normal normal_of(float z)
{
    constexpr bool kShort = sizeof(O) == 2;
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), (kShort ? 0.45f : 0.3f) * 0.70710678f, 1.0f)), g = fast_exp(-0.5f * z * z);
    float p;
    if constexpr (kShort) {
        p = fmaf(t, -0.13586082f, 0.29224834f);
        p = fmaf(p, t, 0.089452292f);
        p = fmaf(p, t, 0.24848109f);
        p = fmaf(p, t, 0.25170138f);
        p = fmaf(p, t, 0.25396823f);
    } else {
        p = fmaf(t, -0.12661661f, 0.47182638f);
        p = fmaf(p, t, -0.48469207f);
        p = fmaf(p, t, 0.51704908f);
        p = fmaf(p, t, -0.074049273f);
        p = fmaf(p, t, 0.2063852f);
        p = fmaf(p, t, 0.15046886f);
        p = fmaf(p, t, 0.17042372f);
        p = fmaf(p, t, 0.16920475f);
    }
    const float tail = 0.5f * (p * t) * g;
    return {z > 0.0f ? 1.0f - tail : tail, 0.39894228f * g};
}
template <class O> __device__ __forceinline__ float act_of(float z, int act)
{
    if (act == SIG_ACT_SILU) return z * sigmoid(z);
    if (act == SIG_ACT_GELU) return z * normal_of<O>(z).below;
    return z;
}
template <class O> __device__ __forceinline__ float slope_of(float z, int act)
{
    if (act == SIG_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    const Normal v = normal_of<O>(z);
    return fmaf(z, v.density, v.below);
}

template <class O, int V> __device__ __forceinline__ void take(const O* p, bool wide, int64_t n, int64_t N, float* to)
{
    if (wide) {
        const Pack<O, V> q = *(const Pack<O, V>*)p;
#pragma unroll
        for (int j = 0; j < V; j++) to[j] = to_float(q.v[j]);
    } else
#pragma unroll
        for (int j = 0; j < V; j++) to[j] = n + j < N ? to_float(p[j]) : 0.0f;
}
template <class O, int V> __device__ __forceinline__ void give(O* p, bool wide, int64_t n, int64_t N, const float* from)
{
    if (wide) {
        store_words<O, V>(p, from);
    } else
#pragma unroll
        for (int j = 0; j < V; j++)
            if (n + j < N) p[j] = from_float<O>(from[j]);
}

// What V neighbouring outputs from n < N on have in common over the tokens
template <class O, int V> struct Columns {
    float bias[V], scale[V];
    int64_t n;
    bool wide;
    __device__ __forceinline__ Columns(const Out& o, int64_t n, int64_t N) : n(n), wide(o.vec && n + V <= N)
    {
#pragma unroll
        for (int j = 0; j < V; j++) {
            bias[j] = 0.0f;
            scale[j] = o.weight_scale ? o.weight_scale[min(n + j, N - 1)] : 1.0f;
        }
        if (o.bias && n < N) take<O, V>((const O*)o.bias + n, wide, n, N, bias);
    }
};

// The residual of V outputs of token m, fetched ahead of the sums
template <class O, int V> __device__ __forceinline__ Words<O, V> residual_of(const Out& o, const Columns<O, V>& c, int64_t m, int64_t N)
{
    const O* p = (const O*)o.residual + m * o.residual_stride + c.n;
    Words<O, V> r;
    if (c.wide) r.w = *(const typename Words<O, V>::Vector*)p;
    else {
        O v[V];
#pragma unroll
        for (int j = 0; j < V; j++) v[j] = p[c.n + j < N ? j : 0];
        __builtin_memcpy(&r.w, v, sizeof(v));
    }
    return r;
}

// What becomes of their sums of token m
template <class O, int V> __device__ __forceinline__ void finish(const Out& o, const Columns<O, V>& c, int64_t m, int64_t N, float* z, const Words<O, V>& r)
{
    const int64_t at = m * N + c.n;
    if (o.x_scale || o.weight_scale) {
        const float xs = o.x_scale ? o.x_scale[m] : 1.0f;
#pragma unroll
        for (int j = 0; j < V; j++) z[j] = z[j] * xs * c.scale[j];
    }
    if (o.bias)
#pragma unroll
        for (int j = 0; j < V; j++) z[j] += c.bias[j];
    if (o.pre) give<O, V>((O*)o.pre + at, c.wide, c.n, N, z);
    if (o.act == SIG_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < V; j++) z[j] = act_of<O>(z[j], SIG_ACT_SILU);
    } else if (o.act == SIG_ACT_GELU)
#pragma unroll
        for (int j = 0; j < V; j++) z[j] = act_of<O>(z[j], SIG_ACT_GELU);
    if (o.residual)
#pragma unroll
        for (int j = 0; j < V; j++) z[j] += r.value(j);
    give<O, V>((O*)o.y + at, c.wide, c.n, N, z);
}

// The sums of a wavefront's tile, 16 FM tokens by 16 FN outputs, to where they belong.  A lane holds four outputs of sixteen tokens' rows; 16 rows at a
// time go through LDS (kPutFloats<FN> of a wavefront's own), after which neighbouring lanes hold neighbouring outputs and a row is whole lines.
template <int FN> constexpr int kPutFloats = 16 * (FN * 16 + 4);
template <class O, int FM, int FN> __device__ __forceinline__ void put(const Tiles& t, const Out& o, float* parts, int split, int64_t m0, int64_t n0, Acc (&acc)[FN][FM], float* lds)
{
    constexpr int V = 16 / sizeof(O), kWide = FN * 16, kPitch = kWide + 4, kLanes = kWide / V, kRows = 64 / kLanes;
    const int lane = threadIdx.x & 63, c = lane % kLanes * V;
    const int64_t N4 = (t.N + 3) / 4 * 4, n = n0 + c;
    const Columns<O, V> columns(o, n, t.N);
    const bool residual = o.residual && t.splits == 1 && n < t.N;
    Words<O, V> next[16 / kRows];                                              // the residual of the next sixteen rows
    auto fetch = [&](int j) {
#pragma unroll
        for (int r = 0; r < 16; r += kRows) next[r / kRows] = residual_of<O, V>(o, columns, min(m0 + j * 16 + r + lane / kLanes, t.M - 1), t.N);
    };
    if (residual) fetch(0);
#pragma unroll
    for (int j = 0; j < FM; j++) {
        Words<O, V> now[16 / kRows];
#pragma unroll
        for (int r = 0; r < 16 / kRows; r++) now[r] = next[r];
        if (residual && j + 1 < FM) fetch(j + 1);
#pragma unroll
        for (int i = 0; i < FN; i++) *(Acc*)(lds + (lane & 15) * kPitch + i * 16 + lane / 16 * 4) = acc[i][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < 16; r += kRows) {
            const int row = r + lane / kLanes;
            const int64_t m = m0 + j * 16 + row;
            float z[V];
#pragma unroll
            for (int k = 0; k < V; k += 4) *(Acc*)(z + k) = *(const Acc*)(lds + row * kPitch + c + k);
            if (m < t.M && n < t.N) {
                if (t.splits > 1) {
                    float* to = parts + ((int64_t)split * t.M + m) * N4 + n;
#pragma unroll
                    for (int k = 0; k < V; k += 4)
                        if (n + k < N4) *(Acc*)(to + k) = *(const Acc*)(z + k);
                } else finish<O, V>(o, columns, m, t.N, z, now[r / kRows]);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// 16 bytes of a row from element k on, zeros from element K on
template <class T> __device__ __forceinline__ Chunk take_chunk(const T* row, int64_t k, int64_t K)
{
    constexpr int E = kChunk / sizeof(T);
    Chunk c;
    if (k + E <= K) {
        __builtin_memcpy(&c, row + k, kChunk);
        return c;
    }
    T v[E];
#pragma unroll
    for (int j = 0; j < E; j++) {
        v[j] = T{};
        if (k + j < K) v[j] = row[k + j];
    }
    __builtin_memcpy(&c, v, kChunk);
    return c;
}

// Sums over the contraction of 16 x 16 products, one chunk a lane of each operand (e4m3: two).  float32 takes four instructions a pair of chunks: all
// pairs' first ones come first, so that none waits for the one before.
template <class T, int FN, int FM, int F> __device__ __forceinline__ void products(const Chunk (&w)[FN][F], const Chunk (&x)[FM][F], Acc (*acc)[FM])
{
#pragma unroll
    for (int q = 0; q < (std::is_same_v<T, float> ? 4 : 1); q++)
#pragma unroll
        for (int j = 0; j < FM; j++)
#pragma unroll
            for (int i = 0; i < FN; i++) {
                if constexpr (std::is_same_v<T, float>) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][0][q]), __uint_as_float(x[j][0][q]), acc[i][j], 0, 0, 0);
                } else if constexpr (std::is_same_v<T, bf16>) {
                    Bf8 a, b;
                    __builtin_memcpy(&a, w[i], 16);
                    __builtin_memcpy(&b, x[j], 16);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc[i][j], 0, 0, 0);
                } else {
                    Int8 a, b;
                    __builtin_memcpy(&a, w[i], 32);
                    __builtin_memcpy(&b, x[j], 32);
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[i][j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);     // block scales of one
                }
            }
}
template <class T> constexpr int kFeed = std::is_same_v<T, e4m3> ? 2 : 1;       // chunks of a row that a step takes


// Workgroups are dealt out to the eight dies in turn: each die gets a run of neighbouring tiles, walked in bands of eight along m
struct Place { int m, n, split; };
__device__ __forceinline__ Place place_of(const Tiles& t)
{
    const uint32_t all = gridDim.x, die = blockIdx.x % 8, q = all / 8, r = all % 8;
    uint32_t id = die * q + min(die, r) + blockIdx.x / 8;
    const uint32_t split = id % t.splits;
    id /= t.splits;
    const uint32_t band = id / (8 * t.n), in = id % (8 * t.n), high = min(8u, (uint32_t)t.m - band * 8);
    return {(int)(band * 8 + in % high), (int)(in / high), (int)split};
}

// Rows of any alignment: a workgroup's tile is 128 tokens by 128 outputs, 64 by 64 a wavefront; chunks pass through registers, where the ends of rows are
// put in order.  16384 x 5460 to 1024 in bfloat16: 272 us (673 TFLOP/s), where rows of 5456 take 189 by aligned_kernel.
template <class T, class O> __global__ __launch_bounds__(256) void product_kernel(Tiles t, const T* x, int64_t ldx, const T* w, int64_t ldw, Out o, float* parts)
{
    constexpr int E = kChunk / sizeof(T), kLoads = kTile * kChunks / 256;
    __shared__ Chunk lds[2][2][kTile * kChunks];
    const Place p = place_of(t);
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wm = wave & 1, wn = wave >> 1;
    const int64_t m0 = (int64_t)p.m * kTile, n0 = (int64_t)p.n * kTile, first = p.split * t.slabs * (kSlab / (int)sizeof(T));
    const int64_t last = min(t.K, first + t.slabs * (kSlab / (int)sizeof(T)));
    Chunk rx[kLoads], rw[kLoads];
    auto load = [&](int64_t k) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int id = threadIdx.x + i * 256, row = id / kChunks;
            const int64_t e = k + (id % kChunks) * E;
            rx[i] = take_chunk(x + min(m0 + row, t.M - 1) * ldx, e, last);
            rw[i] = take_chunk(w + min(n0 + row, t.N - 1) * ldw, e, last);
        }
    };
    auto keep = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int id = threadIdx.x + i * 256, row = id / kChunks, at = row * kChunks + ((id % kChunks) ^ (row & 7));
            lds[buf][0][at] = rx[i];
            lds[buf][1][at] = rw[i];
        }
    };
    Acc acc[4][4] = {};
    load(first);
    keep(0);
    __syncthreads();
    int buf = 0;
    for (int64_t k = first; k < last; k += kSlab / (int)sizeof(T), buf ^= 1) {
        const bool more = k + kSlab / (int)sizeof(T) < last;
        if (more) load(k + kSlab / (int)sizeof(T));
        constexpr int F = kFeed<T>;
#pragma unroll
        for (int s = 0; s < kChunks / 4; s += F) {
            Chunk fx[4][F], fw[4][F];
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int f = 0; f < F; f++) {
                    const int row = i * 16 + (lane & 15), c = (s + f) * 4 + lane / 16;
                    fx[i][f] = lds[buf][0][(wm * 64 + row) * kChunks + (c ^ (row & 7))];
                    fw[i][f] = lds[buf][1][(wn * 64 + row) * kChunks + (c ^ (row & 7))];
                }
            products<T>(fw, fx, acc);
        }
        if (more) keep(buf ^ 1);
        __syncthreads();
    }
    static_assert(4 * kPutFloats<4> * sizeof(float) <= sizeof(lds));
    put<O, 4, 4>(t, o, parts, p.split, m0 + wm * 64, n0 + wn * 64, acc, (float*)lds + wave * kPutFloats<4>);
}

// ---- the same for operands whose rows are multiples of 16 bytes, 16-byte aligned: chunks go from memory to LDS without passing registers, a wavefront's
// load filling 1,024 bytes in lane order; what a lane fetches decides where it lies.
//
// An operand of B rows along the contraction is as above.  One that lies the other way (kAcross: rows of outputs, one for every place of the contraction, as
// the gradients' operands do) comes as 64 (float32: 32) such rows of B outputs a slab, and the LDS reads turn it: a transposing read gives each of sixteen
// lanes four bfloat16 values of its own column; float32 values are read one by one, for which the matrix instructions leave time.  Row r keeps chunk c at place
// c ^ turn(r): the rows that one read touches (four, and the four that lie eight further on; float32: every fourth) are whole multiples of the banks
// apart otherwise.
template <class T, bool kAcross, int B, int kThreads> struct Side {
    static constexpr int E = kChunk / sizeof(T), kStep = kSlab / sizeof(T), kLoads = B * kChunks / kThreads, kRow = kAcross ? B / E : kChunks;     // chunks of a row
    typedef __attribute__((address_space(3))) Chunk Lds;
    const T* base;
    int64_t ld;
    int offset[kLoads], row, width;                                            // width (kAcross): outputs that are there

    static __device__ __forceinline__ int turn(int r) { return (sizeof(T) == 4 ? (r >> 2 & 3) << 2 : ((r & 3) | (r >> 1 & 4)) << 1) & (kRow - 1); }
    // the chunk of row r that this thread fetches
    __device__ __forceinline__ int chunk_of(int r) const
    {
        const int c = (threadIdx.x ^ (kAcross ? turn(r) : r)) & (kRow - 1);
        return kAcross && c * E >= width ? 0 : c;
    }

    // outputs first .. of `outs`; rows and chunks behind the last are others that are there
    __device__ __forceinline__ Side(const T* p, int64_t ld, int64_t first, int64_t outs) : base(p + (kAcross ? first : first * ld)), ld(ld), row(threadIdx.x / kRow), width((int)min(outs - first, (int64_t)B))
    {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int r = row + i * (kThreads / kRow);
            offset[i] = kAcross ? (int)((r * ld + chunk_of(r) * E) * (int)sizeof(T)) : (int)(min((int64_t)r, outs - 1 - first) * ld * (int)sizeof(T));
        }
    }
    __device__ __forceinline__ void fetch(Lds* to, int slab, int64_t K) const
    {
        if constexpr (kAcross) {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (int64_t)slab * kStep * ld), 0, 0x7fffffff, 0x27000);
            const int left = (int)min(K - (int64_t)slab * kStep, (int64_t)kStep);
            if (left == kStep)
#pragma unroll
                for (int i = 0; i < kLoads; i++) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to + i * kThreads, 16, offset[i], 0, 0, 0);
            else
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    const int r = row + i * (kThreads / kRow);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to + i * kThreads, 16, (int)((min(r, left - 1) * ld + chunk_of(r) * E) * (int)sizeof(T)), 0, 0, 0);
                }
        } else {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x27000);
            const int chunk = chunk_of(row), at = (int64_t)slab * kStep + chunk * E < K ? chunk * kChunk : 0;       // beyond the row's end its slab's first chunk
#pragma unroll
            for (int i = 0; i < kLoads; i++) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to + i * kThreads, 16, offset[i] + at, slab * kSlab, 0, 0);
        }
    }
    // zeros behind the end of the contraction, `left` places of the slab being before it (the last one's chunk of a row along the contraction ends in zeros)
    static __device__ __forceinline__ void clear(Chunk* in, int left)
    {
        for (int id = threadIdx.x; id < B * kChunks; id += kThreads)
            if (kAcross ? id / kRow >= left : ((id ^ (id / kRow)) & 7) >= (left + E - 1) / E) in[id] = Chunk{};
    }
    // What a lane feeds for outputs o .. o + 16 N - 1 of the tile at step c of the slab (f: of a feed of kF chunks)
    template <int N, int kF> static __device__ __forceinline__ void read(const Chunk* in, int o, int c, int f, Chunk (&to)[N][kF])
    {
        const int lane = threadIdx.x & 63;
        if constexpr (!kAcross) {
#pragma unroll
            for (int i = 0; i < N; i++) to[i][f] = in[(o + i * 16 + (lane & 15)) * kChunks + ((c * 4 + lane / 16) ^ (lane & 7))];
        } else if constexpr (sizeof(T) == 4) {
            const uint32_t* words = (const uint32_t*)in;
            const int r = c * 16 + lane / 16 * 4;                                            // and the three rows behind it, whose turn is the same
#pragma unroll
            for (int i = 0; i < N; i++)
#pragma unroll
                for (int q = 0; q < 4; q++) to[i][f][q] = words[((r + q) * kRow + ((o / E + i * 4 + (lane & 15) / 4) ^ turn(r))) * 4 + (lane & 3)];
        } else {
            // The compiler would wait for the next slab's loads before a transposing read, which it does not tell from what they write.  So the reads are written
            // out, two or four outputs' at a time with their own wait, while the products of those before are under way.
            static_assert(N % 2 == 0);
            const int r = lane / 16 * 8 + (lane & 15) / 4;                                   // and the row four further on, whose turn is the same
            const uint32_t start = (uint32_t)(uintptr_t)(const Lds*)in + r * kRow * kChunk + (lane & 1) * 8;
            constexpr int kHigh = 4 * kRow * kChunk;
            auto place = [&](int i) { return start + c * (32 * kRow * kChunk) + (((o / E + i * 2 + (lane & 3) / 2) ^ turn(r)) * kChunk); };
            typedef uint64_t Halves __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < N; i += N % 4 ? 2 : 4) {
                uint64_t l0, h0, l1, h1;
                if constexpr (N % 4 == 0) {
                    uint64_t l2, h2, l3, h3;
                    asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\tds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                                 "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\tds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                                 "s_waitcnt lgkmcnt(0)"
                                 : "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1), "=&v"(l2), "=&v"(h2), "=&v"(l3), "=&v"(h3)
                                 : "v"(place(i)), "v"(place(i + 1)), "v"(place(i + 2)), "v"(place(i + 3)), "n"(kHigh));
                    to[i + 2][f] = __builtin_bit_cast(Chunk, Halves{l2, h2});
                    to[i + 3][f] = __builtin_bit_cast(Chunk, Halves{l3, h3});
                } else
                    asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%6\n\tds_read_b64_tr_b16 %2, %5\n\tds_read_b64_tr_b16 %3, %5 offset:%6\n\t"
                                 "s_waitcnt lgkmcnt(0)"
                                 : "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1)
                                 : "v"(place(i)), "v"(place(i + 1)), "n"(kHigh));
                to[i][f] = __builtin_bit_cast(Chunk, Halves{l0, h0});
                to[i + 1][f] = __builtin_bit_cast(Chunk, Halves{l1, h1});
            }
        }
    }
};

template <class T, class O, int B, int WM, int WN, bool kAcrossX, bool kAcrossW>
__global__ __launch_bounds__(WM * WN * 64) void aligned_kernel(Tiles t, const T* x, int64_t ldx, const T* w, int64_t ldw, Out o, float* parts)
{
#ifdef __HIP_DEVICE_COMPILE__                                                  // the host's pass, which makes the launch, drops kernels with buffers and transposing reads
    constexpr int kThreads = WM * WN * 64, FM = B / WM / 16, FN = B / WN / 16, kStep = kSlab / sizeof(T), kStage = 2 * B * kChunks;
    typedef Side<T, kAcrossX, B, kThreads> X;
    typedef Side<T, kAcrossW, B, kThreads> W;
    extern __shared__ Chunk lds[];                                             // two stages of x and weight
    const Place p = place_of(t);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave % WM, wn = wave / WM;
    const int64_t m0 = (int64_t)p.m * B, n0 = (int64_t)p.n * B;
    const int first = (int)(p.split * t.slabs), last = (int)min((int64_t)((t.K + kStep - 1) / kStep), first + t.slabs);
    const X sx(x, ldx, m0, t.M);
    const W sw(w, ldw, n0, t.N);
    auto* base = (__attribute__((address_space(3))) Chunk*)lds + wave * 64;
    Acc acc[FN][FM] = {};
    if (first < last) {
        sx.fetch(base, first, t.K);
        sw.fetch(base + B * kChunks, first, t.K);
    }
    for (int s = first; s < last; s++) {
        const int stage = (s - first) & 1;
        // this slab has landed, and nobody reads the stage that is loaded next any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < last) {
            auto* to = base + (stage ^ 1) * kStage;
            sx.fetch(to, s + 1, t.K);
            sw.fetch(to + B * kChunks, s + 1, t.K);
        }
        Chunk* in = lds + stage * kStage;
        if (const int64_t left = t.K - (int64_t)s * kStep; left < kStep) {
            X::clear(in, (int)left);
            W::clear(in + B * kChunks, (int)left);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        constexpr int F = kFeed<T>;
#pragma unroll
        for (int c = 0; c < kChunks / 4; c += F) {
            // reads that wait for themselves come four outputs at a time, those of the next four while the products of these are under way
            constexpr int G = kAcrossW && FN > 4 ? 4 : FN;
            Chunk fx[FM][F];
#pragma unroll
            for (int f = 0; f < F; f++) X::template read<FM, F>(in, wm * (B / WM), c + f, f, fx);
#pragma unroll
            for (int i = 0; i < FN; i += G) {
                Chunk fw[G][F];
#pragma unroll
                for (int f = 0; f < F; f++) W::template read<G, F>(in + B * kChunks, wn * (B / WN) + i * 16, c + f, f, fw);
                products<T>(fw, fx, acc + i);
                if (G < FN) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    static_assert(WM * WN * kPutFloats<FN> * sizeof(float) <= 2 * kStage * sizeof(Chunk));
    put<O, FM, FN>(t, o, parts, p.split, m0 + wm * (B / WM), n0 + wn * (B / WN), acc, (float*)lds + wave * kPutFloats<FN>);
#endif
}

// ---- few tokens (single tokens of up to 64 streams): 16 FN outputs a workgroup, the contraction over its wavefronts.  Bound by the weights' way from
// memory: operands go to registers as the matrix instructions take them, several steps' loads at once, and the wavefronts' sums meet in LDS once.
template <class T, class O, int FM, int FN, int kW> __global__ __launch_bounds__(kW * 64) void few_kernel(Tiles t, const T* x, int64_t ldx, const T* w, int64_t ldw, Out o)
{
    constexpr int F = kFeed<T>, kStep = 64 * F, U = (FM + FN) * F > 4 ? 2 : 4, kPitch = FN * 16;      // bytes of a row a step
    __shared__ float sums[kW][FM * 16][kPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const Place p = place_of(t);
    const int64_t m0 = (int64_t)p.m * FM * 16, n0 = (int64_t)p.n * FN * 16, bytes = t.K * (int)sizeof(T);
    const char *px[FM], *pw[FN];
#pragma unroll
    for (int j = 0; j < FM; j++) px[j] = (const char*)(x + min(m0 + j * 16 + (lane & 15), t.M - 1) * ldx) + lane / 16 * 16;
#pragma unroll
    for (int i = 0; i < FN; i++) pw[i] = (const char*)(w + min(n0 + i * 16 + (lane & 15), t.N - 1) * ldw) + lane / 16 * 16;
    Acc acc[FN][FM] = {};
    struct { Chunk x[U][FM][F], w[U][FN][F]; } now, next;
    auto load = [&](int64_t k, auto& to) {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int f = 0; f < F; f++) {
                const int64_t at = k + (int64_t)u * kW * kStep + f * 64;
                const bool there = at + lane / 16 * 16 < bytes;                // rows are whole chunks
#pragma unroll
                for (int i = 0; i < FN; i++) to.w[u][i][f] = there ? *(const Chunk*)(pw[i] + at) : Chunk{};
#pragma unroll
                for (int j = 0; j < FM; j++) to.x[u][j][f] = there ? *(const Chunk*)(px[j] + at) : Chunk{};
            }
    };
    int64_t k = (int64_t)wave * kStep;
    if (k < bytes) load(k, now);
    for (; k < bytes; k += (int64_t)kW * kStep * U) {
        if (k + (int64_t)kW * kStep * U < bytes) load(k + (int64_t)kW * kStep * U, next);
#pragma unroll
        for (int u = 0; u < U; u++) products<T>(now.w[u], now.x[u], acc);
        now = next;
    }
#pragma unroll
    for (int j = 0; j < FM; j++)
#pragma unroll
        for (int i = 0; i < FN; i++) *(Acc*)&sums[wave][j * 16 + (lane & 15)][i * 16 + lane / 16 * 4] = acc[i][j];
    __syncthreads();
    for (int id = threadIdx.x; id < FM * 16 * FN * 4; id += kW * 64) {
        const int m = id / (FN * 4), n = id % (FN * 4) * 4;
        if (m0 + m >= t.M || n0 + n >= t.N) continue;
        Acc v = *(const Acc*)&sums[0][m][n];
#pragma unroll
        for (int i = 1; i < kW; i++) v += *(const Acc*)&sums[i][m][n];
        float z[4] = {v[0], v[1], v[2], v[3]};
        const Columns<O, 4> columns(o, n0 + n, t.N);
        Words<O, 4> r{};
        if (o.residual) r = residual_of<O, 4>(o, columns, m0 + m, t.N);
        finish<O, 4>(o, columns, m0 + m, t.N, z, r);
    }
}

// The splits' sums, added up in order, and what becomes of them.  Bound by memory (2107 x 1024, four splits of float32 sums: 9.3 us with a launch of its own)
template <class O> __global__ __launch_bounds__(256) void join_kernel(Tiles t, Out o, const float* parts)
{
    const int64_t quads = (t.N + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= t.M * quads) return;
    Acc v = *(const Acc*)(parts + id * 4);
    for (int s = 1; s < t.splits; s++) v += *(const Acc*)(parts + (s * t.M * quads + id) * 4);
    float z[4] = {v[0], v[1], v[2], v[3]};
    const Columns<O, 4> columns(o, id % quads * 4, t.N);
    Words<O, 4> r{};
    if (o.residual) r = residual_of<O, 4>(o, columns, id / quads, t.N);
    finish<O, 4>(o, columns, id / quads, t.N, z, r);
}

// Rows [R, C] of any alignment to rows of whole chunks, zeros behind the C: 16 bytes a thread.  Bound by memory.
template <class T> __global__ __launch_bounds__(256) void pad_kernel(const T* in, int64_t ld, int64_t R, int64_t C, Chunk* out, uint32_t chunks)
{
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, row = id / chunks, c = id % chunks;
    if (row < R) out[id] = take_chunk(in + row * ld, c * (kChunk / (int)sizeof(T)), C);
}

// The gradient's pass over what comes in: times the activation's slope (pre), rounded to T as the products' other operands are of that type (bfloat16:
// gradients 2.4e-3 off by norm, 1.7e-3 with outputs rounded alone), into rows of whole chunks (flat, `padded` elements apart), and its sums over 64 rows,
// unrounded, for the bias's gradient.  64 rows by 128 bfloat16 or 64 float32 values a workgroup.  Bound by memory: 16384 x 4096 in bfloat16 with GELU's slope 85 us, 4.75 TB/s (by tiles through LDS 109).
template <class T> __global__ __launch_bounds__(256) void slope_kernel(const T* in, int64_t ld, int64_t R, int64_t C, const T* pre, int act, T* flat, int64_t padded, float* sums, int64_t groups, bool vec)
{
    constexpr int V = 16 / sizeof(T), kRows = 4, kWide = 16 * V;
    __shared__ alignas(32) float part[4][kWide];
    const int64_t r0 = (int64_t)(blockIdx.x / groups) * 64 + threadIdx.x / 16, c = (int64_t)(blockIdx.x % groups) * kWide + (threadIdx.x & 15) * V;
    float sum[V] = {};
    if (c < C) {
        Words<T, V> g[kRows], z[kRows];
        auto fetch = [&](const T* p, Words<T, V>& to) {
            if (vec) to.load(p + c);
            else {
                const Chunk q = take_chunk(p, c, C);
                __builtin_memcpy(&to.w, &q, sizeof(q));
            }
        };
#pragma unroll
        for (int i = 0; i < kRows; i++) {
            const int64_t r = min(r0 + i * 16, R - 1);
            fetch(in + r * ld, g[i]);
            if (pre) fetch(pre + r * C, z[i]);
        }
#pragma unroll
        for (int i = 0; i < kRows; i++) {
            if (r0 + i * 16 >= R) break;
            float v[V];
#pragma unroll
            for (int k = 0; k < V; k++) v[k] = g[i].value(k);
            if (pre && act == SIG_ACT_SILU) {
#pragma unroll
                for (int k = 0; k < V; k++) v[k] *= slope_of<T>(z[i].value(k), SIG_ACT_SILU);
            } else if (pre)
#pragma unroll
                for (int k = 0; k < V; k++) v[k] *= slope_of<T>(z[i].value(k), SIG_ACT_GELU);
#pragma unroll
            for (int k = 0; k < V; k++) sum[k] += v[k];
            if (flat) store_words<T, V>(flat + (r0 + i * 16) * padded + c, v);
        }
    }
    if (!sums) return;
#pragma unroll
    for (int k = 0; k < V; k++) {
        sum[k] += __shfl_xor(sum[k], 16);
        sum[k] += __shfl_xor(sum[k], 32);
    }
    if ((threadIdx.x & 63) < 16) store_words<float, V>(&part[threadIdx.x / 64][(threadIdx.x & 15) * V], sum);
    __syncthreads();
    const int64_t n = (int64_t)(blockIdx.x % groups) * kWide + threadIdx.x;
    if (threadIdx.x < kWide && n < C) sums[blockIdx.x / groups * C + n] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

template <class T> __global__ __launch_bounds__(1024) void bias_kernel(const float* sums, int64_t rows, int64_t N, T* grad_bias)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const float s = sum_rows(sums + min(c, N - 1), rows, N);
    if (threadIdx.x < 64 && c < N) grad_bias[c] = from_float<T>(s);
}

size_t parts_bytes(const Tiles& t) { return t.splits > 1 ? (size_t)t.splits * t.M * ((t.N + 3) / 4 * 4) * 4 : 0; }
template <class T, class O, int kSize, int WM, int WN, bool kAcrossX, bool kAcrossW> hipError_t launch(const Tiles& t, const T* x, int64_t ldx, const T* w, int64_t ldw, const Out& o, float* parts, uint32_t blocks, hipStream_t stream)
{
    constexpr int kLds = 2 * 2 * kSize * kSlab;                                // two stages of both operands
    auto kernel = aligned_kernel<T, O, kSize, WM, WN, kAcrossX, kAcrossW>;
    if (kLds > 64 * 1024) {
        hipError_t err = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (err != hipSuccess) return err;
    }
    kernel<<<blocks, WM * WN * 64, kLds, stream>>>(t, x, ldx, w, ldw, o, parts);
    return hipGetLastError();
}

// whole chunks only; a tile's rows and the contraction are reached by 32-bit offsets
bool aligned_rows(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t K, int64_t e)
{
    return (uintptr_t)x % 16 == 0 && (uintptr_t)w % 16 == 0 && ldx * e % 16 == 0 && ldw * e % 16 == 0 && K * e % 16 == 0 && K > 0 &&
           256 * std::max(ldx, ldw) * e + K * e < (1ll << 31);
}

// The launches of a product, whose tiles the caller has found launchable.  aligned: whether aligned_rows holds (operands across: the caller has looked at them).
template <class T, class O, bool kAcrossX = false, bool kAcrossW = false>
hipError_t product(const Tiles& t, bool aligned, const T* x, int64_t ldx, const T* w, int64_t ldw, Out o, float* parts, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(O);
    auto fits = [&](const void* p) { return (uintptr_t)p % 16 == 0; };
    o.vec = t.N % V == 0 && o.residual_stride % V == 0 && fits(o.bias) && fits(o.residual) && fits(o.y) && fits(o.pre);
    const uint32_t blocks = (uint32_t)t.blocks();
    hipError_t err = hipSuccess;
    if (t.few) {
        if constexpr (!kAcrossX && !kAcrossW) {
            auto go = [&](auto kernel) { kernel<<<blocks, kFewThreads, 0, stream>>>(t, x, ldx, w, ldw, o); };
            t.tile == 1 ? go(few_kernel<T, O, 1, 1, kFewThreads / 64>) : t.tile == 2 ? go(few_kernel<T, O, 2, 2, kFewThreads / 64>) : go(few_kernel<T, O, 4, 2, kFewThreads / 64>);
            err = hipGetLastError();
        }
    } else if (!aligned) {
        product_kernel<T, O><<<blocks, 256, 0, stream>>>(t, x, ldx, w, ldw, o, parts);
        err = hipGetLastError();
    } else if (t.tile == 256) {
        if constexpr (sizeof(T) < 4) err = launch<T, O, 256, 4, 2, kAcrossX, kAcrossW>(t, x, ldx, w, ldw, o, parts, blocks, stream);
    } else if (t.tile == 128) err = launch<T, O, 128, 2, 2, kAcrossX, kAcrossW>(t, x, ldx, w, ldw, o, parts, blocks, stream);
    else err = launch<T, O, 64, 2, 2, kAcrossX, kAcrossW>(t, x, ldx, w, ldw, o, parts, blocks, stream);
    if (err != hipSuccess || t.splits == 1) return err;
    join_kernel<O><<<(uint32_t)t.joins(), 256, 0, stream>>>(t, o, parts);
    return hipGetLastError();
}

int bytes_of(int64_t dtype) { return dtype == SIG_F32 ? 4 : dtype == SIG_BF16 ? 2 : 1; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Rows that the aligned kernels read as they lie
bool whole(const void* p, int64_t ld, int64_t cols, int64_t e) { return (uintptr_t)p % 16 == 0 && ld * e % 16 == 0 && cols * e % 16 == 0 && 256 * ld * e < (1ll << 30); }

// Workgroups of the copy of R rows of C values of e bytes into whole chunks
int64_t pad_blocks(int64_t R, int64_t C, int64_t e) { return (R * ((C * e + kChunk - 1) / kChunk) + 255) / 256; }
template <class T> hipError_t pad(const T* in, int64_t ld, int64_t R, int64_t C, T* out, hipStream_t stream)
{
    const int64_t blocks = pad_blocks(R, C, sizeof(T));
    if (blocks) pad_kernel<T><<<(uint32_t)blocks, 256, 0, stream>>>(in, ld, R, C, (Chunk*)out, (uint32_t)((C * (int)sizeof(T) + kChunk - 1) / kChunk));
    return hipGetLastError();
}

// What a forward call keeps in its workspace, in bytes from its start: x and the weight in rows of whole chunks where they are not and the launch's model says
// that the copies (a launch each, read and written at 3 TB/s) cost less than they gain, and the sums of splits.  float32 5000 x 1001 to 1001: 112 us with
// copies, 139 without; 600 x 1554 to 640 stays without (24 us; the model puts its copies at 13).
struct Ahead {
    bool pad_x, pad_w, aligned;
    int64_t padK;
    Tiles tiles;
    size_t x, w, parts, all;
};
Ahead ahead_of(const sig_linear_args& a)
{
    const int e = bytes_of(a.dtype);
    Ahead k{};
    k.padK = a.K;
    k.aligned = aligned_rows(a.x, a.x_stride, a.weight, a.K, a.K, e);
    k.tiles = tiles_of(a.M, a.N, a.K, e, k.aligned);
    size_t at = 0;
    if (const int64_t padK = round_up(a.K, kChunk / e); !k.aligned && 256 * padK * e < (1ll << 30)) {
        const bool x = !whole(a.x, a.x_stride, a.K, e), w = !whole(a.weight, a.K, a.K, e);
        const Tiles u = tiles_of(a.M, a.N, padK, e, true);
        if (u.us + (x ? 4.0 + 2.0 * a.M * padK * e / 3e6 : 0.0) + (w ? 4.0 + 2.0 * a.N * padK * e / 3e6 : 0.0) < k.tiles.us &&
            (!x || launchable(pad_blocks(a.M, a.K, e), 256)) && (!w || launchable(pad_blocks(a.N, a.K, e), 256))) {
            k.pad_x = x;
            k.pad_w = w;
            k.aligned = true;
            k.padK = padK;
            k.tiles = u;
            k.w = x ? (size_t)round_up(a.M * padK * e, 256) : 0;
            at = k.w + (w ? (size_t)round_up(a.N * padK * e, 256) : 0);
        }
    }
    k.parts = at;
    k.all = at + parts_bytes(k.tiles);
    if (k.all) k.all += 16;                                                    // for a workspace whose start is not aligned
    return k;
}

// What the gradient keeps in its workspace: the gradient that comes in where it is multiplied by a slope or not whole chunks, and copies of the weight and
// of x in rows of whole chunks where theirs are not
struct Keep {
    bool pad_x, pad_w;
    int64_t padN, padK;
    Tiles to_x, to_w;                   // of the products that give the gradients of x and of the weight
    size_t flat, x, w, sums, parts, all;
};
Keep keep_of(const sig_linear_args& a)
{
    Keep k;
    const int e = bytes_of(a.dtype);
    k.pad_x = !whole(a.x, a.x_stride, a.K, e);
    k.pad_w = !whole(a.weight, a.K, a.K, e);
    k.padN = round_up(a.N, kChunk / e);
    k.padK = round_up(a.K, kChunk / e);
    size_t at = 0;
    auto take = [&](int64_t n) {
        size_t was = at;
        at += (size_t)round_up(n, 256);
        return was;
    };
    k.flat = take(a.M * k.padN * e);
    k.x = take(k.pad_x ? a.M * k.padK * e : 0);
    k.w = take(k.pad_w ? a.N * k.padK * e : 0);
    k.sums = take((a.M + 63) / 64 * a.N * 4);
    k.to_x = tiles_of(a.M, a.K, a.N, e, true, false);
    k.to_w = tiles_of(a.N, a.K, a.M, e, true, false);
    k.parts = take((int64_t)std::max(parts_bytes(k.to_x), parts_bytes(k.to_w)));
    k.all = at + 16;                                                           // for a workspace whose start is not aligned
    return k;
}

// Workgroups of the pass over the incoming gradient: 64 rows of 256 bytes each
int64_t slope_groups(int64_t C, int64_t e) { return (C * e + 255) / 256; }
int64_t slope_blocks(int64_t R, int64_t C, int64_t e) { return (R + 63) / 64 * slope_groups(C, e); }
template <class T> hipError_t slopes(const T* in, int64_t ld, int64_t R, int64_t C, const T* pre, int act, T* flat, int64_t padded, float* sums, hipStream_t stream)
{
    const int64_t blocks = slope_blocks(R, C, sizeof(T));
    const bool vec = C * sizeof(T) % 16 == 0 && ld * sizeof(T) % 16 == 0 && (uintptr_t)in % 16 == 0 && (uintptr_t)pre % 16 == 0;
    if (blocks) slope_kernel<T><<<(uint32_t)blocks, 256, 0, stream>>>(in, ld, R, C, pre, act, flat, padded, sums, slope_groups(C, sizeof(T)), vec);
    return hipGetLastError();
}

template <class T> hipError_t backward_of(const sig_linear_args& a, const T* gy, int64_t ld, const T* pre, T* gx, T* gw, T* gb, char* ws, hipStream_t stream)
{
    const Keep k = keep_of(a);
    const int64_t e = sizeof(T);
    if (256 * std::max(k.padN, k.padK) * e >= (1ll << 30)) return kTooManyThreads;        // rows of a tile are reached by 32-bit offsets
    if (a.act == SIG_ACT_NONE) pre = nullptr;
    ws += -(uintptr_t)ws & 15;
    T *flat = (T*)(ws + k.flat), *x = (T*)(ws + k.x), *w = (T*)(ws + k.w);
    float *sums = (float*)(ws + k.sums), *parts = (float*)(ws + k.parts);
    gx = a.M ? gx : nullptr;
    const bool copy = (gx || gw) && (pre || !whole(gy, ld, a.N, e));
    const T *g = copy ? flat : gy, *px = k.pad_x ? x : (const T*)a.x, *pw = k.pad_w ? w : (const T*)a.weight;
    const int64_t ldg = copy ? k.padN : ld;
    if (((copy || gb) && !launchable(slope_blocks(a.M, a.N, e), 256)) || (gx && !(k.to_x.launchable() && (!k.pad_w || launchable(pad_blocks(a.N, a.K, e), 256)))) ||
        (gw && !(k.to_w.launchable() && (!k.pad_x || launchable(pad_blocks(a.M, a.K, e), 256)))))
        return kTooManyThreads;
    hipError_t err = hipSuccess;
    if (copy || gb) err = slopes<T>(gy, ld, a.M, a.N, pre, (int)a.act, copy ? flat : nullptr, k.padN, gb ? sums : nullptr, stream);
    if (err == hipSuccess && gb) {
        bias_kernel<T><<<(uint32_t)((a.N + 63) / 64), 1024, 0, stream>>>(sums, (a.M + 63) / 64, a.N, gb);
        err = hipGetLastError();
    }
    Out o{};
    if (err == hipSuccess && gx) {
        if (k.pad_w) err = pad((const T*)a.weight, a.K, a.N, a.K, w, stream);
        o.y = gx;
        if (err == hipSuccess) err = product<T, T, false, true>(k.to_x, true, g, ldg, pw, k.pad_w ? k.padK : a.K, o, parts, stream);
    }
    if (err == hipSuccess && gw) {
        if (k.pad_x) err = pad((const T*)a.x, a.x_stride, a.M, a.K, x, stream);
        o.y = gw;
        if (err == hipSuccess) err = product<T, T, true, true>(k.to_w, true, g, ldg, px, k.pad_x ? k.padK : a.x_stride, o, parts, stream);
    }
    return err;
}

template <class T, class O> hipError_t forward_of(const sig_linear_args& a, void* y, void* pre, char* ws, hipStream_t stream)
{
    const Out o{a.bias, a.residual, a.residual_stride, a.x_scale, a.weight_scale, y, pre, (int)a.act, false};
    const Ahead k = ahead_of(a);
    if (!k.tiles.launchable()) return kTooManyThreads;
    ws += -(uintptr_t)ws & 15;
    T *x = (T*)(ws + k.x), *w = (T*)(ws + k.w);
    hipError_t err = hipSuccess;
    if (k.pad_x) err = pad((const T*)a.x, a.x_stride, a.M, a.K, x, stream);
    if (err == hipSuccess && k.pad_w) err = pad((const T*)a.weight, a.K, a.N, a.K, w, stream);
    if (err != hipSuccess) return err;
    return product<T, O>(k.tiles, k.aligned, k.pad_x ? x : (const T*)a.x, k.pad_x ? k.padK : a.x_stride, k.pad_w ? w : (const T*)a.weight, k.pad_w ? k.padK : a.K, o, (float*)(ws + k.parts), stream);
}

}  // namespace

size_t linear_forward_workspace(const sig_linear_args& a) { return ahead_of(a).all; }
hipError_t linear_forward(const sig_linear_args& a, void* y, void* pre, void* workspace, hipStream_t stream)
{
    char* ws = (char*)workspace;
    if (a.dtype == SIG_BF16) return forward_of<bf16, bf16>(a, y, pre, ws, stream);
    if (a.dtype == SIG_F32) return forward_of<float, float>(a, y, pre, ws, stream);
    return a.out_dtype == SIG_BF16 ? forward_of<e4m3, bf16>(a, y, pre, ws, stream) : forward_of<e4m3, float>(a, y, pre, ws, stream);
}
size_t linear_backward_workspace(const sig_linear_args& a) { return keep_of(a).all; }
hipError_t linear_backward(const sig_linear_args& a, const void* grad_y, int64_t gy_stride, const void* pre, void* grad_x, void* grad_weight, void* grad_bias,
                           void* workspace, hipStream_t stream)
{
    char* ws = (char*)workspace;
    return a.dtype == SIG_BF16 ? backward_of<bf16>(a, (const bf16*)grad_y, gy_stride, (const bf16*)pre, (bf16*)grad_x, (bf16*)grad_weight, (bf16*)grad_bias, ws, stream)
                               : backward_of<float>(a, (const float*)grad_y, gy_stride, (const float*)pre, (float*)grad_x, (float*)grad_weight, (float*)grad_bias, ws, stream);
}

}  // namespace sig
