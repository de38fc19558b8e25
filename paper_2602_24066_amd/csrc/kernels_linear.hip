// Matrix products y = f(x weight^T + bias) + residual over rows of tokens, and their gradient.
//
// One kernel shape for all types: a tile of outputs, both operands row by row along the contraction, 128 bytes of it (a slab) a step, 16 bytes (a
// chunk) an access.  A chunk of 16 rows is what a lane feeds to the matrix instructions: 8 bfloat16 (16x16x32), 4 float32 (four 16x16x4, whose
// order along the contraction is the same for both operands and so does not matter), or, two chunks together, 32 e4m3 (16x16x128).  The weight's rows are
// the instruction's first operand: a lane then holds four neighbouring outputs of one token.
// LDS: row r keeps chunk c at place c ^ (r & 7), so that eight rows' chunks lie in different banks.
// Few tiles and a long contraction: the contraction is split over workgroups, whose float32 sums a second kernel adds up in order.
// The gradient brings both of its products to the same form by transposing what lies the other way.
#include <algorithm>
#include <type_traits>

#include "layer.hpp"

namespace sig {
namespace {

typedef float Acc __attribute__((ext_vector_type(4)));
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef int Int8 __attribute__((ext_vector_type(8)));

constexpr int kSlab = 128, kChunk = 16, kChunks = kSlab / kChunk;      // bytes; bytes; chunks of a slab

struct Out {                            // what becomes of a sum
    const void *bias, *residual;
    int64_t residual_stride;
    const float *x_scale, *weight_scale;
    void *y, *pre;
    int act;
    bool vec;                           // four neighbouring outputs are one access everywhere
};

// f and f': the normal distribution's Phi by the error function
__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == SIG_ACT_SILU) return z * sigmoid(z);
    if (act == SIG_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}
__device__ __forceinline__ float slope_of(float z, int act)
{
    if (act == SIG_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * fast_exp(-0.5f * z * z) * 0.39894228f;
}

template <class O> __device__ __forceinline__ void finish(const Out& o, int64_t m, int64_t n, int64_t N, Acc v)
{
    const bool all = n + 4 <= N;
    const int64_t at = m * N + n;
    float z[4] = {v[0], v[1], v[2], v[3]}, b[4], r[4];
    auto take = [&](const O* p, float* to) {
        if (o.vec && all) {
            const Pack<O, 4> q = *(const Pack<O, 4>*)p;
#pragma unroll
            for (int j = 0; j < 4; j++) to[j] = to_float(q.v[j]);
        } else
#pragma unroll
            for (int j = 0; j < 4; j++) to[j] = n + j < N ? to_float(p[j]) : 0.0f;
    };
    auto give = [&](O* p, const float* from) {
        if (o.vec && all) {
            Pack<O, 4> q;
#pragma unroll
            for (int j = 0; j < 4; j++) q.v[j] = from_float<O>(from[j]);
            *(Pack<O, 4>*)p = q;
        } else
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (n + j < N) p[j] = from_float<O>(from[j]);
    };
    const float xs = o.x_scale ? o.x_scale[m] : 1.0f;
    if (o.x_scale || o.weight_scale)
#pragma unroll
        for (int j = 0; j < 4; j++) z[j] = z[j] * xs * (o.weight_scale ? o.weight_scale[min(n + j, N - 1)] : 1.0f);
    if (o.bias) {
        take((const O*)o.bias + n, b);
#pragma unroll
        for (int j = 0; j < 4; j++) z[j] += b[j];
    }
    if (o.pre) give((O*)o.pre + at, z);
#pragma unroll
    for (int j = 0; j < 4; j++) z[j] = act_of(z[j], o.act);
    if (o.residual) {
        take((const O*)o.residual + m * o.residual_stride + n, r);
#pragma unroll
        for (int j = 0; j < 4; j++) z[j] += r[j];
    }
    give((O*)o.y + at, z);
}

template <class T> struct alignas(sizeof(T)) Loose { T v[kChunk / sizeof(T)]; } __attribute__((packed));

// 16 bytes of a row from element k on, zeros from element K on
template <class T> __device__ __forceinline__ Chunk take_chunk(const T* row, int64_t k, int64_t K, bool aligned)
{
    constexpr int E = kChunk / sizeof(T);
    Chunk c;
    if (k + E <= K) {
        if (aligned) return *(const Chunk*)(row + k);
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

// Sum over the contraction of 16 x 16 products: one chunk a lane of each operand (e4m3: two)
template <class T> __device__ __forceinline__ Acc products(const Chunk* w, const Chunk* x, Acc acc)
{
    if constexpr (std::is_same_v<T, bf16>) {
        Bf8 a, b;
        __builtin_memcpy(&a, w, 16);
        __builtin_memcpy(&b, x, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
    } else if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int j = 0; j < 4; j++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((*w)[j]), __uint_as_float((*x)[j]), acc, 0, 0, 0);
        return acc;
    } else {
        Int8 a, b;
        __builtin_memcpy(&a, w, 32);
        __builtin_memcpy(&b, x, 32);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);     // block scales of one
    }
}
template <class T> constexpr int kFeed = std::is_same_v<T, e4m3> ? 2 : 1;       // chunks of a row that a step takes

struct Tiles { int64_t M, N, K; int m, n, splits; int64_t slabs; };            // tiles along m and n; slabs of a split

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

constexpr int kTile = 128;

// A workgroup's tile is 128 tokens by 128 outputs, 64 by 64 a wavefront.
template <class T, class O> __global__ __launch_bounds__(256) void product_kernel(Tiles t, const T* x, int64_t ldx, const T* w, int64_t ldw, bool aligned, Out o, float* parts)
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
            rx[i] = take_chunk(x + min(m0 + row, t.M - 1) * ldx, e, last, aligned);
            rw[i] = take_chunk(w + min(n0 + row, t.N - 1) * ldw, e, last, aligned);
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
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = products<T>(fw[i], fx[j], acc[i][j]);
        }
        if (more) keep(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int64_t m = m0 + wm * 64 + j * 16 + (lane & 15);
        if (m >= t.M) continue;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t n = n0 + wn * 64 + i * 16 + (lane / 16) * 4;
            if (n >= t.N) continue;
            if (t.splits > 1) *(Acc*)(parts + ((int64_t)p.split * t.M + m) * ((t.N + 3) / 4 * 4) + n) = acc[i][j];
            else finish<O>(o, m, n, t.N, acc[i][j]);
        }
    }
}

// The splits' sums, added up in order, and what becomes of them
template <class O> __global__ __launch_bounds__(256) void join_kernel(Tiles t, Out o, const float* parts)
{
    const int64_t quads = (t.N + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= t.M * quads) return;
    Acc v = *(const Acc*)(parts + id * 4);
    for (int s = 1; s < t.splits; s++) v += *(const Acc*)(parts + (s * t.M * quads + id) * 4);
    finish<O>(o, id / quads, id % quads * 4, t.N, v);
}

// [R, C] to [C, padded R], zeros behind R.  pre: the gradient that comes in is multiplied by the activation's slope first, rounded to T, and kept
// in its own order too (flat); sums: its sums over the rows of a tile, before rounding, for the bias's gradient.
template <class T> __global__ __launch_bounds__(256) void turn_kernel(const T* in, int64_t ld, int64_t R, int64_t C, const T* pre, int act, T* flat, T* turned, int64_t padded,
                                                                       float* sums, int64_t tiles_c)
{
    __shared__ T tile[64][64 + 4 / sizeof(T)];
    __shared__ float part[4][64];
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * 64, c0 = (int64_t)(blockIdx.x % tiles_c) * 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int64_t c = c0 + lane;
    float sum = 0.0f;
    for (int i = wave; i < 64; i += 4) {
        const int64_t r = r0 + i;
        float v = 0.0f;
        if (r < R && c < C) {
            v = to_float(in[r * ld + c]);
            if (pre) {
                v *= slope_of(to_float(pre[r * C + c]), act);
                if (flat) flat[r * C + c] = from_float<T>(v);
            }
            sum += v;
        }
        tile[i][lane] = from_float<T>(v);
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (sums && wave == 0 && c < C) sums[blockIdx.x / tiles_c * C + c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    if (turned)
        for (int i = wave; i < 64; i += 4)
            if (c0 + i < C && r0 + lane < padded) turned[(c0 + i) * padded + r0 + lane] = tile[lane][i];
}

template <class T> __global__ __launch_bounds__(1024) void bias_kernel(const float* sums, int64_t rows, int64_t N, T* grad_bias)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const float s = sum_rows(sums + min(c, N - 1), rows, N);
    if (threadIdx.x < 64 && c < N) grad_bias[c] = from_float<T>(s);
}

Tiles tiles_of(int64_t M, int64_t N, int64_t K, int e)
{
    Tiles t{M, N, K, (int)((M + kTile - 1) / kTile), (int)((N + kTile - 1) / kTile), 1, 0};
    const int64_t slabs = std::max<int64_t>(1, (K * e + kSlab - 1) / kSlab), tiles = (int64_t)t.m * t.n;
    int64_t splits = 1;
    if (tiles && tiles < 256) splits = std::max<int64_t>(1, std::min<int64_t>({512 / tiles, slabs / 8, 32}));
    t.slabs = (slabs + splits - 1) / splits;
    t.splits = (int)((slabs + t.slabs - 1) / t.slabs);
    return t;
}
size_t parts_bytes(const Tiles& t) { return t.splits > 1 ? (size_t)t.splits * t.M * ((t.N + 3) / 4 * 4) * 4 : 0; }

template <class T, class O> hipError_t product(const Tiles& t, const T* x, int64_t ldx, const T* w, int64_t ldw, Out o, float* parts, hipStream_t stream)
{
    const int64_t blocks = (int64_t)t.m * t.n * t.splits, e = sizeof(T);
    if (!launchable(blocks, 256)) return kTooManyThreads;
    const bool aligned = (uintptr_t)x % 16 == 0 && (uintptr_t)w % 16 == 0 && ldx * e % 16 == 0 && ldw * e % 16 == 0;
    const int q = 4 * sizeof(O);
    auto fits = [&](const void* p) { return (uintptr_t)p % q == 0; };
    o.vec = t.N % 4 == 0 && o.residual_stride % 4 == 0 && fits(o.bias) && fits(o.residual) && fits(o.y) && fits(o.pre);
    product_kernel<T, O><<<(uint32_t)blocks, 256, 0, stream>>>(t, x, ldx, w, ldw, aligned, o, parts);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || t.splits == 1) return err;
    const int64_t joins = (t.M * ((t.N + 3) / 4) + 255) / 256;
    if (!launchable(joins, 256)) return kTooManyThreads;
    join_kernel<O><<<(uint32_t)joins, 256, 0, stream>>>(t, o, parts);
    return hipGetLastError();
}

int bytes_of(int64_t dtype) { return dtype == SIG_F32 ? 4 : dtype == SIG_BF16 ? 2 : 1; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// What the gradient keeps in its workspace, in bytes from its start
struct Keep {
    Tiles gx, gw;                       // grad_x = g weight, contraction N; grad_weight = g^T x, contraction M
    int64_t padN, padM;
    size_t flat, turned_g, turned_w, turned_x, sums, parts, all;
};
Keep keep_of(const sig_linear_args& a)
{
    Keep k;
    const int e = bytes_of(a.dtype);
    k.padN = round_up(a.N, 64);
    k.padM = round_up(a.M, 64);
    k.gx = tiles_of(a.M, a.K, a.N, e);
    k.gw = tiles_of(a.N, a.K, a.M, e);
    size_t at = 0;
    auto take = [&](int64_t n) {
        size_t was = at;
        at += (size_t)round_up(n, 256);
        return was;
    };
    k.flat = take(a.act ? a.M * a.N * e : 0);
    k.turned_g = take(a.N * k.padM * e);
    k.turned_w = take(a.K * k.padN * e);
    k.turned_x = take(a.K * k.padM * e);
    k.sums = take((a.M + 63) / 64 * a.N * 4);
    k.parts = take((int64_t)std::max(parts_bytes(k.gx), parts_bytes(k.gw)));
    k.all = at;
    return k;
}

template <class T> hipError_t turn(const T* in, int64_t ld, int64_t R, int64_t C, const T* pre, int act, T* flat, T* turned, int64_t padded, float* sums, hipStream_t stream)
{
    const int64_t tiles_c = (C + 63) / 64, blocks = (R + 63) / 64 * tiles_c;
    if (!launchable(blocks, 256)) return kTooManyThreads;
    if (blocks) turn_kernel<T><<<(uint32_t)blocks, 256, 0, stream>>>(in, ld, R, C, pre, act, flat, turned, padded, sums, tiles_c);
    return hipGetLastError();
}

template <class T> hipError_t backward_of(const sig_linear_args& a, const T* gy, int64_t ld, const T* pre, T* gx, T* gw, T* gb, char* ws, hipStream_t stream)
{
    const Keep k = keep_of(a);
    if (a.act == SIG_ACT_NONE) pre = nullptr;
    T *flat = (T*)(ws + k.flat), *turned_g = (T*)(ws + k.turned_g), *turned_w = (T*)(ws + k.turned_w), *turned_x = (T*)(ws + k.turned_x);
    float *sums = (float*)(ws + k.sums), *parts = (float*)(ws + k.parts);
    hipError_t err = hipSuccess;
    if (pre || gw || gb) err = turn<T>(gy, ld, a.M, a.N, pre, (int)a.act, gx ? flat : nullptr, gw ? turned_g : nullptr, k.padM, gb ? sums : nullptr, stream);
    if (err == hipSuccess && gb) {
        bias_kernel<T><<<(uint32_t)((a.N + 63) / 64), 1024, 0, stream>>>(sums, (a.M + 63) / 64, a.N, gb);
        err = hipGetLastError();
    }
    if (err == hipSuccess && gx && a.M) {
        err = turn<T>((const T*)a.weight, a.K, a.N, a.K, nullptr, 0, nullptr, turned_w, k.padN, nullptr, stream);
        Out o{};
        o.y = gx;
        if (err == hipSuccess) err = product<T, T>(k.gx, pre ? flat : gy, pre ? a.N : ld, turned_w, k.padN, o, parts, stream);
    }
    if (err == hipSuccess && gw) {
        err = turn<T>((const T*)a.x, a.x_stride, a.M, a.K, nullptr, 0, nullptr, turned_x, k.padM, nullptr, stream);
        Out o{};
        o.y = gw;
        if (err == hipSuccess) err = product<T, T>(k.gw, turned_g, k.padM, turned_x, k.padM, o, parts, stream);
    }
    return err;
}

template <class T, class O> hipError_t forward_of(const sig_linear_args& a, void* y, void* pre, float* parts, hipStream_t stream)
{
    const Out o{a.bias, a.residual, a.residual_stride, a.x_scale, a.weight_scale, y, pre, (int)a.act, false};
    return product<T, O>(tiles_of(a.M, a.N, a.K, sizeof(T)), (const T*)a.x, a.x_stride, (const T*)a.weight, a.K, o, parts, stream);
}

}  // namespace

size_t linear_forward_workspace(const sig_linear_args& a) { return parts_bytes(tiles_of(a.M, a.N, a.K, bytes_of(a.dtype))); }
hipError_t linear_forward(const sig_linear_args& a, void* y, void* pre, void* workspace, hipStream_t stream)
{
    float* parts = (float*)workspace;
    if (a.dtype == SIG_BF16) return forward_of<bf16, bf16>(a, y, pre, parts, stream);
    if (a.dtype == SIG_F32) return forward_of<float, float>(a, y, pre, parts, stream);
    return a.out_dtype == SIG_BF16 ? forward_of<e4m3, bf16>(a, y, pre, parts, stream) : forward_of<e4m3, float>(a, y, pre, parts, stream);
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
