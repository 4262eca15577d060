// Softmax cross entropy of tokens over a large vocabulary, and its gradient,
// behind the C ABI of include/hscale.h, without keeping the logits:
//
//   l_tv = x_t . w_v,  lse_t = log sum_v exp(l_tv),  loss_t = lse_t - l_t,target
//   g_tv = weight_t (exp(l_tv - lse_t) - [v = target]),  dX = g W,  dW = g^T X
//
// The loss takes one pass of matrix products whose tiles end as a maximum and
// a sum of exponentials per token; the gradient computes the logits again, a
// piece of the vocabulary at a time, and only that piece of g is held.  Of few
// tokens and words the logits go through memory, so that k can be split.
//
// g meets the products as two bf16 parts, the second what the rounding of the
// first left: within 2^-17 of it.  In one part its rounding errs alike in all of
// a row's terms wherever the softmax is not spread thin, by up to 0.4 of what
// the one rounding of dX and dW to bf16 errs.  Both parts multiply the same W
// and X, one after the other into the same sums, which is twice the matrix work
// of the two products.  The largest weight c stays out of the parts, whose
// range then does not depend on it:
//
//   h_tv = weight_t / c (exp(l_tv - lse_t) - [v = target]), in two parts,
//   dX = c (h W),  dW = c (h^T X).

#include "checks.h"
#include "matmul.h"

#include <algorithm>

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int64_t kMaxWidth = (int64_t)1 << 21;   // of a token's vector
constexpr int64_t kMaxTokens = (int64_t)1 << 24;
constexpr int64_t kMaxVocab = (int64_t)1 << 24;
constexpr int64_t kMaxLogits = (int64_t)1 << 38;  // one launch's tiles: below 2^32 threads


__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// (maximum, sum of exponentials relative to it) of two parts; a part without
// terms is (-inf, 0).
__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    if (m == -INFINITY) return make_float2(m, a.y + b.y);  // keeps the NaN of a part that has one
    return make_float2(m, a.y * exp_of(a.x - m) + b.y * exp_of(b.x - m));
}

// The two bf16 values of a word.
__device__ __forceinline__ float low_half(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_half(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

struct LogitArgs {
    Operand W, X;            // [vocab, d], [tokens, d]
    const int64_t *target;   // [tokens]
    unsigned mtiles;
    // loss
    float2 *parts;           // [mtiles, tokens]
    float *at;               // [tokens]: the target's logit
    // gradient: vocabulary from v0 on
    int64_t v0, vocab;       // of the whole
    const float *lse;
    const float *factor;     // [tokens]: weight_t / c, 0 if not scored
    uint16_t *g;             // [2, tokens, ldg]: the parts
    int64_t ldg;
};

// A tile of words x tokens, reduced over its words where it lies: per token a
// maximum and a sum in registers, then over lanes and waves.  Words are the
// tile's rows, so that a lane holds 64 of one token's.  2040 tokens of 4096 over
// 32003 words: 453 to 477 us, 1.18 to 1.12 PFLOP/s (MFMA 0.6 busy); 8192 over
// 128000: 6.8 to 7.0 ms, 1.25 PFLOP/s: the product, at the clock the chip's power
// leaves it.
template <class T>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void loss_tile_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x, gridDim.x, a.mtiles, mt, nt);
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    Acc<T> acc;
    acc.clear();
    tile_product<T, Along, Along>(acc, lds, a.W, m0, a.X, n0, 0, a.X.k);
    const Place<T> at;
    float2 *red = reinterpret_cast<float2 *>(lds);  // [kWM][kBN]
    const int words = a.vocab - m0 < T::kBM ? (int)(a.vocab - m0) : T::kBM;
    const int first = at.m(0, 0);  // element (i, e) is word first + 32 i + 8 (e / 4) + e % 4
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) {
        const int64_t t = n0 + at.n(j);
        const int64_t y = t < a.X.rows ? a.target[t] - m0 : -1;
        const int own = y >= 0 && y < words ? (int)y - first : -1;
        float2 p = make_float2(-INFINITY, 0.0f);
        float hit = 0.0f;
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int k = 32 * i + 8 * (e >> 2) + (e & 3);
                if (k < words - first) p.x = fmaxf(p.x, acc.v[i][j][e]);
                if (k == own) hit = acc.v[i][j][e];
            }
        if (own >= 0 && (own & 4) == 0 && own < 32 * T::kMI) a.at[t] = hit;  // the one lane that holds it
        const float base = p.x == -INFINITY ? 0.0f : p.x;  // logits of -inf alone add nothing
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int k = 32 * i + 8 * (e >> 2) + (e & 3);
                if (k < words - first) p.y += exp_of(acc.v[i][j][e] - base);
            }
        const float2 o = make_float2(__shfl_xor(p.x, 32, 64), __shfl_xor(p.y, 32, 64));
        p = join(p, o);
        if (at.lane < 32) red[at.wm * T::kBN + at.n(j)] = p;
    }
    __syncthreads();
    for (int n = threadIdx.x; n < T::kBN; n += T::kThreads) {
        if (n0 + n >= a.X.rows) continue;
        float2 p = red[n];
#pragma unroll
        for (int w = 1; w < T::kWM; ++w) p = join(p, red[w * T::kBN + n]);
        a.parts[(int64_t)mt * a.X.rows + n0 + n] = p;
    }
}

// Where tokens and words make few tiles of many k, k is split and the logits'
// partial sums [splits, tokens, words] are written: 4 x 500 words of 8192 in one
// tile take 128 stages, one after another.
struct LogitSumArgs {
    Operand W, X;
    unsigned mtiles, tiles;
    int64_t k_split, words;  // words: a multiple of 4
    float *sum;
};

template <class T>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void logit_sum_kernel(const LogitSumArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x % a.tiles, a.tiles, a.mtiles, mt, nt);
    const int64_t split = blockIdx.x / a.tiles;
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    const int64_t k0 = split * a.k_split, k1 = k0 + a.k_split < a.X.k ? k0 + a.k_split : a.X.k;
    Acc<T> acc;
    acc.clear();
    tile_product<T, Along, Along>(acc, lds, a.W, m0, a.X, n0, k0, k1);
    store_sum<T>(acc, a.sum + split * a.X.rows * a.words, m0, a.words, n0, a.X.rows, true, false);
}

__device__ __forceinline__ float4 logits_of(const float4 *sum, int splits, int64_t fours, int64_t id) {
    float4 v = sum[id];
    for (int s = 1; s < splits; ++s) {
        const float4 o = sum[(int64_t)s * fours + id];
        v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
    }
    return v;
}

// The loss of a token per block from them.
__global__ __launch_bounds__(256) void loss_rows(const float4 *__restrict__ sum, int splits, int64_t words,
                                                 const int64_t *__restrict__ target, int64_t vocab,
                                                 float *__restrict__ loss, float *__restrict__ lse) {
    __shared__ float2 red[4];
    __shared__ float at;
    const int64_t t = blockIdx.x, row = words / 4, fours = row * gridDim.x;
    const int64_t y = target[t];
    float2 p = make_float2(-INFINITY, 0.0f);
    for (int64_t k = threadIdx.x; k < row; k += 256) {
        const float4 q = logits_of(sum, splits, fours, t * row + k);
        const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (4 * k + e >= vocab) continue;
            p = join(p, make_float2(v[e], v[e] == v[e] ? 1.0f : v[e]));
            if (4 * k + e == y) at = v[e];
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) p = join(p, make_float2(__shfl_xor(p.x, o, 64), __shfl_xor(p.y, o, 64)));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = p;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) p = join(p, red[w]);
    const float l = p.x + logf(p.y);
    lse[t] = l;
    loss[t] = y >= 0 && y < vocab ? l - at : 0.0f;
}

// 64 tokens per block, four threads to a token.  8192 tokens' 500 parts each (33
// MB) in 22 us: 128 blocks, so their loads' latency bounds it, 8 at a time.
__global__ __launch_bounds__(256) void loss_finish(const float2 *__restrict__ parts, int64_t tiles, int64_t tokens,
                                                   const int64_t *__restrict__ target, int64_t vocab,
                                                   const float *__restrict__ at, float *__restrict__ loss,
                                                   float *__restrict__ lse) {
    __shared__ float2 red[4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * 64 + lane;
    float2 p = make_float2(-INFINITY, 0.0f);
    if (t < tokens)
        for (int64_t k = w; k < tiles; k += 32) {  // 8 loads under way
            float2 q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                q[i] = k + 4 * i < tiles ? parts[(k + 4 * i) * tokens + t] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int i = 0; i < 8; ++i) p = join(p, q[i]);
        }
    red[w][lane] = p;
    __syncthreads();
    if (w != 0 || t >= tokens) return;
#pragma unroll
    for (int k = 1; k < 4; ++k) p = join(p, red[k][lane]);
    const float l = p.x + logf(p.y);
    const int64_t y = target[t];
    lse[t] = l;
    loss[t] = y >= 0 && y < vocab ? l - at[t] : 0.0f;
}

// Both parts of h of a piece of the vocabulary; zeros where a token is not scored
// and beyond the vocabulary.  8192 tokens of 4096 over 11776 words: 0.77 ms, 1.03
// PFLOP/s (MFMA 0.51 busy); the exponentials and 386 MB of h come after the
// products, which the one block that a CU holds cannot overlap.
template <class T>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void loss_slope_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x, gridDim.x, a.mtiles, mt, nt);
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    Acc<T> acc;
    acc.clear();
    tile_product<T, Along, Along>(acc, lds, a.W, m0, a.X, n0, 0, a.X.k);
    const Place<T> at;
    const int64_t v1 = a.vocab - a.v0 - m0;
    const int words = v1 < T::kBM ? (int)v1 : T::kBM;
    const int first = at.m(0, 0);  // element (i, e) is word first + 32 i + 8 (e / 4) + e % 4
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) {
        const int64_t t = n0 + at.n(j);
        const bool in = t < a.X.rows;
        const int64_t y = in ? a.target[t] : -1;
        const bool scored = y >= 0 && y < a.vocab;
        const float w = in ? a.factor[t] : 0.0f, l = in ? a.lse[t] : 0.0f;
        const int64_t yl = y - a.v0 - m0;
        const int own = scored && yl >= 0 && yl < words ? (int)yl - first : -1;
        const int some = w != 0.0f ? words - first : 0;
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int k = 32 * i + 8 * (e >> 2) + (e & 3);
                const float p = exp_of(acc.v[i][j][e] - l) - (k == own ? 1.0f : 0.0f);
                acc.v[i][j][e] = k < some ? w * p : 0.0f;
            }
    }
    store_bf16<T>(acc, lds, a.g, a.ldg, m0, a.ldg, n0, a.X.rows, true);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j)
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const uint32_t r = bf16_pair(acc.v[i][j][e], acc.v[i][j][e + 1]);
                acc.v[i][j][e] -= low_half(r);
                acc.v[i][j][e + 1] -= high_half(r);
            }
    store_bf16<T>(acc, lds, a.g + a.X.rows * a.ldg, a.ldg, m0, a.ldg, n0, a.X.rows, true);
}

__device__ __forceinline__ float block_max(float v, float *red) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v = fmaxf(v, __shfl_xor(v, o, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    __syncthreads();
    return v;
}

// The largest finite |weight| of the scored tokens, kMost parts of it.
__device__ __forceinline__ float scored_most(const int64_t *target, const float *weight, int64_t first, int64_t tokens,
                                             int64_t step, int64_t vocab) {
    __shared__ float red[4];
    float v = 0.0f;
    for (int64_t t = first; t < tokens; t += step) {
        const int64_t y = target[t];
        const float w = fabsf(weight[t]);
        if (y >= 0 && y < vocab && w < INFINITY) v = fmaxf(v, w);
    }
    return block_max(v, red);
}

__global__ __launch_bounds__(256) void weight_most(const int64_t *__restrict__ target,
                                                   const float *__restrict__ weight, int64_t tokens, int64_t vocab,
                                                   float *__restrict__ most) {
    const float v = scored_most(target, weight, (int64_t)blockIdx.x * 256 + threadIdx.x, tokens, kMost * 256, vocab);
    if (threadIdx.x == 0) most[blockIdx.x] = v;
}

// Their largest, in a block of 256; 1 where no weight counts.
__device__ __forceinline__ float largest(const float *most) {
    __shared__ float red[4];
    const float c = block_max(most[threadIdx.x], red);
    return c == 0.0f ? 1.0f : c;
}

__device__ __forceinline__ float factor_of(int64_t y, float w, int64_t vocab, float c) {
    return y < 0 || y >= vocab ? 0.0f : w / c;
}

// h from the logits' partial sums, four words a thread.
__global__ __launch_bounds__(256) void slope_rows(const float4 *__restrict__ sum, int splits, int64_t tokens,
                                                  int64_t words, int64_t vocab, const int64_t *__restrict__ target,
                                                  const float *__restrict__ lse, const float *__restrict__ factor,
                                                  uint2 *__restrict__ g) {
    const int64_t row = words / 4, fours = tokens * row, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < fours; id += stride) {
        const int64_t t = id / row, v0 = (id - t * row) * 4, y = target[t];
        const float4 q = logits_of(sum, splits, fours, id);
        const float w = factor[t], l = lse[t], x[4] = {q.x, q.y, q.z, q.w};
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = exp_of(x[e] - l) - (v0 + e == y ? 1.0f : 0.0f);
            h[e] = w != 0.0f && v0 + e < vocab ? w * p : 0.0f;
        }
        const uint2 r = make_uint2(bf16_pair(h[0], h[1]), bf16_pair(h[2], h[3]));
        g[id] = r;
        g[fours + id] = make_uint2(bf16_pair(h[0] - low_half(r.x), h[1] - high_half(r.x)),
                                   bf16_pair(h[2] - low_half(r.y), h[3] - high_half(r.y)));
    }
}

// The stages of the second part of g, which lies behind the first: the same k
// of P again.
template <class T, Layout LP, Layout LQ>
struct SecondPart {
    static constexpr bool kAny = true;
    using SP = Stage<LP, T::kBM, T::kWaves, T::kK>;
    using SQ = Stage<LQ, T::kBN, T::kWaves, T::kK>;
    int stages;

    const Operand &P;
    Operand Q;
    int64_t m0, n0, k0, k1;
    bool begun = false;

    __device__ __forceinline__ SecondPart(const Operand &p, int64_t m, const Operand &q, int64_t part, int64_t n,
                                          int64_t from, int64_t to)
        : stages((int)((to - from + T::kK - 1) / T::kK)), P(p), Q(q), m0(m), n0(n), k0(from), k1(to) {
        Q.p = static_cast<const uint16_t *>(q.p) + part;
    }
    __device__ __forceinline__ void set(SP &sp, SQ &sq, bool some) {
        if (!some) {  // stages past the last
            sp.left = sq.left = 0;
            return;
        }
        if (begun) return;
        begun = true;
        const Place<T> at;
        sp.init(P, m0, k0, k1, at.wm + at.wn * T::kWM, at.lane);
        sq.init(Q, n0, k0, k1, at.wm + at.wn * T::kWM, at.lane);
    }
};

// dX and dW of such a piece, both parts: 1.27 and 1.31 ms, 1.24 and 1.21 PFLOP/s
// at MFMA 0.65 busy and 1.8 GHz, where a library product as large as one of the
// parts of 32000 words reaches 1.39.
struct DxArgs {
    Operand W, g;    // W [vocab piece, d] across, g [2, tokens, piece]
    unsigned mtiles, tiles;
    int64_t k_split;
    bool add;
    float *sum;      // [splits, tokens, d]
};

template <class T>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void loss_dx_kernel(const DxArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x % a.tiles, a.tiles, a.mtiles, mt, nt);
    const int64_t split = blockIdx.x / a.tiles;
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    const int64_t k0 = split * a.k_split, k1 = k0 + a.k_split < a.g.k ? k0 + a.k_split : a.g.k;
    Acc<T> acc;
    acc.clear();
    if (k0 < k1)  // a last piece may have fewer splits
        tile_product<T, Across, Along>(acc, lds, a.W, m0, a.g, n0, k0, k1,
                                       SecondPart<T, Across, Along>(a.W, m0, a.g, a.g.rows * a.g.ld, n0, k0, k1));
    store_sum<T>(acc, a.sum + split * a.g.rows * a.W.rows, m0, a.W.rows, n0, a.g.rows, true, a.add);
}

// Adds the splits and rounds.
__global__ __launch_bounds__(256) void loss_dx_finish(const float4 *__restrict__ sum, int splits, int64_t fours,
                                                      int64_t d, const float *__restrict__ most,
                                                      uint16_t *__restrict__ dX, int64_t lddx) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    const float c = largest(most);
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < fours; id += stride) {
        float4 v = sum[id];
        for (int s = 1; s < splits; ++s) {
            const float4 o = sum[(int64_t)s * fours + id];
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const int64_t t = id / (d / 4), m = id % (d / 4) * 4;
        *reinterpret_cast<uint2 *>(dX + t * lddx + m) =
            make_uint2(bf16_pair(v.x * c, v.y * c), bf16_pair(v.z * c, v.w * c));
    }
}

// Every token's weight / c, and X with zeros in the rows that are not scored,
// so that what lies there does not meet the zeros of h in a product.  Of few
// tokens each block finds the largest weight itself and the first leaves it in
// `most`, which saves a launch.
template <bool few>
__global__ __launch_bounds__(256) void scored_rows(const uint16_t *__restrict__ X, int64_t ldx, int64_t tokens,
                                                   int64_t d, const int64_t *__restrict__ target,
                                                   const float *__restrict__ weight, int64_t vocab,
                                                   float *__restrict__ most, float *__restrict__ factor,
                                                   u32x4 *__restrict__ S) {
    const int64_t stride = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    float c;
    if constexpr (few) {
        c = scored_most(target, weight, threadIdx.x, tokens, 256, vocab);
        if (blockIdx.x == 0) most[threadIdx.x] = threadIdx.x == 0 ? c : 0.0f;
        c = c == 0.0f ? 1.0f : c;
    } else {
        c = largest(most);
    }
    for (int64_t t = first; t < tokens; t += stride) factor[t] = factor_of(target[t], weight[t], vocab, c);
    if (!S) return;
    const int64_t words = d / 8, total = tokens * words;
    for (int64_t id = first; id < total; id += stride) {
        const int64_t t = id / words, k = id - t * words;
        const int64_t y = target[t];
        u32x4 v = {0, 0, 0, 0};
        if (y >= 0 && y < vocab && weight[t] != 0.0f) v = *reinterpret_cast<const u32x4 *>(X + t * ldx + k * 8);
        S[id] = v;
    }
}

__global__ __launch_bounds__(256) void clear_kernel(uint2 *__restrict__ p, int64_t n) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < n; id += stride) p[id] = make_uint2(0u, 0u);
}

struct DwArgs {
    Operand X, g;    // X [tokens, d] across, g [2, tokens, piece] across
    const float *most;
    unsigned mtiles;
    int64_t cols;    // rows of dW in this piece
    uint16_t *dW;    // [cols, d]
    bool wide;
};

template <class T>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void loss_dw_kernel(const DwArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x, gridDim.x, a.mtiles, mt, nt);
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    Acc<T> acc;
    acc.clear();
    tile_product<T, Across, Across>(acc, lds, a.X, m0, a.g, n0, 0, a.g.k,
                                    SecondPart<T, Across, Across>(a.X, m0, a.g, a.g.k * a.g.ld, n0, 0, a.g.k));
    float c = a.most[threadIdx.x & 63];
    for (int i = 64; i < kMost; i += 64) c = fmaxf(c, a.most[i + (threadIdx.x & 63)]);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) c = fmaxf(c, __shfl_xor(c, o, 64));
    store_bf16<T>(acc, lds, a.dW, a.X.rows, m0, a.X.rows, n0, a.cols, a.wide, c == 0.0f ? 1.0f : c);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

#define loss_tile_kernel_of(T) loss_tile_kernel<T>
#define logit_sum_kernel_of(T) logit_sum_kernel<T>
#define loss_slope_kernel_of(T) loss_slope_kernel<T>
#define loss_dx_kernel_of(T) loss_dx_kernel<T>
#define loss_dw_kernel_of(T) loss_dw_kernel<T>

// The logits' partial sums of `words` (a multiple of 4).
int logit_sums(const void *X, int64_t tokens, int64_t d, int64_t ldx, const void *W, int64_t vocab, int64_t words,
               const Split &p, float *sum, hipStream_t stream) {
    LogitSumArgs a{};
    a.W = Operand{W, d, vocab, d};
    a.X = Operand{X, ldx, tokens, d};
    a.mtiles = (unsigned)cdiv(words, p.side_m());
    a.tiles = (unsigned)p.units(words, tokens);
    a.k_split = p.k;
    a.words = words;
    a.sum = sum;
    LAUNCH_TILES(logit_sum_kernel_of, Large, p.size, a.tiles * (unsigned)p.splits, stream, a);
    return launch_status();
}

// Tokens whose weights each block of scored_rows reads for itself.  A launch
// before it costs 3.3 us of a call over 384 tokens of 1024; for 2048 tokens of
// 4096 it takes 19 us so, 13 in two launches.
constexpr int64_t kFewWeights = 512;

bool loss_sizes_ok(int64_t tokens, int64_t d, int64_t vocab) {
    return tokens >= 0 && tokens <= kMaxTokens && d >= 0 && d % 16 == 0 && d <= kMaxWidth && vocab >= 0 &&
           vocab <= kMaxVocab && tokens * vocab <= kMaxLogits;
}

}  // namespace

extern "C" {

size_t hscale_token_loss_workspace_bytes(int64_t tokens, int64_t d, int64_t vocab) {
    if (!loss_sizes_ok(tokens, d, vocab) || tokens == 0 || d == 0 || vocab == 0) return 0;
    return most_loss(tokens, d, vocab);
}

int hscale_token_loss(const void *X, int64_t tokens, int64_t d, int64_t ldx, const void *W, int64_t vocab,
                      const int64_t *target, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                      hipStream_t stream) {
    if (!loss_sizes_ok(tokens, d, vocab) || (tokens > 1 && (ldx < d || ldx > kMaxWidth))) return HSCALE_ERR_SHAPE;
    if (tokens == 0) return HSCALE_OK;
    if (d == 0 || vocab == 0) return HSCALE_ERR_SHAPE;
    if (!X || !W || !target || !loss || !lse || !workspace) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(W, 16) || !aligned(target, 8) ||
        !aligned(loss, 4) || !aligned(lse, 4) || !aligned(workspace, 256))
        return HSCALE_ERR_ALIGN;
    const LossPlan p = loss_plan(tokens, d, vocab);
    const size_t need = most_loss(tokens, d, vocab);
    if (workspace_bytes < need) return HSCALE_ERR_WORKSPACE;
    const Range w[] = {{loss, (size_t)tokens * 4}, {lse, (size_t)tokens * 4}, {workspace, p.total}};
    const Range r[] = {{X, span(tokens, ldx, d, 2)}, {W, (size_t)vocab * d * 2}, {target, (size_t)tokens * 8}};
    if (any_overlap(w, 3, r, 3)) return HSCALE_ERR_OVERLAP;
    if (p.tile.splits > 1) {
        const int64_t words = cdiv(vocab, 4) * 4;
        float *sum = static_cast<float *>(workspace);
        if (const int st = logit_sums(X, tokens, d, ldx, W, vocab, words, p.tile, sum, stream)) return st;
        hipLaunchKernelGGL(loss_rows, dim3((unsigned)tokens), dim3(256), 0, stream,
                           reinterpret_cast<const float4 *>(sum), p.tile.splits, words, target, vocab, loss, lse);
        return launch_status();
    }
    LogitArgs a{};
    a.W = Operand{W, d, vocab, d};
    a.X = Operand{X, ldx, tokens, d};
    a.target = target;
    a.parts = static_cast<float2 *>(workspace);
    a.at = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.parts);
    a.vocab = vocab;
    a.mtiles = (unsigned)cdiv(vocab, p.tile.side_m());
    LAUNCH_TILES(loss_tile_kernel_of, Large, p.tile.size, p.tile.units(vocab, tokens), stream, a);
    if (const int st = launch_status()) return st;
    hipLaunchKernelGGL(loss_finish, dim3((unsigned)cdiv(tokens, 64)), dim3(256), 0, stream, a.parts,
                       (int64_t)a.mtiles, tokens, target, vocab, a.at, loss, lse);
    return launch_status();
}

size_t hscale_token_loss_grad_workspace_bytes(int64_t tokens, int64_t d, int64_t vocab) {
    if (!loss_sizes_ok(tokens, d, vocab) || tokens == 0 || d == 0 || vocab == 0) return 0;
    return most_loss_grad(tokens, d, vocab, true);
}

int hscale_token_loss_grad(const void *X, int64_t tokens, int64_t d, int64_t ldx, const void *W, int64_t vocab,
                           const int64_t *target, const float *lse, const float *weight, void *dX, int64_t lddx,
                           void *dW, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!loss_sizes_ok(tokens, d, vocab) ||
        (tokens > 1 && (ldx < d || ldx > kMaxWidth || (dX && lddx < d))))
        return HSCALE_ERR_SHAPE;
    if (tokens == 0 && (!dW || d == 0 || vocab == 0)) return HSCALE_OK;
    if (d == 0 || vocab == 0) return HSCALE_ERR_SHAPE;
    if (tokens == 0) {
        if (!aligned(dW, 8)) return HSCALE_ERR_ALIGN;
        hipLaunchKernelGGL(clear_kernel, dim3(grid_for(vocab * d / 4, 256)), dim3(256), 0, stream,
                           static_cast<uint2 *>(dW), vocab * d / 4);
        return launch_status();
    }
    if (!X || !W || !target || !lse || !weight || !workspace) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(W, 16) || !aligned(target, 8) ||
        !aligned(lse, 4) || !aligned(weight, 4) || !aligned(dX, 8) || (dX && tokens > 1 && lddx % 4 != 0) ||
        !aligned(dW, 8) || !aligned(workspace, 256))
        return HSCALE_ERR_ALIGN;
    const LossGradPlan p = loss_grad_plan(tokens, d, vocab, dW != nullptr);
    const size_t need = most_loss_grad(tokens, d, vocab, dW != nullptr);
    if (workspace_bytes < need) return HSCALE_ERR_WORKSPACE;
    const Range w[] = {{dX, dX ? span(tokens, lddx, d, 2) : 0}, {dW, dW ? (size_t)vocab * d * 2 : 0},
                       {workspace, p.total}};
    const Range r[] = {{X, span(tokens, ldx, d, 2)}, {W, (size_t)vocab * d * 2}, {target, (size_t)tokens * 8},
                       {lse, (size_t)tokens * 4}, {weight, (size_t)tokens * 4}};
    if (any_overlap(w, 3, r, 5)) return HSCALE_ERR_OVERLAP;

    char *ws = static_cast<char *>(workspace);
    uint16_t *g = reinterpret_cast<uint16_t *>(ws);
    float *sum = reinterpret_cast<float *>(ws + p.g);
    u32x4 *rows = dW ? reinterpret_cast<u32x4 *>(ws + p.g + p.sum) : nullptr;
    float *factor = reinterpret_cast<float *>(ws + p.g + p.sum + p.rows);
    float *most = reinterpret_cast<float *>(ws + p.g + p.sum + p.rows + p.factor);
    if (tokens > kFewWeights) {
        hipLaunchKernelGGL(weight_most, dim3(kMost), dim3(256), 0, stream, target, weight, tokens, vocab, most);
        if (const int st = launch_status()) return st;
    }
    hipLaunchKernelGGL(tokens > kFewWeights ? scored_rows<false> : scored_rows<true>, dim3(grid_for(dW ? tokens * d / 8 : tokens, 256)), dim3(256), 0, stream,
                       static_cast<const uint16_t *>(X), ldx, tokens, d, target, weight, vocab, most, factor, rows);
    if (const int st = launch_status()) return st;
    for (int64_t v0 = 0; v0 < vocab; v0 += p.piece) {
        const int64_t cols = std::min(p.piece, vocab - v0), ldg = cdiv(cols, kPieceStep) * kPieceStep;
        const uint16_t *Wp = static_cast<const uint16_t *>(W) + v0 * d;
        if (p.logits.splits > 1) {
            if (const int st = logit_sums(X, tokens, d, ldx, W, vocab, ldg, p.logits, sum, stream)) return st;
            hipLaunchKernelGGL(slope_rows, dim3(grid_for(tokens * ldg / 4, 256)), dim3(256), 0, stream,
                               reinterpret_cast<const float4 *>(sum), p.logits.splits, tokens, ldg, vocab, target, lse,
                               factor, reinterpret_cast<uint2 *>(g));
            if (const int st = launch_status()) return st;
        } else {
            LogitArgs a{};
            a.W = Operand{Wp, d, cols, d};
            a.X = Operand{X, ldx, tokens, d};
            a.target = target;
            a.v0 = v0;
            a.vocab = vocab;
            a.lse = lse;
            a.factor = factor;
            a.g = g;
            a.ldg = ldg;
            const Split logits = slope_plan(ldg, tokens, d);
            a.mtiles = (unsigned)(ldg / logits.side_m());
            LAUNCH_TILES(loss_slope_kernel_of, Large, logits.size, logits.units(ldg, tokens), stream, a);
            if (const int st = launch_status()) return st;
        }
        if (dX) {
            DxArgs x{};
            x.W = Operand{Wp, d, d, cols};
            x.g = Operand{g, ldg, tokens, ldg};
            x.mtiles = (unsigned)cdiv(d, p.dx.side_m());
            x.tiles = (unsigned)p.dx.units(d, tokens);
            x.k_split = p.dx.k;
            x.add = v0 > 0;
            x.sum = sum;
            LAUNCH_TILES(loss_dx_kernel_of, Large, p.dx.size, x.tiles * (unsigned)p.dx.splits, stream, x);
            if (const int st = launch_status()) return st;
        }
        if (dW) {
            DwArgs b{};
            b.X = Operand{rows, d, d, tokens};
            b.g = Operand{g, ldg, ldg, tokens};
            b.most = most;
            const Split rows_of = dw_plan(d, cols, tokens);
            b.mtiles = (unsigned)cdiv(d, rows_of.side_m());
            b.cols = cols;
            b.dW = static_cast<uint16_t *>(dW) + v0 * d;
            b.wide = aligned(dW, 16);
            LAUNCH_TILES(loss_dw_kernel_of, LargeAcross, rows_of.size, rows_of.units(d, cols), stream, b);
            if (const int st = launch_status()) return st;
        }
    }
    if (dX) {
        const int64_t fours = tokens * d / 4;
        hipLaunchKernelGGL(loss_dx_finish, dim3(grid_for(fours, 256)), dim3(256), 0, stream,
                           reinterpret_cast<const float4 *>(sum), p.dx.splits, fours, d, most,
                           static_cast<uint16_t *>(dX), lddx);
        return launch_status();
    }
    return HSCALE_OK;
}

}  // extern "C"
