// A stored NVFP4 layer in use, behind the C ABI of include/hscale.h: its
// product with activations beside the low-rank adapters of many requests,
// activation checkpoints in 8 bits, and the gradients of the adapted layer at
// such a checkpoint.
//
//   y_t  = s_g W^ x_t + alpha_a B_a (A_a x_t)          a = adapter of token t
//   v_t  = alpha_a B_a^T dy_t,   u_t = alpha_a A_a x_t
//   dx_t = s_g W^T dy_t + A_a^T v_t
//   dA_a = sum_t v_t x_t^T,      dB_a = sum_t dy_t u_t^T     over its tokens
//
// An E2M1 value has 2 significant bits and an E4M3 scale 4, so with the power
// of two of s_g = f 2^e (1 <= f < 2) W^ is exact in bf16: the products with W^
// are bf16 products accumulated in fp32, and f multiplies the sum.  u and v are kept as two bf16 parts
// (within 2^-16), so that nothing of the adapters' part is rounded to 8 bits
// before the result is.

#include "matmul.h"

#include <algorithm>

namespace {

constexpr int kCkBlock = 128;               // activations per checkpoint scale
constexpr float kCkTiny = 0x1p-100f;        // smallest magnitude a block is scaled for
constexpr int kMaxRank = 256;
constexpr int kMaxAdapters = 4096;
constexpr int64_t kMaxWidth = (int64_t)1 << 21;   // in, out: a tile's rows are addressed in 32 bits
constexpr int64_t kMaxTokens = (int64_t)1 << 24;
constexpr int kNoAdapter = -1;

// Adapter of token t, or kNoAdapter where the number is none.
__device__ __forceinline__ int adapter_of(const int32_t *ids, int count, int64_t t) {
    if (!ids) return 0;
    const int a = ids[t];
    return a >= 0 && a < count ? a : kNoAdapter;
}

// The smallest adapter above `after` among tokens t0 .. t1 - 1, INT_MAX when
// there is none; the same in all lanes of a wave.
__device__ __forceinline__ int next_adapter(const int32_t *ids, int count, int64_t t0, int64_t t1, int after) {
    int least = INT_MAX;
    for (int64_t t = t0 + (threadIdx.x & 63); t < t1; t += 64) {
        const int a = adapter_of(ids, count, t);
        if (a > after && a < least) least = a;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
    return __builtin_amdgcn_readfirstlane(least);
}

// ---------------------------------------------------------------------------
// Stored weights as bf16
// ---------------------------------------------------------------------------

// Two E2M1 values of byte K of `src` times l, as a pair of bf16: exact.
template <int K>
__device__ __forceinline__ uint32_t stored_pair(uint32_t src, float l) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(src, 1.0f, K);
    return __builtin_amdgcn_perm(__float_as_uint(v[1] * l), __float_as_uint(v[0] * l), 0x07060302);
}

__device__ __forceinline__ u32x4 stored_eight(uint32_t src, float l) {
    return u32x4{stored_pair<0>(src, l), stored_pair<1>(src, l), stored_pair<2>(src, l), stored_pair<3>(src, l)};
}

// W^ [groups * 16] with 2^e in place of s_g, one group per thread.
__global__ __launch_bounds__(256) void stored_to_bf16(const uint8_t *__restrict__ codes,
                                                      const uint2 *__restrict__ packed, int64_t groups, float two_e,
                                                      u32x4 *__restrict__ W) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += stride) {
        const float l = e4m3fn_value(codes[g]) * two_e;
        const uint2 p = packed[g];
        W[2 * g] = stored_eight(p.x, l);
        W[2 * g + 1] = stored_eight(p.y, l);
    }
}

// ---------------------------------------------------------------------------
// Activation checkpoints in 8 bits
// ---------------------------------------------------------------------------

// Eight bf16 values of a 16-byte word as fp32.
__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}

// Eight checkpointed values restored: bf16(q s), one rounding.
__device__ __forceinline__ u32x4 restore8(uint2 q, float s) {
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = k < 2 ? q.x : q.y;
        const float a = (float)(int8_t)(w >> (16 * (k & 1))) * s;
        const float b = (float)(int8_t)(w >> (16 * (k & 1) + 8)) * s;
        r[k] = bf16_pair(a, b);
    }
    return r;
}

// A thread per 8 values, 16 threads per block of 128 (the last of a row may
// be shorter): s = fp32(m fp32(1/127)) with m = max(|x|, 2^-100), and
// q = rint(fp32(x fp32(127 / m))).
__global__ __launch_bounds__(256) void pack_kernel(const uint16_t *__restrict__ X, int64_t tokens, int64_t in,
                                                   int64_t ldx, uint2 *__restrict__ q, float *__restrict__ scale) {
    const int64_t blocks = (in + kCkBlock - 1) / kCkBlock, total = tokens * blocks * 16;
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t blk = id >> 4, t = blk / blocks, b = blk - t * blocks;
        const int64_t c = b * kCkBlock + (id & 15) * 8;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (c < in) unpack8(*reinterpret_cast<const u32x4 *>(X + t * ldx + c), x);
        float m = kCkTiny;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(x[k]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 16));
        const float inv = 127.0f / m;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int v = (int)__builtin_rintf(x[k] * inv);
            w[k >> 2] |= (uint32_t)(v & 0xFF) << (8 * (k & 3));
        }
        if (c < in) q[(t * in + c) >> 3] = make_uint2(w[0], w[1]);
        if ((id & 15) == 0) scale[blk] = m * (1.0f / 127.0f);
    }
}

__global__ __launch_bounds__(256) void unpack_kernel(const uint2 *__restrict__ q, const float *__restrict__ scale,
                                                     int64_t tokens, int64_t in, uint16_t *__restrict__ X,
                                                     int64_t ldx, bool wide) {
    const int64_t blocks = (in + kCkBlock - 1) / kCkBlock, total = tokens * blocks * 16;
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t blk = id >> 4, t = blk / blocks, b = blk - t * blocks;
        const int64_t c = b * kCkBlock + (id & 15) * 8;
        if (c >= in) continue;
        const u32x4 v = restore8(q[(t * in + c) >> 3], scale[blk]);
        uint16_t *x = X + t * ldx + c;
        if (wide) {
            *reinterpret_cast<u32x4 *>(x) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
        }
    }
}

// ---------------------------------------------------------------------------
// Down to the rank: p[t, j] = sum_k z[t, k] A_a[j, k]
// ---------------------------------------------------------------------------

// Activations as bf16 rows, or as a checkpoint.
struct Rows {
    const void *p;       // bf16 [tokens, width] at ld, or int8 [tokens, width]
    const float *scale;  // of a checkpoint, else NULL
    int64_t ld;
};

struct ShrinkArgs {
    Rows z;
    int64_t tokens, width;  // width % 16 == 0
    const uint16_t *A;      // [count, rank, width]
    int count, rank, rank_pad;
    const int32_t *ids;
    int64_t k_split;        // of a split, a multiple of 64
    float *partial;         // [splits, tokens, rank_pad]
};

// 32 tokens x 32 ranks x one split of k per block, of which each of 4 waves
// takes every fourth 16 k; one pass for each adapter that the tokens have
// (ordinals z, z + slots, ...).  Rows of other adapters are computed and not
// stored, so no value of another request enters a token's result.
template <bool kCheckpoint>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkArgs a, int slots) {
    __shared__ float red[3][32 * 33];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * 32, t1 = t0 + 32 < a.tokens ? t0 + 32 : a.tokens;
    const int64_t k0 = (int64_t)blockIdx.y * a.k_split;
    const int64_t k1 = k0 + a.k_split < a.width ? k0 + a.k_split : a.width;
    const int rank_tiles = a.rank_pad / 32;
    const int j0 = (int)(blockIdx.z % rank_tiles) * 32, slot = blockIdx.z / rank_tiles;
    const int64_t t = t0 + (lane & 31);
    const bool t_ok = t < t1;
    const int own = t_ok ? adapter_of(a.ids, a.count, t) : kNoAdapter;
    const int j = j0 + (lane & 31);
    int adapter = -1;
    for (int nth = 0;; ++nth) {
        adapter = next_adapter(a.ids, a.count, t0, t1, adapter);
        if (adapter == INT_MAX) break;
        if (nth % slots != slot) continue;
        const uint16_t *Arow = a.A + ((int64_t)adapter * a.rank + j) * a.width;
        f32x16 acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
        for (int64_t k = k0 + wave * 16; k < k1; k += 64) {
            const int64_t c = k + 8 * (lane >> 5);
            u32x4 fa = {0, 0, 0, 0}, fz = {0, 0, 0, 0};
            if (j < a.rank) fa = *reinterpret_cast<const u32x4 *>(Arow + c);
            if (t_ok) {
                if (kCheckpoint)
                    fz = restore8(
                        *reinterpret_cast<const uint2 *>(reinterpret_cast<const int8_t *>(a.z.p) + t * a.width + c),
                        a.z.scale[t * ((a.width + kCkBlock - 1) / kCkBlock) + c / kCkBlock]);
                else
                    fz = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint16_t *>(a.z.p) + t * a.z.ld + c);
            }
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa),
                                                          __builtin_bit_cast(bf16x8, fz), acc, 0, 0, 0);
        }
        __syncthreads();
        if (wave > 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) red[wave - 1][(lane >> 5) * 16 * 33 + e * 33 + (lane & 31)] = acc[e];
        }
        __syncthreads();
        if (wave == 0 && own == adapter) {
            float *dst = a.partial + ((int64_t)blockIdx.y * a.tokens + t) * a.rank_pad + j0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float4 v;
                float *f = &v.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = (lane >> 5) * 16 * 33 + (4 * q + e) * 33 + (lane & 31);
                    f[e] = ((acc[4 * q + e] + red[0][at]) + red[1][at]) + red[2][at];
                }
                *reinterpret_cast<float4 *>(dst + 8 * q + 4 * (lane >> 5)) = v;
            }
        }
    }
}

// alpha / f times the sum of the splits (f multiplies the result that takes it),
// or alpha times it, as two bf16 parts: low[t, j] and
// low[t, rank_pad + j].  Tokens without an adapter are left as they are; what
// reads `low` skips them.
__global__ __launch_bounds__(256) void shrink_finish(const float *__restrict__ partial, int splits, int64_t tokens,
                                                     int rank, int rank_pad, const float *__restrict__ alpha, float f,
                                                     const int32_t *__restrict__ ids, int count,
                                                     uint16_t *__restrict__ low) {
    const int64_t total = tokens * rank_pad, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t t = id / rank_pad;
        const int j = (int)(id - t * rank_pad);
        const int a = adapter_of(ids, count, t);
        if (a == kNoAdapter) continue;
        float v = 0.0f;
        if (j < rank) {
            for (int s = 0; s < splits; ++s) v += partial[(int64_t)s * total + id];
            if (alpha) v *= alpha[a];
            v /= f;
        }
        const uint32_t hi = bf16_rne(v);
        low[t * 2 * rank_pad + j] = (uint16_t)hi;
        low[t * 2 * rank_pad + rank_pad + j] = (uint16_t)bf16_rne(v - bf16_value(hi));
    }
}

// ---------------------------------------------------------------------------
// The layer with its adapters, many tokens
// ---------------------------------------------------------------------------

struct LowRank {
    const uint16_t *low;    // [tokens, 2 rank_pad]: two bf16 parts
    const uint16_t *other;  // forward: B [count, out, rank]; backward: A [count, rank, in]
    int64_t other_size;     // elements of one adapter
    int64_t ld;
    int count, rank, rank_pad;
    const int32_t *ids;
};

// The stages that add other_a (low_n) for the tokens n of a tile to its
// products: for each adapter that the tile's tokens have, k runs over the rank
// twice, once for each part of low.  Tokens of other adapters enter as zeros.
template <class T, Layout LP>
struct LowRankStages {
    static constexpr bool kAny = true;
    using SP = Stage<LP, T::kBM, T::kWaves, T::kK>;
    using SQ = Stage<Along, T::kBN, T::kWaves, T::kK>;
    int stages;

    const LowRank &w;
    int64_t m0, prows, n0, n1;
    int wave, lane;
    int tile[T::kBN / 64];       // adapters of the tile's tokens, over the wave
    int copied[SQ::kCopies];     // of the rows that this lane copies
    int adapter = -1, step = 0;  // of the next stage

    __device__ __forceinline__ LowRankStages(const LowRank &low, int64_t m, int64_t rows, int64_t n, int64_t tokens)
        : stages(0), w(low), m0(m), prows(rows - m < T::kBM ? rows - m : T::kBM), n0(n),
          n1(n + T::kBN < tokens ? n + T::kBN : tokens) {
        const Place<T> at;
        wave = at.wm + at.wn * T::kWM;
        lane = at.lane;
        if (!w.low) return;
#pragma unroll
        for (int i = 0; i < T::kBN / 64; ++i) tile[i] = of(i * 64 + lane);
#pragma unroll
        for (int i = 0; i < SQ::kCopies; ++i) copied[i] = of(SQ::row_of(i, wave, lane));
        for (int a = next(-1); a != INT_MAX; a = next(a)) stages += per_adapter();
    }
    __device__ __forceinline__ int of(int row) const {
        return n0 + row < n1 ? adapter_of(w.ids, w.count, n0 + row) : kNoAdapter;
    }
    __device__ __forceinline__ int per_adapter() const { return (2 * w.rank_pad + T::kK - 1) / T::kK; }
    __device__ __forceinline__ int next(int after) const {
        int least = INT_MAX;
#pragma unroll
        for (int i = 0; i < T::kBN / 64; ++i)
            if (tile[i] > after) least = min(least, tile[i]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
        return __builtin_amdgcn_readfirstlane(least);
    }
    // Column of the adapter's rank that k of its stages stands for, or none.
    __device__ __forceinline__ int column(int k) const {
        const int j = k >= w.rank_pad ? k - w.rank_pad : k;
        return k < 2 * w.rank_pad && j < w.rank ? j : -1;
    }
    __device__ __forceinline__ void set(SP &sp, SQ &sq, bool some) {
        if (!some) {  // stages past the last
            sp.left = sq.left = 0;
            return;
        }
        if (step == 0) adapter = next(adapter);
        const int k0 = step * T::kK, deep = 2 * w.rank_pad;
        step = step + 1 == per_adapter() ? 0 : step + 1;
        const uint16_t *P = w.other + (int64_t)adapter * w.other_size + (LP == Along ? m0 * w.ld : m0);
        sp.base = reinterpret_cast<const char *>(P);
        sp.left = LP == Along ? ((prows - 1) * w.ld + w.rank) * 2 : ((w.rank - 1) * w.ld + prows) * 2;
        sq.base = reinterpret_cast<const char *>(w.low + n0 * deep);
        sq.left = (n1 - n0) * deep * 2;
        sp.k_left = sq.k_left = INT_MAX;
#pragma unroll
        for (int i = 0; i < SP::kCopies; ++i) {
            const int row = SP::row_of(i, wave, lane), c = SP::at(row, lane);
            const int j = column(LP == Along ? k0 + c * 8 : k0 + row);
            const bool ok = j >= 0 && (LP == Along ? row : c * 8) < prows;
            const int64_t at = LP == Along ? row * w.ld + j : j * w.ld + c * 8;
            sp.off[i] = ok ? (uint32_t)(at * 2) : kNoRead;
        }
#pragma unroll
        for (int i = 0; i < SQ::kCopies; ++i) {
            const int row = SQ::row_of(i, wave, lane), k = k0 + SQ::at(row, lane) * 8;
            sq.off[i] = k < deep && copied[i] == adapter ? (uint32_t)((row * deep + k) * 2) : kNoRead;
        }
    }
};

struct LayerArgs {
    Operand W, X;  // m: the layer's other side, n: tokens
    float scale;
    LowRank low;   // low.low NULL: no adapters
    uint16_t *Y;   // [tokens, m] at ldy
    int64_t ldy;
    bool wide;
    unsigned mtiles;
};

template <class T, Layout LW>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void layer_kernel(const LayerArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x, gridDim.x, a.mtiles, mt, nt);
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    Acc<T> acc;
    acc.clear();
    tile_product<T, LW, Along>(acc, lds, a.W, m0, a.X, n0, 0, a.X.k,
                               LowRankStages<T, LW>(a.low, m0, a.W.rows, n0, a.X.rows));
    store_bf16<T>(acc, lds, a.Y, a.ldy, m0, a.W.rows, n0, a.X.rows, a.wide, a.scale);
}

// ---------------------------------------------------------------------------
// The layer with its adapters, few tokens
// ---------------------------------------------------------------------------

struct FewArgs {
    const uint8_t *codes;
    const uint8_t *packed;
    int64_t out, in;
    const uint16_t *X;
    int64_t tokens, ldx;
    int64_t k_split;  // a multiple of 128
    float *partial;   // [splits, tokens, out]
};

// 64 output rows (16 per wave) x one split of k x 16 kNT tokens.  A lane
// takes 32 consecutive weights of a row at a time, four MFMA steps: which k
// meets which place in a step does not matter, as both operands agree.
template <int kNT>
__global__ __launch_bounds__(256) void few_kernel(const FewArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 64 + wave * 16 + (lane & 15);
    const int64_t t0 = (int64_t)blockIdx.z * 16 * kNT;
    const bool row_ok = row < a.out;
    const int64_t k0 = (int64_t)blockIdx.y * a.k_split;
    const int64_t k1 = k0 + a.k_split < a.in ? k0 + a.k_split : a.in;
    f32x4 acc[kNT];
#pragma unroll
    for (int n = 0; n < kNT; ++n) acc[n] = f32x4{0, 0, 0, 0};
    const uint8_t *prow = a.packed + row * (a.in / 2);
    const uint8_t *crow = a.codes + row * (a.in / kGroup);
    for (int64_t k = k0 + (lane >> 4) * 32; k - (lane >> 4) * 32 < k1; k += 128) {
        uint2 p[2] = {{0, 0}, {0, 0}};
        float l[2] = {0.0f, 0.0f};
#pragma unroll
        for (int g = 0; g < 2; ++g)
            if (row_ok && k + 16 * g < k1) {
                p[g] = *reinterpret_cast<const uint2 *>(prow + (k + 16 * g) / 2);
                l[g] = e4m3fn_value(crow[(k + 16 * g) / kGroup]);
            }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x4 w = stored_eight(q & 1 ? p[q >> 1].y : p[q >> 1].x, l[q >> 1]);
#pragma unroll
            for (int n = 0; n < kNT; ++n) {
                const int64_t t = t0 + n * 16 + (lane & 15);
                u32x4 x = {0, 0, 0, 0};
                if (t < a.tokens && k + 8 * q < k1)
                    x = *reinterpret_cast<const u32x4 *>(a.X + t * a.ldx + k + 8 * q);
                acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w),
                                                                 __builtin_bit_cast(bf16x8, x), acc[n], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        const int64_t t = t0 + n * 16 + (lane & 15);
        const int64_t m = (int64_t)blockIdx.x * 64 + wave * 16 + 4 * (lane >> 4);
        if (t >= a.tokens) continue;
        float *dst = a.partial + ((int64_t)blockIdx.y * a.tokens + t) * a.out;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (m + e < a.out) dst[m + e] = acc[n][e];
    }
}

struct FewFinishArgs {
    const float *partial;  // [splits, tokens, out]
    int splits;
    int64_t tokens, out;
    float s_g;
    const float *low;      // [low_splits, tokens, rank_pad], NULL: no adapters
    int low_splits, rank, rank_pad, count;
    const uint16_t *B;     // [count, out, rank]
    const float *alpha;
    const int32_t *ids;
    uint16_t *Y;
    int64_t ldy;
};

// 256 outputs of one token per block: the sum of the splits, and B_a u in fp32.
__global__ __launch_bounds__(256) void few_finish(const FewFinishArgs a) {
    __shared__ float u[kMaxRank];
    const int64_t t = blockIdx.y, m = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int id = a.low ? adapter_of(a.ids, a.count, t) : kNoAdapter;
    if (id != kNoAdapter) {
        if ((int)threadIdx.x < a.rank) {
            float v = 0.0f;
            for (int s = 0; s < a.low_splits; ++s)
                v += a.low[((int64_t)s * a.tokens + t) * a.rank_pad + threadIdx.x];
            u[threadIdx.x] = a.alpha ? v * a.alpha[id] : v;
        }
        __syncthreads();
    }
    if (m >= a.out) return;
    float y = 0.0f;
    for (int s = 0; s < a.splits; ++s) y += a.partial[((int64_t)s * a.tokens + t) * a.out + m];
    y *= a.s_g;
    if (id != kNoAdapter) {
        const uint16_t *b = a.B + ((int64_t)id * a.out + m) * a.rank;
        for (int j = 0; j < a.rank; j += 8) {
            float v[8];
            unpack8(*reinterpret_cast<const u32x4 *>(b + j), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) y = fmaf(v[e], u[j + e], y);
        }
    }
    a.Y[t * a.ldy + m] = (uint16_t)bf16_rne(y);
}

// ---------------------------------------------------------------------------
// Gradients of the adapters: G_a[j, c] = sum_t low[t, j] z[t, c]
// ---------------------------------------------------------------------------

struct OuterArgs {
    Rows z;
    int64_t tokens, width;
    const uint16_t *low;  // [tokens, 2 rank_pad]
    int count, rank, rank_pad;
    const int32_t *ids;
    int64_t t_split;      // of a split, a multiple of 64
    float *partial;       // [splits, count, rank, width]
};

constexpr int kOuterCols = 128, kOuterTokens = 64;

// 128 columns x 32 ranks of one adapter x one split of the tokens.  Stages of
// 64 tokens, laid out as Stage<Across>; tokens of other adapters are not
// read and enter as zeros, stages without any are skipped.
template <bool kCheckpoint>
__global__ __launch_bounds__(256) void outer_kernel(const OuterArgs a) {
    using SZ = Stage<Across, kOuterCols, 4, kOuterTokens>;
    using SL = Stage<Across, 64, 4, kOuterTokens>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[SZ::kBytes + SL::kBytes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c0 = (int64_t)blockIdx.x * kOuterCols;
    const int rank_tiles = a.rank_pad / 32;
    const int j0 = (int)(blockIdx.y % rank_tiles) * 32, adapter = blockIdx.y / rank_tiles;
    const int64_t t0 = (int64_t)blockIdx.z * a.t_split;
    const int64_t t1 = t0 + a.t_split < a.tokens ? t0 + a.t_split : a.tokens;
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    for (int64_t s = t0; s < t1; s += kOuterTokens) {
        const bool mine = s + lane < t1 && adapter_of(a.ids, a.count, s + lane) == adapter;
        const uint64_t mask = __ballot(mine);
        if (mask == 0) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 16 threads of 8 columns to a token
            const int row = i * 16 + (threadIdx.x >> 4), col = (threadIdx.x & 15) * 8;
            u32x4 v = {0, 0, 0, 0};
            if ((mask >> row & 1) && c0 + col < a.width) {
                const int64_t t = s + row, c = c0 + col;
                if (kCheckpoint)
                    v = restore8(
                        *reinterpret_cast<const uint2 *>(reinterpret_cast<const int8_t *>(a.z.p) + t * a.width + c),
                        a.z.scale[t * ((a.width + kCkBlock - 1) / kCkBlock) + c / kCkBlock]);
                else
                    v = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint16_t *>(a.z.p) + t * a.z.ld + c);
            }
            *reinterpret_cast<u32x4 *>(lds + row * SZ::kRowBytes +
                                       (((col >> 5) ^ SZ::across_swizzle(row)) << 6) + (col & 31) * 2) = v;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // 8 threads to a token: 4 of the first part's 32 ranks, 4 of the second's
            const int row = i * 32 + (threadIdx.x >> 3), part = (threadIdx.x >> 2) & 1, j = (threadIdx.x & 3) * 8;
            u32x4 v = {0, 0, 0, 0};
            if (mask >> row & 1)
                v = *reinterpret_cast<const u32x4 *>(a.low + (s + row) * 2 * a.rank_pad + part * a.rank_pad + j0 + j);
            *reinterpret_cast<u32x4 *>(lds + SZ::kBytes + row * SL::kRowBytes +
                                       ((part ^ SL::across_swizzle(row)) << 6) + j * 2) = v;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kOuterTokens / 16; ++kk) {
            const bf16x8 fz = SZ::read(lds, SZ::read_offset(wave * 32, kk, lane));
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const bf16x8 fl = SL::read(lds + SZ::kBytes, SL::read_offset(part * 32, kk, lane));
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fz, fl, acc, 0, 0, 0);
            }
        }
        __syncthreads();
    }
    const int j = j0 + (lane & 31);
    if (j >= a.rank) return;
    float *dst = a.partial + (((int64_t)blockIdx.z * a.count + adapter) * a.rank + j) * a.width;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t c = c0 + wave * 32 + 8 * q + 4 * (lane >> 5);
        if (c < a.width)
            *reinterpret_cast<float4 *>(dst + c) =
                make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    }
}

// `scale` times the sum of the splits as bf16: dA [count, rank, width] as it lies, or
// dB [count, columns, rank] (columns <= width) transposed.
template <bool kTransposed>
__global__ __launch_bounds__(256) void outer_finish(const float *__restrict__ partial, int splits, int64_t count,
                                                    int rank, int64_t width, int64_t columns, float scale,
                                                    uint16_t *__restrict__ G) {
    const int64_t total = count * rank * width, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        int64_t src = id, c = 0;
        if (kTransposed) {
            const int64_t a = id / (rank * width), r = id - a * rank * width;
            c = r / rank;
            src = (a * rank + r % rank) * width + c;
            if (c >= columns) continue;
            float v = 0.0f;
            for (int s = 0; s < splits; ++s) v += partial[(int64_t)s * total + src];
            G[(a * columns + c) * rank + r % rank] = (uint16_t)bf16_rne(v * scale);
        } else {
            float v = 0.0f;
            for (int s = 0; s < splits; ++s) v += partial[(int64_t)s * total + src];
            G[id] = (uint16_t)bf16_rne(v * scale);
        }
    }
}

// B [count, out, rank] as [count, rank, width], width >= out, zeros beyond.
__global__ __launch_bounds__(256) void turn_kernel(const uint16_t *__restrict__ B, int64_t count, int64_t out,
                                                   int rank, int64_t width, uint16_t *__restrict__ T) {
    const int64_t total = count * rank * width, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t c = id % width, aj = id / width, a = aj / rank, j = aj % rank;
        T[id] = c < out ? B[(a * out + c) * rank + j] : (uint16_t)0;
    }
}

// Rows of `width` >= out columns, zeros beyond.
__global__ __launch_bounds__(256) void widen_kernel(const uint16_t *__restrict__ S, int64_t ld, int64_t tokens,
                                                    int64_t out, int64_t width, uint16_t *__restrict__ D) {
    const int64_t total = tokens * width, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t c = id % width, t = id / width;
        D[id] = c < out ? S[t * ld + c] : (uint16_t)0;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------


constexpr int kTargetBlocks = 1024;
constexpr int64_t kFewTokens = 64;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int rank_pad(int rank) { return (rank + 31) / 32 * 32; }

struct Low {
    int64_t k_split;
    int splits, slots;
};

// Splits of k for the product down to the rank: as many as fill the chip, of
// at least 256 k.
inline Low low_plan(int64_t tokens, int64_t width, int count, int rank) {
    Low p;
    const int64_t tiles = cdiv(tokens, 32) * (rank_pad(rank) / 32);
    const int64_t fill = std::max<int64_t>(1, 4 * kTargetBlocks / tiles);
    p.slots = (int)std::min<int64_t>(std::min<int64_t>(count, 8), std::min(tokens, fill));
    const int64_t blocks = tiles * p.slots;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(cdiv(kTargetBlocks, blocks), cdiv(width, 256)));
    p.k_split = cdiv(cdiv(width, want), 64) * 64;
    p.splits = (int)cdiv(width, p.k_split);
    return p;
}

inline size_t low_partial_bytes(const Low &p, int64_t tokens, int rank) {
    return round_up((size_t)p.splits * tokens * rank_pad(rank) * 4, 256);
}

inline size_t low_bytes(int64_t tokens, int rank) { return round_up((size_t)tokens * 2 * rank_pad(rank) * 2, 256); }

struct Adapters {
    int count, rank;
    const uint16_t *A, *B;
    const float *alpha;
    const int32_t *ids;
};

int shrink(const Rows &z, int64_t tokens, int64_t width, const uint16_t *A, const Adapters &ad, const Low &p,
           float *partial, hipStream_t stream) {
    const ShrinkArgs a{z, tokens, width, A, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, p.k_split, partial};
    const dim3 grid((unsigned)cdiv(tokens, 32), (unsigned)p.splits, (unsigned)(rank_pad(ad.rank) / 32 * p.slots));
    if (z.scale)
        hipLaunchKernelGGL((shrink_kernel<true>), grid, dim3(256), 0, stream, a, p.slots);
    else
        hipLaunchKernelGGL((shrink_kernel<false>), grid, dim3(256), 0, stream, a, p.slots);
    return launch_status();
}

int shrink_to_low(const Rows &z, int64_t tokens, int64_t width, const uint16_t *A, const Adapters &ad, const Low &p,
                  float f, float *partial, uint16_t *low, hipStream_t stream) {
    if (const int st = shrink(z, tokens, width, A, ad, p, partial, stream)) return st;
    hipLaunchKernelGGL(shrink_finish, dim3(grid_for(tokens * rank_pad(ad.rank), 256)), dim3(256), 0, stream, partial,
                       p.splits, tokens, ad.rank, rank_pad(ad.rank), ad.alpha, f, ad.ids, ad.count, low);
    return launch_status();
}

// The 256 x 256 tile where its blocks fill the chip at least once.
template <Layout LW>
int layer(LayerArgs a, hipStream_t stream) {
    const int64_t m = a.W.rows, n = a.X.rows;
    const int64_t large = cdiv(m, Large::kBM) * cdiv(n, Large::kBN);
    if (large >= 256) {
        a.mtiles = (unsigned)cdiv(m, Large::kBM);
        hipLaunchKernelGGL((layer_kernel<Large, LW>), dim3((unsigned)large), dim3(Large::kThreads), 0, stream, a);
    } else {
        a.mtiles = (unsigned)cdiv(m, Small::kBM);
        hipLaunchKernelGGL((layer_kernel<Small, LW>), dim3((unsigned)(a.mtiles * cdiv(n, Small::kBN))),
                           dim3(Small::kThreads), 0, stream, a);
    }
    return launch_status();
}

struct FewPlan {
    int64_t k_split;
    int splits;
};

inline FewPlan few_plan(int64_t in, int64_t out) {
    const int64_t blocks = cdiv(out, 64);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(cdiv(kTargetBlocks, blocks), cdiv(in, 512)));
    FewPlan p;
    p.k_split = cdiv(cdiv(in, want), 128) * 128;
    p.splits = (int)cdiv(in, p.k_split);
    return p;
}

bool sizes_ok(int64_t tokens, int64_t in, int64_t out) {
    return tokens >= 0 && tokens <= kMaxTokens && in >= 0 && in % kGroup == 0 && in <= kMaxWidth && out >= 0 &&
           out <= kMaxWidth;
}

bool adapters_ok(int32_t count, int32_t rank) {
    return count >= 0 && count <= kMaxAdapters && (count == 0 || (rank >= 8 && rank <= kMaxRank && rank % 8 == 0));
}

struct LinearPlan {
    bool few;
    FewPlan base;
    Low low;
    size_t weights, partial, low_partial, low_parts, total;
};

LinearPlan linear_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank) {
    LinearPlan p{};
    p.few = tokens <= kFewTokens;
    if (p.few) {
        p.base = few_plan(in, out);
        p.partial = round_up((size_t)p.base.splits * tokens * out * 4, 256);
    } else {
        p.weights = round_up((size_t)out * in * 2, 256);
    }
    if (count > 0) {
        p.low = low_plan(tokens, in, count, rank);
        p.low_partial = low_partial_bytes(p.low, tokens, rank);
        if (!p.few) p.low_parts = low_bytes(tokens, rank);
    }
    p.total = p.weights + p.partial + p.low_partial + p.low_parts;
    return p;
}

struct GradPlan {
    int64_t width;  // columns of dY as the kernels read it
    bool widen;
    Low v, u;
    int64_t split_a, split_b;
    int splits_a, splits_b;
    size_t weights, dy, turned, low_partial, low, outer, total;
};

// Splits of the tokens for the adapters' gradients.
inline void outer_plan(int64_t tokens, int64_t width, int count, int rank, int64_t &split, int &splits) {
    const int64_t blocks = cdiv(width, kOuterCols) * (rank_pad(rank) / 32) * count;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(cdiv(kTargetBlocks, blocks), cdiv(tokens, 256)));
    split = cdiv(cdiv(tokens, want), kOuterTokens) * kOuterTokens;
    splits = (int)cdiv(tokens, split);
}

GradPlan grad_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank, bool widen) {
    GradPlan p{};
    p.width = cdiv(out, 16) * 16;
    p.widen = widen;
    p.weights = round_up((size_t)out * in * 2, 256);
    p.dy = widen ? round_up((size_t)tokens * p.width * 2, 256) : 0;
    p.turned = round_up((size_t)count * rank * p.width * 2, 256);
    p.v = low_plan(tokens, p.width, count, rank);
    p.u = low_plan(tokens, in, count, rank);
    p.low_partial = std::max(low_partial_bytes(p.v, tokens, rank), low_partial_bytes(p.u, tokens, rank));
    p.low = low_bytes(tokens, rank);
    outer_plan(tokens, in, count, rank, p.split_a, p.splits_a);
    outer_plan(tokens, p.width, count, rank, p.split_b, p.splits_b);
    p.outer = round_up(std::max((size_t)p.splits_a * in, (size_t)p.splits_b * p.width) * count * rank * 4, 256);
    p.total = p.weights + p.dy + p.turned + p.low_partial + 2 * p.low + p.outer;
    return p;
}

// dY is read as it lies when its rows are whole 16-byte words of whole groups.
bool needs_widening(const void *dY, int64_t out, int64_t lddy) {
    return out % 16 != 0 || lddy % 8 != 0 || !aligned(dY, 16);
}

// What the adapters' arrays must be; fills `ad` (count 0 for none).
int check_adapters(const hscale_adapters *w, Adapters &ad) {
    ad = Adapters{};
    if (!w || w->count == 0) return HSCALE_OK;
    if (!adapters_ok(w->count, w->rank)) return HSCALE_ERR_SHAPE;
    if (!w->A || !w->B) return HSCALE_ERR_NULL;
    if (!aligned(w->A, 16) || !aligned(w->B, 16) || !aligned(w->alpha, 4) || !aligned(w->adapter, 4))
        return HSCALE_ERR_ALIGN;
    ad = Adapters{w->count, w->rank, static_cast<const uint16_t *>(w->A), static_cast<const uint16_t *>(w->B),
                  w->alpha, w->adapter};
    return HSCALE_OK;
}

// s = f 2^e with 1 <= f < 2.
inline void split_scale(float s, float &f, float &two_e) {
    int e;
    f = 2.0f * std::frexp(s, &e);
    two_e = std::ldexp(1.0f, e - 1);
}

struct Range {
    const void *p;
    size_t n;
};

// Whether one of the written ranges meets a read one or another written one.
bool any_overlap(const Range *w, int nw, const Range *r, int nr) {
    for (int i = 0; i < nw; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlaps(w[i].p, w[i].n, w[j].p, w[j].n)) return true;
        for (int j = 0; j < nr; ++j)
            if (overlaps(w[i].p, w[i].n, r[j].p, r[j].n)) return true;
    }
    return false;
}

int stored_weights(const uint8_t *codes, const uint8_t *packed, int64_t out, int64_t in, float two_e, void *W,
                   hipStream_t stream) {
    const int64_t groups = out * (in / kGroup);
    hipLaunchKernelGGL(stored_to_bf16, dim3(grid_for(groups, 256)), dim3(256), 0, stream, codes,
                       reinterpret_cast<const uint2 *>(packed), groups, two_e, static_cast<u32x4 *>(W));
    return launch_status();
}

}  // namespace

extern "C" {

int hscale_pack_activations(const void *X, int64_t tokens, int64_t in, int64_t ldx, int8_t *q, float *scale,
                            hipStream_t stream) {
    if (!sizes_ok(tokens, in, 0) || (tokens > 1 && ldx < in)) return HSCALE_ERR_SHAPE;
    if (tokens == 0 || in == 0) return HSCALE_OK;
    if (!X || !q || !scale) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(q, 8) || !aligned(scale, 4))
        return HSCALE_ERR_ALIGN;
    const int64_t blocks = cdiv(in, kCkBlock);
    const Range w[] = {{q, (size_t)tokens * in}, {scale, (size_t)tokens * blocks * 4}};
    const Range r[] = {{X, span(tokens, ldx, in, 2)}};
    if (any_overlap(w, 2, r, 1)) return HSCALE_ERR_OVERLAP;
    hipLaunchKernelGGL(pack_kernel, dim3(grid_for(tokens * blocks * 16, 256)), dim3(256), 0, stream,
                       static_cast<const uint16_t *>(X), tokens, in, ldx, reinterpret_cast<uint2 *>(q), scale);
    return launch_status();
}

int hscale_unpack_activations(const int8_t *q, const float *scale, int64_t tokens, int64_t in, void *X, int64_t ldx,
                              hipStream_t stream) {
    if (!sizes_ok(tokens, in, 0) || (tokens > 1 && ldx < in)) return HSCALE_ERR_SHAPE;
    if (tokens == 0 || in == 0) return HSCALE_OK;
    if (!X || !q || !scale) return HSCALE_ERR_NULL;
    if (!aligned(X, 2) || !aligned(q, 8) || !aligned(scale, 4)) return HSCALE_ERR_ALIGN;
    const int64_t blocks = cdiv(in, kCkBlock);
    const Range w[] = {{X, span(tokens, ldx, in, 2)}};
    const Range r[] = {{q, (size_t)tokens * in}, {scale, (size_t)tokens * blocks * 4}};
    if (any_overlap(w, 1, r, 2)) return HSCALE_ERR_OVERLAP;
    hipLaunchKernelGGL(unpack_kernel, dim3(grid_for(tokens * blocks * 16, 256)), dim3(256), 0, stream,
                       reinterpret_cast<const uint2 *>(q), scale, tokens, in, static_cast<uint16_t *>(X), ldx,
                       aligned(X, 16) && (tokens == 1 || ldx % 8 == 0));
    return launch_status();
}

size_t hscale_adapted_linear_workspace_bytes(int64_t tokens, int64_t in, int64_t out, int32_t count, int32_t rank) {
    if (!sizes_ok(tokens, in, out) || !adapters_ok(count, rank) || tokens == 0 || in == 0 || out == 0) return 0;
    return linear_plan(tokens, in, out, count, rank).total;
}

int hscale_adapted_linear(const void *X, int64_t tokens, int64_t in, int64_t ldx, int64_t out, float global_scale,
                          const uint8_t *scale_codes, const uint8_t *packed_e2m1, const hscale_adapters *adapters,
                          void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!sizes_ok(tokens, in, out) || (tokens > 1 && (ldx < in || ldx > kMaxWidth || ldy < out)))
        return HSCALE_ERR_SHAPE;
    if (tokens == 0 || out == 0) return HSCALE_OK;
    if (in == 0) return HSCALE_ERR_SHAPE;
    if (!scale_ok(global_scale)) return HSCALE_ERR_SCALE;
    Adapters ad;
    if (const int st = check_adapters(adapters, ad)) return st;
    if (!X || !scale_codes || !packed_e2m1 || !Y || !workspace) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(packed_e2m1, 8) || !aligned(Y, 2) ||
        !aligned(workspace, 256))
        return HSCALE_ERR_ALIGN;
    const LinearPlan p = linear_plan(tokens, in, out, ad.count, ad.rank);
    if (workspace_bytes < p.total) return HSCALE_ERR_WORKSPACE;
    const size_t low_size = (size_t)ad.count * ad.rank * 2;
    const Range w[] = {{Y, span(tokens, ldy, out, 2)}, {workspace, p.total}};
    const Range r[] = {{X, span(tokens, ldx, in, 2)}, {scale_codes, (size_t)out * (in / kGroup)},
                       {packed_e2m1, (size_t)out * (in / 2)}, {ad.A, low_size * in}, {ad.B, low_size * out},
                       {ad.alpha, ad.alpha ? (size_t)ad.count * 4 : 0}, {ad.ids, ad.ids ? (size_t)tokens * 4 : 0}};
    if (any_overlap(w, 2, r, 7)) return HSCALE_ERR_OVERLAP;

    char *ws = static_cast<char *>(workspace);
    const Rows x{X, nullptr, ldx};
    uint16_t *y = static_cast<uint16_t *>(Y);
    if (p.few) {
        float *partial = reinterpret_cast<float *>(ws), *low = reinterpret_cast<float *>(ws + p.partial);
        if (ad.count)
            if (const int st = shrink(x, tokens, in, ad.A, ad, p.low, low, stream)) return st;
        const FewArgs a{scale_codes, packed_e2m1, out, in, static_cast<const uint16_t *>(X), tokens, ldx,
                        p.base.k_split, partial};
        const int nt = tokens <= 16 ? 1 : tokens <= 32 ? 2 : 4;
        const dim3 grid((unsigned)cdiv(out, 64), (unsigned)p.base.splits, (unsigned)cdiv(tokens, 16 * nt));
        if (nt == 1)
            hipLaunchKernelGGL((few_kernel<1>), grid, dim3(256), 0, stream, a);
        else if (nt == 2)
            hipLaunchKernelGGL((few_kernel<2>), grid, dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((few_kernel<4>), grid, dim3(256), 0, stream, a);
        if (const int st = launch_status()) return st;
        const FewFinishArgs f{partial, p.base.splits, tokens, out, global_scale, ad.count ? low : nullptr,
                              p.low.splits, ad.rank, rank_pad(ad.rank), ad.count, ad.B, ad.alpha, ad.ids, y, ldy};
        hipLaunchKernelGGL(few_finish, dim3((unsigned)cdiv(out, 256), (unsigned)tokens), dim3(256), 0, stream, f);
        return launch_status();
    }
    void *W = ws;
    float f, two_e;
    split_scale(global_scale, f, two_e);
    float *partial = reinterpret_cast<float *>(ws + p.weights);
    uint16_t *low = reinterpret_cast<uint16_t *>(ws + p.weights + p.low_partial);
    if (const int st = stored_weights(scale_codes, packed_e2m1, out, in, two_e, W, stream)) return st;
    LayerArgs a{};
    if (ad.count) {
        if (const int st = shrink_to_low(x, tokens, in, ad.A, ad, p.low, f, partial, low, stream)) return st;
        a.low = LowRank{low, ad.B, out * ad.rank, ad.rank, ad.count, ad.rank, rank_pad(ad.rank), ad.ids};
    }
    a.W = Operand{W, in, out, in};
    a.X = Operand{X, ldx, tokens, in};
    a.scale = f;
    a.Y = y;
    a.ldy = ldy;
    a.wide = aligned(Y, 16) && (tokens == 1 || ldy % 8 == 0);
    return layer<Along>(a, stream);
}

size_t hscale_adapted_linear_grad_workspace_bytes(int64_t tokens, int64_t in, int64_t out, int32_t count,
                                                  int32_t rank) {
    if (!sizes_ok(tokens, in, out) || !adapters_ok(count, rank) || count == 0 || tokens == 0 || in == 0 || out == 0)
        return 0;
    return grad_plan(tokens, in, out, count, rank, true).total;
}

int hscale_adapted_linear_grad(const void *dY, int64_t tokens, int64_t out, int64_t lddy, const int8_t *q,
                               const float *scale, int64_t in, float global_scale, const uint8_t *scale_codes,
                               const uint8_t *packed_e2m1, const hscale_adapters *adapters, void *dX, int64_t lddx,
                               void *dA, void *dB, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!sizes_ok(tokens, in, out) || (tokens > 1 && (lddy < out || lddy > kMaxWidth || (dX && lddx < in))))
        return HSCALE_ERR_SHAPE;
    if (!adapters) return HSCALE_ERR_NULL;
    if (adapters->count == 0) return HSCALE_ERR_SHAPE;
    Adapters ad;
    if (const int st = check_adapters(adapters, ad)) return st;
    if (in == 0 || out == 0) return HSCALE_ERR_SHAPE;
    if (!scale_ok(global_scale)) return HSCALE_ERR_SCALE;
    if (!dA || !dB) return HSCALE_ERR_NULL;
    if (!aligned(dA, 2) || !aligned(dB, 2)) return HSCALE_ERR_ALIGN;
    GradPlan p{};
    if (tokens > 0) {
        if (!dY || !q || !scale || !scale_codes || !packed_e2m1 || !workspace) return HSCALE_ERR_NULL;
        if (!aligned(dY, 2) || !aligned(q, 8) || !aligned(scale, 4) || !aligned(packed_e2m1, 8) || !aligned(dX, 2) ||
            !aligned(workspace, 256))
            return HSCALE_ERR_ALIGN;
        p = grad_plan(tokens, in, out, ad.count, ad.rank, needs_widening(dY, out, tokens > 1 ? lddy : 0));
        if (workspace_bytes < p.total) return HSCALE_ERR_WORKSPACE;
    }
    const size_t low_size = (size_t)ad.count * ad.rank * 2;
    const Range w[] = {{dX, dX ? span(tokens, lddx, in, 2) : 0}, {dA, low_size * in}, {dB, low_size * out},
                       {workspace, p.total}};
    const Range r[] = {{dY, span(tokens, lddy, out, 2)}, {q, (size_t)tokens * in},
                       {scale, (size_t)tokens * cdiv(in, kCkBlock) * 4},
                       {scale_codes, (size_t)out * (in / kGroup)}, {packed_e2m1, (size_t)out * (in / 2)},
                       {ad.A, low_size * in}, {ad.B, low_size * out},
                       {ad.alpha, ad.alpha ? (size_t)ad.count * 4 : 0}, {ad.ids, ad.ids ? (size_t)tokens * 4 : 0}};
    if (any_overlap(w, 4, r, 9)) return HSCALE_ERR_OVERLAP;

    char *ws = static_cast<char *>(workspace);
    void *W = ws;
    float f, two_e;
    split_scale(global_scale, f, two_e);
    uint16_t *wide_dy = reinterpret_cast<uint16_t *>(ws += p.weights);
    uint16_t *turned = reinterpret_cast<uint16_t *>(ws += p.dy);
    float *partial = reinterpret_cast<float *>(ws += p.turned);
    uint16_t *v = reinterpret_cast<uint16_t *>(ws += p.low_partial);
    uint16_t *u = reinterpret_cast<uint16_t *>(ws += p.low);
    float *outer = reinterpret_cast<float *>(ws += p.low);
    const Rows x{q, scale, in};
    Rows dy{dY, nullptr, lddy};
    if (tokens > 0) {
        if (p.widen) {
            hipLaunchKernelGGL(widen_kernel, dim3(grid_for(tokens * p.width, 256)), dim3(256), 0, stream,
                               static_cast<const uint16_t *>(dY), lddy, tokens, out, p.width, wide_dy);
            if (const int st = launch_status()) return st;
            dy = Rows{wide_dy, nullptr, p.width};
        }
        hipLaunchKernelGGL(turn_kernel, dim3(grid_for(ad.count * ad.rank * p.width, 256)), dim3(256), 0, stream, ad.B,
                           (int64_t)ad.count, out, ad.rank, p.width, turned);
        if (const int st = launch_status()) return st;
        if (const int st = shrink_to_low(dy, tokens, p.width, turned, ad, p.v, f, partial, v, stream)) return st;
        if (const int st = shrink_to_low(x, tokens, in, ad.A, ad, p.u, 1.0f, partial, u, stream)) return st;
        if (dX) {
            if (const int st = stored_weights(scale_codes, packed_e2m1, out, in, two_e, W, stream)) return st;
            LayerArgs a{};
            a.W = Operand{W, in, in, out};
            a.X = Operand{dy.p, dy.ld, tokens, p.width};
            a.scale = f;
            a.low = LowRank{v, ad.A, in * ad.rank, in, ad.count, ad.rank, rank_pad(ad.rank), ad.ids};
            a.Y = static_cast<uint16_t *>(dX);
            a.ldy = lddx;
            a.wide = aligned(dX, 16) && (tokens == 1 || lddx % 8 == 0);
            if (const int st = layer<Across>(a, stream)) return st;
        }
    }
    auto outer_of = [&](const Rows &z, int64_t width, int64_t columns, const uint16_t *low, int64_t split, int splits,
                        float by, void *G, bool transposed) {
        if (tokens > 0) {
            const OuterArgs a{z, tokens, width, low, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, split, outer};
            const dim3 grid((unsigned)cdiv(width, kOuterCols), (unsigned)(rank_pad(ad.rank) / 32 * ad.count),
                            (unsigned)splits);
            if (z.scale)
                hipLaunchKernelGGL((outer_kernel<true>), grid, dim3(256), 0, stream, a);
            else
                hipLaunchKernelGGL((outer_kernel<false>), grid, dim3(256), 0, stream, a);
            if (const int st = launch_status()) return st;
        }
        const dim3 grid(grid_for((int64_t)ad.count * ad.rank * width, 256));
        if (transposed)
            hipLaunchKernelGGL((outer_finish<true>), grid, dim3(256), 0, stream, outer, splits, (int64_t)ad.count,
                               ad.rank, width, columns, by, static_cast<uint16_t *>(G));
        else
            hipLaunchKernelGGL((outer_finish<false>), grid, dim3(256), 0, stream, outer, splits, (int64_t)ad.count,
                               ad.rank, width, columns, by, static_cast<uint16_t *>(G));
        return launch_status();
    };
    if (const int st = outer_of(x, in, in, v, p.split_a, p.splits_a, f, dA, false)) return st;
    return outer_of(dy, tokens > 0 ? p.width : out, out, u, p.split_b, p.splits_b, 1.0f, dB, true);
}

}  // extern "C"
