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

// Eight checkpointed values restored: bf16(fp32(q s)).  A byte becomes a float
// in one operation if it is unsigned, and (q + 128) s - 128 s in one fma rounds
// to the same fp32(q s), as 128 s is exact.
__device__ __forceinline__ u32x4 restore8(uint32_t lo, uint32_t hi, float s) {
    const float less = -128.0f * s;
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = (k < 2 ? lo : hi) ^ 0x80808080u;
        r[k] = bf16_pair(fmaf((float)(w >> (16 * (k & 1)) & 0xFF), s, less),
                         fmaf((float)(w >> (16 * (k & 1) + 8) & 0xFF), s, less));
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
        const uint2 w = q[(t * in + c) >> 3];
        const u32x4 v = restore8(w.x, w.y, scale[blk]);
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

constexpr int kLowStep = 256;  // k of a split: a multiple of it

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
    int64_t k_split;        // of a split, a multiple of kLowStep
    int slots;
    float *partial;         // [splits, tokens, rank_pad]
};

// 128 tokens (32 a wave) x 32 kMI ranks x one split of k per block, 128 k at a
// time; one pass for each adapter that the 128 tokens have, which reads and
// stores only the rows of its own tokens (the nth adapter by the blocks of slot
// n modulo `slots`; a wave without such a token only keeps step).  Reading z
// bounds it: a lane takes
// its token's k straight into registers while the 128 k before multiply, 16
// bytes at a time (two lanes 32 consecutive ones); the adapter's rows, the
// same for all waves, come through LDS, 16-byte chunk c of row j at c ^ (j % 16).
// Checkpoints are taken 256 k at a time, so that as many bytes are under way.
template <bool kCheckpoint, int kMI>
__global__ __launch_bounds__(256, 2) void shrink_kernel(const ShrinkArgs a) {
    constexpr int kK = kCheckpoint ? 256 : 128, kARow = kK * 2, kABytes = 32 * kMI * kARow;
    constexpr int kLoads = 8;  // 16 bytes a lane: 8 or 16 of the kK / 2 k that it takes
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kABytes];
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * 128, t1 = t0 + 128 < a.tokens ? t0 + 128 : a.tokens;
    const int k0 = (int)(blockIdx.y * a.k_split);
    const int k1 = (int)(k0 + a.k_split < a.width ? k0 + a.k_split : a.width), width = (int)a.width;
    const int stages = (k1 - k0 + kK - 1) / kK;
    const int j0 = (int)(blockIdx.z / a.slots) * 32 * kMI, ranks = a.rank - j0 < 32 * kMI ? a.rank - j0 : 32 * kMI;
    const int trow = wave * 32 + (lane & 31);
    const int64_t t = t0 + trow;
    const int own = t < t1 ? adapter_of(a.ids, a.count, t) : kNoAdapter;
    const int blocks = (width + kCkBlock - 1) / kCkBlock;
    const int64_t zrow = kCheckpoint ? a.width : a.z.ld * 2;  // bytes
    const __amdgpu_buffer_rsrc_t rz = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(reinterpret_cast<const char *>(a.z.p)) + t0 * zrow, 0,
        (int)((t1 - t0 - 1) * zrow + (kCheckpoint ? a.width : a.width * 2)), kRawWord3);
    const float *srow = kCheckpoint ? a.z.scale + t * blocks : nullptr;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * 1024;

    struct Taken {
        u32x4 v[kLoads];
        float s[2];
    } z[2];
    int adapter = -1;
    for (int nth = 0;; ++nth) {
        adapter = next_adapter(a.ids, a.count, t0, t1, adapter);
        if (adapter == INT_MAX) break;
        if (nth % a.slots != (int)(blockIdx.z % a.slots)) continue;
        const bool mine = own == adapter, some = __any(mine);
        const u32x4 ra = raw_buffer(a.A + ((int64_t)adapter * a.rank + j0) * a.width, ranks * a.width * 2);
        auto copy_a = [&](int stage) {
            const int k = k0 + stage * kK;
            constexpr int kLanes = kARow / 16, kRows = 64 / kLanes;  // of a row, in a copy
#pragma unroll
            for (int i = 0; i < kABytes / 4096; ++i) {
                const int row = (wave + 4 * i) * kRows + lane / kLanes;
                const int c = k + ((lane % kLanes) ^ (row & 15)) * 8;
                copy_to_lds(ra, row < ranks && c < k1 ? (uint32_t)((row * width + c) * 2) : kNoRead,
                            lds0 + (stage & 1) * kABytes + i * 4096);
            }
        };
        auto take = [&](Taken &r, int stage) {
            const int k = k0 + stage * kK;
#pragma unroll
            for (int p = 0; p < kLoads; ++p) {
                const int c = k + (kCheckpoint ? p * 32 + h * 16 : p * 16 + h * 8);
                r.v[p] = __builtin_amdgcn_raw_buffer_load_b128(
                    rz, mine && c < k1 ? (uint32_t)(trow * zrow + (kCheckpoint ? c : 2 * c)) : kNoRead, 0, 0);
            }
            if (kCheckpoint) {
#pragma unroll
                for (int p = 0; p < 2; ++p) r.s[p] = mine && k + p * kCkBlock < k1 ? srow[k / kCkBlock + p] : 0.0f;
            }
        };
        f32x16 acc[kMI];
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
        auto multiply = [&](const Taken &r, int stage) {
            const uint8_t *buf = lds + (stage & 1) * kABytes + (lane & 31) * kARow;
#pragma unroll
            for (int q = 0; q < kK / 16; ++q) {
                const int chunk = kCheckpoint ? 4 * (q >> 1) + 2 * h + (q & 1) : 2 * q + h;
                const u32x4 w = r.v[kCheckpoint ? q >> 1 : q];
                const u32x4 x = !kCheckpoint ? w
                                : q & 1      ? restore8(w[2], w[3], r.s[q >> 3])
                                             : restore8(w[0], w[1], r.s[q >> 3]);
#pragma unroll
                for (int i = 0; i < kMI; ++i) {
                    const bf16x8 f = *reinterpret_cast<const bf16x8 *>(buf + i * 32 * kARow +
                                                                       ((chunk ^ (lane & 15)) << 4));
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, __builtin_bit_cast(bf16x8, x), acc[i], 0, 0, 0);
                }
                if (q & 1) __builtin_amdgcn_sched_barrier(0);
            }
        };
        copy_a(0);
        if (some) take(z[0], 0);
        for (int s = 0; s < stages; s += 2) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
                if (s + b < stages) {
                    wait_and_barrier();
                    if (s + b + 1 < stages) {
                        copy_a(s + b + 1);
                        if (some) take(z[1 - b], s + b + 1);
                    }
                    if (some) multiply(z[b], s + b);
                }
        }
        wait_and_barrier();
        if (mine) {
            float *dst = a.partial + ((int64_t)blockIdx.y * a.tokens + t) * a.rank_pad + j0;
#pragma unroll
            for (int i = 0; i < kMI; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (j0 + 32 * i < a.rank_pad)
                        *reinterpret_cast<float4 *>(dst + 32 * i + 8 * q + 4 * h) =
                            make_float4(acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]);
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

    __device__ __forceinline__ LowRankStages(const LowRank &low, bool some, int64_t m, int64_t rows, int64_t n,
                                             int64_t tokens)
        : stages(0), w(low), m0(m), prows(rows - m < T::kBM ? rows - m : T::kBM), n0(n),
          n1(n + T::kBN < tokens ? n + T::kBN : tokens) {
        const Place<T> at;
        wave = at.wm + at.wn * T::kWM;
        lane = at.lane;
        if (!w.low || !some) return;
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
    unsigned mtiles, tiles;
    int64_t k_split;
    float *sum;    // [splits, tokens, m]; NULL: one split, written to Y
};

template <class T, Layout LW>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void layer_kernel(const LayerArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    unsigned mt, nt;
    tile_of_block(blockIdx.x % a.tiles, a.tiles, a.mtiles, mt, nt);
    const int64_t split = blockIdx.x / a.tiles;
    const int64_t m0 = (int64_t)mt * T::kBM, n0 = (int64_t)nt * T::kBN;
    const int64_t k0 = split * a.k_split, k1 = k0 + a.k_split < a.X.k ? k0 + a.k_split : a.X.k;
    Acc<T> acc;
    acc.clear();
    // the adapters' stages with the first split
    tile_product<T, LW, Along>(acc, lds, a.W, m0, a.X, n0, k0, k1,
                               LowRankStages<T, LW>(a.low, split == 0, m0, a.W.rows, n0, a.X.rows));
    if (a.sum)
        store_sum<T>(acc, a.sum + split * a.X.rows * a.W.rows, m0, a.W.rows, n0, a.X.rows, a.W.rows % 4 == 0, false);
    else
        store_bf16<T>(acc, lds, a.Y, a.ldy, m0, a.W.rows, n0, a.X.rows, a.wide, a.scale);
}

// `scale` times the sum of the splits, a token's row per blockIdx.y.
__global__ __launch_bounds__(256) void layer_finish(const float *__restrict__ sum, int splits, int64_t tokens,
                                                    int64_t m, float scale, uint16_t *__restrict__ Y, int64_t ldy) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y, plane = tokens * m;
    if (c >= m) return;
    const float *src = sum + t * m + c;
    uint16_t *dst = Y + t * ldy + c;
    if (m % 4 == 0) {
        float4 v = *reinterpret_cast<const float4 *>(src);
        for (int s = 1; s < splits; ++s) {
            const float4 o = *reinterpret_cast<const float4 *>(src + s * plane);
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const uint32_t lo = bf16_pair(v.x * scale, v.y * scale), hi = bf16_pair(v.z * scale, v.w * scale);
        if ((reinterpret_cast<uintptr_t>(dst) & 7) == 0) {
            *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
        } else {
            dst[0] = (uint16_t)lo, dst[1] = (uint16_t)(lo >> 16), dst[2] = (uint16_t)hi, dst[3] = (uint16_t)(hi >> 16);
        }
        return;
    }
    for (int e = 0; e < 4 && c + e < m; ++e) {
        float v = src[e];
        for (int s = 1; s < splits; ++s) v += src[e + s * plane];
        dst[e] = (uint16_t)bf16_rne(v * scale);
    }
}

// ---------------------------------------------------------------------------
// The layer with its adapters, few tokens
// ---------------------------------------------------------------------------

// Down to the rank for few tokens: 32 tokens x 32 ranks x up to 1024 k per
// block, of which each of 8 waves takes an eighth, and one adapter: the nth,
// in the order of the 32 tokens, that they have.  All of a wave's loads are
// under way at once.
constexpr int kFewLowK = 1024;

struct FewLowArgs {
    const uint16_t *X;
    int64_t tokens, ldx, in;
    const uint16_t *A;  // [count, rank, in]
    int count, rank, rank_pad;
    const int32_t *ids;
    float *partial;     // [splits, tokens, rank_pad]
    int splits, slots;  // blocks: token tiles x rank tiles x splits x slots
};

__device__ __forceinline__ void few_low(const FewLowArgs &a, int block, uint8_t *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slot = block % a.slots, split = block / a.slots % a.splits;
    const int rank_tiles = a.rank_pad / 32, rest = block / a.slots / a.splits;
    const int j = rest % rank_tiles * 32 + (lane & 31);
    const int64_t t0 = (int64_t)(rest / rank_tiles) * 32, t1 = t0 + 32 < a.tokens ? t0 + 32 : a.tokens;
    const int64_t t = t0 + (lane & 31);
    const int own = t < t1 ? adapter_of(a.ids, a.count, t) : kNoAdapter;
    bool first = lane < 32 && own != kNoAdapter;
#pragma unroll
    for (int k = 0; k < 31; ++k)
        if (__builtin_amdgcn_readlane(own, k) == own && lane > k) first = false;
    uint64_t mask = __ballot(first);
    for (int nth = 0; nth < slot; ++nth) mask &= mask - 1;
    if (mask == 0) return;
    const int adapter = __builtin_amdgcn_readlane(own, __builtin_ctzll(mask));
    const uint16_t *Arow = a.A + ((int64_t)adapter * a.rank + j) * a.in;
    const uint16_t *Xrow = a.X + t * a.ldx;
    const int64_t c0 = (int64_t)split * kFewLowK + wave * (kFewLowK / 8) + 8 * (lane >> 5);
    constexpr int kSteps = kFewLowK / 8 / 16;
    u32x4 fa[kSteps], fx[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int64_t c = c0 + 16 * k;
        fa[k] = fx[k] = u32x4{0, 0, 0, 0};
        if (c < a.in && j < a.rank) fa[k] = *reinterpret_cast<const u32x4 *>(Arow + c);
        if (c < a.in && t < t1) fx[k] = *reinterpret_cast<const u32x4 *>(Xrow + c);
    }
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[k]),
                                                      __builtin_bit_cast(bf16x8, fx[k]), acc, 0, 0, 0);
    float *red = reinterpret_cast<float *>(lds);  // [8 waves][16][64]
#pragma unroll
    for (int e = 0; e < 16; ++e) red[(wave * 16 + e) * 64 + lane] = acc[e];
    __syncthreads();
    // Thread (wave w, lane) adds elements 2 w and 2 w + 1 of the lane over the waves.
    if (own != adapter) return;
    float v[2] = {0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 8; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) v[e] += red[(w * 16 + 2 * wave + e) * 64 + lane];
    const int row = 8 * (wave >> 1) + 4 * (lane >> 5) + 2 * (wave & 1);
    *reinterpret_cast<float2 *>(a.partial + ((int64_t)split * a.tokens + t) * a.rank_pad + j - (lane & 31) + row) =
        make_float2(v[0], v[1]);
}

// W^ against few tokens: 128 output rows x 16 kNT tokens x one split of k per
// block.  8 waves: 32 rows each, and each half of a 256-k chunk its own four.
// HBM bounds it for few tokens, the conversion of the weights (about 11 cycles
// for two per lane) and LDS reads of X for 64.  A wave's MFMA operand of
// weights comes straight from memory, 32 consecutive weights a lane: which k
// meets which place in a step does not matter, as both operands agree.  X goes
// through LDS, 16 bytes a lane, row t's 16-byte chunk c at c ^ (t % 16).
constexpr int kFewK = 256, kFewRows = 128;

struct FewArgs {
    const uint8_t *codes;
    const uint8_t *packed;
    int64_t out, in;
    const uint16_t *X;
    int64_t tokens, ldx;
    int64_t k_split;  // a multiple of kFewK
    int row_blocks, splits;
    float *partial;   // [splits, tokens, out]
    int low_blocks;   // the first blocks go down to the rank
    FewLowArgs low;
};

template <bool kEven>  // in % 32 == 0: a lane's two scales are one aligned word
struct FewWeights {
    u32x4 p[2];
    uint32_t c[2];
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t rp, const __amdgpu_buffer_rsrc_t rc,
                                         uint32_t prow, uint32_t crow, uint32_t p16, uint32_t c16, uint32_t k) {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            p[f] = __builtin_amdgcn_raw_buffer_load_b128(rp, prow + f * p16 + k / 2, 0, 0);
            if (kEven) {
                c[f] = __builtin_amdgcn_raw_buffer_load_b16(rc, crow + f * c16 + k / 16, 0, 0);
            } else {
                c[f] = __builtin_amdgcn_raw_buffer_load_b8(rc, crow + f * c16 + k / 16, 0, 0);
                c[f] |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rc, crow + f * c16 + k / 16 + 1, 0, 0) << 8;
            }
        }
    }
};

template <int kNT, bool kEven>
__global__ __launch_bounds__(512, 4) void few_kernel(const FewArgs a) {
    constexpr int kXBytes = 16 * kNT * kFewK * 2;
    constexpr int kLdsBytes = 2 * kXBytes > 8 * 4096 ? 2 * kXBytes : 8 * 4096;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
    if ((int)blockIdx.x < a.low_blocks) {
        few_low(a.low, blockIdx.x, lds);
        return;
    }
    const int block = blockIdx.x - a.low_blocks;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave & 3, half = wave >> 2, g = lane >> 4, l16 = lane & 15;
    const int64_t r0 = (int64_t)(block % a.row_blocks) * kFewRows;
    const int split = block / a.row_blocks % a.splits;
    const int64_t t0 = (int64_t)(block / a.row_blocks / a.splits) * 16 * kNT;
    const int64_t k0 = split * a.k_split, k1 = k0 + a.k_split < a.in ? k0 + a.k_split : a.in;
    const int64_t rows = a.out - r0 < kFewRows ? a.out - r0 : kFewRows;
    const int chunks = (int)((k1 - k0 + kFewK - 1) / kFewK);

    // Weights past a row's end are the next row's, and meet zeros of X; past
    // the block's last row they read as zeros.
    const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(a.packed + r0 * (a.in / 2)), 0, (int)(rows * (a.in / 2)), kRawWord3);
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(a.codes + r0 * (a.in / kGroup)), 0, (int)(rows * (a.in / kGroup)), kRawWord3);
    const uint32_t row = rg * 32 + l16;
    const uint32_t prow = row * (uint32_t)(a.in / 2), crow = row * (uint32_t)(a.in / kGroup);
    const uint32_t p16 = 16 * (uint32_t)(a.in / 2), c16 = 16 * (uint32_t)(a.in / kGroup);
    const uint32_t kl = (uint32_t)k0 + half * 128 + g * 32;

    const int64_t toks = a.tokens - t0 < 16 * kNT ? a.tokens - t0 : 16 * kNT;
    const u32x4 rx = raw_buffer(a.X + t0 * a.ldx, ((toks - 1) * a.ldx + a.in) * 2);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * 1024;
    auto copy_x = [&](int chunk) {  // copy i: rows 2 (wave + 8 i) and the next
        const int64_t k = k0 + (int64_t)chunk * kFewK;
#pragma unroll
        for (int i = 0; i < kNT; ++i) {
            const int t = 2 * (wave + 8 * i) + (lane >> 5), c = (lane & 31) ^ (t & 15);
            const uint32_t off = t < toks && k + c * 8 < k1 ? (uint32_t)((t * a.ldx + k + c * 8) * 2) : kNoRead;
            copy_to_lds(rx, off, lds0 + (chunk & 1) * kXBytes + i * 8192);
        }
    };

    f32x4 acc[2][kNT];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int n = 0; n < kNT; ++n) acc[f][n] = f32x4{0, 0, 0, 0};
    FewWeights<kEven> w[2];
    auto compute = [&](const FewWeights<kEven> &v, int chunk) {
        const uint8_t *x = lds + (chunk & 1) * kXBytes + l16 * (kFewK * 2);
        float l[2][2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            l[f][0] = e4m3fn_value(v.c[f] & 0xFF);
            l[f][1] = e4m3fn_value(v.c[f] >> 8 & 0xFF);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 fx[kNT], fw[2];
#pragma unroll
            for (int n = 0; n < kNT; ++n)
                fx[n] = *reinterpret_cast<const bf16x8 *>(x + n * 16 * (kFewK * 2) +
                                                          (((half * 16 + g * 4 + q) ^ l16) << 4));
#pragma unroll
            for (int f = 0; f < 2; ++f) fw[f] = __builtin_bit_cast(bf16x8, stored_eight(v.p[f][q], l[f][q >> 1]));
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int n = 0; n < kNT; ++n)
                    acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[f], fx[n], acc[f][n], 0, 0, 0);
        }
    };
    // A chunk's weights and X come while the chunk before it multiplies.
    copy_x(0);
    w[0].load(rp, rc, prow, crow, p16, c16, kl);
    for (int i = 0; i < chunks; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (i + h < chunks) {
                wait_and_barrier();
                if (i + h + 1 < chunks) {
                    copy_x(i + h + 1);
                    w[1 - h].load(rp, rc, prow, crow, p16, c16, kl + (i + h + 1) * kFewK);
                }
                compute(w[h], i + h);
            }
        }
    }
    __syncthreads();

    // The two halves of k, then out: a lane holds four consecutive rows of a token.
    float4 *red = reinterpret_cast<float4 *>(lds);  // [4 row groups][2][kNT][64]
    if (half == 1) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
                red[((rg * 2 + f) * kNT + n) * 64 + lane] =
                    make_float4(acc[f][n][0], acc[f][n][1], acc[f][n][2], acc[f][n][3]);
    }
    __syncthreads();
    if (half == 1) return;
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            const float4 o = red[((rg * 2 + f) * kNT + n) * 64 + lane];
            const float v[4] = {acc[f][n][0] + o.x, acc[f][n][1] + o.y, acc[f][n][2] + o.z, acc[f][n][3] + o.w};
            const int64_t t = n * 16 + l16, m = rg * 32 + f * 16 + 4 * g;
            if (t >= toks) continue;
            float *dst = a.partial + ((int64_t)split * a.tokens + t0 + t) * a.out + r0 + m;
            if (m + 4 <= rows && (a.out & 3) == 0) {
                *reinterpret_cast<float4 *>(dst) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (m + e < rows) dst[e] = v[e];
            }
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
    float y = 0.0f;
    if (m < a.out)
        for (int s = 0; s < a.splits; ++s) y += a.partial[((int64_t)s * a.tokens + t) * a.out + m];
    y *= a.s_g;
    if (id != kNoAdapter) {
        const uint16_t *b = a.B + ((int64_t)id * a.out + (m < a.out ? m : 0)) * a.rank;
        u32x4 next = *reinterpret_cast<const u32x4 *>(b);
        if ((int)threadIdx.x < a.rank) {
            float v = 0.0f;
#pragma unroll 4
            for (int s = 0; s < a.low_splits; ++s)
                v += a.low[((int64_t)s * a.tokens + t) * a.rank_pad + threadIdx.x];
            u[threadIdx.x] = a.alpha ? v * a.alpha[id] : v;
        }
        __syncthreads();
        for (int j = 0; j < a.rank; j += 8) {
            float v[8];
            unpack8(next, v);
            if (j + 8 < a.rank) next = *reinterpret_cast<const u32x4 *>(b + j + 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) y = fmaf(v[e], u[j + e], y);
        }
    }
    if (m < a.out) a.Y[t * a.ldy + m] = (uint16_t)bf16_rne(y);
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

constexpr int kOuterCols = 256, kOuterTokens = 64, kOuterThreads = 512;

// 256 columns x 32 kRT ranks of one adapter x one split of the tokens.  Stages
// of 64 tokens through LDS, laid out as Stage<Across>; the next stage's rows
// are under way to registers while one multiplies.  Tokens of other adapters
// are not read and enter as zeros, stages without any are passed over: which
// ones have some is found for many stages at a time, so that a stage's rows
// do not wait for its adapters' numbers.
constexpr int kOuterMasks = 256;

template <bool kCheckpoint, int kRT>
__global__ __launch_bounds__(kOuterThreads, 4) void outer_kernel(const OuterArgs a) {
    using SZ = Stage<Across, kOuterCols, 8, kOuterTokens>;
    using SL = Stage<Across, 64, 8, kOuterTokens>;  // of 32 ranks: both parts
    constexpr int kZ = kCheckpoint ? 2 : 4;         // 16-byte words a thread
    __shared__ __attribute__((aligned(16))) uint8_t lds[SZ::kBytes + kRT * SL::kBytes];
    __shared__ uint64_t masks[kOuterMasks];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int c0 = (int)blockIdx.x * kOuterCols, width = (int)a.width;
    const int groups = (a.rank_pad / 32 + kRT - 1) / kRT;
    const int j0 = (int)(blockIdx.y % groups) * 32 * kRT, adapter = blockIdx.y / groups;
    const int64_t t0 = (int64_t)blockIdx.z * a.t_split;
    const int64_t t1 = t0 + a.t_split < a.tokens ? t0 + a.t_split : a.tokens;
    const int blocks = (width + kCkBlock - 1) / kCkBlock;
    const int64_t zrow = kCheckpoint ? a.width : a.z.ld * 2;  // bytes
    const int lrow = a.rank_pad * 4;

    u32x4 z[kZ], l[kRT];
    float scale[kZ];
    // Where a thread's words lie: 16 (bf16: 32) threads to a token's columns,
    // 8 to its 32 ranks, of which 4 to each part.
    auto z_row = [&](int i) { return kCheckpoint ? i * 32 + (tid >> 4) : i * 16 + (tid >> 5); };
    const int zc = kCheckpoint ? (tid & 15) * 16 : (tid & 31) * 8, l_row = tid >> 3, part = (tid >> 2) & 1;

    // The next stage of a run of stages from `base` that has a token of the
    // adapter, from the gth on: its number, and its rows under way.
    auto fetch = [&](int64_t base, int g, int count) {
        uint64_t mask = 0;
        for (; g < count; ++g) {
            mask = masks[g];
            if (mask) break;
        }
        if (g >= count) return count;
        const int64_t s = base + (int64_t)g * kOuterTokens;
        const int64_t rows = t1 - s < kOuterTokens ? t1 - s : kOuterTokens;
        const __amdgpu_buffer_rsrc_t rz = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char *>(reinterpret_cast<const char *>(a.z.p)) + s * zrow, 0,
            (int)((rows - 1) * zrow + (kCheckpoint ? a.width : a.width * 2)), kRawWord3);
        const __amdgpu_buffer_rsrc_t rl = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint16_t *>(a.low) + s * 2 * a.rank_pad, 0, (int)(rows * lrow), kRawWord3);
#pragma unroll
        for (int i = 0; i < kZ; ++i) {
            const int row = z_row(i), c = c0 + zc;
            const bool some = (mask >> row & 1) && c < width;
            z[i] = __builtin_amdgcn_raw_buffer_load_b128(
                rz, some ? (uint32_t)(row * zrow + (kCheckpoint ? c : 2 * c)) : kNoRead, 0, 0);
            if (kCheckpoint) scale[i] = some ? a.z.scale[(s + row) * blocks + c / kCkBlock] : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < kRT; ++r) {
            const int j = j0 + r * 32 + (tid & 3) * 8;
            const bool some = (mask >> l_row & 1) && j < a.rank_pad;
            l[r] = __builtin_amdgcn_raw_buffer_load_b128(
                rl, some ? (uint32_t)(l_row * lrow + (part * a.rank_pad + j) * 2) : kNoRead, 0, 0);
        }
        return g;
    };
    auto put = [&](int row, int col, u32x4 v) {
        *reinterpret_cast<u32x4 *>(lds + row * SZ::kRowBytes + (((col >> 5) ^ SZ::across_swizzle(row)) << 6) +
                                   (col & 31) * 2) = v;
    };

    f32x16 acc[kRT];
#pragma unroll
    for (int r = 0; r < kRT; ++r)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][e] = 0.0f;
    for (int64_t base = t0; base < t1; base += kOuterMasks * kOuterTokens) {
        const int64_t left = (t1 - base + kOuterTokens - 1) / kOuterTokens;
        const int count = left < kOuterMasks ? (int)left : kOuterMasks;
        __syncthreads();
        for (int g = wave; g < count; g += 8) {
            const int64_t t = base + (int64_t)g * kOuterTokens + lane;
            const uint64_t mask = __ballot(t < t1 && adapter_of(a.ids, a.count, t) == adapter);
            if (lane == 0) masks[g] = mask;
        }
        __syncthreads();
        for (int g = fetch(base, 0, count); g < count;) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kZ; ++i) {
                if (kCheckpoint) {
                    put(z_row(i), zc, restore8(z[i][0], z[i][1], scale[i]));
                    put(z_row(i), zc + 8, restore8(z[i][2], z[i][3], scale[i]));
                } else {
                    put(z_row(i), zc, z[i]);
                }
            }
#pragma unroll
            for (int r = 0; r < kRT; ++r)
                *reinterpret_cast<u32x4 *>(lds + SZ::kBytes + r * SL::kBytes + l_row * SL::kRowBytes +
                                           ((part ^ SL::across_swizzle(l_row)) << 6) + (tid & 3) * 16) = l[r];
            __syncthreads();
            g = fetch(base, g + 1, count);
#pragma unroll
            for (int kk = 0; kk < kOuterTokens / 16; ++kk) {
                const bf16x8 fz = SZ::read(lds, SZ::read_offset(wave * 32, kk, lane));
#pragma unroll
                for (int r = 0; r < kRT; ++r)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const bf16x8 fl = SL::read(lds + SZ::kBytes + r * SL::kBytes, SL::read_offset(p * 32, kk, lane));
                        acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fz, fl, acc[r], 0, 0, 0);
                    }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
        const int j = j0 + r * 32 + (lane & 31);
        if (j >= a.rank) continue;
        float *dst = a.partial + (((int64_t)blockIdx.z * a.count + adapter) * a.rank + j) * a.width;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = c0 + wave * 32 + 8 * q + 4 * (lane >> 5);
            if (c < width)
                *reinterpret_cast<float4 *>(dst + c) =
                    make_float4(acc[r][4 * q], acc[r][4 * q + 1], acc[r][4 * q + 2], acc[r][4 * q + 3]);
        }
    }
}

// `scale` times the sum of the splits as bf16: dA [count, rank, width] as it
// lies, four columns a thread.
__global__ __launch_bounds__(256) void outer_finish(const float4 *__restrict__ partial, int splits, int64_t fours,
                                                    float scale, uint16_t *__restrict__ G) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < fours; id += stride) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int s = 0; s < splits; ++s) {
            const float4 o = partial[(int64_t)s * fours + id];
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const uint32_t lo = bf16_pair(v.x * scale, v.y * scale), hi = bf16_pair(v.z * scale, v.w * scale);
        uint16_t *dst = G + id * 4;
        if ((reinterpret_cast<uintptr_t>(G) & 7) == 0) {
            *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
        } else {
            dst[0] = (uint16_t)lo, dst[1] = (uint16_t)(lo >> 16), dst[2] = (uint16_t)hi, dst[3] = (uint16_t)(hi >> 16);
        }
    }
}

// The same for dB [count, columns, rank], 32 columns of one adapter a block:
// sums in along the columns, out along the ranks.
__global__ __launch_bounds__(256) void outer_finish_turned(const float *__restrict__ partial, int splits,
                                                           int64_t count, int rank, int64_t width, int64_t columns,
                                                           float scale, uint16_t *__restrict__ G) {
    __shared__ float tile[kMaxRank * 33];
    const int64_t c0 = (int64_t)blockIdx.x * 32, a = blockIdx.y, plane = count * rank * width;
    const int64_t c = c0 + (threadIdx.x & 31);
    for (int r = threadIdx.x >> 5; r < rank; r += 8) {
        float v = 0.0f;
        if (c < columns)
            for (int s = 0; s < splits; ++s) v += partial[s * plane + (a * rank + r) * width + c];
        tile[r * 33 + (threadIdx.x & 31)] = v * scale;
    }
    __syncthreads();
    const int n = (int)(columns - c0 < 32 ? columns - c0 : 32) * rank;
    for (int i = threadIdx.x; i < n; i += 256)
        G[(a * columns + c0) * rank + i] = (uint16_t)bf16_rne(tile[i % rank * 33 + i / rank]);
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
constexpr int64_t kFewTokens = 64, kFewBlocks = 512;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int rank_pad(int rank) { return (rank + 31) / 32 * 32; }

struct Low {
    int64_t k_split;
    int splits, slots;
};

// Ranks that a block of the product down to the rank takes.
inline int rank_tile(int rank) { return rank <= 32 ? 32 : 64; }

// Splits of k for the product down to the rank: as many as fill the chip, of
// at least 512 k.
inline Low low_plan(int64_t tokens, int64_t width, int count, int rank) {
    Low p;
    const int64_t blocks = cdiv(tokens, 128) * cdiv(rank, rank_tile(rank));
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kTargetBlocks / blocks, cdiv(width, 2 * kLowStep)));
    p.k_split = cdiv(cdiv(width, want), kLowStep) * kLowStep;
    p.splits = (int)cdiv(width, p.k_split);
    // a slot more costs blocks that find no adapter; few tiles leave room for them
    p.slots = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(count, 8), 2 * kTargetBlocks / (blocks * p.splits)));
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
    const ShrinkArgs a{z, tokens, width, A, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, p.k_split, p.slots,
                       partial};
    const dim3 grid((unsigned)cdiv(tokens, 128), (unsigned)p.splits,
                    (unsigned)(cdiv(ad.rank, rank_tile(ad.rank)) * p.slots));
#define SHRINK(c)                                                                    \
    if (ad.rank <= 32)                                                               \
        hipLaunchKernelGGL((shrink_kernel<c, 1>), grid, dim3(256), 0, stream, a);    \
    else                                                                             \
        hipLaunchKernelGGL((shrink_kernel<c, 2>), grid, dim3(256), 0, stream, a)
    if (z.scale) {
        SHRINK(true);
    } else {
        SHRINK(false);
    }
#undef SHRINK
    return launch_status();
}

int shrink_to_low(const Rows &z, int64_t tokens, int64_t width, const uint16_t *A, const Adapters &ad, const Low &p,
                  float f, float *partial, uint16_t *low, hipStream_t stream) {
    if (const int st = shrink(z, tokens, width, A, ad, p, partial, stream)) return st;
    hipLaunchKernelGGL(shrink_finish, dim3(grid_for(tokens * rank_pad(ad.rank), 256)), dim3(256), 0, stream, partial,
                       p.splits, tokens, ad.rank, rank_pad(ad.rank), ad.alpha, f, ad.ids, ad.count, low);
    return launch_status();
}

inline size_t sum_bytes(const Split &p, int64_t m, int64_t n) {
    return p.splits > 1 ? round_up((size_t)p.splits * m * n * 4, 256) : 0;
}

template <Layout LW>
int layer(LayerArgs a, const Split &p, float *sum, hipStream_t stream) {
    const int64_t m = a.W.rows, n = a.X.rows, side = p.large ? 256 : 128;
    a.mtiles = (unsigned)cdiv(m, side);
    a.tiles = (unsigned)(a.mtiles * cdiv(n, side));
    a.k_split = p.k;
    a.sum = p.splits > 1 ? sum : nullptr;
    const dim3 grid(a.tiles * (unsigned)p.splits);
    if (p.large)
        hipLaunchKernelGGL((layer_kernel<Large, LW>), grid, dim3(Large::kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((layer_kernel<Small, LW>), grid, dim3(Small::kThreads), 0, stream, a);
    if (const int st = launch_status()) return st;
    if (p.splits == 1) return HSCALE_OK;
    // rows of a grid's second dimension: at most 65535 tokens at a time
    for (int64_t t = 0; t < n; t += 65535) {
        const dim3 blocks((unsigned)cdiv(m, 1024), (unsigned)std::min<int64_t>(65535, n - t));
        hipLaunchKernelGGL(layer_finish, blocks, dim3(256), 0, stream, sum + t * m, p.splits, n, m, a.scale,
                           a.Y + t * a.ldy, a.ldy);
        if (const int st = launch_status()) return st;
    }
    return HSCALE_OK;
}

struct FewPlan {
    int64_t k_split;
    int splits, low_splits, low_slots;
};

// Splits of k as far as they fill the chip once; every one costs its partial
// sums once more.
inline FewPlan few_plan(int64_t tokens, int64_t in, int64_t out, int count) {
    FewPlan p;
    const int64_t blocks = cdiv(out, kFewRows) * cdiv(tokens, 64);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kFewBlocks / blocks, cdiv(in, kFewK)));
    p.k_split = cdiv(cdiv(in, want), kFewK) * kFewK;
    p.splits = (int)cdiv(in, p.k_split);
    p.low_splits = (int)cdiv(in, kFewLowK);
    p.low_slots = (int)std::min<int64_t>(count, std::min<int64_t>(tokens, 32));
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
    Split tile;
    size_t weights, partial, low_partial, low_parts, total;
};

LinearPlan linear_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank) {
    LinearPlan p{};
    p.few = tokens <= kFewTokens;
    if (p.few) {
        p.base = few_plan(tokens, in, out, count);
        p.partial = round_up((size_t)p.base.splits * tokens * out * 4, 256);
        if (count > 0) p.low_partial = round_up((size_t)p.base.low_splits * tokens * rank_pad(rank) * 4, 256);
    } else {
        p.weights = round_up((size_t)out * in * 2, 256);
        p.tile = split_plan(out, tokens, in);
        p.partial = sum_bytes(p.tile, out, tokens);
        if (count > 0) {
            p.low = low_plan(tokens, in, count, rank);
            p.low_partial = low_partial_bytes(p.low, tokens, rank);
            p.low_parts = low_bytes(tokens, rank);
        }
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
    Split tile;
    size_t weights, dy, turned, low_partial, low, outer, total;
};

// Splits of the tokens for the adapters' gradients.
inline void outer_plan(int64_t tokens, int64_t width, int count, int rank, int64_t &split, int &splits) {
    const int64_t blocks = cdiv(width, kOuterCols) * cdiv(rank, rank_tile(rank)) * count;
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
    p.tile = split_plan(in, tokens, p.width);
    p.outer = std::max(p.outer, sum_bytes(p.tile, in, tokens));  // in turn
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
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(q, 16) || !aligned(scale, 4))
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
    if (!aligned(X, 2) || !aligned(q, 16) || !aligned(scale, 4)) return HSCALE_ERR_ALIGN;
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
        FewArgs a{scale_codes, packed_e2m1, out, in, static_cast<const uint16_t *>(X), tokens, ldx, p.base.k_split,
                  (int)cdiv(out, kFewRows), p.base.splits, partial, 0, {}};
        if (ad.count) {
            a.low = FewLowArgs{a.X, tokens, ldx, in, ad.A, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, low,
                               p.base.low_splits, p.base.low_slots};
            a.low_blocks = (int)cdiv(tokens, 32) * (rank_pad(ad.rank) / 32) * p.base.low_splits * p.base.low_slots;
        }
        const int nt = (int)std::min<int64_t>(cdiv(tokens, 16), 4);
        const dim3 grid((unsigned)(a.low_blocks + (int64_t)a.row_blocks * a.splits * cdiv(tokens, 16 * nt)));
        const bool even = in % 32 == 0 && aligned(scale_codes, 2);
#define FEW(n)                                                                              \
    if (even)                                                                               \
        hipLaunchKernelGGL((few_kernel<n, true>), grid, dim3(512), 0, stream, a);           \
    else                                                                                    \
        hipLaunchKernelGGL((few_kernel<n, false>), grid, dim3(512), 0, stream, a)
        if (nt == 1) {
            FEW(1);
        } else if (nt == 2) {
            FEW(2);
        } else if (nt == 3) {
            FEW(3);
        } else {
            FEW(4);
        }
#undef FEW
        if (const int st = launch_status()) return st;
        const FewFinishArgs f{partial, p.base.splits, tokens, out, global_scale, ad.count ? low : nullptr,
                              p.base.low_splits, ad.rank, rank_pad(ad.rank), ad.count, ad.B, ad.alpha, ad.ids, y, ldy};
        hipLaunchKernelGGL(few_finish, dim3((unsigned)cdiv(out, 256), (unsigned)tokens), dim3(256), 0, stream, f);
        return launch_status();
    }
    void *W = ws;
    float f, two_e;
    split_scale(global_scale, f, two_e);
    float *sum = reinterpret_cast<float *>(ws += p.weights);
    float *partial = reinterpret_cast<float *>(ws += p.partial);
    uint16_t *low = reinterpret_cast<uint16_t *>(ws + p.low_partial);
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
    return layer<Along>(a, p.tile, sum, stream);
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
        if (!aligned(dY, 2) || !aligned(q, 16) || !aligned(scale, 4) || !aligned(packed_e2m1, 8) || !aligned(dX, 2) ||
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
            if (const int st = layer<Across>(a, p.tile, outer, stream)) return st;
        }
    }
    auto outer_of = [&](const Rows &z, int64_t width, int64_t columns, const uint16_t *low, int64_t split, int splits,
                        float by, void *G, bool transposed) {
        if (tokens > 0) {
            const OuterArgs a{z, tokens, width, low, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, split, outer};
            const dim3 grid((unsigned)cdiv(width, kOuterCols),
                            (unsigned)(cdiv(ad.rank, rank_tile(ad.rank)) * ad.count), (unsigned)splits);
            if (z.scale && ad.rank <= 32)
                hipLaunchKernelGGL((outer_kernel<true, 1>), grid, dim3(kOuterThreads), 0, stream, a);
            else if (z.scale)
                hipLaunchKernelGGL((outer_kernel<true, 2>), grid, dim3(kOuterThreads), 0, stream, a);
            else if (ad.rank <= 32)
                hipLaunchKernelGGL((outer_kernel<false, 1>), grid, dim3(kOuterThreads), 0, stream, a);
            else
                hipLaunchKernelGGL((outer_kernel<false, 2>), grid, dim3(kOuterThreads), 0, stream, a);
            if (const int st = launch_status()) return st;
        }
        if (transposed) {
            hipLaunchKernelGGL(outer_finish_turned, dim3((unsigned)cdiv(columns, 32), (unsigned)ad.count), dim3(256),
                               0, stream, outer, splits, (int64_t)ad.count, ad.rank, width, columns, by,
                               static_cast<uint16_t *>(G));
        } else {
            const int64_t fours = (int64_t)ad.count * ad.rank * width / 4;
            hipLaunchKernelGGL(outer_finish, dim3(grid_for(fours, 256)), dim3(256), 0, stream,
                               reinterpret_cast<const float4 *>(outer), splits, fours, by, static_cast<uint16_t *>(G));
        }
        return launch_status();
    };
    if (const int st = outer_of(x, in, in, v, p.split_a, p.splits_a, f, dA, false)) return st;
    return outer_of(dy, tokens > 0 ? p.width : out, out, u, p.split_b, p.splits_b, 1.0f, dB, true);
}

}  // extern "C"
