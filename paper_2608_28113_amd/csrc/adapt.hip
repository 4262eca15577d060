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
// of two of s_g = f 2^e W^ is exact in bf16: the products with W^
// are bf16 products accumulated in fp32, and f multiplies the sum.  u and v are
// kept as two bf16 parts (within 2^-16), so that nothing of the adapters' part
// is rounded to 8 bits before the result is.
//
// Times below are of one MI355X, whose large copies reach 4.9 TB/s, streaming
// reads 6.9 TB/s and large bf16 products 1.4 to 1.5 PFLOP/s.

#include "checks.h"
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

// Tells the compiler that loads to `v` are done, where wait_and_barrier() has
// waited for them.  It does not see that wait, nor the copies to LDS issued
// behind the loads, and its own wait before v's use would be for those.
__device__ __forceinline__ void landed(u32x4 &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void landed(uint32_t &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void landed(float &v) { asm volatile("" : "+v"(v)); }

// The adapters that up to 64 kN tokens have, one after another, in the order
// in which they come first; the same in all lanes of a wave.
template <int kN>
struct Distinct {
    int id[kN];          // of token 64 i + lane
    uint64_t left[kN];   // tokens whose adapter is still to come
    __device__ __forceinline__ void read(const int32_t *ids, int count, int64_t t0, int64_t t1) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int64_t t = t0 + i * 64 + lane;
            id[i] = t < t1 ? adapter_of(ids, count, t) : kNoAdapter;
        }
        restart();
    }
    __device__ __forceinline__ void restart() {
#pragma unroll
        for (int i = 0; i < kN; ++i) left[i] = __ballot(id[i] != kNoAdapter);
    }
    __device__ __forceinline__ int next() {  // kNoAdapter when there are no more
        int a = kNoAdapter;
#pragma unroll
        for (int i = kN - 1; i >= 0; --i)
            if (left[i]) a = __builtin_amdgcn_readlane(id[i], __builtin_ctzll(left[i]));
        if (a == kNoAdapter) return a;
#pragma unroll
        for (int i = 0; i < kN; ++i) left[i] &= ~__ballot(id[i] == a);
        return a;
    }
};

// ---------------------------------------------------------------------------
// Stored weights as bf16
// ---------------------------------------------------------------------------

// The E4M3 value of a scale code times 2^e, exact and without a branch: the
// code's fields moved to those of an fp32 stand for the value times 2^-120, the
// subnormal ones among them.
__device__ __forceinline__ float scale_value(uint32_t code, int e) {
    return ldexpf(__uint_as_float(code << 20), 120 + e);
}

// Two E2M1 values of byte K of `src` times l, as a pair of bf16: exact.
template <int K>
__device__ __forceinline__ uint32_t stored_pair(uint32_t src, float l) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(src, 1.0f, K);
    return __builtin_amdgcn_perm(__float_as_uint(v[1] * l), __float_as_uint(v[0] * l), 0x07060302);
}

__device__ __forceinline__ u32x4 stored_eight(uint32_t src, float l) {
    return u32x4{stored_pair<0>(src, l), stored_pair<1>(src, l), stored_pair<2>(src, l), stored_pair<3>(src, l)};
}

// W^ [groups * 16] with 2^e in place of s_g, one group per thread.  HBM bounds
// it: 14336 x 4096 in 31 us, 4.8 TB/s of 33 MB read and 117 MB written.  For
// many tokens that is less than converting in every tile of the product, whose
// matrix cores would wait for it.
__global__ __launch_bounds__(256) void stored_to_bf16(const uint8_t *__restrict__ codes,
                                                      const uint2 *__restrict__ packed, int64_t groups, int e,
                                                      u32x4 *__restrict__ W) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += stride) {
        const float l = scale_value(codes[g] & 0x7F, e);
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
// in one operation if it is unsigned; (q + 128) - 128 is exact, and the product
// is rounded once.  (One fma of (q + 128) s and -128 s saves an operation, but
// 128 s passes fp32's range where a block's largest magnitude is one of bf16's
// two largest.)
__device__ __forceinline__ u32x4 restore8(uint32_t lo, uint32_t hi, float s) {
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = (k < 2 ? lo : hi) ^ 0x80808080u;
        r[k] = bf16_pair(((float)(w >> (16 * (k & 1)) & 0xFF) - 128.0f) * s,
                         ((float)(w >> (16 * (k & 1) + 8) & 0xFF) - 128.0f) * s);
    }
    return r;
}

// A thread per 8 values, 16 threads per block of 128 (the last of a row may
// be shorter): s = fp32(m fp32(1/127)) with m = max(|x|, 2^-100), and
// q = rint(fp32(x fp32(127 / m))).  HBM bounds this and the way back: 16384 x
// 14336 in 136 and 111 us, 5.2 and 6.4 TB/s.
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
// 8192 x 4096 at rank 16 in 17 to 20 us (3.9 to 3.4 TB/s); a checkpoint of 8192 x
// 14336 at rank 64 in 95 us (1.3 TB/s of 121 MB; MFMA 0.06 and VALU 0.20 busy, 0.44
// of the waves' time waiting): few and short stages, each of which waits for its
// loads and for the block's barrier.
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
    Distinct<2> adapters;
    adapters.read(a.ids, a.count, t0, t1);
    for (int nth = 0;; ++nth) {
        const int adapter = adapters.next();
        if (adapter == kNoAdapter) break;
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
                    if (some) {
#pragma unroll
                        for (int p = 0; p < kLoads; ++p) landed(z[b].v[p]);
                        if (kCheckpoint) landed(z[b].s[0]), landed(z[b].s[1]);
                    }
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

// The sum over the splits in order, 8 loads under way at a time.
__device__ __forceinline__ float sum_splits(const float *__restrict__ p, int splits, int64_t plane) {
    float v = 0.0f;
    for (int s = 0; s < splits; s += 8) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = s + k < splits ? p[(s + k) * plane] : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) v += w[k];
    }
    return v;
}

// alpha / f times the sum of the splits (f multiplies the result that takes it),
// or alpha times it, as two bf16 parts: low[t, j] and low[t, pad + j].  Tokens without an adapter are left as they are; what
// reads `low` skips them.
__global__ __launch_bounds__(256) void shrink_finish(const float *__restrict__ partial, int splits, int64_t tokens,
                                                     int rank, int rank_pad, int pad, const float *__restrict__ alpha,
                                                     float f,
                                                     const int32_t *__restrict__ ids, int count,
                                                     uint16_t *__restrict__ low) {
    const int64_t total = tokens * pad, stride = (int64_t)gridDim.x * 256;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t t = id / pad;
        const int j = (int)(id - t * pad);
        const int a = adapter_of(ids, count, t);
        if (a == kNoAdapter) continue;
        float v = 0.0f;
        if (j < rank) {
            v = sum_splits(partial + t * rank_pad + j, splits, tokens * rank_pad);
            if (alpha) v *= alpha[a];
            v /= f;
        }
        const uint32_t hi = bf16_rne(v);
        low[t * 2 * pad + j] = (uint16_t)hi;
        low[t * 2 * pad + pad + j] = (uint16_t)bf16_rne(v - bf16_value(hi));
    }
}

// ---------------------------------------------------------------------------
// The layer with its adapters, many tokens
// ---------------------------------------------------------------------------

struct LowRank {
    const uint16_t *low;    // [tokens, 2 pad]: two bf16 parts
    const uint16_t *other;  // forward: B [count, out, rank]; backward: A [count, rank, in]
    int64_t other_size;     // elements of one adapter
    int64_t ld;
    int count, rank, pad;
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
    Distinct<T::kBN / 64> adapters;
    int copied[SQ::kCopies];     // of the rows that this lane copies
    int adapter = kNoAdapter, step = 0;  // of the next stage

    __device__ __forceinline__ LowRankStages(const LowRank &low, bool some, int64_t m, int64_t rows, int64_t n,
                                             int64_t tokens)
        : stages(0), w(low), m0(m), prows(rows - m < T::kBM ? rows - m : T::kBM), n0(n),
          n1(n + T::kBN < tokens ? n + T::kBN : tokens) {
        const Place<T> at;
        wave = at.wm + at.wn * T::kWM;
        lane = at.lane;
        if (!w.low || !some) return;
        adapters.read(w.ids, w.count, n0, n1);
#pragma unroll
        for (int i = 0; i < SQ::kCopies; ++i) {
            const int row = SQ::row_of(i, wave, lane);
            copied[i] = n0 + row < n1 ? adapter_of(w.ids, w.count, n0 + row) : kNoAdapter;
        }
        while (adapters.next() != kNoAdapter) stages += per_adapter();
        adapters.restart();
    }
    __device__ __forceinline__ int per_adapter() const { return (2 * w.pad + T::kK - 1) / T::kK; }
    // Column of the adapter's rank that k of its stages stands for, or none.
    __device__ __forceinline__ int column(int k) const {
        const int j = k >= w.pad ? k - w.pad : k;
        return k < 2 * w.pad && j < w.rank ? j : -1;
    }
    __device__ __forceinline__ void set(SP &sp, SQ &sq, bool some) {
        if (!some) {  // stages past the last
            sp.left = sq.left = 0;
            return;
        }
        if (step == 0) adapter = adapters.next();
        const int k0 = step * T::kK, deep = 2 * w.pad;
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
    // 8192 tokens of 4096 -> 14336 with adapters of rank 16: 790 to 826 us, 1.22 to
    // 1.17 PFLOP/s at MFMA 0.62 busy and 1.87 GHz; the plain product in the same
    // tiles reaches 1.25 to 1.35 as the chip's power lets its clock.
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
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int s = 0; s < splits; s += 4) {  // 4 loads under way
            float4 o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[k] = s + k < splits ? *reinterpret_cast<const float4 *>(src + (s + k) * plane)
                                      : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) v.x += o[k].x, v.y += o[k].y, v.z += o[k].z, v.w += o[k].w;
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
    Distinct<1> adapters;
    adapters.read(a.ids, a.count, t0, t1);
    int adapter = adapters.next();
    for (int nth = 0; nth < slot && adapter != kNoAdapter; ++nth) adapter = adapters.next();
    if (adapter == kNoAdapter) return;
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
// block.  8 waves: 32 rows each, and each half of a chunk of k its own four.
// Latency bounds it: the conversion of the weights (about 11 cycles for two per
// lane) keeps the VALU a fifth to a third busy, and the waves wait for loads
// and for each other.  A wave's MFMA operand of
// weights comes straight from memory, 32 consecutive weights a lane: which k
// meets which place in a step does not matter, as both operands agree.  X goes
// through LDS, 16 bytes a lane, row t's 16-byte chunk c at c ^ (t % 16).
// 1 token of 4096 -> 1024 in 6.6 us; 48 of 4096 -> 14336 with 32 adapters in 24 us
// (33 MB of weights, 5 us of HBM's time; VALU 0.20 busy, 0.54 of the waves' time
// waiting: the 256 blocks that go down to the rank come before the 448 of the
// product, which 512 places do not hold together); 515 of 14336 -> 4096 in 104 us,
// 0.58 PFLOP/s, a fifth of it on the empty columns of the fifth block of 128:
// MFMA 0.31, LDS 0.31, VALU 0.33 busy, which two blocks' waves overlap only in
// part.
struct FewArgs {
    const uint8_t *codes;
    const uint8_t *packed;
    int64_t out, in;
    const uint16_t *X;
    int64_t tokens, ldx;
    int64_t k_split;  // a multiple of kFewK
    int row_blocks, splits;
    int e;            // 2^e in place of s_g = f 2^e
    float *partial;   // [splits, tokens, out]; NULL: one split, f times it written to Y
    float f;
    uint16_t *Y;
    int64_t ldy;
    bool wide;        // rows of Y are 8-byte aligned
    int low_blocks;   // the first blocks go down to the rank (then the adapters' part is few_finish's)
    FewLowArgs low;
    LowRank rank;     // or it is added here: rank.low not NULL
};

template <bool kEven, int kNF, int kDepth>  // kEven: in % 32 == 0, a lane's two scales are one aligned word
struct FewWeights {
    u32x4 p[kNF][kDepth];
    uint32_t c[kNF][kDepth];
    __device__ __forceinline__ void landed_all() {
#pragma unroll
        for (int f = 0; f < kNF; ++f)
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                landed(p[f][d]);
                landed(c[f][d]);
            }
    }
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t rp, const __amdgpu_buffer_rsrc_t rc,
                                         uint32_t prow, uint32_t crow, uint32_t p16, uint32_t c16, uint32_t k0) {
#pragma unroll
        for (int f = 0; f < kNF; ++f)
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                const uint32_t k = k0 + d * 128;
                p[f][d] = __builtin_amdgcn_raw_buffer_load_b128(rp, prow + f * p16 + k / 2, 0, 0);
                if (kEven) {
                    c[f][d] = __builtin_amdgcn_raw_buffer_load_b16(rc, crow + f * c16 + k / 16, 0, 0);
                } else {
                    c[f][d] = __builtin_amdgcn_raw_buffer_load_b8(rc, crow + f * c16 + k / 16, 0, 0);
                    c[f][d] |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rc, crow + f * c16 + k / 16 + 1, 0, 0)
                               << 8;
                }
            }
    }
};

template <int kNT, bool kEven>
__global__ __launch_bounds__(512, kNT <= 4 ? 4 : 2) void few_kernel(const FewArgs a) {
    constexpr int kNF = kFewRows / 64;
    constexpr int kDepth = kNT <= 2 ? 2 : 1;  // 128 k of a half at a time
    constexpr int kK = 256 * kDepth, kXRow = kK * 2, kXBytes = 16 * kNT * kXRow;
    constexpr int kRedBytes = 4 * kNF * kNT * 1024;
    constexpr int kLdsBytes = std::max(std::max(2 * kXBytes, kRedBytes), 8 * 4096);
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
    const int chunks = (int)((k1 - k0 + kK - 1) / kK);

    // Weights past a row's end are the next row's, and meet zeros of X; past
    // the block's last row they read as zeros.
    const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(a.packed + r0 * (a.in / 2)), 0, (int)(rows * (a.in / 2)), kRawWord3);
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(a.codes + r0 * (a.in / kGroup)), 0, (int)(rows * (a.in / kGroup)), kRawWord3);
    const uint32_t row = rg * 16 * kNF + l16;
    const uint32_t prow = row * (uint32_t)(a.in / 2), crow = row * (uint32_t)(a.in / kGroup);
    const uint32_t p16 = 16 * (uint32_t)(a.in / 2), c16 = 16 * (uint32_t)(a.in / kGroup);
    const uint32_t kl = (uint32_t)k0 + half * 128 * kDepth + g * 32;

    const int64_t toks = a.tokens - t0 < 16 * kNT ? a.tokens - t0 : 16 * kNT;
    const u32x4 rx = raw_buffer(a.X + t0 * a.ldx, ((toks - 1) * a.ldx + a.in) * 2);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * 1024;
    auto copy_x = [&](int chunk, int buf) {  // a copy: 2 or 1 rows
        const int64_t k = k0 + (int64_t)chunk * kK;
        constexpr int kLanes = kXRow / 16, kRows = 64 / kLanes;
#pragma unroll
        for (int i = 0; i < kXBytes / 8192; ++i) {
            const int t = (wave + 8 * i) * kRows + lane / kLanes, c = (lane % kLanes) ^ (t & 15);
            const uint32_t off = t < toks && k + c * 8 < k1 ? (uint32_t)((t * a.ldx + k + c * 8) * 2) : kNoRead;
            copy_to_lds(rx, off, lds0 + buf * kXBytes + i * 8192);
        }
    };

    f32x4 acc[kNF][kNT];
#pragma unroll
    for (int f = 0; f < kNF; ++f)
#pragma unroll
        for (int n = 0; n < kNT; ++n) acc[f][n] = f32x4{0, 0, 0, 0};
    FewWeights<kEven, kNF, kDepth> w[2];
    auto compute = [&](const FewWeights<kEven, kNF, kDepth> &v, int buf) {
        const uint8_t *x = lds + buf * kXBytes + l16 * kXRow;
#pragma unroll
        for (int d = 0; d < kDepth; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 fx[kNT], fw[kNF];
#pragma unroll
                for (int n = 0; n < kNT; ++n)
                    fx[n] = *reinterpret_cast<const bf16x8 *>(
                        x + n * 16 * kXRow + (((half * 16 * kDepth + d * 16 + g * 4 + q) ^ l16) << 4));
#pragma unroll
                for (int f = 0; f < kNF; ++f)
                    fw[f] = __builtin_bit_cast(
                        bf16x8,
                        stored_eight(v.p[f][d][q], scale_value(v.c[f][d] >> (8 * (q >> 1)) & 0x7F, a.e)));
#pragma unroll
                for (int f = 0; f < kNF; ++f)
#pragma unroll
                    for (int n = 0; n < kNT; ++n)
                        acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[f], fx[n], acc[f][n], 0, 0, 0);
                if (kNF * kNT > 8) __builtin_amdgcn_sched_barrier(0);  // one step's operands at a time
            }
    };
    // A chunk's weights and X come while the one before it multiplies.  (Two
    // chunks ahead is slower: the LDS for a third takes the second block from
    // the CU.)
    copy_x(0, 0);
    w[0].load(rp, rc, prow, crow, p16, c16, kl);
    for (int i = 0; i < chunks; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (i + h < chunks) {
                wait_and_barrier();
                w[h].landed_all();
                if (i + h + 1 < chunks) {
                    copy_x(i + h + 1, 1 - h);
                    w[1 - h].load(rp, rc, prow, crow, p16, c16, kl + (i + h + 1) * kK);
                }
                compute(w[h], h);
            }
        }
    }
    wait_and_barrier();

    // The adapters' part, once: for each adapter that the tokens have, its rows
    // of B against both parts of low; tokens of others enter as zeros.  The
    // halves take every other adapter.
    if (a.rank.low && split == 0) {
        const LowRank &w = a.rank;
        int own[kNT];
#pragma unroll
        for (int n = 0; n < kNT; ++n)
            own[n] = n * 16 + l16 < toks ? adapter_of(w.ids, w.count, t0 + n * 16 + l16) : kNoAdapter;
        Distinct<(kNT + 3) / 4> adapters;
        adapters.read(w.ids, w.count, t0, t0 + toks);
        int nth = 0;
        for (int adapter = adapters.next(); adapter != kNoAdapter; adapter = adapters.next()) {
            if ((nth++ & 1) != half) continue;
            const uint16_t *B = w.other + adapter * w.other_size + (r0 + row) * w.rank;
            for (int k = g * 8; k < 2 * w.pad; k += 32) {
                const int j = k >= w.pad ? k - w.pad : k;
                u32x4 fw[kNF], fx[kNT];
#pragma unroll
                for (int f = 0; f < kNF; ++f) {
                    fw[f] = u32x4{0, 0, 0, 0};
                    if (j < w.rank && (int64_t)row + f * 16 < rows)
                        fw[f] = *reinterpret_cast<const u32x4 *>(B + f * 16 * w.rank + j);
                }
#pragma unroll
                for (int n = 0; n < kNT; ++n) {
                    fx[n] = u32x4{0, 0, 0, 0};
                    if (own[n] == adapter)
                        fx[n] = *reinterpret_cast<const u32x4 *>(w.low + (t0 + n * 16 + l16) * 2 * w.pad + k);
                }
#pragma unroll
                for (int f = 0; f < kNF; ++f)
#pragma unroll
                    for (int n = 0; n < kNT; ++n)
                        acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[f]),
                                                                            __builtin_bit_cast(bf16x8, fx[n]),
                                                                            acc[f][n], 0, 0, 0);
            }
        }
    }

    // The two halves of k, then out: a lane holds four consecutive rows of a token.
    float4 *red = reinterpret_cast<float4 *>(lds);  // [4 row groups][kNF][kNT][64]
    if (half == 1) {
#pragma unroll
        for (int f = 0; f < kNF; ++f)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
                red[((rg * kNF + f) * kNT + n) * 64 + lane] =
                    make_float4(acc[f][n][0], acc[f][n][1], acc[f][n][2], acc[f][n][3]);
    }
    __syncthreads();
    if (half == 1) return;
#pragma unroll
    for (int f = 0; f < kNF; ++f)
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            const float4 o = red[((rg * kNF + f) * kNT + n) * 64 + lane];
            const float v[4] = {acc[f][n][0] + o.x, acc[f][n][1] + o.y, acc[f][n][2] + o.z, acc[f][n][3] + o.w};
            const int64_t t = n * 16 + l16, m = (rg * kNF + f) * 16 + 4 * g;
            if (t >= toks) continue;
            if (!a.partial) {
                uint16_t *dst = a.Y + (t0 + t) * a.ldy + r0 + m;
                const uint32_t lo = bf16_pair(v[0] * a.f, v[1] * a.f), hi = bf16_pair(v[2] * a.f, v[3] * a.f);
                if (m + 4 <= rows && a.wide) {
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (m + e < rows) dst[e] = (uint16_t)((e < 2 ? lo : hi) >> (16 * (e & 1)));
                }
                continue;
            }
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
    float f;
    const float *low;      // [low_splits, tokens, rank_pad]
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
    const int id = adapter_of(a.ids, a.count, t);
    const int64_t plane = a.tokens * a.out, low_plane = a.tokens * a.rank_pad;
    float y = m < a.out ? sum_splits(a.partial + t * a.out + m, a.splits, plane) * a.f : 0.0f;
    if (id != kNoAdapter) {
        const uint16_t *b = a.B + ((int64_t)id * a.out + (m < a.out ? m : 0)) * a.rank;
        u32x4 next = *reinterpret_cast<const u32x4 *>(b);
        if ((int)threadIdx.x < a.rank) {
            const float v = sum_splits(a.low + t * a.rank_pad + threadIdx.x, a.low_splits, low_plane);
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
    const uint16_t *low;  // [tokens, 2 pad]
    int count, rank, pad;
    const int32_t *ids;
    int64_t t_split;      // of a split, a multiple of 64
    float *partial;       // [splits, count, rank, width]
    // of a single split: the result, `by` times the sums, in place of `partial`
    uint16_t *G;          // dA [count, rank, width], dB [count, columns, rank]
    int64_t columns;
    float by;
};

// 256 columns x 32 kRT ranks of one adapter x one split of the tokens.  Stages
// of 64 tokens through LDS, laid out as Stage<Across>; the next stage's rows
// are under way to registers while one multiplies.  Tokens of other adapters
// are not read and enter as zeros, stages without any are passed over: which
// ones have some is found for many stages at a time, so that a stage's rows
// do not wait for its adapters' numbers.  A checkpoint of 8192 x 14336 (two
// parts of rank 64, four adapters, nearly all tokens of one of them) takes 90 us,
// dY of 8192 x 4096 46: the blocks that have tokens of their adapter are a
// quarter of all, not many more than run at once, and the longest last.  Sharing
// out the stages evenly cost more than that on these tokens (121 and 78 us: every
// block then visits every part of them).
constexpr int kOuterMasks = 256, kOuterThreads = 512;

// Four bf16 values to where they may not be aligned together.
__device__ __forceinline__ void store_four(uint16_t *dst, uint32_t lo, uint32_t hi) {
    if ((reinterpret_cast<uintptr_t>(dst) & 7) == 0) {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
    } else {
        dst[0] = (uint16_t)lo, dst[1] = (uint16_t)(lo >> 16), dst[2] = (uint16_t)hi, dst[3] = (uint16_t)(hi >> 16);
    }
}

template <bool kCheckpoint, int kRT>
__global__ __launch_bounds__(kOuterThreads, 4) void outer_kernel(const OuterArgs a) {
    using SZ = Stage<Across, kOuterCols, 8, kOuterTokens>;
    using SL = Stage<Across, 64, 8, kOuterTokens>;  // of 32 ranks: both parts
    constexpr int kZ = kCheckpoint ? 2 : 4;         // 16-byte words a thread
    __shared__ __attribute__((aligned(16))) uint8_t lds[SZ::kBytes + kRT * SL::kBytes];
    __shared__ uint64_t masks[kOuterMasks];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int c0 = (int)blockIdx.x * kOuterCols, width = (int)a.width;
    const int groups = (a.rank + 32 * kRT - 1) / (32 * kRT);
    const int j0 = (int)(blockIdx.y % groups) * 32 * kRT, adapter = blockIdx.y / groups;
    const int64_t t0 = (int64_t)blockIdx.z * a.t_split;
    const int64_t t1 = t0 + a.t_split < a.tokens ? t0 + a.t_split : a.tokens;
    const int blocks = (width + kCkBlock - 1) / kCkBlock;
    const int64_t zrow = kCheckpoint ? a.width : a.z.ld * 2;  // bytes
    const int lrow = a.pad * 4;

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
            const_cast<uint16_t *>(a.low) + s * 2 * a.pad, 0, (int)(rows * lrow), kRawWord3);
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
            const bool some = (mask >> l_row & 1) && j < a.pad;
            l[r] = __builtin_amdgcn_raw_buffer_load_b128(
                rl, some ? (uint32_t)(l_row * lrow + (part * a.pad + j) * 2) : kNoRead, 0, 0);
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
        if (a.G) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = c0 + wave * 32 + 8 * q + 4 * (lane >> 5);
                const uint32_t lo = bf16_pair(acc[r][4 * q] * a.by, acc[r][4 * q + 1] * a.by);
                const uint32_t hi = bf16_pair(acc[r][4 * q + 2] * a.by, acc[r][4 * q + 3] * a.by);
                if constexpr (kCheckpoint) {
                    if (c < width) store_four(a.G + ((int64_t)adapter * a.rank + j) * width + c, lo, hi);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < a.columns)
                            a.G[((int64_t)adapter * a.columns + c + e) * a.rank + j] =
                                (uint16_t)((e < 2 ? lo : hi) >> (16 * (e & 1)));
                }
            }
            continue;
        }
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
        store_four(G + id * 4, lo, hi);
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
        const float v = c < columns ? sum_splits(partial + (a * rank + r) * width + c, splits, plane) : 0.0f;
        tile[r * 33 + (threadIdx.x & 31)] = v * scale;
    }
    __syncthreads();
    const int n = (int)(columns - c0 < 32 ? columns - c0 : 32) * rank;
    for (int i = threadIdx.x; i < n; i += 256)
        G[(a * columns + c0) * rank + i] = (uint16_t)bf16_rne(tile[i % rank * 33 + i / rank]);
}

// B [count, out, rank] as [count, rank, width], width >= out, zeros beyond: 32
// columns of one adapter a block, whole rows in and runs of columns out.
__global__ __launch_bounds__(256) void turn_kernel(const uint16_t *__restrict__ B, int64_t out, int rank, int64_t width,
                                                   uint16_t *__restrict__ T) {
    __shared__ uint16_t tile[32 * (kMaxRank + 2)];
    const int64_t c0 = (int64_t)blockIdx.x * 32, a = blockIdx.y;
    const int row = rank + 2, words = rank / 8;
    for (int i = threadIdx.x; i < 32 * words; i += 256) {
        const int c = i / words, k = i - c * words;
        u32x4 v = {0, 0, 0, 0};
        if (c0 + c < out) v = *reinterpret_cast<const u32x4 *>(B + (a * out + c0 + c) * rank + k * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t *>(tile + c * row + k * 8 + 2 * e) = v[e];
    }
    __syncthreads();
    const int c = (threadIdx.x & 15) * 2;
    if (c0 + c >= width) return;
    for (int j = threadIdx.x >> 4; j < rank; j += 16)
        *reinterpret_cast<uint32_t *>(T + (a * rank + j) * width + c0 + c) =
            (uint32_t)tile[c * row + j] | (uint32_t)tile[(c + 1) * row + j] << 16;
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
    hipLaunchKernelGGL(shrink_finish, dim3(grid_for(tokens * low_pad(ad.rank), 256)), dim3(256), 0, stream, partial,
                       p.splits, tokens, ad.rank, rank_pad(ad.rank), low_pad(ad.rank), ad.alpha, f, ad.ids, ad.count, low);
    return launch_status();
}

int sum_of_splits(const float *sum, int splits, int64_t tokens, int64_t m, float scale, uint16_t *Y, int64_t ldy,
                  hipStream_t stream) {
    for (int64_t t = 0; t < tokens; t += 65535) {  // as many rows has a grid
        const dim3 blocks((unsigned)cdiv(m, 1024), (unsigned)std::min<int64_t>(65535, tokens - t));
        hipLaunchKernelGGL(layer_finish, blocks, dim3(256), 0, stream, sum + t * m, splits, tokens, m, scale,
                           Y + t * ldy, ldy);
        if (const int st = launch_status()) return st;
    }
    return HSCALE_OK;
}

template <Layout LW>
int layer(LayerArgs a, const Split &p, float *sum, hipStream_t stream) {
    const int64_t m = a.W.rows, n = a.X.rows;
    a.mtiles = (unsigned)cdiv(m, p.side_m());
    a.tiles = (unsigned)p.units(m, n);
    a.k_split = p.k;
    a.sum = p.splits > 1 ? sum : nullptr;
#define LAYER(T) layer_kernel<T, LW>
    LAUNCH_TILES(LAYER, Large, p.size, a.tiles * (unsigned)p.splits, stream, a);
#undef LAYER
    if (const int st = launch_status()) return st;
    return p.splits > 1 ? sum_of_splits(sum, p.splits, n, m, a.scale, a.Y, a.ldy, stream) : HSCALE_OK;
}

bool sizes_ok(int64_t tokens, int64_t in, int64_t out) {
    return tokens >= 0 && tokens <= kMaxTokens && in >= 0 && in % kGroup == 0 && in <= kMaxWidth && out >= 0 &&
           out <= kMaxWidth;
}

bool adapters_ok(int32_t count, int32_t rank) {
    return count >= 0 && count <= kMaxAdapters && (count == 0 || (rank >= 8 && rank <= kMaxRank && rank % 8 == 0));
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

// s = f 2^e with 1 <= f < 2, or more where 2^e would take the largest weight,
// 448 x 6, out of bf16's range.
inline void split_scale(float s, float &f, int &e) {
    constexpr int kMostE = 100;
    f = 2.0f * std::frexp(s, &e);
    --e;
    if (e > kMostE) {
        f = std::ldexp(f, e - kMostE);
        e = kMostE;
    }
}

int stored_weights(const uint8_t *codes, const uint8_t *packed, int64_t out, int64_t in, int e, void *W,
                   hipStream_t stream) {
    const int64_t groups = out * (in / kGroup);
    hipLaunchKernelGGL(stored_to_bf16, dim3(grid_for(groups, 256)), dim3(256), 0, stream, codes,
                       reinterpret_cast<const uint2 *>(packed), groups, e, static_cast<u32x4 *>(W));
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
    return most_linear(tokens, in, out, count, rank);
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
    const LinearPlan p = linear_plan(tokens, in, out, ad.count, ad.rank);
    const size_t need = most_linear(tokens, in, out, ad.count, ad.rank);
    if (!X || !scale_codes || !packed_e2m1 || !Y || (!workspace && need)) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || (tokens > 1 && ldx % 8 != 0) || !aligned(packed_e2m1, 8) || !aligned(Y, 2) ||
        !aligned(workspace, 256))
        return HSCALE_ERR_ALIGN;
    if (workspace_bytes < need) return HSCALE_ERR_WORKSPACE;
    const size_t low_size = (size_t)ad.count * ad.rank * 2;
    const Range w[] = {{Y, span(tokens, ldy, out, 2)}, {workspace, p.total}};
    const Range r[] = {{X, span(tokens, ldx, in, 2)}, {scale_codes, (size_t)out * (in / kGroup)},
                       {packed_e2m1, (size_t)out * (in / 2)}, {ad.A, low_size * in}, {ad.B, low_size * out},
                       {ad.alpha, ad.alpha ? (size_t)ad.count * 4 : 0}, {ad.ids, ad.ids ? (size_t)tokens * 4 : 0}};
    if (any_overlap(w, 2, r, 7)) return HSCALE_ERR_OVERLAP;

    char *ws = static_cast<char *>(workspace);
    const Rows x{X, nullptr, ldx};
    uint16_t *y = static_cast<uint16_t *>(Y);
    float f;
    int e;
    split_scale(global_scale, f, e);
    void *W = ws;
    float *sum = reinterpret_cast<float *>(ws += p.weights);
    float *low_sum = reinterpret_cast<float *>(ws += p.partial);
    uint16_t *low = reinterpret_cast<uint16_t *>(ws + p.low_partial);
    LowRank rank{};
    if (p.low_parts) {
        if (const int st = shrink_to_low(x, tokens, in, ad.A, ad, p.low, f, low_sum, low, stream)) return st;
        rank = LowRank{low, ad.B, out * ad.rank, ad.rank, ad.count, ad.rank, low_pad(ad.rank), ad.ids};
    }
    if (p.few) {
        FewArgs a{};
        a.codes = scale_codes;
        a.packed = packed_e2m1;
        a.out = out, a.in = in;
        a.X = static_cast<const uint16_t *>(X);
        a.tokens = tokens, a.ldx = ldx;
        a.k_split = p.base.k_split;
        a.row_blocks = (int)cdiv(out, kFewRows);
        a.splits = p.base.splits;
        a.e = e, a.f = f;
        a.partial = p.partial ? sum : nullptr;
        a.Y = y, a.ldy = ldy, a.wide = aligned(Y, 8) && (tokens == 1 || ldy % 4 == 0);
        a.rank = rank;
        if (p.base.fused) {
            a.low = FewLowArgs{a.X, tokens, ldx, in, ad.A, ad.count, ad.rank, rank_pad(ad.rank), ad.ids, low_sum,
                               p.base.low_splits, p.base.low_slots};
            a.low_blocks = (int)few_low_blocks(p.base, tokens, ad.rank);
        }
        const int nt = p.base.tile;
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
        } else if (nt == 4) {
            FEW(4);
        } else {
            FEW(8);
        }
#undef FEW
        if (const int st = launch_status()) return st;
        if (!p.base.fused) return p.partial ? sum_of_splits(sum, p.base.splits, tokens, out, f, y, ldy, stream) : HSCALE_OK;
        const FewFinishArgs last{sum, p.base.splits, tokens, out, f, low_sum, p.base.low_splits, ad.rank,
                              rank_pad(ad.rank), ad.count, ad.B, ad.alpha, ad.ids, y, ldy};
        hipLaunchKernelGGL(few_finish, dim3((unsigned)cdiv(out, 256), (unsigned)tokens), dim3(256), 0, stream, last);
        return launch_status();
    }
    if (const int st = stored_weights(scale_codes, packed_e2m1, out, in, e, W, stream)) return st;
    LayerArgs a{};
    a.low = rank;
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
    return most_grad(tokens, in, out, count, rank, true);
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
    size_t need = 0;
    if (tokens > 0) {
        if (!dY || !q || !scale || !scale_codes || !packed_e2m1 || !workspace) return HSCALE_ERR_NULL;
        if (!aligned(dY, 2) || !aligned(q, 16) || !aligned(scale, 4) || !aligned(packed_e2m1, 8) || !aligned(dX, 2) ||
            !aligned(workspace, 256))
            return HSCALE_ERR_ALIGN;
        p = grad_plan(tokens, in, out, ad.count, ad.rank, needs_widening(dY, out, tokens > 1 ? lddy : 0));
        need = most_grad(tokens, in, out, ad.count, ad.rank, p.widen);
        if (workspace_bytes < need) return HSCALE_ERR_WORKSPACE;
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
    float f;
    int e;
    split_scale(global_scale, f, e);
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
        hipLaunchKernelGGL(turn_kernel, dim3((unsigned)cdiv(p.width, 32), (unsigned)ad.count), dim3(256), 0, stream,
                           ad.B, out, ad.rank, p.width, turned);
        if (const int st = launch_status()) return st;
        if (const int st = shrink_to_low(dy, tokens, p.width, turned, ad, p.v, f, partial, v, stream)) return st;
        if (const int st = shrink_to_low(x, tokens, in, ad.A, ad, p.u, 1.0f, partial, u, stream)) return st;
        if (dX) {
            if (const int st = stored_weights(scale_codes, packed_e2m1, out, in, e, W, stream)) return st;
            LayerArgs a{};
            a.W = Operand{W, in, in, out};
            a.X = Operand{dy.p, dy.ld, tokens, p.width};
            a.scale = f;
            a.low = LowRank{v, ad.A, in * ad.rank, in, ad.count, ad.rank, low_pad(ad.rank), ad.ids};
            a.Y = static_cast<uint16_t *>(dX);
            a.ldy = lddx;
            a.wide = aligned(dX, 16) && (tokens == 1 || lddx % 8 == 0);
            if (const int st = layer<Across>(a, p.tile, outer, stream)) return st;
        }
    }
    auto outer_of = [&](const Rows &z, int64_t width, int64_t columns, const uint16_t *low, int64_t split, int splits,
                        float by, void *G, bool transposed) {
        if (tokens > 0) {
            const OuterArgs a{z, tokens, width, low, ad.count, ad.rank, low_pad(ad.rank), ad.ids, split, outer,
                              splits == 1 ? static_cast<uint16_t *>(G) : nullptr, columns, by};
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
            const int st = launch_status();
            if (st || splits == 1) return st;
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
