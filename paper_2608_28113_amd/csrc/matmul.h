// bf16 matrix products on the matrix cores, shared by adapt.hip and loss.hip.
//
//   C[m, n] = sum_k P[m, k] Q[n, k],   P and Q bf16, C in fp32 registers,
//
// for operands stored either with k along a row (row-major [m, k]: `Along`) or
// with k across rows (row-major [k, m]: `Across`), so that a forward product
// and both products of its backward pass read the same arrays as they lie.
// A block computes a kBM x kBN tile; what becomes of it is the caller's
// epilogue.  Consecutive m of one n share a lane, so arrays stored with m
// along a row are written in 8-byte pieces.
#pragma once

#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kRawWord3 = 0x00020000u;   // raw (untyped) buffer, 32-bit data format
constexpr uint32_t kNoRead = 0x7FFF0000u;     // an offset beyond every descriptor: reads zeros
constexpr int64_t kMostBytes = 0x7FF00000;    // of one descriptor
constexpr int kStageK = 64;                   // k per LDS stage

__device__ __forceinline__ u32x4 raw_buffer(const void *p, int64_t bytes) {
    const uint64_t a = reinterpret_cast<uintptr_t>(p);
    const int64_t n = bytes < 0 ? 0 : bytes < kMostBytes ? bytes : kMostBytes;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)n), kRawWord3};
}

// Starts a copy of 16 bytes per lane to LDS at `dst` + 16 x lane; the caller
// waits for vmcnt.  In assembly because the compiler, which cannot tell the
// buffer being filled from the one being read, puts a wait for the builtin's
// copies before LDS reads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(u32x4 rsrc, uint32_t offset, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(dst), "v"(offset), "s"(rsrc)
                 : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ void wait_and_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ uint32_t bf16_rne(float f) {  // NaN stays NaN
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return bf16_rne(a) | (bf16_rne(b) << 16); }

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// One operand: `rows` of m (or n) and `k`, at a leading dimension of `ld`
// elements (a multiple of 8; the array is 16-byte aligned).  The one that lies
// along a row is a multiple of 8 too.  Rows and k beyond read as zeros.
struct Operand {
    const void *p;
    int64_t ld, rows, k;
};

enum Layout { Along, Across };

// Stages of one operand's kRows x kStageK tile in LDS, filled by kWaves waves
// with copies of 1 KB (16 bytes a lane).  Along: a row holds its 64 k (128
// bytes), the 16-byte chunk c at position c ^ ((row / 2) % 8), so that the 16
// rows that an operand read serves at a time fall in 16 different 16-byte
// columns of the banks.  Across: a row holds one k of all kRows (2 kRows
// bytes), its 64-byte chunk c at c ^ (k % 4) (for 64 rows c ^ (k / 2 % 2)), so
// that the four k rows of a transposed read fall in different banks.
template <Layout L, int kRows, int kWaves>
struct Stage {
    static constexpr int kBytes = kRows * kStageK * 2;
    static constexpr int kCopies = kBytes / 1024 / kWaves;  // per wave and stage
    static_assert(kBytes % (1024 * kWaves) == 0, "whole copies per wave");
    static constexpr int kRowBytes = L == Along ? kStageK * 2 : kRows * 2;
    static constexpr int kLanesPerRow = kRowBytes / 16;

    uint32_t off[kCopies];  // of this lane from the stage's first byte
    const char *base;       // of the next stage
    int64_t left;           // bytes from base to the array's end
    int64_t step;           // bytes from stage to stage
    int64_t k_left;
    int chunk;              // Along: the lane's 16-byte chunk of its row

    static __device__ __forceinline__ int across_swizzle(int k) { return kRows == 64 ? (k >> 1) & 1 : k & 3; }

    // The tile at row r0, and k from k0 on.
    __device__ __forceinline__ void init(const Operand &o, int64_t r0, int64_t k0, int64_t k1, int wave, int lane) {
        const int64_t rows = o.rows - r0 < kRows ? o.rows - r0 : kRows;
        k_left = (k1 < o.k ? k1 : o.k) - k0;
        if (L == Along) {
            base = reinterpret_cast<const char *>(o.p) + (r0 * o.ld + k0) * 2;
            left = ((rows - 1) * o.ld + k_left) * 2;
            step = kStageK * 2;
        } else {
            base = reinterpret_cast<const char *>(o.p) + (k0 * o.ld + r0) * 2;
            left = ((k_left - 1) * o.ld + rows) * 2;
            step = kStageK * o.ld * 2;
        }
        if (rows <= 0 || k_left <= 0) left = 0;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = (wave + i * kWaves) * (64 / kLanesPerRow) + lane / kLanesPerRow;
            const int pos = lane % kLanesPerRow;
            if (L == Along) {
                chunk = pos ^ ((row >> 1) & 7);  // the same for every i: kWaves is even
                off[i] = row < rows ? (uint32_t)(row * o.ld * 2 + chunk * 16) : kNoRead;
            } else {
                const int col = ((((pos >> 2) ^ across_swizzle(row)) << 2) | (pos & 3)) * 8;
                off[i] = col < rows ? (uint32_t)(row * o.ld * 2 + col * 2) : kNoRead;
            }
        }
    }

    // Starts the copies of the next stage into LDS address `dst` (of this
    // wave's first copy).
    __device__ __forceinline__ void issue(uint32_t dst) {
        if (L == Along && k_left < kStageK && chunk * 8 >= k_left) {  // k past the end: the row's next values are not read
#pragma unroll
            for (int i = 0; i < kCopies; ++i) off[i] = kNoRead;
        }
        const u32x4 r = raw_buffer(base, left);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(r, off[i], dst + i * kWaves * 1024);
        base += step;
        left -= step;
        k_left -= kStageK;
    }

    // Offset of the 8 k of step kk (16 k) that this lane holds of a 32-row
    // operand block at row r.
    static __device__ __forceinline__ int read_offset(int r, int kk, int lane) {
        if (L == Along) {
            const int row = r + (lane & 31);
            return row * kRowBytes + (((2 * kk + (lane >> 5)) ^ ((row >> 1) & 7)) << 4);
        }
        // A transposed read gives lane p of 16 the four k of column p from a
        // 4-row x 16-column block whose row p / 4 the lane addresses; two
        // reads are the 8 k.
        const int p = lane & 15, g = lane >> 4;
        const int k = kk * 16 + 8 * (g >> 1) + (p >> 2);
        const int byte = r * 2 + 32 * (g & 1) + 8 * (p & 3);
        return k * kRowBytes + ((((byte >> 6) ^ across_swizzle(k)) << 6) | (byte & 63));
    }

    static __device__ __forceinline__ bf16x8 read(const uint8_t *buf, int offset) {
        if (L == Along) return *reinterpret_cast<const bf16x8 *>(buf + offset);
        // Rows k and k + 4: the swizzles agree mod 4, and for 64 rows mod 8 / 2 as well.
        auto *q = (__attribute__((address_space(3))) s16x4 *)(buf + offset);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * kRowBytes / 8);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// A tile: kWM x kWN waves, each of 32 kMI x 32 kNJ accumulators of 32 x 32.
template <int WM, int WN, int MI, int NJ>
struct Tile {
    static constexpr int kWM = WM, kWN = WN, kMI = MI, kNJ = NJ;
    static constexpr int kBM = 32 * WM * MI, kBN = 32 * WN * NJ;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kLds = 2 * (kBM + kBN) * kStageK * 2;  // two stages
};

template <class T>
struct Acc {
    f32x16 v[T::kMI][T::kNJ];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int j = 0; j < T::kNJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[i][j][e] = 0.0f;
    }
    __device__ __forceinline__ void scale(float s) {
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int j = 0; j < T::kNJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[i][j][e] *= s;
    }
};

// This lane's place in a tile: element e of accumulator (i, j) is row
// m(i, e) and column n(j) of the tile.
template <class T>
struct Place {
    int lane, wm, wn;
    __device__ __forceinline__ Place() {
        lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave % T::kWM;
        wn = wave / T::kWM;
    }
    __device__ __forceinline__ int m(int i, int e) const {  // e = 4 q: rows m .. m + 3 are elements e .. e + 3
        return (wm * T::kMI + i) * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
    }
    __device__ __forceinline__ int n(int j) const { return (wn * T::kNJ + j) * 32 + (lane & 31); }
};

// acc += the products over k0 .. k1 of the tile at (m0, n0).  `lds` holds
// T::kLds bytes; all of the block's threads call it, and every wave has left
// the LDS when it returns.
template <class T, Layout LP, Layout LQ>
__device__ __forceinline__ void tile_product(Acc<T> &acc, uint8_t *lds, const Operand &P, int64_t m0,
                                             const Operand &Q, int64_t n0, int64_t k0, int64_t k1) {
    using SP = Stage<LP, T::kBM, T::kWaves>;
    using SQ = Stage<LQ, T::kBN, T::kWaves>;
    constexpr int kStageBytes = SP::kBytes + SQ::kBytes;
    const Place<T> at;
    const int wave = at.wm + at.wn * T::kWM;
    SP sp;
    SQ sq;
    sp.init(P, m0, k0, k1, wave, at.lane);
    sq.init(Q, n0, k0, k1, wave, at.lane);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * 1024;
    const int stages = (int)((k1 - k0 + kStageK - 1) / kStageK);
    auto issue = [&](int buf) {
        sp.issue(lds0 + buf * kStageBytes);
        sq.issue(lds0 + buf * kStageBytes + SP::kBytes);
    };
    if (stages > 0) issue(0);
    for (int s = 0; s < stages; ++s) {
        wait_and_barrier();
        if (s + 1 < stages) issue((s + 1) & 1);
        const uint8_t *buf = lds + (s & 1) * kStageBytes;
#pragma unroll
        for (int kk = 0; kk < kStageK / 16; ++kk) {
            bf16x8 fp[T::kMI], fq[T::kNJ];
#pragma unroll
            for (int i = 0; i < T::kMI; ++i)
                fp[i] = SP::read(buf, SP::read_offset((at.wm * T::kMI + i) * 32, kk, at.lane));
#pragma unroll
            for (int j = 0; j < T::kNJ; ++j)
                fq[j] = SQ::read(buf + SP::kBytes, SQ::read_offset((at.wn * T::kNJ + j) * 32, kk, at.lane));
#pragma unroll
            for (int i = 0; i < T::kMI; ++i)
#pragma unroll
                for (int j = 0; j < T::kNJ; ++j)
                    acc.v[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i], fq[j], acc.v[i][j], 0, 0, 0);
        }
    }
    wait_and_barrier();
}

// The (m tile, n tile) of block b of `total`.  Blocks go to the 8 XCDs
// round-robin; XCD x takes a contiguous range of an order in which kBand m
// tiles of consecutive n tiles are adjacent, so that the blocks an XCD runs
// at once share their operands in its L2.
__device__ __forceinline__ void tile_of_block(unsigned b, unsigned total, unsigned mtiles, unsigned &mt,
                                              unsigned &nt) {
    constexpr unsigned kBand = 4;
    const unsigned per = total / 8, rem = total % 8, x = b % 8;
    const unsigned L = x * per + (x < rem ? x : rem) + b / 8;
    const unsigned ntiles = total / mtiles;
    const unsigned band = mtiles < kBand ? mtiles : kBand;
    const unsigned full = mtiles / band * band;
    const unsigned grp = L / (ntiles * band);
    if (grp * band < full) {
        const unsigned r = L - grp * ntiles * band;
        nt = r / band;
        mt = grp * band + r % band;
    } else {
        const unsigned bt = mtiles - full;
        const unsigned r = L - full * ntiles;
        nt = r / bt;
        mt = full + r % bt;
    }
}

// Writes a tile as bf16 to C[n * ld + m]; `wide`: rows of C are 8-byte
// aligned and m in whole fours.
template <class T>
__device__ __forceinline__ void store_bf16(const Acc<T> &acc, uint16_t *C, int64_t ld, int64_t m0, int64_t rows,
                                           int64_t n0, int64_t cols, bool wide) {
    const Place<T> at;
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) {
        const int64_t n = n0 + at.n(j);
        if (n >= cols) continue;
        uint16_t *row = C + n * ld;
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t m = m0 + at.m(i, 4 * q);
                const f32x16 &a = acc.v[i][j];
                if (wide && m + 4 <= rows) {
                    *reinterpret_cast<uint2 *>(row + m) = make_uint2(bf16_pair(a[4 * q], a[4 * q + 1]),
                                                                     bf16_pair(a[4 * q + 2], a[4 * q + 3]));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (m + e < rows) row[m + e] = (uint16_t)bf16_rne(a[4 * q + e]);
                }
            }
    }
}

}  // namespace
