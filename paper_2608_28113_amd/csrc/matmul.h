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
#include "plan.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kRawWord3 = 0x00020000u;   // raw (untyped) buffer, 32-bit data format
constexpr uint32_t kNoRead = 0x7FFF0000u;     // an offset beyond every descriptor: reads zeros
constexpr int64_t kMostBytes = 0x7FF00000;    // of one descriptor

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

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {  // one conversion
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// One operand: `rows` of m (or n) and `k`, at a leading dimension of `ld`
// elements (a multiple of 8; the array is 16-byte aligned).  The one that lies
// along a row is a multiple of 8 too.  Rows and k beyond read as zeros.
struct Operand {
    const void *p;
    int64_t ld, rows, k;
};

enum Layout { Along, Across };

// Stages of one operand's kRows x kK tile in LDS, filled by kWaves waves with
// copies of 1 KB (16 bytes a lane).  Along: a row holds its 32 or 64 k (64 or
// 128 bytes), the 16-byte chunk c at position c ^ ((row / 4) % 4) or
// c ^ ((row / 2) % 8), so that the 16 rows that an operand read serves at a
// time fall in 16 different 16-byte columns of the banks.  Across: a row holds
// one k of all kRows (2 kRows bytes), its 64-byte chunk c at c ^ (k % 4) (for
// 64 rows c ^ (k / 2 % 2)), so that the four k rows of a transposed read fall
// in different banks.
template <Layout L, int kRows, int kWaves, int kK>
struct Stage {
    static_assert(kK == 32 || kK == 64, "k of a stage");
    static constexpr int kBytes = kRows * kK * 2;
    static constexpr int kCopies = kBytes / 1024 / kWaves;  // per wave and stage
    static_assert(kBytes % (1024 * kWaves) == 0, "whole copies per wave");
    static constexpr int kRowBytes = L == Along ? kK * 2 : kRows * 2;
    static constexpr int kLanesPerRow = kRowBytes / 16;

    uint32_t off[kCopies];  // of this lane from the stage's first byte
    const char *base;       // of the next stage
    int64_t left;           // bytes from base to the array's end
    int64_t step;           // bytes from stage to stage
    int64_t k_left;
    int chunk;              // Along: the lane's 16-byte chunk of its rows

    static __device__ __forceinline__ int along_swizzle(int row) {
        return kK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    }
    static __device__ __forceinline__ int across_swizzle(int k) { return kRows == 64 ? (k >> 1) & 1 : k & 3; }

    // The tile at row r0, and k from k0 on.
    __device__ __forceinline__ void init(const Operand &o, int64_t r0, int64_t k0, int64_t k1, int wave, int lane) {
        const int64_t rows = o.rows - r0 < kRows ? o.rows - r0 : kRows;
        k_left = (k1 < o.k ? k1 : o.k) - k0;
        if (L == Along) {
            base = reinterpret_cast<const char *>(o.p) + (r0 * o.ld + k0) * 2;
            left = ((rows - 1) * o.ld + k_left) * 2;
            step = kK * 2;
        } else {
            base = reinterpret_cast<const char *>(o.p) + (k0 * o.ld + r0) * 2;
            left = ((k_left - 1) * o.ld + rows) * 2;
            step = kK * o.ld * 2;
        }
        if (rows <= 0 || k_left <= 0) left = 0;
        chunk = at(row_of(0, wave, lane), lane);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = row_of(i, wave, lane), c = at(row, lane);
            if (L == Along)
                off[i] = row < rows ? (uint32_t)(row * o.ld * 2 + c * 16) : kNoRead;
            else
                off[i] = c * 8 < rows ? (uint32_t)(row * o.ld * 2 + c * 16) : kNoRead;
        }
    }

    // The LDS row that this lane fills in copy i, and the 16-byte chunk of its
    // row that belongs at the lane's position (Along: the same in every copy).
    static __device__ __forceinline__ int row_of(int i, int wave, int lane) {
        return (wave + i * kWaves) * (64 / kLanesPerRow) + lane / kLanesPerRow;
    }
    static __device__ __forceinline__ int at(int row, int lane) {
        const int pos = lane % kLanesPerRow;
        return L == Along ? pos ^ along_swizzle(row) : (((pos >> 2) ^ across_swizzle(row)) << 2) | (pos & 3);
    }

    // Before the copies of a stage: its descriptor, and k past the end turned
    // into reads of nothing (a row's next values are not read).  Stages past
    // the last are all nothing: zeros, and no memory traffic.
    __device__ __forceinline__ u32x4 begin() {
        if (L == Along && __builtin_amdgcn_readfirstlane(k_left < kK)) {
#pragma unroll
            for (int i = 0; i < kCopies; ++i)
                if (chunk * 8 >= k_left) off[i] = kNoRead;
        }
        return raw_buffer(base, left);
    }
    // Copy i of the stage to LDS address `dst` (of this wave's first copy).
    __device__ __forceinline__ void copy(const u32x4 &r, int i, uint32_t dst) const {
        copy_to_lds(r, off[i], dst + i * kWaves * 1024);
    }
    __device__ __forceinline__ void end() {
        base += step;
        left -= step;
        k_left -= kK;
    }

    // Where this lane finds its 8 k of 16-k step kk of the 32-row operand block
    // i, counted from row r0: place(i, kk) + shift(i, kk), the shift known at
    // compile time and the places few.
        static __device__ __forceinline__ int place(int r0, int which, int lane) {
        if (L == Along) {  // which = kk
            const int row = r0 + (lane & 31);
            return row * kRowBytes + (((2 * which + (lane >> 5)) ^ along_swizzle(row)) << 4);
        }
        // which = i.  A transposed read gives lane p of 16 the four k of
        // column p from a 4-row x 16-column block whose row p / 4 the lane
        // addresses; two reads are the 8 k.
        const int p = lane & 15, g = lane >> 4;
        const int k = 8 * (g >> 1) + (p >> 2);
        const int byte = (r0 + 32 * which) * 2 + 32 * (g & 1) + 8 * (p & 3);
        return k * kRowBytes + ((((byte >> 6) ^ across_swizzle(k)) << 6) | (byte & 63));
    }
    static constexpr __device__ __forceinline__ int shift(int i, int kk) {
        return L == Along ? i * 32 * kRowBytes : kk * 16 * kRowBytes;
    }
    static constexpr __device__ __forceinline__ int which(int i, int kk) { return L == Along ? kk : i; }
    static __device__ __forceinline__ int read_offset(int r, int kk, int lane) {
        return place(r, L == Along ? kk : 0, lane) + shift(0, kk);
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

// A tile: WM x WN waves, each of MI x NJ accumulators of 32 x 32, and a ring of
// R stages of K in LDS, whose copies are spread over W steps of 16 k.
template <int WM, int WN, int MI, int NJ, int K, int R, int W>
struct Tile {
    static constexpr int kWM = WM, kWN = WN, kMI = MI, kNJ = NJ, kK = K, kRing = R, kSpread = W;
    static constexpr int kBM = 32 * WM * MI, kBN = 32 * WN * NJ;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kLds = R * (kBM + kBN) * K * 2;
    static constexpr int kBlocks = 160 * 1024 / kLds;  // per CU
    static constexpr int kOccupancy = kWaves * kBlocks / 4 < 1 ? 1 : kWaves * kBlocks / 4;
    static_assert(W >= 1 && W <= K / 16 && R >= 2, "copies end before the stage that waits for them");
};

typedef Tile<2, 2, 4, 4, 64, 2, 2> Large;        // 256 x 256
typedef Tile<2, 2, 4, 2, 64, 3, 2> Middle;       // 256 x 128
typedef Tile<2, 2, 2, 2, 64, 4, 2> Small;        // 128 x 128: its ring hides latency where blocks are few
typedef Tile<2, 4, 4, 2, 32, 4, 2> LargeAcross;  // 256 x 256 for two operands across, in eight waves: four run out of registers
// Launches KERNEL(tile) in the plan's tile.
#define LAUNCH_TILES(KERNEL, LARGE, size, blocks, stream, ...)                                                    \
    do {                                                                                                          \
        if ((size) == kLarge)                                                                                     \
            hipLaunchKernelGGL((KERNEL(LARGE)), dim3((unsigned)(blocks)), dim3(LARGE::kThreads), 0, stream,       \
                               __VA_ARGS__);                                                                      \
        else if ((size) == kMiddle)                                                                               \
            hipLaunchKernelGGL((KERNEL(Middle)), dim3((unsigned)(blocks)), dim3(Middle::kThreads), 0, stream,     \
                               __VA_ARGS__);                                                                      \
        else                                                                                                      \
            hipLaunchKernelGGL((KERNEL(Small)), dim3((unsigned)(blocks)), dim3(Small::kThreads), 0, stream,       \
                               __VA_ARGS__);                                                                      \
    } while (0)

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

template <int N>
__device__ __forceinline__ void wait_copies_and_barrier() {  // all but the last N copies, and own reads
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

// Stages beyond those of the two operands, for tile_product: none.
struct NoMore {
    static constexpr bool kAny = false;
};

// acc += the products over k0 .. k1 of the tile at (m0, n0), and those of the
// `more.stages` stages that more.set(sp, sq) points the copies at.  `lds`
// holds T::kLds bytes; all of the block's threads call it, and every wave has
// left the LDS when it returns.
template <class T, Layout LP, Layout LQ, class More>
__device__ __forceinline__ void tile_product(Acc<T> &acc, uint8_t *lds, const Operand &P, int64_t m0,
                                             const Operand &Q, int64_t n0, int64_t k0, int64_t k1, More more) {
    using SP = Stage<LP, T::kBM, T::kWaves, T::kK>;
    using SQ = Stage<LQ, T::kBN, T::kWaves, T::kK>;
    constexpr int kStageBytes = SP::kBytes + SQ::kBytes;
    constexpr int kCopies = SP::kCopies + SQ::kCopies;  // of a wave and stage
    constexpr int R = T::kRing, W = T::kSpread, kSteps = T::kK / 16, kMfmas = T::kMI * T::kNJ;
    constexpr int kUnits = T::kMI + T::kNJ;
    const Place<T> at;
    const int wave = at.wm + at.wn * T::kWM;
    SP sp;
    SQ sq;
    sp.init(P, m0, k0, k1, wave, at.lane);
    sq.init(Q, n0, k0, k1, wave, at.lane);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * 1024;
    const int own = (int)((k1 - k0 + T::kK - 1) / T::kK);
    int stages = own, begun = 0;
    if constexpr (More::kAny) stages += more.stages;
    if (stages <= 0) return;
    u32x4 rp, rq;
    auto begin = [&]() {
        if constexpr (More::kAny) {
            if (begun >= own) more.set(sp, sq, begun < stages);
            ++begun;
        }
        rp = sp.begin();
        rq = sq.begin();
    };
    auto copy = [&](int c, int buf) {  // copy c of the stage begun
        const uint32_t dst = lds0 + buf * kStageBytes;
        if (c < SP::kCopies)
            sp.copy(rp, c, dst);
        else
            sq.copy(rq, c - SP::kCopies, dst + SP::kBytes);
    };
    auto end = [&]() {
        sp.end();
        sq.end();
    };
    int pp[LP == Along ? kSteps : T::kMI], pq[LQ == Along ? kSteps : T::kNJ];
#pragma unroll
    for (int k = 0; k < (LP == Along ? kSteps : T::kMI); ++k) pp[k] = SP::place(at.wm * T::kMI * 32, k, at.lane);
#pragma unroll
    for (int k = 0; k < (LQ == Along ? kSteps : T::kNJ); ++k) pq[k] = SQ::place(at.wn * T::kNJ * 32, k, at.lane);
    bf16x8 fp[2][T::kMI], fq[2][T::kNJ];
    auto read_unit = [&](const uint8_t *buf, int kk, int u) {  // operand block u of step kk
        if (u < T::kMI)
            fp[kk & 1][u] = SP::read(buf, pp[SP::which(u, kk)] + SP::shift(u, kk));
        else
            fq[kk & 1][u - T::kMI] =
                SQ::read(buf + SP::kBytes, pq[SQ::which(u - T::kMI, kk)] + SQ::shift(u - T::kMI, kk));
    };

    // Two sets of operand registers: each 16-k step's operands are read while
    // the step before it multiplies, across stages too.  At a stage's last
    // step its operands are in registers, so after the waits (own reads done,
    // own copies of the next stage landed) and the barrier its buffer takes
    // the stage kRing further on.  Those copies are started one by one
    // between the MFMAs of that step and of the next W - 1: in one go they
    // fill the memory pipeline's queue, and the wave stands before it.
    constexpr int kFirst = kCopies / W;  // copies in a stage's last step
#pragma unroll
    for (int s = 0; s < R; ++s) {
        begin();
#pragma unroll
        for (int c = 0; c < (s < R - 1 ? kCopies : kFirst); ++c) copy(c, s);
        if (s < R - 1 || W == 1) end();
    }
    wait_copies_and_barrier<(R - 2) * kCopies + kFirst>();
#pragma unroll
    for (int u = 0; u < kUnits; ++u) read_unit(lds, 0, u);
    int cur = 0, prev = R - 1;
    for (int s = 0; s < stages; ++s) {
        const int next = cur + 1 == R ? 0 : cur + 1;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const bool last = kk == kSteps - 1;
            if (last) {
                wait_copies_and_barrier<(R - 2) * kCopies>();
            }
            // after the last stage: old values that nothing uses
            const uint8_t *from = lds + (last ? next : cur) * kStageBytes;
            const int w = last ? 0 : kk + 1;  // step of the window
            const int c0 = w < W ? kCopies * w / W : 0, c1 = w < W ? kCopies * (w + 1) / W : 0;
#pragma unroll
            for (int q = 0; q < kMfmas; ++q) {
                const int i = q % T::kMI, j = q / T::kMI;
                acc.v[i][j] =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[kk & 1][i], fq[kk & 1][j], acc.v[i][j], 0, 0, 0);
                if (last && q == 0) begin();  // behind an MFMA, not before it
#pragma unroll
                for (int u = 0; u < kUnits; ++u)
                    if (u * kMfmas / (2 * kUnits) == q) read_unit(from, last ? 0 : kk + 1, u);
#pragma unroll
                for (int c = 0; c < kCopies; ++c)
                    if (c >= c0 && c < c1 && (2 * (c - c0) + 1) * kMfmas / (2 * (c1 - c0)) == q)
                        copy(c, last ? cur : prev);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (w == W - 1) end();
        }
        prev = cur;
        cur = next;
    }
    wait_and_barrier();
}

template <class T, Layout LP, Layout LQ>
__device__ __forceinline__ void tile_product(Acc<T> &acc, uint8_t *lds, const Operand &P, int64_t m0,
                                             const Operand &Q, int64_t n0, int64_t k0, int64_t k1) {
    tile_product<T, LP, LQ>(acc, lds, P, m0, Q, n0, k0, k1, NoMore{});
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

// Writes `scale` times a tile as bf16 to C[n * ld + m], for m below `rows` and
// n below `cols`.  Accumulators hold four consecutive m of 32 rows n at a time; written
// like that, every store is 32 pieces of 16 bytes, and the 128 KB of a 256 x
// 256 tile take longer than 600 of its k.  So the tile goes through LDS, 16
// bytes of a row at chunk position c ^ (n % 32) (of the row's chunks), and out
// in whole rows.  `wide`: C and its rows are 16-byte aligned; else element by
// element.
template <class T>
__device__ __forceinline__ void store_bf16(const Acc<T> &acc, uint8_t *lds, uint16_t *C, int64_t ld, int64_t m0,
                                           int64_t rows, int64_t n0, int64_t cols, bool wide, float scale = 1.0f) {
    const Place<T> at;
    constexpr int kRow = T::kBM * 2, kChunks = kRow / 16;
    static_assert(T::kBN * kRow <= T::kLds, "the tile fits the ring");
    if (wide) {
#pragma unroll
        for (int j = 0; j < T::kNJ; ++j) {
            const int n = at.n(j);
#pragma unroll
            for (int i = 0; i < T::kMI; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int m = at.m(i, 4 * q);
                    const f32x16 &a = acc.v[i][j];
                    *reinterpret_cast<uint2 *>(lds + n * kRow + (((m >> 3) ^ (n & 31 & (kChunks - 1))) << 4) +
                                               (m & 4) * 2) =
                        make_uint2(bf16_pair(a[4 * q] * scale, a[4 * q + 1] * scale),
                                   bf16_pair(a[4 * q + 2] * scale, a[4 * q + 3] * scale));
                }
        }
        __syncthreads();
        const int c = threadIdx.x % kChunks;
        const int64_t m = m0 + c * 8;
        uint16_t *dst = C + n0 * ld + m;
        for (int n = threadIdx.x / kChunks; n < T::kBN; n += T::kThreads / kChunks) {
            if (n0 + n >= cols) break;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + n * kRow + ((c ^ (n & 31 & (kChunks - 1))) << 4));
            if (m + 8 <= rows) {
                *reinterpret_cast<u32x4 *>(dst + n * ld) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (m + e < rows) dst[n * ld + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) {
        const int64_t n = n0 + at.n(j);
        if (n >= cols) continue;
        uint16_t *row = C + n * ld;
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t m = m0 + at.m(i, e);
                if (m < rows) row[m] = (uint16_t)bf16_rne(acc.v[i][j][e] * scale);
            }
    }
}

// Writes a tile to a partial sum S[n, rows], or adds it to what is there.
// `fours`: rows is a multiple of 4.
template <class T>
__device__ __forceinline__ void store_sum(const Acc<T> &acc, float *S, int64_t m0, int64_t rows, int64_t n0,
                                          int64_t cols, bool fours, bool add) {
    const Place<T> at;
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) {
        const int64_t n = n0 + at.n(j);
        if (n >= cols) continue;
#pragma unroll
        for (int i = 0; i < T::kMI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t m = m0 + at.m(i, 4 * q);
                float *dst = S + n * rows + m;
                const f32x16 &a = acc.v[i][j];
                if (fours && m < rows) {
                    float4 v = add ? *reinterpret_cast<float4 *>(dst) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    v.x += a[4 * q], v.y += a[4 * q + 1], v.z += a[4 * q + 2], v.w += a[4 * q + 3];
                    *reinterpret_cast<float4 *>(dst) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (m + e < rows) dst[e] = (add ? dst[e] : 0.0f) + a[4 * q + e];
                }
            }
    }
}

}  // namespace
