// Layers of stored NVFP4 experts for a few tokens, behind the C ABI of
// include/hscale.h: routing, and the experts' products.
//
//   w_tj = exp(l_te - max) / sum,  e = e_tj the j-th largest logit of token t
//   h_s  = silu(s_g G_e x_t) * (s_u U_e x_t)        of slot s = (t, j)
//   y_t  = sum_j w_tj s_d D_e h_s
//
// A weight's E2M1 value times its E4M3 scale has at most 6 significant bits, so
// with the power of two of a matrix's global scale it is exact in bf16: the
// products are bf16 products accumulated in fp32, and the rest of the global
// scale multiplies the sum.  h is kept as two bf16 parts (within 2^-16), so
// that nothing is rounded to 8 bits before y is.
//
// Times below are of one MI355X, whose large copies reach 4.9 TB/s, streaming
// reads 6.9 TB/s and large bf16 products 1.4 to 1.5 PFLOP/s.

#include "checks.h"
#include "expert_plan.h"
#include "matmul.h"
#include "stored.h"

#include <algorithm>

namespace {

constexpr int kNoExpert = -1;

// ---------------------------------------------------------------------------
// Routing
// ---------------------------------------------------------------------------

// A number that orders as the logit does, 0 for what is never chosen: -inf and
// NaN.  -0 and +0 are equal.
__device__ __forceinline__ uint32_t choice_key(float l) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(l + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The largest of a wave's numbers, in all its lanes: within 16 lanes, then over
// the rows of 16.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    uint32_t o;
#define MAX_OF(ctrl, rows)                                                                          \
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false);                   \
    v = o > v ? o : v
    MAX_OF(0x111, 0xF);  // row_shr:1, 2, 4, 8
    MAX_OF(0x112, 0xF);
    MAX_OF(0x114, 0xF);
    MAX_OF(0x118, 0xF);
    MAX_OF(0x142, 0xA);  // row_bcast:15, 31
    MAX_OF(0x143, 0xC);
#undef MAX_OF
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// A wave per token, kN logits a lane.  k rounds of the wave's largest key, each
// taken out where it first lies; the softmax is relative to the first.  48
// tokens of 64 experts take 2.8 us, a launch; 8190 of 160 6.9, bound by vector
// instructions: 370 a wave, eight waves a SIMD, are 4.9 us of issue (4.3 and
// 13.7 us with the largest key by shuffles of 64 bits).
template <int kN, bool kWide>
__global__ __launch_bounds__(256) void route_kernel(const void *__restrict__ logits, int64_t tokens, int experts,
                                                    int64_t ld, int k, bool normalize, int32_t *__restrict__ expert,
                                                    float *__restrict__ weight) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= tokens) return;
    float l[kN];
    uint32_t key[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int e = i * 64 + lane;
        l[i] = -INFINITY;
        if (e < experts)
            l[i] = kWide ? static_cast<const float *>(logits)[t * ld + e]
                         : bf16_value(static_cast<const uint16_t *>(logits)[t * ld + e]);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) key[i] = choice_key(l[i]);
    uint32_t mine = 0;      // lane j holds the j-th choice
    int which = kNoExpert;
    for (int j = 0; j < k; ++j) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < kN; ++i) best = key[i] > best ? key[i] : best;
        best = wave_max(best);
        if (best == 0) break;  // fewer than k can be chosen
        int at = -1;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const uint64_t mask = __ballot(key[i] == best);
            if (at < 0 && mask) {
                at = i * 64 + __builtin_ctzll(mask);
                if (lane == (at & 63)) key[i] = 0;
            }
        }
        if (lane == j) mine = best, which = at;
    }
    const float v = __uint_as_float(mine & 0x80000000u ? mine & 0x7FFFFFFFu : ~mine);
    const float top = which == kNoExpert ? 0.0f : v, first = __shfl(top, 0);
    const float p = which == kNoExpert ? 0.0f : expf(v - first);
    // Over all experts too where the k alone are asked for: a NaN anywhere shows.
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < kN; ++i)
        if (!(l[i] == -INFINITY)) all += expf(l[i] - first);
    all = wave_sum(all);
    const float some = wave_sum(p);
    if (lane >= k) return;
    expert[t * k + lane] = which;
    weight[t * k + lane] = all != all ? all : which == kNoExpert ? 0.0f : p / (normalize ? some : all);
}

// ---------------------------------------------------------------------------
// Which slots an expert has
// ---------------------------------------------------------------------------

__device__ __forceinline__ int expert_of(const int32_t *ids, int experts, int s) {
    const int e = ids[s];
    return e >= 0 && e < experts ? e : kNoExpert;
}

// Many slots, sorted by expert once: a block of 1024 counts the slots of each
// expert, adds the counts up and puts every slot at its place.  In which order
// an expert's slots lie comes from atomics and changes no result: a slot's sums
// do not depend on its neighbours.
__global__ __launch_bounds__(1024) void share_kernel(const int32_t *__restrict__ ids, int slots, int experts, int most,
                                                     int32_t *__restrict__ order, Share *__restrict__ shares,
                                                     int max_shares) {
    __shared__ int count[kMaxExperts], place[kMaxExperts], wave_slots[16], wave_shares[16];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    count[e] = 0;
    __syncthreads();
    for (int s = e; s < slots; s += 1024) {
        const int x = expert_of(ids, experts, s);
        if (x != kNoExpert) atomicAdd(&count[x], 1);
    }
    __syncthreads();
    const int n = count[e], pieces = (n + most - 1) / most;
    int a = n, b = pieces;  // inclusive sums over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int pa = __shfl_up(a, o), pb = __shfl_up(b, o);
        if (lane >= o) a += pa, b += pb;
    }
    if (lane == 63) wave_slots[wave] = a, wave_shares[wave] = b;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) a += wave_slots[w], b += wave_shares[w];
        total += wave_shares[w];
    }
    place[e] = a - n;
    for (int i = 0; i < pieces; ++i)
        shares[b - pieces + i] = Share{e, a - n + i * most, n - i * most < most ? n - i * most : most};
    for (int i = total + e; i < max_shares; i += 1024) shares[i] = Share{kNoExpert, 0, 0};
    __syncthreads();
    for (int s = e; s < slots; s += 1024) {
        const int x = expert_of(ids, experts, s);
        if (x != kNoExpert) order[atomicAdd(&place[x], 1)] = s;
    }
}

// ---------------------------------------------------------------------------
// The experts' products
// ---------------------------------------------------------------------------

struct Matrices {  // of all experts
    const float *scale;
    const uint8_t *codes, *packed;
};

struct ExpertArgs {
    Matrices w[2];     // gate and up, or down
    int64_t rows, k;   // of a matrix
    const uint16_t *in;
    int64_t ld;        // elements from one row of `in` to the next (of a slot's two parts: twice their width)
    int64_t in_bytes;
    const int32_t *ids;
    const float *weight;
    int slots, choices, experts;
    const int32_t *order;  // with many slots
    const Share *shares;
    uint16_t *H;       // [slots, 2, rows]: gate and up
    float *P;          // [splits, slots, rows]: down
    int split;         // steps of a split of k: down
};

// s = f 2^e with 1 <= f < 2, or more where 2^e would take the largest weight
// out of bf16's range.
__device__ __forceinline__ void split_device_scale(float s, float &f, float &two_e) {
    constexpr int kMostE = 100;
    int e = (int)(__float_as_uint(s) >> 23 & 0xFF) - 127;
    e = e > kMostE ? kMostE : e < -126 ? -126 : e;
    two_e = ldexpf(1.0f, e);
    f = ldexpf(s, -e);
}

// The slots of a block's expert.  Up to 256 in all each wave finds them itself:
// of one block for each expert, or for each slot where those are fewer (there
// the block of an expert's first slot stays).
struct Found {
    int expert, count, first;  // first: in `order`, of many slots
    uint64_t mask[kBlockSlots / 64];
    bool many;

    __device__ __forceinline__ bool find(const ExpertArgs &a, int y) {
        const int lane = threadIdx.x & 63;
        many = a.shares != nullptr;
        if (many) {
            const Share s = a.shares[y];
            expert = s.expert, count = s.count, first = s.first;
            return count > 0;
        }
        int id[kBlockSlots / 64];
#pragma unroll
        for (int i = 0; i < kBlockSlots / 64; ++i)
            id[i] = i * 64 + lane < a.slots ? a.ids[i * 64 + lane] : kNoExpert;
        expert = a.slots <= a.experts ? expert_of(a.ids, a.experts, y) : y;
        if (expert == kNoExpert) return false;
        count = 0;
        int at = -1;  // the expert's first slot
#pragma unroll
        for (int i = 0; i < kBlockSlots / 64; ++i) {
            mask[i] = __ballot(id[i] == expert);
            if (at < 0 && mask[i]) at = i * 64 + __builtin_ctzll(mask[i]);
            count += __popcll(mask[i]);
        }
        return count > 0 && (a.slots > a.experts || at == y);
    }
    // The c0 + lane th slot, -1 past the last.  `list` is the wave's own.
    __device__ __forceinline__ int slot(const ExpertArgs &a, int c0, int *list) const {
        const int lane = threadIdx.x & 63;
        if (many) return c0 + lane < count ? a.order[first + c0 + lane] : -1;
        int before = -c0;
#pragma unroll
        for (int i = 0; i < kBlockSlots / 64; ++i) {
            const int n = before + __popcll(mask[i] & (((uint64_t)1 << lane) - 1));
            if ((mask[i] >> lane & 1) && n >= 0 && n < 64) list[n] = i * 64 + lane;
            before += __popcll(mask[i]);
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int got = c0 + lane < count ? list[lane] : -1;
        __builtin_amdgcn_wave_barrier();
        return got;
    }
};

// Gate, up and silu: a lane's four rows of a slot's h, in two bf16 parts.
__device__ __forceinline__ void store_hidden(uint16_t *h, int64_t rows, const float (&gate)[4], const float (&up)[4]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float v = gate[q] / (1.0f + expf(-gate[q])) * up[q];
        hi[q] = bf16_rne(v);
        const float rest = v - bf16_value(hi[q]);
        lo[q] = fabsf(rest) < INFINITY ? bf16_rne(rest) : 0;  // where v itself rounds to infinity
    }
    *reinterpret_cast<uint2 *>(h) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
    *reinterpret_cast<uint2 *>(h + rows) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
}

__device__ __forceinline__ void own_writes_and_barrier() {  // loads stay under way
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// 16 kRT rows of gate and the same of up (or 32 kRT of down) a wave, x up to
// kTok slots of one expert.  kW of the block's four waves share their rows: each
// takes every kWth step of k, and they add up through LDS.
//
// Reading the weights bounds it while slots are few: 64 tokens over 128 experts
// of 4096 x 1536 take 178 and 120 us, 5.1 and 3.8 TB/s; 37 over 8 of 4096 x 14336
// 109 and 69, 4.9 and 3.8; one token over two of these 33 and 20, 4.0 and 3.4.
// With many it is the loads' return path, 0.62 and 0.57 busy, beside the
// conversion of the weights (VALU 0.36 and 0.24) and the products (MFMA 0.21 and
// 0.25), which two waves a SIMD overlap only in part: 512 tokens over 64 experts
// of 2048 x 1024, 48 slots each, 57 and 48 us.  Four sets of weights under way in place of two measured equal
// there, 256 k of weights with 128 of the rows 138 us a call for 130.
//
// A wave's operand of weights comes straight from memory, 32 consecutive weights
// of a row a lane (which k meets which place in a step does not matter, as both
// operands agree).  The slots' rows go through LDS, 16-byte chunk c of row t at
// c ^ (t % 16), two buffers of kW steps: straight from memory each wave's reads
// of them kept the return path of loads 92 % busy, and a wait for them was one
// for the weights behind them too.  Rows of a buffer that no slot has are columns
// of the product that nothing reads.
//
// Scales are taken for four of the wave's steps at once, 16 bytes a lane, and
// read back from LDS two at a time: as 2-byte loads for each step they took a
// quarter of the time (64 tokens of 4096 over 128 experts of 1536: 363 us with
// them, 275 without any scales).
template <bool kDown, int kTok, int kRT, int kW, int kStep>
__global__ __launch_bounds__(256, !kDown && kTok == 16 && kW == 1 ? 4 : kTok == 64 && kW == 4 ? 1 : 2) void expert_kernel(const ExpertArgs a) {
    constexpr int kNT = (kTok + 15) / 16, kSets = 2 * kRT, kMats = kDown ? 1 : 2, kParts = kDown ? 2 : 1;
    constexpr int kRows = kDown ? 32 * kRT : 16 * kRT;  // of a wave
    constexpr int kHalves = kStep / 128, kRowBytes = kStep * 2, kStepBytes = kTok * kRowBytes;
    constexpr int kRowLanes = kStep / 8, kCopyRows = 256 / kRowLanes;  // threads of a row, rows of a copy
    constexpr int kBuffer = kW * kParts * kStepBytes, kCopies = kBuffer / 4096;  // 16 bytes a thread
    static_assert(kBuffer % 4096 == 0, "whole copies");
    constexpr int kSums = kW > 1 ? 4 * kSets * kNT * 1024 : 0;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kBuffer > kSums ? 2 * kBuffer : kSums];
    __shared__ int list[4][64];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = wave % kW;
    const int64_t r0 = ((int64_t)blockIdx.x * (4 / kW) + wave / kW) * kRows;
    const int rows = (int)(a.rows - r0 < 0 ? 0 : a.rows - r0 < kRows ? a.rows - r0 : kRows);
    const int K = (int)a.k;

    Found own;
    if (!own.find(a, blockIdx.y)) return;
    const int expert = __builtin_amdgcn_readfirstlane(own.expert), count = __builtin_amdgcn_readfirstlane(own.count);

    float f[2], two_e[2];
    const uint8_t *packed[2], *codes[2];
#pragma unroll
    for (int m = 0; m < kMats; ++m) {
        split_device_scale(a.w[m].scale[expert], f[m], two_e[m]);
        const int64_t row = (int64_t)expert * a.rows + (rows ? r0 : 0);
        packed[m] = a.w[m].packed + row * (K / 2);
        codes[m] = a.w[m].codes + row * (K / 16);
    }
    const uint32_t prow = (uint32_t)(l16 * (K / 2) + g * 16), crow = (uint32_t)(l16 * (K / 16) + g * (kStep / 16) * kW);
    const int step0 = kDown ? (int)blockIdx.z * a.split : 0;
    const int steps = kDown && step0 + a.split < (K + kStep - 1) / kStep ? step0 + a.split : (K + kStep - 1) / kStep;
    const int rounds = (steps - step0 + kW - 1) / kW;
    const int read = rows > 0 ? steps : 0;  // a wave behind the last row only keeps step

    struct Weights {  // 32 of each 128 of a row's
        u32x4 p[kSets][kHalves];
    };
    // What lies past the last k meets zeros of the slots' rows; steps past the
    // last are not read.
    auto load_weights = [&](Weights &w, int step) {
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            const int m = kDown ? 0 : s / kRT, tile = kDown ? s : s % kRT;
            const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<uint8_t *>(packed[m]) + step * (kStep / 2), 0,
                step < read ? rows * (K / 2) - step * (kStep / 2) : 0, kRawWord3);
            const uint32_t p = prow + tile * 16 * (K / 2);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) w.p[s][h] = __builtin_amdgcn_raw_buffer_load_b128(rp, p + 64 * h, 0, 0);
        }
    };
    // Rows of scales lie at any byte: whole words from the one that the first byte
    // is in to the one that the last is in, put in place when they are written.
    constexpr int kScaleWords = kStep / 64;
    struct Scales {  // of one of four steps
        uint32_t c[kSets][kScaleWords + 1];
    };
    auto load_scales = [&](Scales &w, int step) {
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            const int m = kDown ? 0 : s / kRT, tile = kDown ? s : s % kRT;
            const uintptr_t from = reinterpret_cast<uintptr_t>(codes[m]) + step * (kStep / 16);
            const int bytes = rows * (K / 16) - step * (kStep / 16) + (int)(from & 3);
            const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(
                reinterpret_cast<void *>(from & ~(uintptr_t)3), 0, step < read ? (bytes + 3) & ~3 : 0, kRawWord3);
            const uint32_t c = (crow + tile * 16 * (K / 16) + (uint32_t)(from & 3)) & ~3u;
            if constexpr (kScaleWords == 4) {
                const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rc, c, 0, 0);
#pragma unroll
                for (int q = 0; q < 4; ++q) w.c[s][q] = v[q];
            } else {
                const auto v = __builtin_amdgcn_raw_buffer_load_b64(rc, c, 0, 0);
                w.c[s][0] = v[0], w.c[s][1] = v[1];
            }
            w.c[s][kScaleWords] = __builtin_amdgcn_raw_buffer_load_b32(rc, c + 4 * kScaleWords, 0, 0);
        }
    };
    constexpr int kScaleRow = kStep / 4 + kStep / 16, kScaleSet = 16 * kScaleRow;  // a row in other banks than its neighbours
    __shared__ __attribute__((aligned(16))) uint8_t scale_lds[4 * kSets * kScaleSet];
    uint8_t *scales = scale_lds + wave * kSets * kScaleSet;  // the wave's own
    auto write_scales = [&](const Scales &w) {
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            const uint32_t by = crow + (uint32_t)reinterpret_cast<uintptr_t>(codes[kDown ? 0 : s / kRT]);
            uint32_t v[kScaleWords];
#pragma unroll
            for (int q = 0; q < kScaleWords; ++q) v[q] = __builtin_amdgcn_alignbyte(w.c[s][q + 1], w.c[s][q], by & 3);
            __builtin_memcpy(__builtin_assume_aligned(scales + s * kScaleSet + l16 * kScaleRow + g * (kStep / 16), kStep / 16),
                             v, kStep / 16);
        }
    };
    // What lies behind a row's last scale may be of another array: an E4M3 NaN
    // would not vanish beside the zeros of the slots' rows, and becomes a number.
    auto scale_of = [](float l) { return __builtin_amdgcn_fmed3f(l, -448.0f, 448.0f); };
    const __amdgpu_buffer_rsrc_t rx =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.in), 0, (int)a.in_bytes, kRawWord3);

    for (int c0 = 0; c0 < count; c0 += kTok) {
        // Loads are waited for in the order in which they were issued: what the
        // loop's first round needs comes first.
        Weights w[2];
        Scales c;
        load_scales(c, step0 + part);
        load_weights(w[0], step0 + part);
        __builtin_amdgcn_sched_barrier(0);
        const int held = own.slot(a, c0, list[wave]);
        // A thread's places in a buffer: a chunk of rows tid / kRowLanes, kCopyRows further on, ...
        constexpr int kOfRows = kTok > kCopyRows ? kTok / kCopyRows : 1;  // copies of a step's rows
        const int chunk0 = tid % kRowLanes, row0 = tid / kRowLanes;
        uint32_t from[kOfRows];
#pragma unroll
        for (int i = 0; i < kOfRows; ++i) {
            const int row = row0 % kTok + kCopyRows * i;
            const int slot = __shfl(held, row);
            from[i] = slot < 0 ? kNoRead
                               : (uint32_t)((kDown ? slot : slot / a.choices) * a.ld * 2) + ((chunk0 ^ (row & 15)) << 4);
        }
        struct Rows {
            u32x4 v[kCopies];
        };
        auto load_rows = [&](Rows &x, int round) {
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                // Units of kTok rows: the steps of the round, part by part.
                const int unit = kTok < kCopyRows ? (i * kCopyRows + row0) / kTok : i / kOfRows, of = i % kOfRows;
                const int step = step0 + round * kW + unit / kParts;
                const int chunk = chunk0 ^ ((row0 % kTok + kCopyRows * of) & 15);
                const bool past = step * kStep + chunk * 8 >= K;
                const uint32_t at = from[of] + (uint32_t)(step * kRowBytes + unit % kParts * K * 2);
                x.v[i] = __builtin_amdgcn_raw_buffer_load_b128(rx, past || from[of] == kNoRead ? kNoRead : at, 0, 0);
            }
        };
        auto write_rows = [&](const Rows &x, int round) {
#pragma unroll
            for (int i = 0; i < kCopies; ++i)
                *reinterpret_cast<u32x4 *>(lds + (round & 1) * kBuffer + i * 4096 + tid * 16) = x.v[i];
        };
        f32x4 acc[kSets][kNT];
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
            for (int n = 0; n < kNT; ++n) acc[s][n] = f32x4{0, 0, 0, 0};

        Rows x;
        load_rows(x, 0);
        __builtin_amdgcn_sched_barrier(0);
        write_scales(c);
        write_rows(x, 0);
        load_rows(x, 1);
        __builtin_amdgcn_sched_barrier(0);
        load_weights(w[1], step0 + kW + part);
        own_writes_and_barrier();
        const int row = l16 % kTok;
        for (int first = 0; first < rounds; first += 4) {
            load_scales(c, step0 + (first + 4) * kW + part);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int round = first + d;
                if (d == 0 || round < rounds) {  // a branch that jumps over no load leaves their order known
                    const uint8_t *buf = lds + (d & 1) * kBuffer + part * kParts * kStepBytes + row * kRowBytes;
                    const uint8_t *from = scales + l16 * kScaleRow + d * (kStep / 16) + g * 2;
                    uint32_t code[kSets][kHalves];
#pragma unroll
                    for (int s = 0; s < kSets; ++s)
#pragma unroll
                        for (int h = 0; h < kHalves; ++h)
                            code[s][h] = *reinterpret_cast<const uint16_t *>(from + s * kScaleSet + 8 * h);
#pragma unroll
                    for (int i = 0; i < kStep / 32; ++i) {
                        bf16x8 fx[kNT][kParts];
#pragma unroll
                        for (int n = 0; n < kNT; ++n)
#pragma unroll
                            for (int p = 0; p < kParts; ++p)
                                fx[n][p] = *reinterpret_cast<const bf16x8 *>(
                                    buf + p * kStepBytes + n * 16 * kRowBytes +
                                    (((i / 4 * 16 + 4 * g + i % 4) ^ row) << 4));
#pragma unroll
                        for (int s = 0; s < kSets; ++s) {
                            const float l = scale_of(i & 2 ? __builtin_amdgcn_cvt_f32_fp8(code[s][i / 4], 1)
                                                           : __builtin_amdgcn_cvt_f32_fp8(code[s][i / 4], 0));
                            const bf16x8 fw = __builtin_bit_cast(
                                bf16x8, scaled_eight(w[d & 1].p[s][i / 4][i % 4], two_e[kDown ? 0 : s / kRT], l));
#pragma unroll
                            for (int n = 0; n < kNT; ++n)
#pragma unroll
                                for (int p = 0; p < kParts; ++p)
                                    acc[s][n] =
                                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw, fx[n][p], acc[s][n], 0, 0, 0);
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                write_rows(x, round + 1);
                load_rows(x, round + 2);
                __builtin_amdgcn_sched_barrier(0);
                load_weights(w[d & 1], step0 + (round + 2) * kW + part);
                if (d == 3) write_scales(c);
                own_writes_and_barrier();
            }
        }

        // A lane holds four consecutive rows of a slot.
        int slot[kNT];
#pragma unroll
        for (int n = 0; n < kNT; ++n) slot[n] = n * 16 + l16 < kTok ? __shfl(held, n * 16 + l16) : -1;
        auto out = [&](int s, int n, float4 v, float4 o) {
            const int at = s * 16 + 4 * g;
            if (slot[n] < 0 || at >= rows) return;
            if constexpr (kDown) {
                const float by = a.weight[slot[n]];
                *reinterpret_cast<float4 *>(a.P + ((int64_t)blockIdx.z * a.slots + slot[n]) * a.rows + r0 + at) =
                    make_float4(v.x * f[0] * by, v.y * f[0] * by, v.z * f[0] * by, v.w * f[0] * by);
            } else {
                const float gate[4] = {v.x * f[0], v.y * f[0], v.z * f[0], v.w * f[0]};
                const float up[4] = {o.x * f[1], o.y * f[1], o.z * f[1], o.w * f[1]};
                store_hidden(a.H + (int64_t)slot[n] * 2 * a.rows + r0 + at, a.rows, gate, up);
            }
        };
        constexpr int kOuts = kDown ? kSets : kRT;  // tiles of 16 rows
        auto four = [&](int s, int n) { return make_float4(acc[s][n][0], acc[s][n][1], acc[s][n][2], acc[s][n][3]); };
        if constexpr (kW == 1) {
#pragma unroll
            for (int s = 0; s < kOuts; ++s)
#pragma unroll
                for (int n = 0; n < kNT; ++n) out(s, n, four(s, n), four(kDown ? s : kRT + s, n));
        } else {
            float4 *red = reinterpret_cast<float4 *>(lds);  // [4 waves][kSets * kNT][64]
#pragma unroll
            for (int s = 0; s < kSets; ++s)
#pragma unroll
                for (int n = 0; n < kNT; ++n) red[(wave * kSets * kNT + s * kNT + n) * 64 + lane] = four(s, n);
            own_writes_and_barrier();
            auto sum = [&](int unit) {
                const float4 *from = red + (wave / kW * kW * kSets * kNT + unit) * 64 + lane;
                float4 v = from[0];
#pragma unroll
                for (int q = 1; q < kW; ++q) {
                    const float4 o = from[q * kSets * kNT * 64];
                    v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
                }
                return v;
            };
#pragma unroll
            for (int s = 0; s < kOuts; ++s)
#pragma unroll
                for (int n = 0; n < kNT; ++n)
                    if ((s * kNT + n) % kW == part)
                        out(s, n, sum(s * kNT + n), kDown ? float4{} : sum((kRT + s) * kNT + n));
            own_writes_and_barrier();
        }
    }
}

// Y[t] = the sum over the splits of k of the token's slots, both in their order;
// four outputs a thread.  A slot without an expert adds its weight times 0; what
// lies in its place is read with the others', so that all are under way at once,
// and left out.
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ P, int splits, int64_t slots,
                                                   const int32_t *__restrict__ ids, const float *__restrict__ weight,
                                                   int choices, int experts, int64_t out, uint16_t *__restrict__ Y,
                                                   int64_t ldy, bool wide) {
    const int64_t t = blockIdx.y, m = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (m >= out) return;
    constexpr int kAhead = 8;
    float y[4] = {0, 0, 0, 0};
    const float *p = P + t * choices * out + m;
    int j = 0, z = 0;
    while (z < splits) {
        float4 a[kAhead];
        float other[kAhead];  // in its place, if there is no expert
        bool none[kAhead], some[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            some[q] = z < splits;
            const int jq = some[q] ? j : 0;
            a[q] = *reinterpret_cast<const float4 *>(p + ((some[q] ? z : 0) * slots + jq) * out);
            none[q] = expert_of(ids, experts, (int)(t * choices) + jq) == kNoExpert;
            other[q] = z == 0 ? weight[t * choices + jq] * 0.0f : 0.0f;
            if (++j == choices) j = 0, ++z;
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            if (!some[q]) continue;
            y[0] += none[q] ? other[q] : a[q].x, y[1] += none[q] ? other[q] : a[q].y;
            y[2] += none[q] ? other[q] : a[q].z, y[3] += none[q] ? other[q] : a[q].w;
        }
    }
    uint16_t *dst = Y + t * ldy + m;
    const uint32_t lo = bf16_pair(y[0], y[1]), hi = bf16_pair(y[2], y[3]);
    if (wide) {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
    } else {
        dst[0] = (uint16_t)lo, dst[1] = (uint16_t)(lo >> 16), dst[2] = (uint16_t)hi, dst[3] = (uint16_t)(hi >> 16);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

int check_matrix(const hscale_experts *w) {
    if (!w || !w->global_scale || !w->scale_codes || !w->packed_e2m1) return HSCALE_ERR_NULL;
    if (!aligned(w->global_scale, 4) || !aligned(w->packed_e2m1, 8)) return HSCALE_ERR_ALIGN;
    return HSCALE_OK;
}

Matrices matrices(const hscale_experts *w) { return Matrices{w->global_scale, w->scale_codes, w->packed_e2m1}; }

template <bool kDown, int kTok, int kRT, int kW, int kStep = 256>
int launch_experts(const ExpertArgs &a, int shares, int splits, hipStream_t stream) {
    const dim3 grid((unsigned)cdiv(a.rows, (kDown ? 32 : 16) * kRT * (4 / kW)), (unsigned)shares, (unsigned)splits);
    hipLaunchKernelGGL((expert_kernel<kDown, kTok, kRT, kW, kStep>), grid, dim3(256), 0, stream, a);
    return launch_status();
}

int gate_and_up(const ExpertArgs &a, int shares, int tile, int waves, hipStream_t stream) {
    if (tile == 4 && waves == 2) return launch_experts<false, 4, 1, 2>(a, shares, 1, stream);
    if (tile <= 16)
        return waves == 2 ? launch_experts<false, 16, 1, 2>(a, shares, 1, stream)
                          : launch_experts<false, 16, 1, 1>(a, shares, 1, stream);
    if (tile == 32)
        return waves == 4 ? launch_experts<false, 32, 1, 4, 128>(a, shares, 1, stream)
                          : launch_experts<false, 32, 1, 1>(a, shares, 1, stream);
    return waves == 4 ? launch_experts<false, 64, 1, 4, 128>(a, shares, 1, stream)
                      : launch_experts<false, 64, 2, 1, 128>(a, shares, 1, stream);
}

int down_product(const ExpertArgs &a, int shares, int tile, int splits, hipStream_t stream) {
    if (tile == 4) return launch_experts<true, 4, 1, 1>(a, shares, splits, stream);
    if (tile == 16) return launch_experts<true, 16, 1, 1>(a, shares, splits, stream);
    if (tile == 64) return launch_experts<true, 64, 2, 1, 128>(a, shares, splits, stream);
    return launch_experts<true, 32, 2, 1, 128>(a, shares, splits, stream);
}

}  // namespace

extern "C" {

int hscale_route_tokens(const void *logits, int32_t type, int64_t tokens, int32_t experts, int64_t ld, int32_t k,
                        int32_t normalize, int32_t *expert, float *weight, hipStream_t stream) {
    if (tokens < 0 || tokens > kMaxTokens || experts < 1 || experts > kMaxExperts || k < 1 || k > kMaxChoices ||
        k > experts || (type != HSCALE_BF16 && type != HSCALE_F32) || (tokens > 1 && ld < experts))
        return HSCALE_ERR_SHAPE;
    if (tokens == 0) return HSCALE_OK;
    if (!logits || !expert || !weight) return HSCALE_ERR_NULL;
    const size_t size = type == HSCALE_F32 ? 4 : 2;
    if (!aligned(logits, size) || !aligned(expert, 4) || !aligned(weight, 4)) return HSCALE_ERR_ALIGN;
    const Range w[] = {{expert, (size_t)tokens * k * 4}, {weight, (size_t)tokens * k * 4}};
    const Range r[] = {{logits, span(tokens, ld, experts, size)}};
    if (any_overlap(w, 2, r, 1)) return HSCALE_ERR_OVERLAP;
    const dim3 grid((unsigned)cdiv(tokens, 4));
#define ROUTE(n)                                                                                                     \
    if (type == HSCALE_F32)                                                                                          \
        hipLaunchKernelGGL((route_kernel<n, true>), grid, dim3(256), 0, stream, logits, tokens, experts, ld, k,      \
                           normalize != 0, expert, weight);                                                          \
    else                                                                                                             \
        hipLaunchKernelGGL((route_kernel<n, false>), grid, dim3(256), 0, stream, logits, tokens, experts, ld, k,     \
                           normalize != 0, expert, weight)
    if (experts <= 64) {
        ROUTE(1);
    } else if (experts <= 128) {
        ROUTE(2);
    } else if (experts <= 192) {
        ROUTE(3);
    } else if (experts <= 256) {
        ROUTE(4);
    } else {
        ROUTE(16);
    }
#undef ROUTE
    return launch_status();
}

size_t hscale_expert_layer_workspace_bytes(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k) {
    if (!layer_sizes_ok(tokens, in, hidden, experts, k) || tokens == 0 || in == 0 || hidden == 0) return 0;
    return layer_space(tokens, in, hidden, experts, k).total;
}

int hscale_expert_layer(const void *X, int64_t tokens, int64_t in, int64_t ldx, int64_t hidden, int32_t experts,
                        const hscale_experts *gate, const hscale_experts *up, const hscale_experts *down,
                        const int32_t *expert, const float *weight, int32_t k, void *Y, int64_t ldy, void *workspace,
                        size_t workspace_bytes, hipStream_t stream) {
    if (!layer_sizes_ok(tokens, in, hidden, experts, k) ||
        (tokens > 1 && (ldx < in || ldx > kMaxWidth || ldy < in)))
        return HSCALE_ERR_SHAPE;
    if (tokens == 0) return HSCALE_OK;
    if (in == 0 || hidden == 0) return HSCALE_ERR_SHAPE;
    if (tokens == 1) ldx = ldy = in;
    for (const hscale_experts *w : {gate, up, down})
        if (const int st = check_matrix(w)) return st;
    if (!X || !expert || !weight || !Y || !workspace) return HSCALE_ERR_NULL;
    if (!aligned(X, 16) || ldx % 8 != 0 || !aligned(expert, 4) || !aligned(weight, 4) || !aligned(Y, 2) ||
        !aligned(workspace, 256))
        return HSCALE_ERR_ALIGN;
    const LayerSpace space = layer_space(tokens, in, hidden, experts, k);
    if (workspace_bytes < space.total) return HSCALE_ERR_WORKSPACE;
    const size_t matrix = (size_t)experts * in * hidden;
    const Range w[] = {{Y, span(tokens, ldy, in, 2)}, {workspace, space.total}};
    const Range r[] = {{X, span(tokens, ldx, in, 2)},
                       {expert, (size_t)tokens * k * 4},
                       {weight, (size_t)tokens * k * 4},
                       {gate->global_scale, (size_t)experts * 4},
                       {gate->scale_codes, matrix / 16},
                       {gate->packed_e2m1, matrix / 2},
                       {up->global_scale, (size_t)experts * 4},
                       {up->scale_codes, matrix / 16},
                       {up->packed_e2m1, matrix / 2},
                       {down->global_scale, (size_t)experts * 4},
                       {down->scale_codes, matrix / 16},
                       {down->packed_e2m1, matrix / 2}};
    if (any_overlap(w, 2, r, 12)) return HSCALE_ERR_OVERLAP;

    char *ws = static_cast<char *>(workspace);
    uint16_t *H = reinterpret_cast<uint16_t *>(ws);
    float *P = reinterpret_cast<float *>(ws += space.h);
    int32_t *order = reinterpret_cast<int32_t *>(ws += space.p);
    Share *shares = reinterpret_cast<Share *>(ws + space.order);
    const LayerPlan plan = plan_layer(tokens, in, hidden, experts, k, ldx);
    for (int64_t t0 = 0; t0 < tokens; t0 += plan.piece) {
        const int64_t n = std::min(plan.piece, tokens - t0);
        const PiecePlan piece = plan_piece(plan, n, experts, k);
        const int32_t *ids = expert + t0 * k;
        if (piece.many) {
            hipLaunchKernelGGL(share_kernel, dim3(1), dim3(1024), 0, stream, ids, piece.slots, (int)experts, piece.tile,
                               order, shares, piece.shares);
            if (const int st = launch_status()) return st;
        }
        ExpertArgs a{};
        a.w[0] = matrices(gate);
        a.w[1] = matrices(up);
        a.rows = hidden, a.k = in;
        a.in = static_cast<const uint16_t *>(X) + t0 * ldx;
        a.ld = ldx;
        a.in_bytes = (int64_t)span(n, ldx, in, 2);
        a.ids = ids;
        a.weight = weight + t0 * k;
        a.slots = piece.slots, a.choices = k, a.experts = experts;
        a.order = piece.many ? order : nullptr;
        a.shares = piece.many ? shares : nullptr;
        a.H = H;
        a.P = P;
        if (const int st = gate_and_up(a, piece.shares, piece.tile, plan.waves, stream)) return st;
        a.w[0] = a.w[1] = matrices(down);
        a.rows = in, a.k = hidden;
        a.in = H;
        a.ld = 2 * hidden;
        a.in_bytes = (int64_t)piece.slots * hidden * 4;
        a.split = plan.split * (piece.tile >= 32 ? 2 : 1);  // steps of 128 there
        if (const int st = down_product(a, piece.shares, piece.tile, plan.splits, stream)) return st;
        uint16_t *y = static_cast<uint16_t *>(Y) + t0 * ldy;
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)cdiv(in, 1024), (unsigned)n), dim3(256), 0, stream, P, plan.splits,
                           (int64_t)piece.slots, ids, a.weight, (int)k, (int)experts, in, y, ldy, aligned(y, 8) && ldy % 4 == 0);
        if (const int st = launch_status()) return st;
    }
    return HSCALE_OK;
}

}  // extern "C"
