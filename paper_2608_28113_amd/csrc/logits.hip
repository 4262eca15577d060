// What a request's rules change its logits by before a token is chosen, behind
// the C ABI of include/hscale.h:
//
//   l = l > 0 ? l (1 / r) : l r    of words in the history
//   l = l - f count - p            of words in the answer
//   l = l + bias,  l = -inf        where the mask forbids a word
//
// Times below are of one MI355X, whose large copies reach 4.9 TB/s.

#include "checks.h"

#include <algorithm>
#include <tuple>

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 24, kMostVocab = (int64_t)1 << 24;
constexpr int64_t kMostHistory = (int64_t)1 << 30;
constexpr uint32_t kInPrompt = 0x80000000u;  // beside a word's count in the answer

struct LogitArgs {
    hscale_logit_rules r;
    const void *logits;
    void *out;
    int64_t rows, vocab, ld, ldo;
    bool penalties;
};

__device__ __forceinline__ int clamped(const int32_t *p, int64_t row, int64_t least, int64_t most) {
    return p ? (int)(p[row] < least ? least : p[row] > most ? most : p[row]) : -1;
}

// Rows lie at any alignment of their type; loads and stores of 16 bytes need
// none of their own here.
template <class T>
__device__ __forceinline__ T load_any(const void *p) {
    T v;
    __builtin_memcpy(&v, p, sizeof(T));
    return v;
}

struct Eight {  // words of one row
    u32x4 v[2];  // bf16: the first alone
};

template <bool kWide>
__device__ __forceinline__ void unpack(const Eight &w, float (&l)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (kWide) {
            l[q] = __uint_as_float(w.v[0][q]), l[q + 4] = __uint_as_float(w.v[1][q]);
        } else {
            l[2 * q] = __uint_as_float(w.v[0][q] << 16), l[2 * q + 1] = __uint_as_float(w.v[0][q] & 0xFFFF0000u);
        }
    }
}

// kWords words of one row per block, eight a thread at a time.  Their counts in
// the row's history are made in LDS, by integer additions whose order does not
// show; every block of a row reads the whole history, while its logits are under
// way.  64 rows of 128000 bf16 logits with 2000 words said, biases and masks take
// 13.7 us, of which 4 are a launch's own (33 MB in and out); 256 of fp32 in a
// grammar 59 us, 4.5 TB/s, a copy's rate; 16 rows with 32768 words said 11.4 us,
// each history read by 16 blocks.
template <bool kWide, int kWords, int kThreads>
__global__ __launch_bounds__(kThreads) void adjust_kernel(const LogitArgs a) {
    constexpr int kSize = kWide ? 4 : 2, kUnits = kWords / (8 * kThreads), kAhead = 4;
    static_assert(kUnits * 8 * kThreads == kWords, "whole units");
    __shared__ __attribute__((aligned(16))) uint32_t said[kWords];
    const int tid = threadIdx.x;
    const int64_t v0 = (int64_t)blockIdx.x * kWords;
    const int words = (int)(a.vocab - v0 < kWords ? a.vocab - v0 : kWords);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const char *src = static_cast<const char *>(a.logits) + (row * a.ld + v0) * kSize;
        char *dst = static_cast<char *>(a.out) + (row * a.ldo + v0) * kSize;
        // The history's first words, then the logits, under way together.
        const int most = a.penalties ? (int)a.r.history_length : 0;
        const int32_t *h = a.r.history + row * a.r.history_ld;
        u32x4 w[kAhead];
        auto load_words = [&](int i0) {
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                const int i = i0 + (b * kThreads + tid) * 4;
                if (i + 4 <= most) w[b] = load_any<u32x4>(h + i);
            }
        };
        load_words(0);
        Eight x[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int v = (u * kThreads + tid) * 8;
            if (v + 8 > words) continue;
            x[u].v[0] = load_any<u32x4>(src + v * kSize);
            if (kWide) x[u].v[1] = load_any<u32x4>(src + v * kSize + 16);
        }
        const int length = a.penalties && a.r.length ? clamped(a.r.length, row, 0, most) : most;
        if (length > 0) {
            const int prompt = a.r.prompt ? clamped(a.r.prompt, row, 0, most) : 0;
#pragma unroll
            for (int i = 0; i < kWords; i += 4 * kThreads)
                *reinterpret_cast<u32x4 *>(said + i + tid * 4) = u32x4{0, 0, 0, 0};
            __syncthreads();
            auto count = [&](int i, int32_t word) {
                const uint32_t at = (uint32_t)word - (uint32_t)v0;
                if (i >= length || word < 0 || at >= (uint32_t)words) return;
                if (i < prompt)
                    atomicOr(&said[at], kInPrompt);
                else
                    atomicAdd(&said[at], 1u);
            };
            for (int i0 = 0; i0 < length; i0 += kAhead * 4 * kThreads) {
                if (i0 > 0) load_words(i0);
#pragma unroll
                for (int b = 0; b < kAhead; ++b) {
                    const int i = i0 + (b * kThreads + tid) * 4;
                    if (i + 4 <= most) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) count(i + q, (int32_t)w[b][q]);
                    } else {
                        for (int q = i; q < most; ++q) count(q, h[q]);  // the last ones, three at most
                    }
                }
            }
            __syncthreads();
        }
        const float rho = a.r.repetition ? a.r.repetition[row] : 1.0f, inv = 1.0f / rho;
        const float frequency = a.r.frequency ? a.r.frequency[row] : 0.0f;
        const float presence = a.r.presence ? a.r.presence[row] : 0.0f;
        const int bias_row = !a.r.bias ? -1 : a.r.bias_row ? a.r.bias_row[row] : 0;
        const int mask_row = !a.r.mask ? -1 : a.r.mask_row ? a.r.mask_row[row] : 0;
        const float *bias = bias_row >= 0 && bias_row < a.r.biases ? a.r.bias + bias_row * a.vocab + v0 : nullptr;
        const uint8_t *mask = mask_row >= 0 && mask_row < a.r.masks
                                  ? reinterpret_cast<const uint8_t *>(a.r.mask + mask_row * ((a.vocab + 31) / 32)) + v0 / 8
                                  : nullptr;
        // A division for each word would take most of the time.
        auto penalized = [&](float l, uint32_t n) {
            l *= l > 0.0f ? inv : rho;
            const uint32_t c = n & ~kInPrompt;
            return c ? l - frequency * (float)c - presence : l;
        };
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int v = (u * kThreads + tid) * 8;
            if (v >= words) continue;
            const int n = words - v < 8 ? words - v : 8;
            const uint32_t bits = mask ? mask[v >> 3] : 0xFFu;
            float l[8], b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (n == 8) {
                unpack<kWide>(x[u], l);
                if (bias) {
                    const u32x4 x0 = load_any<u32x4>(bias + v), x1 = load_any<u32x4>(bias + v + 4);
#pragma unroll
                    for (int q = 0; q < 4; ++q) b[q] = __uint_as_float(x0[q]), b[q + 4] = __uint_as_float(x1[q]);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    l[q] = 0.0f;
                    if (q >= n) continue;
                    if (kWide)
                        l[q] = reinterpret_cast<const float *>(src)[v + q];
                    else
                        l[q] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(src)[v + q] << 16);
                    if (bias) b[q] = bias[v + q];
                }
            }
            u32x4 n0{0, 0, 0, 0}, n1{0, 0, 0, 0};
            if (length > 0) {
                n0 = *reinterpret_cast<const u32x4 *>(said + v);
                n1 = *reinterpret_cast<const u32x4 *>(said + v + 4);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const uint32_t said_q = q < 4 ? n0[q & 3] : n1[q & 3];
                if (said_q) l[q] = penalized(l[q], said_q);
            }
            if (bias) {
#pragma unroll
                for (int q = 0; q < 8; ++q) l[q] += b[q];
            }
            if (mask) {
#pragma unroll
                for (int q = 0; q < 8; ++q) l[q] = bits >> q & 1 ? l[q] : -INFINITY;
            }
            if (kWide) {
                if (n == 8) {
                    __builtin_memcpy(dst + v * 4, l, 32);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < n) reinterpret_cast<float *>(dst)[v + q] = l[q];
                }
            } else {
                uint16_t w[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) w[q] = __builtin_bit_cast(uint16_t, (__bf16)l[q]);
                if (n == 8) {
                    __builtin_memcpy(dst + v * 2, w, 16);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < n) reinterpret_cast<uint16_t *>(dst)[v + q] = w[q];
                }
            }
        }
        if (gridDim.y < a.rows) __syncthreads();
    }
}

template <bool kWide, int kWords, int kThreads>
int launch_adjust(const LogitArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.vocab + kWords - 1) / kWords), (unsigned)std::min<int64_t>(a.rows, 65535));
    hipLaunchKernelGGL((adjust_kernel<kWide, kWords, kThreads>), grid, dim3(kThreads), 0, stream, a);
    return launch_status();
}

// Blocks of a row read its whole history each, so a long one goes to fewer and
// larger blocks (its length on the host is the most that a row may have).  In
// us with bf16 logits, blocks of 2048, 4096, 8192 words by 512 threads and by 1024:
//   1 row of 128000, 1000 said       3.6   4.4   4.6   4.4
//   1 row of 128000, 16384 said      7.4   8.4   6.7   5.6
//   64 rows of 128000, 1000 said    12.8  11.9  12.2  15.5
//   64 rows of 128000, 16384 said   29.5  22.9  20.2  24.1
template <bool kWide>
int adjust(const LogitArgs &a, hipStream_t stream) {
    const bool few = a.rows * a.vocab <= (int64_t)1 << 21;
    if (a.penalties && a.r.history_length > 4096)
        return few ? launch_adjust<kWide, 8192, 1024>(a, stream) : launch_adjust<kWide, 8192, 512>(a, stream);
    return few ? launch_adjust<kWide, 2048, 256>(a, stream) : launch_adjust<kWide, 4096, 256>(a, stream);
}

}  // namespace

extern "C" {

int hscale_adjust_logits(const hscale_logit_rules *rules, const void *logits, int32_t type, int64_t rows, int64_t vocab,
                         int64_t ld, void *out, int64_t ldo, hipStream_t stream) {
    if (rows < 0 || rows > kMostRows || vocab < 0 || vocab > kMostVocab ||
        (type != HSCALE_BF16 && type != HSCALE_F32) || (rows > 1 && (ld < vocab || ldo < vocab)))
        return HSCALE_ERR_SHAPE;
    if (!rules) return HSCALE_ERR_NULL;
    const hscale_logit_rules &r = *rules;
    const bool penalties = r.repetition || r.frequency || r.presence;
    if ((r.history || penalties) && (r.history_length < 0 || r.history_length > kMostHistory ||
                                     (rows > 1 && r.history_ld < r.history_length)))
        return HSCALE_ERR_SHAPE;
    for (const auto &[p, n, at] : {std::make_tuple((const void *)r.bias, r.biases, r.bias_row),
                                   std::make_tuple((const void *)r.mask, r.masks, r.mask_row)})
        if (p && (n < 0 || n > (1 << 24) || (!at && n != 1))) return HSCALE_ERR_SHAPE;
    if (rows == 0 || vocab == 0) return HSCALE_OK;
    if (!logits || !out || (penalties && !r.history && r.history_length > 0)) return HSCALE_ERR_NULL;
    const size_t size = type == HSCALE_F32 ? 4 : 2;
    if (!aligned(logits, size) || !aligned(out, size)) return HSCALE_ERR_ALIGN;
    for (const void *p : {(const void *)r.history, (const void *)r.length, (const void *)r.prompt,
                          (const void *)r.repetition, (const void *)r.frequency, (const void *)r.presence,
                          (const void *)r.bias, (const void *)r.bias_row, (const void *)r.mask,
                          (const void *)r.mask_row})
        if (!aligned(p, 4)) return HSCALE_ERR_ALIGN;
    const size_t each = (size_t)rows * 4;
    const Range w[] = {{out, span(rows, ldo, vocab, size)}};
    const Range in[] = {{out == logits && (rows == 1 || ldo == ld) ? nullptr : logits, span(rows, ld, vocab, size)},
                        {r.history, span(rows, r.history_ld, r.history_length, 4)},
                        {r.length, each},
                        {r.prompt, each},
                        {r.repetition, each},
                        {r.frequency, each},
                        {r.presence, each},
                        {r.bias, (size_t)r.biases * vocab * 4},
                        {r.bias_row, each},
                        {r.mask, (size_t)r.masks * ((vocab + 31) / 32) * 4},
                        {r.mask_row, each}};
    for (const Range &x : in)
        if (x.p && overlaps(w[0].p, w[0].n, x.p, x.n)) return HSCALE_ERR_OVERLAP;
    const LogitArgs a{r, logits, out, rows, vocab, ld, ldo, penalties && r.history_length > 0};
    return type == HSCALE_F32 ? adjust<true>(a, stream) : adjust<false>(a, stream);
}

}  // extern "C"
