// What a request's rules change its logits by before a token is chosen, behind
// the C ABI of include/hscale.h:
//
//   l = l > 0 ? l / r : l r        of words in the history
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

// kWords words of one row per block.  Their counts in the row's history are
// made in LDS, by integer additions whose order does not show; every block of a
// row reads the whole history.
template <bool kWide, int kWords>
__global__ __launch_bounds__(256) void adjust_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t said[kWords];
    const int tid = threadIdx.x;
    const int64_t v0 = (int64_t)blockIdx.x * kWords;
    const int words = (int)(a.vocab - v0 < kWords ? a.vocab - v0 : kWords);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        int length = 0;
        if (a.penalties) {
            const int most = (int)a.r.history_length;
            length = a.r.length ? clamped(a.r.length, row, 0, most) : most;
            const int prompt = a.r.prompt ? clamped(a.r.prompt, row, 0, most) : 0;
            if (length > 0) {
                for (int i = tid * 4; i < kWords; i += 1024)
                    *reinterpret_cast<u32x4 *>(said + i) = u32x4{0, 0, 0, 0};
                __syncthreads();
                const int32_t *h = a.r.history + row * a.r.history_ld;
                auto count = [&](int i, int32_t word) {
                    const uint32_t at = (uint32_t)word - (uint32_t)v0;
                    if (word < 0 || at >= (uint32_t)words) return;
                    if (i < prompt)
                        atomicOr(&said[at], kInPrompt);
                    else
                        atomicAdd(&said[at], 1u);
                };
                int i = tid * 4;
                for (; i + 4 <= length; i += 1024) {
                    const u32x4 w = load_any<u32x4>(h + i);
#pragma unroll
                    for (int q = 0; q < 4; ++q) count(i + q, (int32_t)w[q]);
                }
                for (; i < length; ++i) count(i, h[i]);  // the last ones, three at most
                __syncthreads();
            }
        }
        const float rho = a.r.repetition ? a.r.repetition[row] : 1.0f;
        const float frequency = a.r.frequency ? a.r.frequency[row] : 0.0f;
        const float presence = a.r.presence ? a.r.presence[row] : 0.0f;
        const int bias_row = !a.r.bias ? -1 : a.r.bias_row ? a.r.bias_row[row] : 0;
        const int mask_row = !a.r.mask ? -1 : a.r.mask_row ? a.r.mask_row[row] : 0;
        const float *bias = bias_row >= 0 && bias_row < a.r.biases ? a.r.bias + bias_row * a.vocab + v0 : nullptr;
        const uint8_t *mask = mask_row >= 0 && mask_row < a.r.masks
                                  ? reinterpret_cast<const uint8_t *>(a.r.mask + mask_row * ((a.vocab + 31) / 32)) + v0 / 8
                                  : nullptr;
        auto changed = [&](float l, uint32_t n, float b, bool allowed) {
            if (n) {
                if (a.r.repetition) l = l > 0.0f ? l / rho : l * rho;
                const uint32_t c = n & ~kInPrompt;
                if (c) {
                    if (a.r.frequency) l -= frequency * (float)c;
                    if (a.r.presence) l -= presence;
                }
            }
            if (bias) l += b;
            return allowed ? l : -INFINITY;
        };
        constexpr int kSize = kWide ? 4 : 2;
        const char *src = static_cast<const char *>(a.logits) + (row * a.ld + v0) * kSize;
        char *dst = static_cast<char *>(a.out) + (row * a.ldo + v0) * kSize;
        for (int v = tid * 8; v < words; v += 2048) {
            const int n = words - v < 8 ? words - v : 8;
            float l[8], b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            const uint32_t bits = mask ? mask[v >> 3] : 0xFFu;
            if (n == 8) {
                if (kWide) {
                    const u32x4 x = load_any<u32x4>(src + v * 4), y = load_any<u32x4>(src + v * 4 + 16);
#pragma unroll
                    for (int q = 0; q < 4; ++q) l[q] = __uint_as_float(x[q]), l[q + 4] = __uint_as_float(y[q]);
                } else {
                    const u32x4 x = load_any<u32x4>(src + v * 2);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        l[2 * q] = __uint_as_float(x[q] << 16), l[2 * q + 1] = __uint_as_float(x[q] & 0xFFFF0000u);
                }
                if (bias) {
                    const u32x4 x = load_any<u32x4>(bias + v), y = load_any<u32x4>(bias + v + 4);
#pragma unroll
                    for (int q = 0; q < 4; ++q) b[q] = __uint_as_float(x[q]), b[q + 4] = __uint_as_float(y[q]);
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
            if (length > 0) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(said + v), y = *reinterpret_cast<const u32x4 *>(said + v + 4);
#pragma unroll
                for (int q = 0; q < 8; ++q) l[q] = changed(l[q], q < 4 ? x[q & 3] : y[q & 3], b[q], bits >> q & 1);
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) l[q] = changed(l[q], 0, b[q], bits >> q & 1);
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
        __syncthreads();
    }
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
    constexpr int kFew = 2048, kMany = 8192;
    const bool few = rows * vocab <= (int64_t)256 * kMany;
    const dim3 grid((unsigned)((vocab + (few ? kFew : kMany) - 1) / (few ? kFew : kMany)),
                    (unsigned)std::min<int64_t>(rows, 65535));
    if (type == HSCALE_F32 && few)
        hipLaunchKernelGGL((adjust_kernel<true, kFew>), grid, dim3(256), 0, stream, a);
    else if (type == HSCALE_F32)
        hipLaunchKernelGGL((adjust_kernel<true, kMany>), grid, dim3(256), 0, stream, a);
    else if (few)
        hipLaunchKernelGGL((adjust_kernel<false, kFew>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((adjust_kernel<false, kMany>), grid, dim3(256), 0, stream, a);
    return launch_status();
}

}  // extern "C"
