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
#include "matmul.h"
#include "stored.h"

#include <algorithm>

namespace {

constexpr int kMaxExperts = 1024;
constexpr int kMaxChoices = 32;
constexpr int64_t kMaxWidth = (int64_t)1 << 21;
constexpr int64_t kMaxTokens = (int64_t)1 << 24;
constexpr int kNoExpert = -1;

// ---------------------------------------------------------------------------
// Routing
// ---------------------------------------------------------------------------

// A number that orders as (logit, lowest index first), 0 for what is never
// chosen: -inf and NaN.  -0 and +0 are equal.
__device__ __forceinline__ uint64_t choice_key(float l, int e) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(l + 0.0f);
    return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~e;
}

// A wave per token, kN logits a lane.  k rounds of the wave's largest key, each
// taken out where it lies; the softmax is relative to the first.
template <int kN, bool kWide>
__global__ __launch_bounds__(256) void route_kernel(const void *__restrict__ logits, int64_t tokens, int experts,
                                                    int64_t ld, int k, bool normalize, int32_t *__restrict__ expert,
                                                    float *__restrict__ weight) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= tokens) return;
    float l[kN];
    uint64_t key[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int e = i * 64 + lane;
        l[i] = -INFINITY;
        if (e < experts)
            l[i] = kWide ? static_cast<const float *>(logits)[t * ld + e]
                         : bf16_value(static_cast<const uint16_t *>(logits)[t * ld + e]);
        key[i] = choice_key(l[i], e);
    }
    float top = 0.0f, all = 0.0f, some = 0.0f, mine = 0.0f;
    int which = kNoExpert;  // lane j holds the j-th choice
    for (int j = 0; j < k; ++j) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) best = key[i] > best ? key[i] : best;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor((unsigned long long)best, o);
            best = other > best ? other : best;
        }
        if (best == 0) break;  // fewer than k can be chosen
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (key[i] == best) key[i] = 0;
        const uint32_t u = (uint32_t)(best >> 32);
        const float v = __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
        if (j == 0) top = v;
        const float p = expf(v - top);
        some += p;
        if (lane == j) which = (int)~(uint32_t)best, mine = p;
    }
    // Over all experts too where the k alone are asked for: a NaN anywhere shows.
#pragma unroll
    for (int i = 0; i < kN; ++i)
        if (!(l[i] == -INFINITY)) all += expf(l[i] - top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    if (lane >= k) return;
    expert[t * k + lane] = which;
    weight[t * k + lane] = all != all ? all : which == kNoExpert ? 0.0f : mine / (normalize ? some : all);
}

// ---------------------------------------------------------------------------
// Which slots an expert has
// ---------------------------------------------------------------------------

constexpr int kBlockSlots = 256;  // up to so many, each block finds its expert's slots itself

__device__ __forceinline__ int expert_of(const int32_t *ids, int experts, int s) {
    const int e = ids[s];
    return e >= 0 && e < experts ? e : kNoExpert;
}

// Up to 16 kNT slots of one expert; count 0: none.
struct Share {
    int expert, first, count;
};

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
    float *P;          // [slots, rows]: down
};

// s = f 2^e with 1 <= f < 2, or more where 2^e would take the largest weight
// out of bf16's range.
__device__ __forceinline__ void split_device_scale(float s, float &f, int &e) {
    constexpr int kMostE = 100;
    e = (int)(__float_as_uint(s) >> 23 & 0xFF) - 127;
    e = e > kMostE ? kMostE : e < -126 ? -126 : e;
    f = ldexpf(s, -e);
}

// 16 kRT rows of gate and of up (or 32 kRT of down) x up to 16 kNT slots of one
// expert per block.  Its four waves take every fourth 128 k and add up through
// LDS.  A wave's MFMA operand of weights comes straight from memory, 32
// consecutive weights a lane: which k meets which place in a step does not
// matter, as both operands agree.  The slots' rows come from L2 the same way;
// each is read by one wave of the block.
template <bool kDown, int kRT, int kNT, bool kEven>
__global__ __launch_bounds__(256) void expert_kernel(const ExpertArgs a) {
    constexpr int kSets = 2 * kRT, kMats = kDown ? 1 : 2, kParts = kDown ? 2 : 1;
    constexpr int kRows = kDown ? 32 * kRT : 16 * kRT;  // of a matrix
    constexpr int kStep = 128, kDepth = 2;
    __shared__ __attribute__((aligned(16))) float4 red[4][kSets * kNT][64];
    __shared__ int list[kBlockSlots];
    __shared__ int found[4];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r0 = (int64_t)blockIdx.x * kRows;
    const int rows = (int)(a.rows - r0 < kRows ? a.rows - r0 : kRows);
    const int K = (int)a.k;

    int expert, count;
    if (a.shares) {
        const Share s = a.shares[blockIdx.y];
        expert = s.expert, count = s.count;
        if (count == 0) return;
        if (tid < count) list[tid] = a.order[s.first + tid];
    } else {
        const int own = tid < a.slots ? expert_of(a.ids, a.experts, tid) : kNoExpert;
        // As many blocks as slots: that of an expert's first slot.  Else one of each expert.
        expert = a.slots <= a.experts ? expert_of(a.ids, a.experts, blockIdx.y) : (int)blockIdx.y;
        if (expert == kNoExpert) return;
        const uint64_t mask = __ballot(own == expert);
        if (lane == 0) found[wave] = __popcll(mask);
        __syncthreads();
        int before = __popcll(mask & (((uint64_t)1 << lane) - 1));
        count = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before += found[w];
            count += found[w];
        }
        if (own == expert) list[before] = tid;
        __syncthreads();
        if (count == 0 || (a.slots <= a.experts && list[0] != (int)blockIdx.y)) return;
    }
    __syncthreads();
    expert = __builtin_amdgcn_readfirstlane(expert);
    count = __builtin_amdgcn_readfirstlane(count);

    float f[2];
    int e[2];
    __amdgpu_buffer_rsrc_t rp[2], rc[2];
#pragma unroll
    for (int m = 0; m < kMats; ++m) {
        split_device_scale(a.w[m].scale[expert], f[m], e[m]);
        const int64_t row = (int64_t)expert * a.rows + r0;
        rp[m] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.w[m].packed) + row * (K / 2), 0,
                                                  rows * (K / 2), kRawWord3);
        rc[m] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.w[m].codes) + row * (K / 16), 0,
                                                  rows * (K / 16), kRawWord3);
    }
    const __amdgpu_buffer_rsrc_t rx =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.in), 0, (int)a.in_bytes, kRawWord3);
    const uint32_t prow = (uint32_t)(l16 * (K / 2) + g * 16), crow = (uint32_t)(l16 * (K / 16) + g * 2);

    struct Weights {
        u32x4 p[kSets];
        uint32_t c[kSets];
    };
    struct Inputs {
        u32x4 x[kNT][kParts][4];
    };
    auto load_weights = [&](Weights &w, int step) {
        const uint32_t k = step * kStep;
        const uint32_t skip = (int)(k + g * 32) < K ? 0 : kNoRead;
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            const int m = kDown ? 0 : s / kRT, tile = kDown ? s : s % kRT;
            const uint32_t c = crow + tile * 16 * (K / 16) + k / 16 + skip;
            w.p[s] = __builtin_amdgcn_raw_buffer_load_b128(rp[m], prow + tile * 16 * (K / 2) + k / 2 + skip, 0, 0);
            if (kEven) {
                w.c[s] = __builtin_amdgcn_raw_buffer_load_b16(rc[m], c, 0, 0);
            } else {
                w.c[s] = __builtin_amdgcn_raw_buffer_load_b8(rc[m], c, 0, 0);
                w.c[s] |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rc[m], c + 1, 0, 0) << 8;
            }
        }
    };

    const int steps = (K + kStep - 1) / kStep;
    for (int c0 = 0; c0 < count; c0 += 16 * kNT) {
        uint32_t xrow[kNT];
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            const int i = c0 + n * 16 + l16;
            xrow[n] = kNoRead;
            if (i < count) xrow[n] = (uint32_t)((kDown ? list[i] : list[i] / a.choices) * a.ld * 2) + g * 64;
        }
        f32x4 acc[kSets][kNT];
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
            for (int n = 0; n < kNT; ++n) acc[s][n] = f32x4{0, 0, 0, 0};
        auto load_inputs = [&](Inputs &x, int step) {
            const int k = step * kStep + g * 32;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t skip = k + i * 8 < K ? 0 : kNoRead;
#pragma unroll
                for (int n = 0; n < kNT; ++n)
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const uint32_t at = xrow[n] + (uint32_t)(step * kStep * 2 + i * 16 + p * K * 2);
                        x.x[n][p][i] = __builtin_amdgcn_raw_buffer_load_b128(rx, skip ? kNoRead : at, 0, 0);
                    }
            }
        };
        auto multiply = [&](const Weights &w, const Inputs &x) {
#pragma unroll
            for (int s = 0; s < kSets; ++s) {
                const int m = kDown ? 0 : s / kRT;
                const float l[2] = {scale_value(w.c[s] & 0x7F, e[m]), scale_value(w.c[s] >> 8 & 0x7F, e[m])};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bf16x8 fw = __builtin_bit_cast(bf16x8, stored_eight(w.p[s][i], l[i >> 1]));
#pragma unroll
                    for (int n = 0; n < kNT; ++n)
#pragma unroll
                        for (int p = 0; p < kParts; ++p)
                            acc[s][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                fw, __builtin_bit_cast(bf16x8, x.x[n][p][i]), acc[s][n], 0, 0, 0);
                }
            }
        };
        // Loads past the last step read nothing.
        Weights w[kDepth];
        if constexpr (kNT * kParts <= 2) {
            Inputs x[kDepth];
#pragma unroll
            for (int d = 0; d < kDepth; ++d) load_weights(w[d], wave + 4 * d), load_inputs(x[d], wave + 4 * d);
            for (int step = wave; step < steps; step += 4 * kDepth) {
#pragma unroll
                for (int d = 0; d < kDepth; ++d) {
                    multiply(w[d], x[d]);
                    load_weights(w[d], step + 4 * (d + kDepth));
                    load_inputs(x[d], step + 4 * (d + kDepth));
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) load_weights(w[d], wave + 4 * d);
            for (int step = wave; step < steps; step += 4 * kDepth) {
#pragma unroll
                for (int d = 0; d < kDepth; ++d) {
                    Inputs x;
                    load_inputs(x, step + 4 * d);
                    multiply(w[d], x);
                    load_weights(w[d], step + 4 * (d + kDepth));
                }
            }
        }

        // The four quarters of k, then out: a lane holds four consecutive rows of a slot.
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
                red[wave][s * kNT + n][lane] = make_float4(acc[s][n][0], acc[s][n][1], acc[s][n][2], acc[s][n][3]);
        __syncthreads();
        auto sum = [&](int unit) {
            float4 v = red[0][unit][lane];
#pragma unroll
            for (int q = 1; q < 4; ++q) {
                const float4 o = red[q][unit][lane];
                v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
            }
            return v;
        };
        constexpr int kUnits = (kDown ? kSets : kRT) * kNT;
        for (int u = wave; u < kUnits; u += 4) {
            const int tile = u / kNT, i = c0 + (u % kNT) * 16 + l16;
            const int row = tile * 16 + 4 * g;
            if (i >= count || row >= rows) continue;
            const int64_t slot = list[i];
            if constexpr (kDown) {
                const float4 v = sum(u);
                const float by = a.weight[slot];
                *reinterpret_cast<float4 *>(a.P + slot * a.rows + r0 + row) =
                    make_float4(v.x * f[0] * by, v.y * f[0] * by, v.z * f[0] * by, v.w * f[0] * by);
            } else {
                const float4 vg = sum(u), vu = sum(kRT * kNT + u);
                const float gate[4] = {vg.x * f[0], vg.y * f[0], vg.z * f[0], vg.w * f[0]};
                const float up[4] = {vu.x * f[1], vu.y * f[1], vu.z * f[1], vu.w * f[1]};
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float h = gate[q] / (1.0f + expf(-gate[q])) * up[q];
                    hi[q] = bf16_rne(h);
                    const float rest = h - bf16_value(hi[q]);
                    lo[q] = fabsf(rest) < INFINITY ? bf16_rne(rest) : 0;  // where h itself rounds to infinity
                }
                uint16_t *h = a.H + slot * 2 * a.rows + r0 + row;
                *reinterpret_cast<uint2 *>(h) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
                *reinterpret_cast<uint2 *>(h + a.rows) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
            }
        }
        __syncthreads();
    }
}

// Y[t] = the sum of the token's slots in their order; eight outputs a thread.
// A slot without an expert adds its weight times 0.
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ P, const int32_t *__restrict__ ids,
                                                   const float *__restrict__ weight, int choices, int experts,
                                                   int64_t out, uint16_t *__restrict__ Y, int64_t ldy, bool wide) {
    const int64_t t = blockIdx.y, m = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (m >= out) return;
    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int j = 0; j < choices; ++j) {
        const int64_t s = t * choices + j;
        if (expert_of(ids, experts, (int)s) == kNoExpert) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] += weight[s] * 0.0f;
            continue;
        }
        const float4 a = *reinterpret_cast<const float4 *>(P + s * out + m);
        const float4 b = *reinterpret_cast<const float4 *>(P + s * out + m + 4);
        y[0] += a.x, y[1] += a.y, y[2] += a.z, y[3] += a.w;
        y[4] += b.x, y[5] += b.y, y[6] += b.z, y[7] += b.w;
    }
    uint16_t *dst = Y + t * ldy + m;
    const u32x4 v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])};
    if (wide) {
        *reinterpret_cast<u32x4 *>(dst) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) dst[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int kPieceSlots = 4096;  // a call of more goes piece by piece

bool layer_sizes_ok(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k) {
    return tokens >= 0 && tokens <= kMaxTokens && in >= 0 && in % kGroup == 0 && in <= kMaxWidth && hidden >= 0 &&
           hidden % kGroup == 0 && hidden <= kMaxWidth && experts >= 1 && experts <= kMaxExperts && k >= 1 &&
           k <= kMaxChoices;
}

// Tokens of a piece: its rows of X and of h are addressed in 32 bits.
int64_t piece_tokens(int64_t hidden, int32_t k, int64_t ldx) {
    int64_t n = kPieceSlots / k;
    n = std::min(n, ((int64_t)1 << 29) / std::max<int64_t>(1, ldx));
    return std::max<int64_t>(1, std::min(n, ((int64_t)1 << 28) / (hidden * k)));
}

struct LayerSpace {
    size_t h, p, order, shares, total;
};

LayerSpace layer_space(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k) {
    const int64_t slots = std::min(tokens, piece_tokens(hidden, k, 1)) * k;
    LayerSpace s{};
    s.h = round_256((size_t)(slots * hidden * 4));
    s.p = round_256((size_t)(slots * in * 4));
    s.order = round_256((size_t)slots * 4);
    s.shares = round_256((size_t)(slots + experts) * sizeof(Share));
    s.total = s.h + s.p + s.order + s.shares;
    return s;
}

int check_matrix(const hscale_experts *w) {
    if (!w || !w->global_scale || !w->scale_codes || !w->packed_e2m1) return HSCALE_ERR_NULL;
    if (!aligned(w->global_scale, 4) || !aligned(w->packed_e2m1, 8)) return HSCALE_ERR_ALIGN;
    return HSCALE_OK;
}

Matrices matrices(const hscale_experts *w) { return Matrices{w->global_scale, w->scale_codes, w->packed_e2m1}; }

template <bool kDown, int kRT, int kNT>
void launch_experts(const ExpertArgs &a, int shares, bool even, hipStream_t stream) {
    const dim3 grid((unsigned)cdiv(a.rows, (kDown ? 32 : 16) * kRT), (unsigned)shares);
    if (even)
        hipLaunchKernelGGL((expert_kernel<kDown, kRT, kNT, true>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((expert_kernel<kDown, kRT, kNT, false>), grid, dim3(256), 0, stream, a);
}

template <bool kDown>
int experts_product(const ExpertArgs &a, int shares, int tiles, hipStream_t stream) {
    bool even = a.k % 32 == 0;
    for (int m = 0; m < (kDown ? 1 : 2); ++m) even = even && aligned(a.w[m].codes, 2);
    if (tiles == 1)
        launch_experts<kDown, 1, 1>(a, shares, even, stream);
    else if (tiles == 2)
        launch_experts<kDown, 1, 2>(a, shares, even, stream);
    else
        launch_experts<kDown, 2, 4>(a, shares, even, stream);
    return launch_status();
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
    const int64_t piece = piece_tokens(hidden, k, ldx);
    for (int64_t t0 = 0; t0 < tokens; t0 += piece) {
        const int64_t n = std::min(piece, tokens - t0);
        const int slots = (int)(n * k);
        const int32_t *ids = expert + t0 * k;
        // Columns of 16 slots: as many as an expert's share, on average, is likely to need.
        const int tiles = slots <= 2 * experts ? 1 : slots <= 16 * experts ? 2 : 4;
        int count = std::min(slots, (int)experts);
        const bool many = slots > kBlockSlots;
        if (many) {
            count = std::min(slots, slots / (16 * tiles) + (int)experts);
            hipLaunchKernelGGL(share_kernel, dim3(1), dim3(1024), 0, stream, ids, slots, (int)experts, 16 * tiles,
                               order, shares, count);
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
        a.slots = slots, a.choices = k, a.experts = experts;
        a.order = many ? order : nullptr;
        a.shares = many ? shares : nullptr;
        a.H = H;
        a.P = P;
        if (const int st = experts_product<false>(a, count, tiles, stream)) return st;
        a.w[0] = a.w[1] = matrices(down);
        a.rows = in, a.k = hidden;
        a.in = H;
        a.ld = 2 * hidden;
        a.in_bytes = (int64_t)slots * hidden * 4;
        if (const int st = experts_product<true>(a, count, tiles, stream)) return st;
        uint16_t *y = static_cast<uint16_t *>(Y) + t0 * ldy;
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)cdiv(in, 2048), (unsigned)n), dim3(256), 0, stream, P, ids,
                           a.weight, (int)k, (int)experts, in, y, ldy, aligned(y, 16) && ldy % 8 == 0);
        if (const int st = launch_status()) return st;
    }
    return HSCALE_OK;
}

}  // extern "C"
