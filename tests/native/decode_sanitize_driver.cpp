// Host-side memory and undefined-behaviour check of the workspaces and argument
// validation behind routing, the layer of stored experts and the rules on
// logits, built with sanitizers for the host only.  Every call fails validation
// or is empty, so nothing reaches the GPU.
#include <cstdint>
#include <cstdio>

#include "hscale.h"

static void *at(uint64_t a) { return reinterpret_cast<void *>(a); }

int main() {
    const int64_t sizes[] = {-1, 0, 1, 15, 16, 17, 64, 1024, 4096, 14336, 1 << 20, 1 << 21, (1 << 21) + 16,
                             1 << 24, (1 << 24) + 1, INT64_MAX};
    const int32_t counts[] = {INT32_MIN, -1, 0, 1, 3, 32, 33, 1024, 1025, INT32_MAX};
    const uint64_t A = 1ull << 44;  // addresses that no call reads
    const auto u8 = [&](int k) { return static_cast<uint8_t *>(at(k * A)); };
    const auto f32 = [&](int k) { return static_cast<float *>(at(k * A)); };
    const auto i32 = [&](int k) { return static_cast<int32_t *>(at(k * A)); };
    const hscale_experts m{f32(7), u8(8), u8(9)};
    double total = 0.0;
    int bad = 0;
    for (int64_t t : sizes)
        for (int64_t n : sizes)
            for (int32_t e : counts)
                for (int32_t k : counts) {
                    for (int64_t h : sizes) {
                        total += (double)hscale_expert_layer_workspace_bytes(t, n, h, e, k);
                        bad |= hscale_expert_layer(at(A), t, n, n, h, e, &m, &m, &m, i32(2), f32(3), k, at(4 * A), n,
                                                   at(5 * A + 1), SIZE_MAX, nullptr) == 0 && t != 0;
                    }
                    bad |= hscale_route_tokens(at(A + 1), k == 3, t, e, n, k, 1, i32(2), f32(3), nullptr) == 0 && t != 0;
                }
    for (int64_t r : sizes)
        for (int64_t v : sizes)
            for (int64_t l : sizes)
                for (int32_t b : counts) {
                    const hscale_logit_rules rules{i32(10), l, l, i32(11), i32(12), f32(13), f32(14), f32(15), f32(16), b,
                                                   nullptr, reinterpret_cast<uint32_t *>(u8(17)), b, nullptr};
                    bad |= hscale_adjust_logits(&rules, at(A + 1), 1, r, v, v, at(2 * A), v, nullptr) == 0 && r != 0 && v != 0;
                }
    if (bad || total <= 0.0) return 1;
    std::printf("sanitize driver: ok\n");
    return 0;
}
