// Host-side memory and undefined-behaviour check of the plans and argument
// validation behind the adapted layer and the token loss, built with
// -fsanitize=address,undefined for the host only.  Workspaces are asked for
// sizes from one to the limits and beyond; every other call fails validation
// or is empty, so nothing reaches the GPU.
#include <cstdint>
#include <cstdio>

#include "hscale.h"

static void *at(uint64_t a) { return reinterpret_cast<void *>(a); }

int main() {
    const int64_t sizes[] = {-1, 0, 1, 15, 16, 17, 64, 65, 1024, 1040, 4096, 14336, 1 << 20, 1 << 21, (1 << 21) + 16,
                             1 << 24, (1 << 24) + 1, INT64_MAX};
    const int32_t counts[] = {-1, 0, 1, 3, 4096, 4097, INT32_MAX}, ranks[] = {-8, 0, 8, 40, 256, 264, INT32_MAX};
    double total = 0.0;
    for (int64_t t : sizes)
        for (int64_t n : sizes)
            for (int64_t m : sizes) {
                total += (double)hscale_token_loss_workspace_bytes(t, n, m);
                total += (double)hscale_token_loss_grad_workspace_bytes(t, n, m);
                for (int32_t c : counts)
                    for (int32_t r : ranks) {
                        total += (double)hscale_adapted_linear_workspace_bytes(t, n, m, c, r);
                        total += (double)hscale_adapted_linear_grad_workspace_bytes(t, n, m, c, r);
                    }
            }
    int bad = total <= 0.0;

    const uint64_t A = 1ull << 40;  // addresses that no call reads
    const auto u8 = [&](int k) { return static_cast<uint8_t *>(at(k * A)); };
    const auto f32 = [&](int k) { return static_cast<float *>(at(k * A)); };
    const auto i64 = [&](int k) { return static_cast<int64_t *>(at(k * A)); };
    const auto i8 = [&](int k) { return static_cast<int8_t *>(at(k * A)); };
    hscale_adapters ad{3, 8, at(20 * A), at(21 * A), nullptr, static_cast<int32_t *>(at(22 * A))};
    const size_t most = SIZE_MAX;
    for (int64_t t : sizes)
        for (int64_t n : sizes)
            for (int64_t m : sizes) {
                // a workspace that is one byte off its alignment, or none
                bad |= hscale_adapted_linear(at(A), t, n, n, m, 1e-3f, u8(2), u8(3), &ad, at(4 * A), m, at(5 * A + 1),
                                             most, nullptr) == 0 && t > 0 && m > 0;
                bad |= hscale_adapted_linear_grad(at(A), t, m, m, i8(2), f32(3), n, 1e-3f, u8(4), u8(5), &ad,
                                                  at(6 * A), n, at(7 * A), at(8 * A), at(9 * A + 1), most, nullptr) == 0;
                bad |= hscale_token_loss(at(A), t, n, n, at(2 * A), m, i64(3), f32(4), f32(5), at(6 * A + 1), most,
                                         nullptr) == 0 && t > 0;
                if (t != 0)
                    bad |= hscale_token_loss_grad(at(A), t, n, n, at(2 * A), m, i64(3), f32(4), f32(5), at(6 * A), n,
                                                  at(7 * A), at(8 * A + 1), most, nullptr) == 0;
                bad |= hscale_pack_activations(at(A + 2), t, n, n, i8(2), f32(3), nullptr) == 0 && t > 0 && n > 0;
                bad |= hscale_unpack_activations(i8(2), f32(3), t, n, at(A + 1), n, nullptr) == 0 && t > 0 && n > 0;
            }
    for (int32_t c : counts)
        for (int32_t r : ranks) {
            ad.count = c, ad.rank = r;
            bad |= hscale_adapted_linear(at(A), 5, 64, 64, 7, 1e-3f, u8(2), u8(3), &ad, at(4 * A), 7, nullptr, 0,
                                         nullptr) == 0;
        }
    if (bad) return 1;
    std::puts("sanitize driver: ok");
    return 0;
}
