// Driver for the sanitizer build of the host code of the operators around the mixer: their checks, workspace sizes and launch
// plans over a grid of sizes.  This program runs where there is no GPU: a valid call ends at its launch with SLA_ERR_HIP.
#include <cstdio>

#include "sla.h"

static int failures = 0;
static void expect(bool ok, const char* what, int a, int b, int c) {
    if (!ok) {
        ++failures;
        std::printf("%s (%d, %d, %d)\n", what, a, b, c);
    }
}

int main() {
    void* A = (void*)(uintptr_t)(1 << 20);
    const float* F = (const float*)A;
    float* G = (float*)A;
    const int32_t* I = (const int32_t*)A;
    auto reached = [](int rc) { return rc == SLA_OK || rc == SLA_ERR_HIP; };
    const int sizes[] = {0, 1, 2, 7, 64, 1000, 16384, 1 << 20, 1 << 29};
    for (int T : sizes)
        for (int B : {0, 1, 3})
            for (int d = -8; d <= 520; d += 8) {
                const bool fits = (int64_t)B * T <= (int64_t)1 << 30;
                for (int heads : {1, 3, 16, 1024}) {
                    for (int rot : {0, 2, 30, 32, d - 2, d, d + 2})
                        for (int flags : {0, SLA_FLAG_HEAD_MAJOR, SLA_FLAG_ADJACENT_PAIRS}) {
                            sla_rotary_params p{SLA_BF16, B, T, heads, 1, d, rot, flags, 1.f};
                            const int rc = sla_rotary(&p, A, A, (const double*)A, nullptr, nullptr, A, A, nullptr);
                            const bool ok = fits && d >= 8 && d <= 512 && rot >= 2 && rot <= d;
                            expect(ok ? reached(rc) : rc == SLA_ERR_SHAPE, "rotary", T, d, rot);
                        }
                    for (int flags : {0, SLA_FLAG_HEAD_WEIGHTS}) {
                        sla_norm_gate_params p{SLA_F32, B, T, heads, d, SLA_GATE_SILU, flags, 1e-5f};
                        const bool ok = fits && d >= 8 && d <= 512;
                        const int rc = sla_norm_gate(&p, A, A, F, nullptr, A, nullptr);
                        expect(ok ? reached(rc) : rc == SLA_ERR_SHAPE, "norm_gate", T, d, heads);
                        const size_t n = sla_norm_gate_backward_workspace_bytes(&p, 0);
                        expect((n > 0) == (ok && B > 0 && T > 0), "norm_gate workspace", T, d, heads);
                        const int rb = sla_norm_gate_backward(&p, A, A, F, A, nullptr, A, A, G, A, n, nullptr);
                        expect(ok ? reached(rb) : rb == SLA_ERR_SHAPE, "norm_gate backward", T, d, heads);
                        if (n)
                            expect(sla_norm_gate_backward(&p, A, A, F, A, nullptr, A, A, G, A, n - 1, nullptr) == SLA_ERR_WORKSPACE,
                                   "norm_gate workspace too small", T, d, heads);
                    }
                }
                for (int D : {d, 31 * d}) {
                    sla_join_norm_params p{SLA_BF16, SLA_F32, B, T, D, 0.5f, 1e-5f};
                    const bool ok = fits && D >= 8 && D <= 16384;
                    const int rc = sla_join_norm(&p, A, A, F, F, F, I, A, A, nullptr);
                    expect(D >= 8 && D <= 16384 ? reached(rc) : rc == SLA_ERR_SHAPE, "join_norm packed", T, D, B);
                    const size_t n = sla_join_norm_backward_workspace_bytes(&p, 0);
                    expect((n > 0) == (ok && B > 0 && T > 0), "join_norm workspace", T, D, B);
                    const int rb = sla_join_norm_backward(&p, A, A, F, F, F, A, A, nullptr, A, A, G, G, G, A, n, nullptr);
                    expect(ok ? reached(rb) : rb == SLA_ERR_SHAPE, "join_norm backward", T, D, B);
                }
            }
    std::printf("%d failures\n", failures);
    return failures != 0;
}
