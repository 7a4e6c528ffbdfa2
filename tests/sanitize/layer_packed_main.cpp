// Driver for the sanitizer build of the host code of the operators around the mixer on packed batches: sizes of workspaces and
// refusals for few and many sequences.  This program runs where there is no GPU: a valid call ends at its launch with SLA_ERR_HIP.
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
    for (int T : {0, 1, 7, 4096, 1 << 20, 1 << 30, (1 << 30) + 1, 2147483647})
        for (int B : {0, 1, 1024, 1025, 1 << 17, 2147483647})
            for (int d : {8, 40, 128, 512, 8200, 16384}) {
                const bool fits = T <= 1 << 30, work = B > 0 && T > 0;
                sla_join_norm_params j{SLA_BF16, SLA_F32, B, T, d, 0.5f, 1e-5f};
                const size_t n = sla_join_norm_backward_workspace_bytes(&j, 1);
                expect((n > 0) == (fits && work), "join_norm workspace", T, B, d);
                const int rj = sla_join_norm_backward(&j, A, A, F, F, F, A, A, I, A, A, G, G, G, A, n, nullptr);
                expect(fits ? reached(rj) : rj == SLA_ERR_SHAPE, "join_norm backward", T, B, d);
                if (n)
                    expect(sla_join_norm_backward(&j, A, A, F, F, F, A, A, I, A, A, G, G, G, A, n - 1, nullptr) == SLA_ERR_WORKSPACE,
                           "join_norm workspace too small", T, B, d);
                if (d > 512) continue;
                sla_rotary_params r{SLA_BF16, B, T, 4, 1, d, 2, 0, 1.f};
                const int rr = sla_rotary(&r, A, A, (const double*)A, nullptr, I, A, A, nullptr);
                expect(fits ? reached(rr) : rr == SLA_ERR_SHAPE, "rotary", T, B, d);
                for (int flags : {0, SLA_FLAG_HEAD_WEIGHTS}) {
                    sla_norm_gate_params p{SLA_F32, B, T, 4, d, SLA_GATE_SILU, flags, 1e-5f};
                    const size_t m = sla_norm_gate_backward_workspace_bytes(&p, 1);
                    expect((m > 0) == (fits && work), "norm_gate workspace", T, B, d);
                    const int rg = sla_norm_gate_backward(&p, A, A, F, A, I, A, A, G, A, m, nullptr);
                    expect(fits ? reached(rg) : rg == SLA_ERR_SHAPE, "norm_gate backward", T, B, d);
                    if (m)
                        expect(sla_norm_gate_backward(&p, A, A, F, A, I, A, A, G, A, m - 1, nullptr) == SLA_ERR_WORKSPACE,
                               "norm_gate workspace too small", T, B, d);
                }
            }
    std::printf("%d failures\n", failures);
    return failures != 0;
}
