// Rotary positions for gfx950: every pair (a, b) of a head's first `rotary` elements is turned by the angle
// th = position * frequency and scaled by the magnitude m,
//     a' = m (a cos th - b sin th),   b' = m (a sin th + b cos th);
// the gradient is the same turn by -th (the turn's transpose), so one kernel serves both.  RetNet's queries and keys are
// turned like this in front of the recurrence of Sec. 5.1; with a relative angle per token the products q . k see only the
// distance between two tokens.
//
// A streaming pass: 3 flops an element.  The angles are made here instead of read from a table: a thread keeps its pairs'
// frequencies, and the cosines of a token serve all of its heads that the thread walks.  An angle is reduced to a quarter
// turn in fp64 (position * frequency / 2 pi minus its nearest multiple of 1/4: exact but for the product's rounding of
// 2^-53), so far positions cost no accuracy; sine and cosine of what is left, |x| <= pi/4, are their Taylor polynomials.
#include "sla_row_ops.h"

namespace sla {

namespace {

using namespace row_ops;

constexpr int kThreads = 256;
constexpr int kHeadsAhead = 4;  // heads whose loads a thread has in flight
constexpr int kMaxHeads = 1024, kMaxWidth = 512;

struct RotaryArgs {
    const void *q, *k;
    void *qo, *ko;
    const double* freq;
    const int32_t *positions, *cu;
    int B, T, Hq, Hk, d, r;
    int pieces;       // threads that share one head of a token
    int head_lanes;   // heads of a token that are worked on at the same time
    int tokens;       // tokens of a workgroup
    int per_token;    // positions: one per token, else one per sequence
    int head_major;
    float magnitude;
    float sign;       // -1: turn back
};

// cos and sin of 2 pi t, times the magnitude
__device__ __forceinline__ void turn(double t, float m, float sign, float& c, float& s) {
    const double q = __builtin_rint(4.0 * t);
    const float x = (float)__builtin_fma(-0.25, q, t) * 6.28318530717958648f, z = x * x;
    const int k = (int)q;
    const float sp = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
    const float cp = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
    const float cc = (k & 1) ? sp : cp, ss = (k & 1) ? cp : sp;
    c = m * (((k + 1) & 2) ? -cc : cc);
    s = m * sign * ((k & 2) ? -ss : ss);
}

__device__ __forceinline__ float load1(const void* x, size_t off, bool bf16) {
    return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)x)[off] << 16) : ((const float*)x)[off];
}
__device__ __forceinline__ void store1(void* y, size_t off, float f, bool bf16) {
    if (bf16) {
        ((uint16_t*)y)[off] = __builtin_bit_cast(uint16_t, (__bf16)f);
    } else {
        ((float*)y)[off] = f;
    }
}

// The sequence that token n of a packed batch lies in: the last b with cu[b] <= n.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int64_t n) {
    int lo = 0, hi = B;  // cu[lo] <= n < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= n) lo = mid; else hi = mid;
    }
    return lo;
}

// ADJ: pairs (2i, 2i+1), a thread turns the four pairs of eight adjacent elements.  Otherwise pairs (i, i + r/2), a thread
// turns V of them: eight where r/2 is a multiple of eight, so that both halves are read 16 bytes at a time, else one (2-byte
// accesses, 64 adjacent ones a wave).  Elements from r on are copied, V (or eight) at a time; in place they stay.
template <bool BF16, bool ADJ, int V>
__global__ __launch_bounds__(512) void sla_rotary_kernel(RotaryArgs a) {
    constexpr int P = ADJ ? 4 : V;  // pairs of a thread
    const int turned = ADJ ? (a.r + 7) / 8 : a.r / 2 / V;
    int tl, hl, c;
    {
        const int x = threadIdx.x / a.pieces;
        c = threadIdx.x - x * a.pieces;
        if (a.head_major) {  // adjacent threads on adjacent tokens of a head
            hl = x / a.tokens;
            tl = x - hl * a.tokens;
        } else {
            tl = x / a.head_lanes;
            hl = x - tl * a.head_lanes;
        }
    }
    if (tl >= a.tokens || hl >= a.head_lanes) return;
    const bool turns = c < turned;
    const int off0 = ADJ ? 8 * c : (turns ? V * c : a.r + V * (c - turned)), off1 = a.r / 2 + off0;
    double f[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = P * c + i;
        f[i] = turns && p < a.r / 2 ? a.freq[p] * 0.15915494309189533577 : 0.0;
    }
    int64_t first, end;
    token_range(a.cu, a.B, a.cu ? (int64_t)a.T : (int64_t)a.B * a.T, first, end);
    const int heads = a.Hq + a.Hk;
    for (int64_t n = first + (int64_t)blockIdx.x * a.tokens + tl; n < end; n += (int64_t)gridDim.x * a.tokens) {
        int64_t b, t;
        if (a.cu) {
            b = sequence_of(a.cu, a.B, n);
            t = n - a.cu[b];
        } else {
            b = (uint32_t)n / (uint32_t)a.T;
            t = n - b * a.T;
        }
        double pos;
        if (a.per_token)
            pos = a.positions[n];
        else
            pos = (double)(t + (a.positions ? a.positions[b] : 0));
        float cs[P], sn[P];
#pragma unroll
        for (int i = 0; i < P; ++i) turn(pos * f[i], a.magnitude, a.sign, cs[i], sn[i]);
        for (int h0 = hl; h0 < heads; h0 += a.head_lanes * kHeadsAhead) {
            float x[kHeadsAhead][8], y[kHeadsAhead][8];
            const void* src[kHeadsAhead];
            void* dst[kHeadsAhead];
            size_t row[kHeadsAhead];
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                const int h = h0 + u * a.head_lanes;
                if (h >= heads) break;
                const bool isk = h >= a.Hq;
                const int H = isk ? a.Hk : a.Hq, hh = isk ? h - a.Hq : h;
                src[u] = isk ? a.k : a.q;
                dst[u] = isk ? a.ko : a.qo;
                row[u] = (a.head_major ? ((size_t)b * H + hh) * a.T + t : (size_t)n * H + hh) * a.d;
                if constexpr (ADJ || V == 8) {
                    load8<BF16>(src[u], row[u] + off0, x[u]);
                    if (!ADJ && turns) load8<BF16>(src[u], row[u] + off1, y[u]);
                } else {
                    x[u][0] = load1(src[u], row[u] + off0, BF16);
                    if (turns) y[u][0] = load1(src[u], row[u] + off1, BF16);
                }
            }
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                if (h0 + u * a.head_lanes >= heads) break;
                if constexpr (ADJ) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = x[u][2 * i], o = x[u][2 * i + 1];
                        const bool in = 4 * c + i < a.r / 2;
                        x[u][2 * i] = in ? e * cs[i] - o * sn[i] : e;
                        x[u][2 * i + 1] = in ? e * sn[i] + o * cs[i] : o;
                    }
                    store8<BF16>(dst[u], row[u] + off0, x[u]);
                } else {
                    if (turns) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float e = x[u][i], o = y[u][i];
                            x[u][i] = e * cs[i] - o * sn[i];
                            y[u][i] = e * sn[i] + o * cs[i];
                        }
                    }
                    if constexpr (V == 8) {
                        store8<BF16>(dst[u], row[u] + off0, x[u]);
                        if (turns) store8<BF16>(dst[u], row[u] + off1, y[u]);
                    } else {
                        store1(dst[u], row[u] + off0, x[u][0], BF16);
                        if (turns) store1(dst[u], row[u] + off1, y[u][0], BF16);
                    }
                }
            }
        }
    }
}

int check_rotary(const sla_rotary_params* p, const void* q, const void* k, const double* freq, const int32_t* positions,
                 const int32_t* cu, const void* qo, const void* ko) {
    if (!p) return SLA_ERR_NULL;
    if (p->dtype != SLA_F32 && p->dtype != SLA_BF16) return SLA_ERR_UNSUPPORTED;
    if (p->flags & ~(SLA_FLAG_HEAD_MAJOR | SLA_FLAG_ADJACENT_PAIRS | SLA_FLAG_TOKEN_POSITIONS)) return SLA_ERR_UNSUPPORTED;
    if (p->B < 0 || p->T < 0 || p->Hq < 1 || p->Hk < 0 || p->Hq > kMaxHeads || p->Hk > kMaxHeads) return SLA_ERR_SHAPE;
    if (p->d < 8 || p->d > kMaxWidth || (p->d & 7) || p->rotary < 2 || p->rotary > p->d || (p->rotary & 1)) return SLA_ERR_SHAPE;
    if ((cu ? (int64_t)p->T : (int64_t)p->B * p->T) > (int64_t)1 << 30) return SLA_ERR_SHAPE;
    if (cu && (p->flags & SLA_FLAG_HEAD_MAJOR)) return SLA_ERR_UNSUPPORTED;  // packed batches are [T,H,d]
    if ((p->flags & SLA_FLAG_TOKEN_POSITIONS) && !positions && p->B > 0 && p->T > 0) return SLA_ERR_NULL;
    if ((p->Hk > 0) != (k != nullptr) && p->B > 0 && p->T > 0) return SLA_ERR_NULL;
    if ((k != nullptr) != (ko != nullptr)) return SLA_ERR_NULL;
    if (p->B > 0 && p->T > 0 && (!q || !qo || !freq)) return SLA_ERR_NULL;
    const void* ptrs[] = {q, k, qo, ko};
    for (const void* x : ptrs)
        if (!aligned(x, 16)) return SLA_ERR_ALIGN;
    if (!aligned(freq, 8) || !aligned(positions, 4) || !aligned(cu, 4)) return SLA_ERR_ALIGN;
    return SLA_OK;
}

int rotary(const sla_rotary_params* p, const void* q, const void* k, const double* freq, const int32_t* positions,
           const int32_t* cu, void* qo, void* ko, float sign, hipStream_t stream) {
    const int rc = check_rotary(p, q, k, freq, positions, cu, qo, ko);
    if (rc != SLA_OK) return rc;
    if (p->B == 0 || p->T == 0) return SLA_OK;
    const bool adj = p->flags & SLA_FLAG_ADJACENT_PAIRS;
    const bool wide = adj || p->rotary % 16 == 0;
    RotaryArgs a{q, k, qo, ko, freq, positions, cu, p->B, p->T, p->Hq, p->Hk, p->d, p->rotary};
    a.per_token = (p->flags & SLA_FLAG_TOKEN_POSITIONS) != 0;
    a.head_major = (p->flags & SLA_FLAG_HEAD_MAJOR) != 0;
    a.magnitude = p->magnitude;
    a.sign = sign;
    a.pieces = adj ? p->d / 8 : (wide ? p->rotary / 16 + (p->d - p->rotary) / 8 : p->d - p->rotary / 2);
    const int64_t tokens = cu ? p->T : (int64_t)p->B * p->T;
    const int heads = p->Hq + p->Hk;
    const int threads = a.pieces > kThreads ? 512 : kThreads;
    int each = kHeadsAhead;  // heads a thread walks: fewer while that leaves compute units without work
    while (each > 1 && tokens * a.pieces * ((heads + each - 1) / each) < (int64_t)kComputeUnits * 512) each /= 2;
    a.head_lanes = (heads + each - 1) / each;
    if (a.head_lanes * a.pieces > threads) a.head_lanes = threads / a.pieces;
    a.tokens = threads / (a.head_lanes * a.pieces);
    const int64_t blocks = (tokens + a.tokens - 1) / a.tokens;
    const dim3 grid((unsigned)(blocks < kComputeUnits * 64 ? blocks : kComputeUnits * 64));
#define SLA_ROT(BF, ADJ, V) hipLaunchKernelGGL((sla_rotary_kernel<BF, ADJ, V>), grid, dim3(threads), 0, stream, a)
    if (p->dtype == SLA_BF16) {
        if (adj) SLA_ROT(true, true, 8); else if (wide) SLA_ROT(true, false, 8); else SLA_ROT(true, false, 1);
    } else {
        if (adj) SLA_ROT(false, true, 8); else if (wide) SLA_ROT(false, false, 8); else SLA_ROT(false, false, 1);
    }
#undef SLA_ROT
    return hipGetLastError() == hipSuccess ? SLA_OK : SLA_ERR_HIP;
}

}  // namespace

}  // namespace sla

extern "C" {

int sla_rotary(const sla_rotary_params* p, const void* q, const void* k, const double* frequencies,
               const int32_t* positions, const int32_t* cu_seqlens, void* q_out, void* k_out, void* stream) {
    return sla::rotary(p, q, k, frequencies, positions, cu_seqlens, q_out, k_out, 1.f, (hipStream_t)stream);
}

int sla_rotary_backward(const sla_rotary_params* p, const void* dq_out, const void* dk_out, const double* frequencies,
                        const int32_t* positions, const int32_t* cu_seqlens, void* dq, void* dk, void* stream) {
    return sla::rotary(p, dq_out, dk_out, frequencies, positions, cu_seqlens, dq, dk, -1.f, (hipStream_t)stream);
}

}  // extern "C"
