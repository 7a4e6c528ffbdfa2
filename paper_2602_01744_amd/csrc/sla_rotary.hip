// Rotary positions for gfx950: every pair (a, b) of a head's first `rotary` elements is turned by the angle
// th = position * frequency and scaled by the magnitude m,
//     a' = m (a cos th - b sin th),   b' = m (a sin th + b cos th);
// the gradient is the same turn by -th (the turn's transpose), so one kernel serves both.  RetNet's queries and keys are
// turned like this in front of the recurrence of Sec. 5.1; with a relative angle per token the products q . k see only the
// distance between two tokens.
//
// A streaming pass of 3 flops an element, bound by memory.  Measured in bf16 (a large copy reaches 5.4 TB/s, more where the
// last-level cache holds part of it): B=8 T=2048 16+16 heads of 128, 268 MB, 45 us; T=65536 32+32 heads, 2.1 GB, 397 us.
//
// The angles are made here instead of read from a table: a thread keeps its pairs' frequencies, and the cosines of a token
// serve all of its heads that the thread walks.  An angle is reduced to a quarter turn in fp64 (position * frequency / 2 pi
// minus its nearest multiple of 1/4: exact but for the product's rounding of 2^-53), so far positions cost no accuracy; sine
// and cosine of what is left, |x| <= pi/4, are their Taylor polynomials.
#include "sla_row_ops.h"

namespace sla {

namespace {

using namespace row_ops;

constexpr int kThreads = 256;    // a head takes at most 73 of them
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
// turns eight of them, or copies eight of the elements from r on.  ODD: r/2 is no multiple of eight, so the second half and what
// is copied begin anywhere, and the last pairs and elements that make no eight have a thread each (bf16, B=4 T=2048 16+16 heads
// of 128 with 100 elements turned: 30.6 us, 134 MB; a thread for every pair, 2 bytes at a time: 61 us).
template <bool BF16, bool ADJ, bool ODD>
__global__ __launch_bounds__(kThreads) void sla_rotary_kernel(RotaryArgs a) {
    constexpr int P = ADJ ? 4 : 8;  // pairs of a thread
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
    // the thread's first element, its pairs (0: it copies), and whether it has a single pair or element
    int off, pairs;
    bool single = false;
    if (ADJ) {
        off = 8 * c;
        pairs = a.r / 2 - 4 * c;
        pairs = pairs < 0 ? 0 : (pairs > 4 ? 4 : pairs);
    } else {
        const int half = a.r / 2, rest = a.d - a.r, wide = half / 8, wide_copies = rest / 8;
        int q = c;
        if (q < wide) {
            off = 8 * q;
            pairs = 8;
        } else if ((q -= wide) < wide_copies) {
            off = a.r + 8 * q;
            pairs = 0;
        } else if ((q -= wide_copies) < half % 8) {
            off = 8 * wide + q;
            pairs = 1;
            single = true;
        } else {
            off = a.r + 8 * wide_copies + q - half % 8;
            pairs = 0;
            single = true;
        }
    }
    const int off1 = off + a.r / 2;
    double f[P];
#pragma unroll
    for (int i = 0; i < P; ++i) f[i] = i < pairs ? a.freq[(ADJ ? 4 * c : off) + i] * 0.15915494309189533577 : 0.0;
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
            Raw8<BF16> rx[kHeadsAhead], ry[kHeadsAhead];
            float x1[kHeadsAhead], y1[kHeadsAhead];
            auto at = [&](int u, const void* q, const void* k, const void*& base) {  // the head's row in q or k
                const int h = h0 + u * a.head_lanes;
                const bool isk = h >= a.Hq;
                const int H = isk ? a.Hk : a.Hq, hh = isk ? h - a.Hq : h;
                base = isk ? k : q;
                return (a.head_major ? ((size_t)b * H + hh) * a.T + t : (size_t)n * H + hh) * a.d;
            };
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                if (h0 + u * a.head_lanes >= heads) break;
                const void* src;
                const size_t row = at(u, a.q, a.k, src);
                if (ODD && single) {
                    x1[u] = load1(src, row + off, BF16);
                    if (pairs) y1[u] = load1(src, row + off1, BF16);
                } else if constexpr (ODD) {
                    fetch8_anywhere(src, row + off, rx[u]);
                    if (pairs) fetch8_anywhere(src, row + off1, ry[u]);
                } else {
                    fetch8(src, row + off, rx[u]);
                    if (!ADJ && pairs) fetch8(src, row + off1, ry[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                if (h0 + u * a.head_lanes >= heads) break;
                const void* to;
                const size_t row = at(u, a.qo, a.ko, to);
                void* dst = const_cast<void*>(to);
                if (ODD && single) {
                    const float e = x1[u], o = y1[u];
                    store1(dst, row + off, pairs ? e * cs[0] - o * sn[0] : e, BF16);
                    if (pairs) store1(dst, row + off1, e * sn[0] + o * cs[0], BF16);
                    continue;
                }
                float x[8], y[8];
                unpack8(rx[u], x);
                if constexpr (ADJ) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = x[2 * i], o = x[2 * i + 1];
                        x[2 * i] = i < pairs ? e * cs[i] - o * sn[i] : e;
                        x[2 * i + 1] = i < pairs ? e * sn[i] + o * cs[i] : o;
                    }
                    store8<BF16>(dst, row + off, x);
                } else {
                    if (pairs) {
                        unpack8(ry[u], y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float e = x[i], o = y[i];
                            x[i] = e * cs[i] - o * sn[i];
                            y[i] = e * sn[i] + o * cs[i];
                        }
                    }
                    if constexpr (ODD) {
                        store8_anywhere<BF16>(dst, row + off, x);
                        if (pairs) store8_anywhere<BF16>(dst, row + off1, y);
                    } else {
                        store8<BF16>(dst, row + off, x);
                        if (pairs) store8<BF16>(dst, row + off1, y);
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
    const int half = p->rotary / 2, rest = p->d - p->rotary;
    const bool odd = !adj && half % 8 != 0;
    RotaryArgs a{q, k, qo, ko, freq, positions, cu, p->B, p->T, p->Hq, p->Hk, p->d, p->rotary};
    a.per_token = (p->flags & SLA_FLAG_TOKEN_POSITIONS) != 0;
    a.head_major = (p->flags & SLA_FLAG_HEAD_MAJOR) != 0;
    a.magnitude = p->magnitude;
    a.sign = sign;
    a.pieces = adj ? p->d / 8 : half / 8 + rest / 8 + half % 8 + rest % 8;  
    const int64_t tokens = cu ? p->T : (int64_t)p->B * p->T;
    const int heads = p->Hq + p->Hk;
    // Heads a thread walks: their turns share one set of angles.  bf16, B=8 T=2048 16+16 heads of 128: 2, 4, 8, 16, 32 heads
    // 57.1, 48.0, 45.3, 55.0, 55.1 us, head-major 64.4, 51.1, 46.9, 44.9, 45.0 us; B=4 T=4096 32+4 heads 85.5, 56.1, 54.1,
    // 55.1, 59.4 us.  Fewer while that leaves less than two waves a SIMD.
    int each = 8;
    while (each > 1 && tokens * a.pieces * ((heads + each - 1) / each) < (int64_t)kComputeUnits * 512) each /= 2;
    a.head_lanes = (heads + each - 1) / each;
    if (a.head_lanes * a.pieces > kThreads) a.head_lanes = kThreads / a.pieces;
    a.tokens = kThreads / (a.head_lanes * a.pieces);
    const int64_t blocks = (tokens + a.tokens - 1) / a.tokens;
    const dim3 grid((unsigned)(blocks < kComputeUnits * 64 ? blocks : kComputeUnits * 64));
#define SLA_ROT(BF, ADJ, ODD) hipLaunchKernelGGL((sla_rotary_kernel<BF, ADJ, ODD>), grid, dim3(kThreads), 0, stream, a)
    if (p->dtype == SLA_BF16) {
        if (adj) SLA_ROT(true, true, false); else if (odd) SLA_ROT(true, false, true); else SLA_ROT(true, false, false);
    } else {
        if (adj) SLA_ROT(false, true, false); else if (odd) SLA_ROT(false, false, true); else SLA_ROT(false, false, false);
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
