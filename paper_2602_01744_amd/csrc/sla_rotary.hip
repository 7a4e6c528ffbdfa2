// Rotary positions for gfx950: every pair (a, b) of a head's first `rotary` elements is turned by the angle
// th = position * frequency and scaled by the magnitude m,
//     a' = m (a cos th - b sin th),   b' = m (a sin th + b cos th);
// the gradient is the same turn by -th (the turn's transpose), so one kernel serves both.  RetNet's queries and keys are
// turned like this in front of the recurrence of Sec. 5.1; with a relative angle per token the products q . k see only the
// distance between two tokens.
//
// A streaming pass of 3 flops an element, bound by memory.  Measured in bf16 (a large copy reaches 5.4 TB/s, more where the
// last-level cache holds part of it): B=8 T=2048 16+16 heads of 128, 268 MB, 45 us; T=65536 32+32 heads, 2.1 GB, 378 us.
//
// The angles are made here instead of read from a table: a lane forms one to four of a token's, and every head of the token
// that the wave walks takes them.  An angle is reduced to a quarter turn in fp64: position * frequency / 2 pi minus its
// nearest multiple of 1/4, a difference that is exact; 1 / 2 pi and the two products are rounded by 2^-53 each, so the angle is off
// by less than 2^-51 of itself, under fp32's 2^-24 up to 2^27 radians.  Sine and cosine of what is left, |x| <= pi/4, are their
// Taylor polynomials of degree 9 and 10, off by less than 2.5e-9 and 2e-10 of them.
#include "sla_row_ops.h"

namespace sla {

namespace {

using namespace row_ops;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kHeadsAhead = 4;  // heads whose loads a lane has in flight
constexpr int kMaxHeads = 1024, kMaxWidth = 512;

enum { kAdjacent, kHalves, kHalvesAnywhere };

struct RotaryArgs {
    const void *q, *k;
    void *qo, *ko;
    const double* freq;
    const int32_t *positions, *cu;
    int B, T, Hq, Hk, d, r;
    int pieces;       // lanes of a head, eight elements each
    int wave_heads;   // heads and tokens that a wave works on at a time
    int wave_tokens;
    int groups;       // waves that share a token's heads
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

// The sequence that token n of a packed batch lies in: the last b with cu[b] <= n.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int64_t n) {
    int lo = 0, hi = B;  // cu[lo] <= n < cu[hi]
    while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);  // the sum of two ends may pass 2^31
        if (cu[mid] <= n) lo = mid; else hi = mid;
    }
    return lo;
}

// A wave's LDS accesses are carried out in their order; this keeps the compiler from changing it.
__device__ __forceinline__ void order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// A lane holds eight adjacent elements of a head, so that all of memory moves in aligned pieces of 16 bytes.  kAdjacent: its
// four pairs (2i, 2i+1).  kHalves: pairs (i, i + r/2); an element's partner lies r/2 further or back in the row, which the wave
// passes through LDS; r/2 a multiple of eight, so that a lane's partners are one piece, or else (kHalvesAnywhere) eight elements
// that may begin anywhere and belong to both halves (100 of 128 elements turned, B=4 T=2048 16+16 heads, 134 MB, cold: 24 us;
// lanes that read both elements of their pairs from memory, wherever they lie: 45 us, and 26 for the 24.7 us of aligned
// halves).  The lanes on a token form its angles together, each at most four (one where
// four heads or more are worked on at a time), and read their own from LDS.
template <bool BF16, int MODE>
__global__ __launch_bounds__(kThreads) void sla_rotary_kernel(RotaryArgs a) {
    constexpr int U = kHeadsAhead, P = MODE == kAdjacent ? 4 : 8;  // P: angles that a lane applies
    // the angles of a wave's tokens: at most 64 / pieces tokens of at most 4 pieces + 4 places
    __shared__ __align__(16) float2 angles[kWaves][512];
    __shared__ __align__(16) unsigned char exchange[MODE == kAdjacent ? 16 : kWaves * U * 64 * 8 * (BF16 ? 2 : 4)];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int slot = lane / a.pieces, c = lane - slot * a.pieces;
    const int ts = slot / a.wave_heads, hs = slot - ts * a.wave_heads;
    const int w = blockIdx.x * kWaves + wv, tile = w / a.groups, grp = w - tile * a.groups;
    const int tiles = gridDim.x * kWaves / a.groups;  // whole ones; the last waves of the grid may make no more
    if (ts >= a.wave_tokens || tile >= tiles) return;
    const int half = a.r / 2, sharers = a.wave_heads * a.pieces, self = hs * a.pieces + c;
    float2* const mine = angles[wv] + ts * ((half + 7) & ~7);
    double f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = self + i * sharers < half ? a.freq[self + i * sharers] * 0.15915494309189533577 : 0.0;
    int pair[P], partner[MODE == kHalvesAnywhere ? 8 : 1];
    float side[P];  // which of its pair an element is: -1 the first, 1 the second, 0 of no pair (kAdjacent: 1 or 0)
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (MODE == kAdjacent) {
            pair[i] = 4 * c + i;
            side[i] = pair[i] < half ? 1.f : 0.f;
        } else {
            const int e = 8 * c + i;
            side[i] = e < half ? -1.f : e < a.r ? 1.f : 0.f;
            pair[i] = e < half ? e : e - half;
            if (MODE == kHalvesAnywhere) partner[i] = e < half ? e + half : e < a.r ? e - half : e;
        }
        if (side[i] == 0.f) pair[i] = MODE == kHalves ? i : 0;
    }
    if (MODE == kHalves) partner[0] = 8 * c < half ? 8 * c + half : 8 * c < a.r ? 8 * c - half : 8 * c;
    int64_t first, end;
    token_range(a.cu, a.B, a.cu ? (int64_t)a.T : (int64_t)a.B * a.T, first, end);
    const int heads = a.Hq + a.Hk, next = a.wave_heads * a.groups;
    const int64_t step = (int64_t)tiles * a.wave_tokens;
    for (int64_t n = first + (int64_t)tile * a.wave_tokens + ts; n < end; n += step) {
        int64_t b = 0, t = 0;
        if (!a.cu) {
            b = (uint32_t)n / (uint32_t)a.T;
            t = n - b * a.T;
        } else if (!a.per_token) {
            b = sequence_of(a.cu, a.B, n);
            t = n - (a.cu[b] > 0 ? a.cu[b] : 0);  // a start in front of the tensors is their first token
        }
        double pos;
        if (a.per_token)
            pos = a.positions[n];
        else
            pos = (double)(t + (a.positions ? a.positions[b] : 0));
        order();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i * sharers >= half) break;
            float co, si;
            turn(pos * f[i], a.magnitude, a.sign, co, si);
            if (self + i * sharers < half) mine[self + i * sharers] = float2{co, si};
        }
        order();
        float cs[P], sn[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float2 v = mine[MODE == kHalvesAnywhere ? pair[i] : pair[0] + i];
            cs[i] = v.x;
            sn[i] = MODE == kAdjacent ? v.y : v.y * side[i];
        }
        for (int h0 = grp * a.wave_heads + hs; h0 < heads; h0 += next * U) {
            Raw8<BF16> r[U];
            auto at = [&](int u, const void* q, const void* k, const void*& base) {  // the head's row in q or k
                const int h = h0 + u * next;
                const bool isk = h >= a.Hq;
                const int H = isk ? a.Hk : a.Hq, hh = isk ? h - a.Hq : h;
                base = isk ? k : q;
                return (a.head_major ? ((size_t)b * H + hh) * a.T + t : (size_t)n * H + hh) * a.d + 8 * c;
            };
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h0 + u * next >= heads) break;
                const void* src;
                const size_t off = at(u, a.q, a.k, src);
                fetch8(src, off, r[u]);
            }
            if (MODE != kAdjacent) {
                order();
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (h0 + u * next < heads) put8(exchange, ((wv * U + u) * 64 + lane) * 8, r[u]);
                order();
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h0 + u * next >= heads) break;
                const void* to;
                const size_t off = at(u, a.qo, a.ko, to);
                float x[8];
                unpack8(r[u], x);
                if constexpr (MODE == kAdjacent) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = x[2 * i], o = x[2 * i + 1];
                        x[2 * i] = side[i] != 0.f ? e * cs[i] - o * sn[i] : e;
                        x[2 * i + 1] = side[i] != 0.f ? e * sn[i] + o * cs[i] : o;
                    }
                } else {
                    const int row = ((wv * U + u) * 64 + slot * a.pieces) * 8;
                    float y[8];
                    if constexpr (MODE == kHalves) {
                        load8<BF16>(exchange, row + partner[0], y);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            y[i] = BF16 ? __uint_as_float((uint32_t)((const uint16_t*)exchange)[row + partner[i]] << 16)
                                        : ((const float*)exchange)[row + partner[i]];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = side[i] != 0.f ? x[i] * cs[i] + y[i] * sn[i] : x[i];
                }
                store8<BF16>(const_cast<void*>(to), off, x);
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
    RotaryArgs a{q, k, qo, ko, freq, positions, cu, p->B, p->T, p->Hq, p->Hk, p->d, p->rotary};
    a.per_token = (p->flags & SLA_FLAG_TOKEN_POSITIONS) != 0;
    a.head_major = (p->flags & SLA_FLAG_HEAD_MAJOR) != 0;
    a.magnitude = p->magnitude;
    a.sign = sign;
    a.pieces = p->d / 8;
    const int64_t tokens = cu ? p->T : (int64_t)p->B * p->T;
    const int heads = p->Hq + p->Hk, slots = 64 / a.pieces;
    // A wave lies on adjacent heads of a token, or head-major on adjacent tokens of a head; on more tokens where there are few
    // heads, so that it has several loads under way (bf16, B=15 T=11073 4+1 heads of 64: 41.8 us instead of 71.5 with the five
    // heads of one token).
    a.wave_heads = a.head_major ? 1 : heads / kHeadsAhead;
    a.wave_heads = a.wave_heads < 1 ? 1 : (a.wave_heads < slots ? a.wave_heads : slots);
    a.wave_tokens = slots / a.wave_heads;
    const int64_t tiles = (tokens + a.wave_tokens - 1) / a.wave_tokens;
    const int steps = (heads + a.wave_heads - 1) / a.wave_heads;
    // Steps of a wave over a token's heads, which share its angles.  bf16, at most 4, 8, 12, 16: B=8 T=2048 16+16 heads of 128 51.7,
    // 45.4, 45.1, 45.9 us, head-major 63.3, 50.9, 48.1, 47.0; B=4 T=4096 32+4 heads 70.2, 61.3, 54.1, 54.2 us; T=65536 32+32 heads
    // 410, 380, 378, 394 us.  Fewer while that leaves less than two waves a SIMD.
    int each = 12;
    while (each > 1 && tiles * ((steps + each - 1) / each) < (int64_t)kComputeUnits * 8) each /= 2;
    a.groups = (steps + each - 1) / each;
    int64_t waves = tiles * a.groups;
    const int64_t most = (int64_t)kComputeUnits * 256;
    if (waves > most) waves = most;
    const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves));
#define SLA_ROT(BF, MODE) hipLaunchKernelGGL((sla_rotary_kernel<BF, MODE>), grid, dim3(kThreads), 0, stream, a)
    if (p->dtype == SLA_BF16) {
        if (adj) SLA_ROT(true, kAdjacent); else if (p->rotary % 16 == 0) SLA_ROT(true, kHalves); else SLA_ROT(true, kHalvesAnywhere);
    } else {
        if (adj) SLA_ROT(false, kAdjacent); else if (p->rotary % 16 == 0) SLA_ROT(false, kHalves); else SLA_ROT(false, kHalvesAnywhere);
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
