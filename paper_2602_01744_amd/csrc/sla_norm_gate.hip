// The read-out behind the mixer for gfx950: every head's output vector x (width dv) divided by its root mean square,
// weighted and gated, as RetNet, GLA and the delta rule's blocks do in front of the output projection,
//     r = 1 / sqrt(mean(x^2) + eps),  n = x r,  y = n w act(g)          act: SiLU, sigmoid, or no gate
// and its gradients for the cotangent dy of y, from x and g again (nothing is kept from the forward call),
//     dn = dy w act(g),  dx = r (dn - n mean(dn n)),  dg = dy n w act'(g),  dw = sum over tokens of dy n act(g).
//
// Streaming passes over 3 (backward 5) tensors, a few tens of flops an element, bound by memory.  Measured in bf16 (a large copy
// reaches 5.4 TB/s, more where the last-level cache holds part of it): T=65536 16 heads of 128, 805 MB, 142 us; gradients B=8
// T=4096 16 heads of 128, 671 MB, 131 to 136 us.  A head's vector lies in dv/8 lanes (a power of
// two of them is set aside), eight elements each, so its sums are a few lane exchanges and nothing is read twice.  A wave
// covers as many heads of a token as divide H, then several tokens: a lane keeps to one head, whose weights stay in
// registers.  dw is summed in a fixed order: a lane's tokens in fp32 registers, then, in 64 bits, the lanes of a workgroup through
// LDS and, in a second kernel, the workgroups' partial sums (fp32 in memory); no atomics, so results do not change from run to run.
#include "sla_row_ops.h"

namespace sla {

namespace {

using namespace row_ops;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxHeads = 1024, kMaxWidth = 512;
constexpr int kForwardAhead = 2;  // rows whose loads a lane has in flight
enum { kNone = SLA_GATE_NONE, kSilu = SLA_GATE_SILU, kSigmoid = SLA_GATE_SIGMOID };

struct GateArgs {
    const void *x, *g, *dy;
    const float* w;
    void *y, *dx, *dg;
    float* part;
    const int32_t* cu;
    int B, T, H, dv;
    int lanes;        // lanes of a head
    int wave_heads;   // heads of a wave (64 / lanes / wave_heads tokens at a time)
    int groups;       // groups of wave_heads heads
    int head_major;   // x, dx are [B,H,T,dv]
    int per_head;     // w is [H,dv]
    float eps, inv_dv;
};

// p = 1 / (1 + exp(-g)) and rest = 1 - p, which a difference would lose where the gate is open: both from e = exp(-|g|).  In fp32
// (EXACT) what the product |g| log2 e loses to rounding, up to |g| 2^-24 of e, comes back as a factor (not where e leaves the normal
// range), and the reciprocal has a Newton step: 5 steps of 2^-24 in all.  bf16 needs neither: at most 2^-17, half a step is 2^-9.
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float g, float& rest) {
    const float m = fabsf(g), t = -m * lane_ops::kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    if (EXACT) {
        const float lost = __builtin_fmaf(m, -1.92596299e-8f, __builtin_fmaf(m, -lane_ops::kLog2e, -t));  // log2 e = kLog2e + 1.926e-8
        e = t > -126.f ? __builtin_fmaf(e * 0.693147181f, lost, e) : e;
    }
    const float d = 1.f + e;
    float near = __builtin_amdgcn_rcpf(d);
    if (EXACT) near = __builtin_fmaf(near, __builtin_fmaf(-d, near, 1.f), near);
    const float far = e * near;
    rest = g < 0.f ? near : far;
    return g < 0.f ? far : near;
}
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float g) {
    float rest;
    if (EXACT) return sigmoid<true>(g, rest);
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-g * lane_ops::kLog2e));
}

// Where a lane works: head h, piece e of it, tokens first + its slot, then every `step`-th.
struct Place {
    int h, e;
    bool live;
    int64_t n, end, step;
};
__device__ __forceinline__ Place place(const GateArgs& a) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int grp = blockIdx.x % a.groups, slot = lane / a.lanes, tokens = 64 / a.lanes / a.wave_heads;
    Place p;
    p.e = lane % a.lanes;
    p.h = grp * a.wave_heads + slot % a.wave_heads;
    p.live = 8 * p.e < a.dv;
    int64_t first;
    token_range(a.cu, a.B, a.cu ? (int64_t)a.T : (int64_t)a.B * a.T, first, p.end);
    p.n = first + ((int64_t)(blockIdx.x / a.groups) * kWaves + wv) * tokens + slot / a.wave_heads;
    p.step = (int64_t)(gridDim.x / a.groups) * kWaves * tokens;
    return p;
}

__device__ __forceinline__ size_t offset_x(const GateArgs& a, const Place& p, int64_t n) {
    if (!a.head_major) return ((size_t)n * a.H + p.h) * a.dv + 8 * p.e;
    const uint32_t b = (uint32_t)n / (uint32_t)a.T, t = (uint32_t)n - b * a.T;
    return (((size_t)b * a.H + p.h) * a.T + t) * a.dv + 8 * p.e;
}
__device__ __forceinline__ size_t offset_y(const GateArgs& a, const Place& p, int64_t n) {
    return ((size_t)n * a.H + p.h) * a.dv + 8 * p.e;
}

__device__ __forceinline__ void load_weights(const GateArgs& a, const Place& p, float (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    if (a.w && p.live) load8<false>(a.w, (a.per_head ? (size_t)p.h * a.dv : 0) + 8 * p.e, w);
}

template <bool BF16, int GATE>
__global__ __launch_bounds__(kThreads) void sla_norm_gate_kernel(GateArgs a) {
    constexpr int U = kForwardAhead;
    const Place p = place(a);
    float w[8];
    load_weights(a, p, w);
    // every lane of a wave makes the same number of steps: the sums below take all of them
    const int64_t wave_first = __builtin_amdgcn_readfirstlane((int)p.n);
    for (int64_t m = wave_first, n0 = p.n; m < p.end; m += U * p.step, n0 += U * p.step) {
        float x[U][8], g[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t n = n0 + u * p.step;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = g[u][i] = 0.f;
            if (p.live && n < p.end) {
                load8<BF16>(a.x, offset_x(a, p, n), x[u]);
                if (GATE != kNone) load8<BF16>(a.g, offset_y(a, p, n), g[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t n = n0 + u * p.step;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[u][i] * x[u][i];
            const float r = inverse_root(lanes_sum(s, a.lanes) * a.inv_dv + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = x[u][i] * r * w[i];
                if (GATE == kSilu) v *= g[u][i] * sigmoid<!BF16>(g[u][i]);
                if (GATE == kSigmoid) v *= sigmoid<!BF16>(g[u][i]);
                x[u][i] = v;
            }
            if (p.live && n < p.end) store8<BF16>(a.y, offset_y(a, p, n), x[u]);
        }
    }
}

template <bool BF16, int GATE>
__global__ __launch_bounds__(kThreads) void sla_norm_gate_backward_kernel(GateArgs a) {
    __shared__ float red[kThreads * 8];
    const Place p = place(a);
    float w[8], dw[8];
    load_weights(a, p, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] = 0.f;
    Raw8<BF16> xr{}, gr{}, yr{};
    auto fetch = [&](int64_t n) {
        if (!p.live || n >= p.end) return;
        const size_t oy = offset_y(a, p, n);
        fetch8(a.x, offset_x(a, p, n), xr);
        fetch8(a.dy, oy, yr);
        if (GATE != kNone) fetch8(a.g, oy, gr);
    };
    fetch(p.n);
    const int64_t wave_first = __builtin_amdgcn_readfirstlane((int)p.n);
    for (int64_t m = wave_first, n = p.n; m < p.end; m += p.step, n += p.step) {
        float x[8], g[8], dy[8], dn[8];
        const bool row = p.live && n < p.end;  // where not, the lane holds some other row: nothing of it is stored or summed
        unpack8(xr, x);
        unpack8(yr, dy);
        unpack8(gr, g);
        fetch(n + p.step);  // the next row's loads are under way while this one is worked on
        float s = 0.f, c = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float act = 1.f;
            if (GATE != kNone) {
                // g becomes the gate's derivative.  SiLU's is a sum beside which 1 - q may be a difference: in bf16 it is, which
                // leaves the pass bound by memory (B=8 T=4096 16 heads of 128: 133 us, and 148 with the other form).
                float rest;
                const float q = BF16 && GATE == kSilu ? sigmoid<false>(g[i]) : sigmoid<!BF16>(g[i], rest);
                if (BF16 && GATE == kSilu) rest = 1.f - q;
                act = GATE == kSilu ? g[i] * q : q;
                g[i] = GATE == kSilu ? q * (1.f + g[i] * rest) : q * rest;
            }
            dn[i] = dy[i] * act;  // the weight comes later: the sum for dw takes it without
            s += x[i] * x[i];
            c += dn[i] * w[i] * x[i];
        }
        const float r = inverse_root(lanes_sum(s, a.lanes) * a.inv_dv + a.eps);
        const float mean = lanes_sum(c, a.lanes) * r * a.inv_dv;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float n_ = x[i] * r;
            if (row) dw[i] += dn[i] * n_;  // a row that is not there has no finite n where eps is 0
            if (GATE != kNone) g[i] *= dy[i] * n_ * w[i];
            x[i] = r * (dn[i] * w[i] - n_ * mean);
        }
        if (row) {
            store8<BF16>(a.dx, offset_x(a, p, n), x);
            if (GATE != kNone) store8<BF16>(a.dg, offset_y(a, p, n), g);
        }
    }
    if (!a.part) return;
    // the workgroup's tokens (and, for shared weights, heads): its waves' lanes of the same piece, added in order
#pragma unroll
    for (int i = 0; i < 8; ++i) red[threadIdx.x * 8 + i] = dw[i];
    __syncthreads();
    const int heads = a.per_head ? a.wave_heads : 1, slots = kThreads / a.lanes;
    for (int j = threadIdx.x; j < heads * a.dv; j += kThreads) {
        const int hh = j / a.dv, col = j - hh * a.dv;
        double sum = 0.0;  // up to 256 slots one after the other
        for (int q = hh; q < slots; q += heads) sum += red[(q * a.lanes + col / 8) * 8 + col % 8];
        const float s = (float)sum;
        const size_t blk = blockIdx.x / a.groups, grp = blockIdx.x % a.groups;
        if (a.per_head)
            a.part[(blk * a.H + grp * heads + hh) * a.dv + col] = s;
        else
            a.part[(size_t)blockIdx.x * a.dv + col] = s;
    }
}

int64_t tokens_of(const sla_norm_gate_params& p, bool packed) { return packed ? p.T : (int64_t)p.B * p.T; }

// The sizes and types of a call or of a query for one.
int check_sizes(const sla_norm_gate_params* p, bool packed) {
    if (!p) return SLA_ERR_NULL;
    if (p->dtype != SLA_F32 && p->dtype != SLA_BF16) return SLA_ERR_UNSUPPORTED;
    if (p->gate < kNone || p->gate > kSigmoid) return SLA_ERR_UNSUPPORTED;
    if (p->flags & ~(SLA_FLAG_HEAD_MAJOR | SLA_FLAG_HEAD_WEIGHTS)) return SLA_ERR_UNSUPPORTED;
    if (packed && (p->flags & SLA_FLAG_HEAD_MAJOR)) return SLA_ERR_UNSUPPORTED;  // packed batches are [T,H,dv]
    if (p->B < 0 || p->T < 0 || p->H < 1 || p->H > kMaxHeads) return SLA_ERR_SHAPE;
    if (p->dv < 8 || p->dv > kMaxWidth || (p->dv & 7) || !(p->eps >= 0.f)) return SLA_ERR_SHAPE;
    return tokens_of(*p, packed) > (int64_t)1 << 30 ? SLA_ERR_SHAPE : SLA_OK;
}

int check_norm_gate(const sla_norm_gate_params* p, const void* g, const float* w, const int32_t* cu) {
    const int rc = check_sizes(p, cu != nullptr);
    if (rc != SLA_OK) return rc;
    if (p->B > 0 && p->T > 0 && (p->gate != kNone) != (g != nullptr)) return SLA_ERR_NULL;
    if ((p->flags & SLA_FLAG_HEAD_WEIGHTS) && !w) return SLA_ERR_NULL;
    if (!aligned(g, 16) || !aligned(w, 16) || !aligned(cu, 4)) return SLA_ERR_ALIGN;
    return SLA_OK;
}

void layout(const sla_norm_gate_params& p, GateArgs& a) {
    a.B = p.B; a.T = p.T; a.H = p.H; a.dv = p.dv;
    a.eps = p.eps;
    a.inv_dv = 1.f / p.dv;
    a.head_major = (p.flags & SLA_FLAG_HEAD_MAJOR) != 0;
    a.per_head = (p.flags & SLA_FLAG_HEAD_WEIGHTS) != 0;
    a.lanes = 1;
    while (a.lanes * 8 < p.dv) a.lanes *= 2;
    a.wave_heads = 1;
    while (a.wave_heads * 2 * a.lanes <= 64 && p.H % (a.wave_heads * 2) == 0) a.wave_heads *= 2;
    a.groups = p.H / a.wave_heads;
}

// Workgroups for `tokens` tokens, a multiple of a.groups: one row a lane, at most `most` of them (one group each at least).
unsigned workgroups(const GateArgs& a, int64_t tokens, int64_t most) {
    const int64_t each = (int64_t)kWaves * (64 / a.lanes / a.wave_heads);  // tokens of a workgroup and step
    int64_t n = (tokens + each - 1) / each;
    const int64_t cap = most / a.groups > 1 ? most / a.groups : 1;
    return (unsigned)((n < cap ? n : cap) * a.groups);
}

constexpr int64_t kBackwardGroups = kComputeUnits * 4;  // workgroups, and with them partial sums of dw

// Bytes of the partial sums that so many workgroups of the backward leave.
size_t sums_bytes(const GateArgs& a, unsigned blocks) {
    return (a.per_head ? (size_t)(blocks / a.groups) * a.H : blocks) * (size_t)a.dv * sizeof(float);
}

}  // namespace

}  // namespace sla

extern "C" {

int sla_norm_gate(const sla_norm_gate_params* p, const void* x, const void* g, const float* w, const int32_t* cu_seqlens,
                  void* y, void* stream) {
    using namespace sla;
    const int rc = check_norm_gate(p, g, w, cu_seqlens);
    if (rc != SLA_OK) return rc;
    const bool work = p->B > 0 && p->T > 0;
    if (work && (!x || !y)) return SLA_ERR_NULL;
    if (!aligned(x, 16) || !aligned(y, 16)) return SLA_ERR_ALIGN;
    if (!work) return SLA_OK;
    GateArgs a{};
    layout(*p, a);
    a.x = x; a.g = g; a.w = w; a.y = y; a.cu = cu_seqlens;
    // bf16 rows that lie apart in x want fewer workgroups that walk on: head-major, with 4, 8, 16 and 64 a compute unit, B=8 T=2048 16
    // heads of 128 37.0, 37.9, 38.0, 46 us, B=8 T=4096 4 heads of 256 37.4, 39.5, 40.1, 44, 8 of 64 18.9, 19.3, 21.8, 21.3, 2 of 512
    // 36.1, 40.0, 39.5, 44, B=16384 T=1 16 of 128 35.1, 35.6, 37.6, 43; only a single long row differs, T=65536 149, 154, 160, 143.
    // fp32 rows are twice as long and want what token-major ones do: with 4, 16 and 64, B=4 T=2048 16 of 128 38.2, 35.3, 34.1 us, B=8
    // T=2048 8 of 128 36.5, 35.0, 33.3, B=8 T=4096 2 of 256 35.8, 35.5, 34.1, B=4 T=2048 32 of 64 37.0, 36.3, 35.3; only B=4 T=4096 4 of
    // 256 differs, 35.3, 37.6, 37.5.  Token-major bf16, T=65536 16 heads of 128: 151 us with 8 and 142 with 64.
    const dim3 grid(workgroups(a, tokens_of(*p, cu_seqlens), kComputeUnits * (a.head_major && p->dtype == SLA_BF16 ? 4 : 64)));
#define SLA_NG(BF, G) hipLaunchKernelGGL((sla_norm_gate_kernel<BF, G>), grid, dim3(kThreads), 0, (hipStream_t)stream, a)
    if (p->dtype == SLA_BF16) {
        if (p->gate == kNone) SLA_NG(true, kNone); else if (p->gate == kSilu) SLA_NG(true, kSilu); else SLA_NG(true, kSigmoid);
    } else {
        if (p->gate == kNone) SLA_NG(false, kNone); else if (p->gate == kSilu) SLA_NG(false, kSilu); else SLA_NG(false, kSigmoid);
    }
#undef SLA_NG
    return hipGetLastError() == hipSuccess ? SLA_OK : SLA_ERR_HIP;
}

size_t sla_norm_gate_backward_workspace_bytes(const sla_norm_gate_params* p, int packed) {
    using namespace sla;
    if (!p) return 0;
    sla_norm_gate_params q = *p;
    q.gate = kNone;  // says nothing about the sums
    if (check_sizes(&q, packed != 0) != SLA_OK || p->B == 0 || p->T == 0) return 0;
    GateArgs a{};
    layout(*p, a);
    return sums_bytes(a, workgroups(a, tokens_of(*p, packed != 0), kBackwardGroups));
}

int sla_norm_gate_backward(const sla_norm_gate_params* p, const void* x, const void* g, const float* w, const void* dy,
                           const int32_t* cu_seqlens, void* dx, void* dg, float* dw, void* workspace,
                           size_t workspace_bytes, void* stream) {
    using namespace sla;
    const int rc = check_norm_gate(p, g, w, cu_seqlens);
    if (rc != SLA_OK) return rc;
    const bool work = p->B > 0 && p->T > 0;
    if (work && (!x || !dy || !dx || (g != nullptr) != (dg != nullptr))) return SLA_ERR_NULL;
    if ((w != nullptr) != (dw != nullptr)) return SLA_ERR_NULL;
    const void* ptrs[] = {x, dy, dx, dg, dw, workspace};
    for (const void* q : ptrs)
        if (!aligned(q, 16)) return SLA_ERR_ALIGN;
    GateArgs a{};
    layout(*p, a);
    const int width = a.per_head ? a.H * a.dv : a.dv;
    if (!work) return dw ? launch_column_sums(nullptr, 0, 1, width, dw, nullptr, nullptr, nullptr, nullptr, (hipStream_t)stream) : SLA_OK;
    const unsigned blocks = workgroups(a, tokens_of(*p, cu_seqlens != nullptr), kBackwardGroups);
    if (dw && (!workspace || workspace_bytes < sums_bytes(a, blocks))) return SLA_ERR_WORKSPACE;
    a.x = x; a.g = g; a.w = w; a.dy = dy; a.dx = dx; a.dg = dg; a.cu = cu_seqlens;
    a.part = dw ? (float*)workspace : nullptr;
#define SLA_NG(BF, G) \
    hipLaunchKernelGGL((sla_norm_gate_backward_kernel<BF, G>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, a)
    if (p->dtype == SLA_BF16) {
        if (p->gate == kNone) SLA_NG(true, kNone); else if (p->gate == kSilu) SLA_NG(true, kSilu); else SLA_NG(true, kSigmoid);
    } else {
        if (p->gate == kNone) SLA_NG(false, kNone); else if (p->gate == kSilu) SLA_NG(false, kSilu); else SLA_NG(false, kSigmoid);
    }
#undef SLA_NG
    if (hipGetLastError() != hipSuccess) return SLA_ERR_HIP;
    if (!dw) return SLA_OK;
    return launch_column_sums((const float*)workspace, (int)(a.per_head ? blocks / a.groups : blocks), 1, width, dw, nullptr,
                              nullptr, nullptr, nullptr, (hipStream_t)stream);
}

}  // extern "C"
