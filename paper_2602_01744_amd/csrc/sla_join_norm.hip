// The residual stream between two blocks of a layer stack for gfx950: a block's output h joins the stream x, behind a norm
// of its own if it has one, and the next block's input is the stream's norm, in one pass,
//     u = h  or  h / rms(h) * w_after,    x' = x + scale * c * u,    y = x' / rms(x') * w_before      rms(v) = sqrt(mean(v^2) + eps)
// (c a scale per channel, or 1), and the gradients from x' for the cotangents dy of y and dx' of x',
//     n = x' r,  dn = dy w_before,  dX = dx' + r (dn - n mean(dn n))           dx = dX,  dw_before = sum dy n
//     m = h r_h, P = sum scale dX m,  dm = scale dX c w_after                  dw_after = c P,  dc = w_after P
//     dh = r_h (dm - m mean(dm m))         or, without the norm behind the block, dh = scale dX c,  dc = sum scale dX h.
//
// Streaming passes over 4 (backward up to 6) tensors, bound by memory.  A row of the stream lies in the registers of one to
// sixteen waves, eight elements a lane (sixteen in rows over 8192), from its first read to its last write, so nothing is read
// twice; a sum over it is a few lane exchanges and, where waves share the row, one exchange through LDS.  x' goes into y before
// it is rounded to the stream's type.  The backward's workgroups walk over rows with the sums for w_before and P in registers
// and leave one partial sum each; a second kernel adds these, in 64 bits and a fixed order: no atomics, so results do not change
// from run to run.  Measured (a large copy reaches 5.4 TB/s, more where the last-level cache holds part of it): bf16, 32768 rows
// of 1024 with both norms, 268 MB, 48 us; gradients of 16384 rows of 2048, fp32 stream, both norms and a scale, 604 MB, 120 us.
// Rows over 8192 stay at half of that rate: one workgroup fills a compute unit without room to load ahead.
#include "sla_row_ops.h"

namespace sla {

namespace {

using namespace row_ops;

constexpr int kMaxWidth = 16384;
constexpr int kForwardWaves = 4, kBackwardWaves = 8;  // of a workgroup, where a row takes no more

struct JoinArgs {
    const void *x, *h, *dy, *dxo;
    const float *w_after, *channel, *w_before;
    void *xo, *y, *dx, *dh;
    float* part;
    const int32_t* cu;
    int64_t tokens;
    int B, D;
    int row_waves;   // waves of a row
    int rows;        // rows of a workgroup
    float scale, eps, inv_d;
};

// Sums of N values over the lanes of a row, to all of them; every wave of the workgroup takes part the same number of times.
// `flip` alternates between two halves of the exchange buffer, so that one barrier a sum is enough.
template <int N>
__device__ __forceinline__ void row_sums(float (&s)[N], int row_waves, float* red, int& flip) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = lanes_sum(s[i], 64);
    if (row_waves == 1) return;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    float* r = red + flip * 16 * 4;
    flip ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) r[wv * 4 + i] = s[i];
    }
    __syncthreads();
    const int w0 = wv / row_waves * row_waves;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = 0.f;
        for (int w = 0; w < row_waves; ++w) t += r[(w0 + w) * 4 + i];
        s[i] = t;
    }
}

// A row of a tensor, the same in a whole wave.  It is held in scalar registers: a lane's address is then 32 bits beside it, where
// the compiler would else keep one of 64 for each tensor and piece across the walk over rows.
template <bool BF16, typename P>
__device__ __forceinline__ P* row_of(P* x, int64_t n, int D) {
    uint64_t at = (uint64_t)x + (size_t)n * D * (BF16 ? 2 : 4);
    asm("" : "+s"(at));
    return (P*)(__attribute__((address_space(1))) P*)at;
}

template <bool XBF, bool HBF, int V>
__global__ __launch_bounds__(1024) void sla_join_norm_kernel(JoinArgs a) {
    __shared__ float red[2 * 16 * 4];
    int flip = 0;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slot = wv / a.row_waves;
    const uint32_t col = ((wv - slot * a.row_waves) * 64 + (threadIdx.x & 63)) * 8, next = a.row_waves * 64 * 8, D = a.D;
    int64_t first, end;
    token_range(a.cu, a.B, a.tokens, first, end);
    for (int64_t r0 = first + (int64_t)blockIdx.x * a.rows; r0 < end; r0 += (int64_t)gridDim.x * a.rows) {
        const int64_t n = r0 + slot;
        float x[V][8], h[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] = h[v][i] = 0.f;
            const uint32_t j = col + v * next;
            if (j < D && n < end) {
                load8<XBF>(row_of<XBF>(a.x, n, a.D), j, x[v]);
                if (a.h) load8<HBF>(row_of<HBF>(a.h, n, a.D), j, h[v]);
            }
        }
        if (a.h) {
            float rh = a.scale;
            if (a.w_after) {
                float s[1] = {0.f};
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[0] += h[v][i] * h[v][i];
                row_sums(s, a.row_waves, red, flip);
                rh *= inverse_root(s[0] * a.inv_d + a.eps);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t j = col + v * next;
                if (j >= D) continue;
                float w[8], c[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = c[i] = 1.f;
                if (a.w_after) load8<false>(a.w_after, j, w);
                if (a.channel) load8<false>(a.channel, j, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] += h[v][i] * rh * w[i] * c[i];
                if (n < end) store8<XBF>(row_of<XBF>(a.xo, n, a.D), j, x[v]);
            }
        }
        if (a.y) {
            float s[1] = {0.f};
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] += x[v][i] * x[v][i];
            row_sums(s, a.row_waves, red, flip);
            const float r = inverse_root(s[0] * a.inv_d + a.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t j = col + v * next;
                if (j >= D || n >= end) continue;
                float w[8];
                load8<false>(a.w_before, j, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] *= r * w[i];
                store8<HBF>(row_of<HBF>(a.y, n, a.D), j, x[v]);
            }
        }
    }
}

// Adds eight sums to those in LDS that the thread keeps there, and clears them.
__device__ __forceinline__ void add_to(float* at, float (&f)[8]) {
    float u[8];
    load8<false>(at, 0, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] += f[i];
        f[i] = 0.f;
    }
    store8<false>(at, 0, u);
}

// Rows up to 8192 (V = 1): the weights stay in registers, and the next row's loads are under way while a row is worked on (4096
// rows of 8192, fp32 stream: 95 -> 88 us).  Wider ones (V = 2) have registers for neither, and their sums over tokens move to LDS.
template <bool XBF, bool HBF, int V>
__global__ __launch_bounds__(1024) void sla_join_norm_backward_kernel(JoinArgs a) {
    extern __shared__ __align__(16) float red[];  // the exchange buffer; after it [V == 1 ? rows - 1 : 1][planes][row_waves * 64 * 8 * V] sums
    float* lds = red + 2 * 16 * 4;
    int flip = 0;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slot = wv / a.row_waves;
    const uint32_t col = ((wv - slot * a.row_waves) * 64 + (threadIdx.x & 63)) * 8, next = a.row_waves * 64 * 8, D = a.D;
    const bool reads_h = a.w_after || a.channel;
    const int planes = reads_h ? 2 : 1, width = next * V;
    Raw8<XBF> x_[V], dxo_[V];
    Raw8<HBF> dy_[V], h_[V];
    float wb[8], cw[8], pw[8], pp[8];
    // w_before (0 without dy), and scale * channel * w_after, at piece v; past the row's end nothing is read
    auto before = [&](int v, float (&w)[8]) {
        const uint32_t j = col + v * next;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.f;
        if (a.dy && j < D) load8<false>(row_of<false>(a.w_before, 0, 0), j, w);
    };
    auto after = [&](int v, float (&w)[8]) {
        const uint32_t j = col + v * next;
        float u[8], c[8];
        if constexpr (V == 1) {  // both loads under way at a time
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = c[i] = 1.f;
            if (a.w_after && j < D) load8<false>(row_of<false>(a.w_after, 0, 0), j, u);
            if (a.channel && j < D) load8<false>(row_of<false>(a.channel, 0, 0), j, c);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = a.scale * u[i] * c[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = a.scale;
            auto times = [&](const float* t) {
                if (!t || j >= D) return;
                load8<false>(row_of<false>(t, 0, 0), j, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] *= u[i];
            };
            times(a.w_after);
            times(a.channel);
        }
    };
    auto fetch = [&](int64_t n) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t j = col + v * next;
            if (j >= D) continue;
            if (a.dy) {
                fetch8(row_of<XBF>(a.x, n, a.D), j, x_[v]);
                fetch8(row_of<HBF>(a.dy, n, a.D), j, dy_[v]);
            }
            if (a.dxo) fetch8(row_of<XBF>(a.dxo, n, a.D), j, dxo_[v]);
            if (reads_h) fetch8(row_of<HBF>(a.h, n, a.D), j, h_[v]);
        }
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        x_[v] = {}; dxo_[v] = {}; dy_[v] = {}; h_[v] = {};  // what is never fetched counts as zero
    }
    int64_t first, end;
    token_range(a.cu, a.B, a.tokens, first, end);
    const int64_t step = (int64_t)gridDim.x * a.rows;
    int64_t r0 = first + (int64_t)blockIdx.x * a.rows;
    if (V == 1 && r0 + slot < end) fetch(r0 + slot);  // ahead of the weights, whose way from memory is as long
#pragma unroll
    for (int i = 0; i < 8; ++i) pw[i] = pp[i] = 0.f;
    if (V == 1) {
        before(0, wb);
        after(0, cw);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (V > 1 && a.part) {
            store8<false>(lds, col + v * next, pw);
            if (reads_h) store8<false>(lds, width + col + v * next, pp);
        }
    }
    for (; r0 < end; r0 += step) {
        const int64_t n = r0 + slot;
        const bool there = n < end;  // where not, the lanes hold some other row: nothing of it is stored or summed
        if (V > 1 && there) fetch(n);
        float dx[V][8], h[V][8];
        float s[3] = {0.f, 0.f, 0.f};
        Raw8<XBF> xr[V];
        Raw8<HBF> yr[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float x[8], dy[8];
            if (V > 1) before(v, wb);
            xr[v] = x_[v];
            yr[v] = dy_[v];
            unpack8(xr[v], x);
            unpack8(yr[v], dy);
            unpack8(dxo_[v], dx[v]);
            unpack8(h_[v], h[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[0] += x[i] * x[i];
                s[1] += dy[i] * wb[i] * x[i];
                s[2] += h[v][i] * h[v][i];
            }
        }
        if (V == 1 && n + step < end) fetch(n + step);
        row_sums(s, a.row_waves, red, flip);
        const float rh = a.w_after ? inverse_root(s[2] * a.inv_d + a.eps) : 1.f;
        if (a.dy) {
            const float r = inverse_root(s[0] * a.inv_d + a.eps), mean = s[1] * r * a.inv_d;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t j = col + v * next;
                float x[8], dy[8];
                if (V > 1) before(v, wb);
                unpack8(xr[v], x);
                unpack8(yr[v], dy);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float n_ = x[i] * r;
                    if (there) pw[i] += dy[i] * n_;
                    dx[v][i] += r * (dy[i] * wb[i] - n_ * mean);
                }
                if (V > 1 && a.part) add_to(lds + j, pw);
                if (j < D && there) store8<XBF>(row_of<XBF>(a.dx, n, a.D), j, dx[v]);
            }
        }
        if (!a.dh) continue;
        float t[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (V > 1) after(v, cw);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[v][i] *= rh;
                if (there) pp[i] += dx[v][i] * h[v][i];
                dx[v][i] *= cw[i];
                t[0] += dx[v][i] * h[v][i];
            }
            if (V > 1 && a.part && reads_h) add_to(lds + width + col + v * next, pp);
        }
        if (a.w_after) row_sums(t, a.row_waves, red, flip);
        const float mean = a.w_after ? t[0] * a.inv_d : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t j = col + v * next;
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[v][i] = rh * (dx[v][i] - h[v][i] * mean);
            if (j < D && there) store8<HBF>(row_of<HBF>(a.dh, n, a.D), j, dx[v]);
        }
    }
    if (!a.part) return;
    // one partial sum a workgroup: the rows beside the first leave theirs in LDS
    if (V == 1 && slot > 0) {
        store8<false>(lds, (size_t)(slot - 1) * planes * width + col, pw);
        if (planes == 2) store8<false>(lds, (size_t)((slot - 1) * planes + 1) * width + col, pp);
    }
    __syncthreads();
    if (slot > 0) return;
    float* out = a.part + (size_t)blockIdx.x * planes * a.D;
    const int others = V == 1 ? a.rows - 1 : 1;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t j = col + v * next;
        if (j >= D) continue;
        float u[8];
        if (V > 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] = pp[i] = 0.f;
        }
        for (int q = 0; q < others; ++q) {
            load8<false>(lds, (size_t)q * planes * width + j, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] += u[i];
            if (planes == 2) {
                load8<false>(lds, (size_t)(q * planes + 1) * width + j, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) pp[i] += u[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) pp[i] *= a.scale;
        store8<false>(out, j, pw);
        if (planes == 2) store8<false>(out, a.D + j, pp);
    }
}

// A workgroup sums 16 adjacent columns of a plane in 64 bits: 64 threads a column, four of them in a wave.
constexpr int kSumColumns = 16, kSumRows = 64;
__global__ __launch_bounds__(kSumColumns * kSumRows) void sla_column_sums_kernel(const float* part, int nparts, int planes, int width,
                                                                               float* out0, float* out1, const float* by1,
                                                                               float* out2, const float* by2) {
    __shared__ double red[kSumRows / 4][kSumColumns];
    const int c = threadIdx.x % kSumColumns, rr = threadIdx.x / kSumColumns, wv = threadIdx.x >> 6;
    const int per_plane = (width + kSumColumns - 1) / kSumColumns;
    const int plane = blockIdx.x / per_plane, j = (blockIdx.x - plane * per_plane) * kSumColumns + c;
    double s = 0.0;
    if (j < width) {
#pragma unroll 8
        for (int n = rr; n < nparts; n += kSumRows) s += part[((size_t)n * planes + plane) * width + j];
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (threadIdx.x % 64 < kSumColumns) red[wv][c] = s;
    __syncthreads();
    if (rr > 0 || j >= width) return;
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kSumRows / 4; ++w) s += red[w][c];
    if (plane == 0) {
        if (out0) out0[j] = (float)s;
    } else {
        if (out1) out1[j] = (float)(by1 ? s * by1[j] : s);
        if (out2) out2[j] = (float)(by2 ? s * by2[j] : s);
    }
}

int64_t tokens_of(const sla_join_norm_params& p, bool packed) { return packed ? p.T : (int64_t)p.B * p.T; }

// The sizes and types of a call or of a query for one.
int check_sizes(const sla_join_norm_params* p, bool packed) {
    if (!p) return SLA_ERR_NULL;
    if ((p->dtype != SLA_F32 && p->dtype != SLA_BF16) || (p->x_dtype != SLA_F32 && p->x_dtype != SLA_BF16)) return SLA_ERR_UNSUPPORTED;
    if (p->dtype == SLA_F32 && p->x_dtype == SLA_BF16) return SLA_ERR_UNSUPPORTED;  // the stream is never narrower than the blocks
    if (p->B < 0 || p->T < 0 || p->D < 8 || p->D > kMaxWidth || (p->D & 7) || !(p->eps >= 0.f)) return SLA_ERR_SHAPE;
    return tokens_of(*p, packed) > (int64_t)1 << 30 ? SLA_ERR_SHAPE : SLA_OK;
}

int check_join(const sla_join_norm_params* p, const int32_t* cu) {
    const int rc = check_sizes(p, cu != nullptr);
    return rc == SLA_OK && !aligned(cu, 4) ? SLA_ERR_ALIGN : rc;
}

// How a row lies over lanes: one piece of eight a lane and as many waves as that takes (bf16, 16384 rows of 2048 with one, two
// and four pieces 45.5, 47.7, 51.8 us; fp32 stream 78, 81, 92 us), or two pieces in rows over 8192.  More rows share a
// workgroup of `waves` waves where theirs leave room.
struct Split {
    int v, row_waves, rows, threads;
};
Split split(int D, int waves) {
    Split s{1, 1, 1, 64 * waves};
    while (s.row_waves < 16 && s.row_waves * 64 * 8 < D) s.row_waves *= 2;
    if (s.row_waves * 64 * 8 < D) s.v = 2;
    if (s.row_waves < waves) s.rows = waves / s.row_waves; else s.threads = 64 * s.row_waves;
    return s;
}

// Launches with more than the 64 KB of LDS that a kernel gets without asking.
template <typename F>
bool allow_lds(F kernel, size_t lds) {
    if (lds <= 64 * 1024 || hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess)
        return true;
    (void)hipGetLastError();
    return false;
}

// Workgroups of the backward, each of which leaves a partial sum: as many as are at work at a time.
unsigned backward_workgroups(const Split& s, int64_t tokens) {
    const int64_t n = (tokens + s.rows - 1) / s.rows, most = kComputeUnits * (s.threads == 1024 ? 1 : 2);
    return (unsigned)(n < most ? n : most);
}

// Bytes of the partial sums that so many workgroups leave (one plane of two may stay unused).
size_t sums_bytes(unsigned blocks, int D) { return (size_t)blocks * 2 * D * sizeof(float); }

}  // namespace

int launch_column_sums(const float* part, int nparts, int planes, int width, float* out0, float* out1, const float* by1,
                       float* out2, const float* by2, hipStream_t stream) {
    const unsigned per_plane = (unsigned)((width + kSumColumns - 1) / kSumColumns);
    hipLaunchKernelGGL(sla_column_sums_kernel, dim3(per_plane * planes), dim3(kSumColumns * kSumRows), 0, stream, part,
                       nparts, planes, width, out0, out1, by1, out2, by2);
    return hipGetLastError() == hipSuccess ? SLA_OK : SLA_ERR_HIP;
}

}  // namespace sla

extern "C" {

int sla_join_norm(const sla_join_norm_params* p, const void* x, const void* h, const float* w_after, const float* channel_scale,
                  const float* w_before, const int32_t* cu_seqlens, void* x_out, void* y, void* stream) {
    using namespace sla;
    const int rc = check_join(p, cu_seqlens);
    if (rc != SLA_OK) return rc;
    const bool work = p->B > 0 && p->T > 0;
    if (work && (!x || (!h && !y))) return SLA_ERR_NULL;
    if (work && ((h != nullptr) != (x_out != nullptr) || (y != nullptr) != (w_before != nullptr))) return SLA_ERR_NULL;
    if (work && !h && (w_after || channel_scale)) return SLA_ERR_NULL;
    const void* ptrs[] = {x, h, w_after, channel_scale, w_before, x_out, y};
    for (const void* q : ptrs)
        if (!aligned(q, 16)) return SLA_ERR_ALIGN;
    if (!work) return SLA_OK;
    JoinArgs a{};
    a.x = x; a.h = h; a.w_after = w_after; a.channel = channel_scale; a.w_before = w_before; a.xo = x_out; a.y = y;
    a.cu = cu_seqlens; a.tokens = tokens_of(*p, cu_seqlens); a.B = p->B; a.D = p->D;
    a.scale = p->scale; a.eps = p->eps; a.inv_d = 1.f / p->D;
    const Split s = split(p->D, kForwardWaves);
    a.row_waves = s.row_waves; a.rows = s.rows;
    const int64_t blocks = (a.tokens + s.rows - 1) / s.rows;
    const dim3 grid((unsigned)(blocks < kComputeUnits * 64 ? blocks : kComputeUnits * 64));
#define SLA_JN(X, Y, V) hipLaunchKernelGGL((sla_join_norm_kernel<X, Y, V>), grid, dim3(s.threads), 0, (hipStream_t)stream, a)
#define SLA_JN_V(X, Y) \
    if (s.v == 1) SLA_JN(X, Y, 1); else SLA_JN(X, Y, 2)
    if (p->dtype == SLA_F32) { SLA_JN_V(false, false); }
    else if (p->x_dtype == SLA_F32) { SLA_JN_V(false, true); }
    else { SLA_JN_V(true, true); }
#undef SLA_JN_V
#undef SLA_JN
    return hipGetLastError() == hipSuccess ? SLA_OK : SLA_ERR_HIP;
}

size_t sla_join_norm_backward_workspace_bytes(const sla_join_norm_params* p, int packed) {
    using namespace sla;
    if (check_sizes(p, packed != 0) != SLA_OK || p->B == 0 || p->T == 0) return 0;
    return sums_bytes(backward_workgroups(split(p->D, kBackwardWaves), tokens_of(*p, packed != 0)), p->D);
}

int sla_join_norm_backward(const sla_join_norm_params* p, const void* x_out, const void* h, const float* w_after,
                           const float* channel_scale, const float* w_before, const void* dy, const void* dx_out,
                           const int32_t* cu_seqlens, void* dx, void* dh, float* dw_after, float* dchannel_scale,
                           float* dw_before, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sla;
    const int rc = check_join(p, cu_seqlens);
    if (rc != SLA_OK) return rc;
    const bool work = p->B > 0 && p->T > 0, reads_h = w_after || channel_scale;
    // dy with the norm's weight and everything that flows from it; without it dx would be dx_out itself
    if ((dy != nullptr) != (w_before != nullptr) || (w_before != nullptr) != (dw_before != nullptr)) {
        if (work || (w_before != nullptr) != (dw_before != nullptr)) return SLA_ERR_NULL;
    }
    if ((w_after != nullptr) != (dw_after != nullptr) || (channel_scale != nullptr) != (dchannel_scale != nullptr)) return SLA_ERR_NULL;
    if (work && ((dy != nullptr) != (dx != nullptr) || (dy && !x_out) || (!dy && !dx_out))) return SLA_ERR_NULL;
    if (work && ((reads_h && (!h || !dh)) || (!dx && !dh))) return SLA_ERR_NULL;
    const void* ptrs[] = {x_out, h, w_after, channel_scale, w_before, dy, dx_out, dx, dh, dw_after, dchannel_scale, dw_before, workspace};
    for (const void* q : ptrs)
        if (!aligned(q, 16)) return SLA_ERR_ALIGN;
    const bool sums = dw_before || dw_after || dchannel_scale;
    const int planes = reads_h ? 2 : 1;
    if (!work)
        return sums ? launch_column_sums(nullptr, 0, planes, p->D, dw_before, dw_after, nullptr, dchannel_scale, nullptr, (hipStream_t)stream)
                    : SLA_OK;
    const Split s = split(p->D, kBackwardWaves);
    const unsigned blocks = backward_workgroups(s, tokens_of(*p, cu_seqlens != nullptr));
    if (sums && (!workspace || workspace_bytes < sums_bytes(blocks, p->D))) return SLA_ERR_WORKSPACE;
    JoinArgs a{};
    a.x = x_out; a.h = h; a.w_after = w_after; a.channel = channel_scale; a.w_before = w_before; a.dy = dy; a.dxo = dx_out;
    a.dx = dx; a.dh = dh; a.part = sums ? (float*)workspace : nullptr;
    a.cu = cu_seqlens; a.tokens = tokens_of(*p, cu_seqlens); a.B = p->B; a.D = p->D;
    a.scale = p->scale; a.eps = p->eps; a.inv_d = 1.f / p->D;
    a.row_waves = s.row_waves; a.rows = s.rows;
    const size_t lds = (2 * 16 * 4 + (size_t)(s.v == 1 ? s.rows - 1 : 1) * planes * s.row_waves * 64 * 8 * s.v) * sizeof(float);
#define SLA_JN(X, Y, V)                                                                                                 \
    do {                                                                                                                \
        const auto kernel = sla_join_norm_backward_kernel<X, Y, V>;                                                       \
        if (!allow_lds(kernel, lds)) return SLA_ERR_HIP;                                                                 \
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(s.threads), lds, (hipStream_t)stream, a);                          \
    } while (0)
#define SLA_JN_V(X, Y) \
    if (s.v == 1) SLA_JN(X, Y, 1); else SLA_JN(X, Y, 2)
    if (p->dtype == SLA_F32) { SLA_JN_V(false, false); }
    else if (p->x_dtype == SLA_F32) { SLA_JN_V(false, true); }
    else { SLA_JN_V(true, true); }
#undef SLA_JN_V
#undef SLA_JN
    if (hipGetLastError() != hipSuccess) return SLA_ERR_HIP;
    if (!sums) return SLA_OK;
    return launch_column_sums((const float*)workspace, (int)blocks, planes, p->D, dw_before, dw_after, channel_scale, dchannel_scale,
                              w_after, (hipStream_t)stream);
}

}  // extern "C"
