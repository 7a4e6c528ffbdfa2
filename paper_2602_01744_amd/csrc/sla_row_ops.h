// Rows of eight-element pieces, reductions over the lanes of a row, and the second stage of sums over tokens, as the
// kernels around the mixer use them (rotary positions, read-out norm, residual join).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sla.h"
#include "sla_lane_ops.h"

namespace sla {
namespace row_ops {

using lane_ops::f4;
using lane_ops::u4;

// The chip the library is built for; sizes of grids and workspaces must not depend on the current device.
constexpr int kComputeUnits = 256;

// Eight elements as they lie in memory, for loads that are waited for later.
template <bool BF16>
struct Raw8;
template <>
struct Raw8<true> {
    u4 v;
};
template <>
struct Raw8<false> {
    f4 a, b;
};
__device__ __forceinline__ void fetch8(const void* x, size_t off, Raw8<true>& r) { r.v = *(const u4*)((const uint16_t*)x + off); }
__device__ __forceinline__ void fetch8(const void* x, size_t off, Raw8<false>& r) {
    r.a = *(const f4*)((const float*)x + off);
    r.b = *(const f4*)((const float*)x + off + 4);
}
__device__ __forceinline__ void put8(void* x, size_t off, const Raw8<true>& r) { *(u4*)((uint16_t*)x + off) = r.v; }
__device__ __forceinline__ void put8(void* x, size_t off, const Raw8<false>& r) {
    *(f4*)((float*)x + off) = r.a;
    *(f4*)((float*)x + off + 4) = r.b;
}
__device__ __forceinline__ void unpack8(const Raw8<true>& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = lane_ops::bf_lo(r.v[i]);
        f[2 * i + 1] = lane_ops::bf_hi(r.v[i]);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<false>& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = r.a[i];
        f[4 + i] = r.b[i];
    }
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* x, size_t off, float (&f)[8]) {
    Raw8<BF16> r;
    fetch8(x, off, r);
    unpack8(r, f);
}

template <bool BF16>
__device__ __forceinline__ void store8(void* y, size_t off, const float (&f)[8]) {
    if constexpr (BF16) {
        u4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = lane_ops::pack2(f[2 * i], f[2 * i + 1]);
        *(u4*)((uint16_t*)y + off) = v;
    } else {
        *(f4*)((float*)y + off) = f4{f[0], f[1], f[2], f[3]};
        *(f4*)((float*)y + off + 4) = f4{f[4], f[5], f[6], f[7]};
    }
}

// Sum over groups of `lanes` adjacent lanes (a power of two, the same in the whole wave), to all of them, the same bits in
// each.  Every lane of the wave takes part.
__device__ __forceinline__ float lanes_sum(float s, int lanes) {
    if (lanes > 1) s += lane_ops::dpp<0xB1>(s);   // quad_perm [1,0,3,2]
    if (lanes > 2) s += lane_ops::dpp<0x4E>(s);   // quad_perm [2,3,0,1]
    if (lanes > 4) s += lane_ops::dpp<0x141>(s);  // row_half_mirror
    if (lanes > 8) s += lane_ops::dpp<0x140>(s);  // row_mirror
    if (lanes > 16) {
        const lane_ops::u2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        s = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if (lanes > 32) {
        const lane_ops::u2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        s = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    return s;
}

// 1 / sqrt(x): the hardware's, within one unit of the last place, and a Newton step; 0 and infinity keep the hardware's.  Values
// under the normal range, which the instruction takes for 0, are scaled into it first: by ldexp, which costs the join's gradients of
// rows over 8192 two spilled registers (factors chosen by a condition 14, and 11 % of their time).
__device__ __forceinline__ float inverse_root(float x) {
    const int s = x < 0x1p-126f ? 32 : 0;
    const float y = ldexpf(__builtin_amdgcn_rsqf(ldexpf(x, 2 * s)), s);
    const float z = __builtin_fmaf(0.5f * y, __builtin_fmaf(-x * y, y, 1.f), y);
    return y > 0.f && y < INFINITY ? z : y;
}

// The tokens a packed call works on: from the first sequence's start to the last one's end, inside [0, T]; all without
// cu_seqlens.
__device__ __forceinline__ void token_range(const int32_t* cu, int B, int64_t tokens, int64_t& first, int64_t& end) {
    first = 0;
    end = tokens;
    if (cu) {
        const int64_t a = cu[0], b = cu[B];
        first = a < 0 ? 0 : (a > tokens ? tokens : a);
        end = b < first ? first : (b > tokens ? tokens : b);
    }
}

inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace row_ops

// Second stage of sums over tokens: with s_p[j] = sum over the nparts parts of part[n][p][j] (planes p of `width` floats),
// in a fixed order: out0 = s_0;  with two planes also out1 = s_1 * by1 and out2 = s_1 * by2 (a NULL factor is 1, a NULL
// output is left out).  nparts == 0 writes zeros.
int launch_column_sums(const float* part, int nparts, int planes, int width, float* out0, float* out1, const float* by1,
                       float* out2, const float* by2, hipStream_t stream);

}  // namespace sla
