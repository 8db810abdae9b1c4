// dReLU's activations in 8 bits: max(0, gate) and max(0, up), all that its
// gradient needs of them.  They have no sign, so a code is 4 bits of exponent
// and 4 of mantissa; 0 stands for "not positive", so the set of neurons that
// the gradient passes is exact.  Blocks of 16 columns of a row (what four lanes hold
// of a 16 x 16 product) share a byte E0, the exponent of their largest, at least 15:
//   t(v) = the fp32 bits of v, rounded to 4 bits of mantissa, >> 19
//          (16 x biased exponent + mantissa)
//   E0 = max(15, largest t >> 4),  code = max(1, t - 16 E0 + 240)
// Half a step is 2^-5 of the value (e4m3: 2^-4); what lies below 33/32 x 2^-15 of the
// largest's power of two comes out as 17/16 x 2^-15 of it.  A code's value has 5
// significant bits: bf16 holds it exactly, its bits are t << 3.
#pragma once

#include <hip/hip_runtime.h>

#include "ts_device.h"

namespace ts {

constexpr int kKeepBlock = 16;  // columns per exponent byte

// 16 x exponent + mantissa of max(0, v), rounded to nearest even; a finite value
// to the largest finite one at most.  0 where v is not positive (or NaN), and
// for the smallest subnormals, whose code is 1 all the same.
__device__ __forceinline__ int keep_steps(float v) {
    uint32_t b = __float_as_uint(v > 0.f ? v : 0.f);
    b = b < 0x7F800000u ? min(b, 0x7F7BFFFFu) : b;
    return (int)((b + 0x3FFFFu + ((b >> 19) & 1u)) >> 19);
}
__device__ __forceinline__ uint32_t keep_code(float v, int t, int e0) {
    return v > 0.f ? (uint32_t)max(t - 16 * e0 + 240, 1) : 0u;
}
// The value of a code (no block has a code that leads outside of fp32).
__device__ __forceinline__ float keep_value(uint32_t code, int e0) {
    return code ? __uint_as_float((code + 16u * (uint32_t)e0 - 240u) << 19) : 0.f;
}

// The largest of the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ int max_over_rows(int v) {
    const auto a = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
    const int m = max((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap((unsigned)m, (unsigned)m, false, false);
    return max((int)b[0], (int)b[1]);
}

// Four columns of gate and of up of a block that lanes l, l ^ 16, ... share:
// eight codes, gate's and up's in turn, and the two exponent bytes.  `in`: the
// columns exist.
__device__ __forceinline__ uint2 keep_four(f32x4 g, f32x4 u, bool in, uint32_t *exps) {
    int tg[4], tu[4], mg = 0, mu = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        tg[v] = keep_steps(g[v]);
        tu[v] = keep_steps(u[v]);
        mg = max(mg, tg[v]);
        mu = max(mu, tu[v]);
    }
    const int eg = max(15, max_over_rows(in ? mg : 0) >> 4), eu = max(15, max_over_rows(in ? mu : 0) >> 4);
    uint32_t c[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) c[v] = keep_code(g[v], tg[v], eg) | keep_code(u[v], tu[v], eu) << 8;
    *exps = (uint32_t)eg | (uint32_t)eu << 8;
    return uint2{c[0] | c[1] << 16, c[2] | c[3] << 16};
}

// Their values.
__device__ __forceinline__ void keep_values4(uint2 codes, uint32_t exps, f32x4 &g, f32x4 &u) {
    const int eg = exps & 255, eu = exps >> 8 & 255;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const uint32_t c = (v < 2 ? codes.x : codes.y) >> 16 * (v & 1);
        g[v] = keep_value(c & 255u, eg);
        u[v] = keep_value(c >> 8 & 255u, eu);
    }
}

}  // namespace ts
