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

#include <type_traits>

#include "ts_device.h"

namespace ts {

constexpr int kKeepBlock = 16;  // columns per exponent byte

// t of positive bits b (0: of what is not positive), a finite value's only up to
// the largest if SAT.
template <bool SAT>
__device__ __forceinline__ int keep_steps(uint32_t b) {
    if constexpr (SAT) b = b < 0x7F800000u ? min(b, 0x7F7BFFFFu) : b;
    return (int)((b + 0x3FFFFu + ((b >> 19) & 1u)) >> 19);
}

// V columns of gate and of up, whose block of 16 is in 16 / V neighbouring lanes: their
// codes, gate's and up's in turn, four columns a pair of words, the block's two exponent
// bytes, and c = max(0, gate) max(0, up).  `in`: the columns exist.  16 instructions a
// column (with comparisons instead of the median and the check for what overflows
// once a block, 32).
template <int V>
__device__ __forceinline__ uint32_t keep_codes(const float (&g)[V], const float (&u)[V], bool in, uint2 (&codes)[V / 4],
                                               float (&c)[V]) {
    uint32_t bg[V], bu[V];
    int tg[V], tu[V], mg, mu;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float x = fmaxf(g[v], 0.f), y = fmaxf(u[v], 0.f);  // (NaN: 0)
        c[v] = x * y;
        bg[v] = __float_as_uint(x);
        bu[v] = __float_as_uint(y);
    }
    auto steps = [&](auto sat) {
        mg = mu = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            tg[v] = keep_steps<decltype(sat)::value>(bg[v]);
            tu[v] = keep_steps<decltype(sat)::value>(bu[v]);
            mg = max(mg, tg[v]);
            mu = max(mu, tu[v]);
        }
        mg = in ? mg : 0;
        mu = in ? mu : 0;
        auto over = [&](auto ctrl) {
            mg = max(mg, __builtin_amdgcn_update_dpp(0, mg, decltype(ctrl)::value, 0xF, 0xF, false));
            mu = max(mu, __builtin_amdgcn_update_dpp(0, mu, decltype(ctrl)::value, 0xF, 0xF, false));
        };
        over(std::integral_constant<int, 0xB1>{});                        // quad_perm [1,0,3,2]
        if constexpr (V == 4) over(std::integral_constant<int, 0x4E>{});  // quad_perm [2,3,0,1]
    };
    steps(std::false_type{});
    if (__any(max(mg, mu) >= 0xFF0)) {
        // values that round to 2^128, infinities (times what is not positive: 0)
        steps(std::true_type{});
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = bg[v] && bu[v] ? c[v] : 0.f;
    }
    const int eg = max(15, mg >> 4), eu = max(15, mu >> 4), kg = 16 * eg - 240, ku = 16 * eu - 240;
    // max(1, t - k) where b > 0, otherwise (t = 0) 0: the middle one of t - k, 1 and b
    auto code = [](int t, int k, uint32_t b) { return (uint32_t)max(min(max(t - k, 1), (int)b), min(t - k, 1)); };
#pragma unroll
    for (int v = 0; v < V; v += 4) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = code(tg[v + i], kg, bg[v + i]) | code(tu[v + i], ku, bu[v + i]) << 8;
        codes[v / 4] = uint2{q[0] | q[1] << 16, q[2] | q[3] << 16};
    }
    return (uint32_t)eg | (uint32_t)eu << 8;
}

// Four columns' codes as values (of a code 0: some finite number), and which codes are
// not 0.  (No block has a code that leads outside of
// fp32.)
__device__ __forceinline__ void keep_values4(uint2 codes, uint32_t exps, float *g, float *u, bool *gate_on, bool *up_on) {
    const uint32_t kg = (16u * (exps & 255u) - 240u) << 19, ku = (16u * (exps >> 8 & 255u) - 240u) << 19;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const uint32_t c = v < 2 ? codes.x : codes.y, a = c >> 16 * (v & 1) & 255u, b = c >> (16 * (v & 1) + 8) & 255u;
        gate_on[v] = a != 0u;
        up_on[v] = b != 0u;
        g[v] = __uint_as_float((a << 19) + kg);
        u[v] = __uint_as_float((b << 19) + ku);
    }
}

}  // namespace ts
