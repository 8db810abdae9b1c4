// The router's balance loss: counts per expert, the loss over the softmax of all
// experts, the squared log-sum (z) term, and the logits' gradient.
//
//   n tokens count, p = softmax of a token's logits, lse = log sum exp of them,
//   f_e = counts[e] / (K n), P_e = sum_t p[t][e] / n
//   loss[0] = E sum_e f_e P_e, loss[1] = sum_t lse^2 / n
//   d_logits[t][e] = p (d0 E / n (f_e - sum_j f_j p_j) + d1 2 / n lse)
//
// Bytes and latency: the logits are read once forward and once backward.  L lanes of
// a wave hold a token, four experts each, so that a load is 16 bytes a lane and
// a wave has 64 / L tokens' chains side by side.  Sums go lane, wave, workgroup, grid in
// a fixed order: the same bits on every run.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>

#include "ts_device.h"
#include "ts_group.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

namespace {

constexpr int kBalThreads = 1024, kBalWaves = kBalThreads / 64;  // loss
constexpr int kMaxBalBlocks = 256;
constexpr int kGradThreads = 256, kGradWaves = kGradThreads / 64;

struct BalArgs {
    const float *logits = nullptr;
    const int32_t *idx = nullptr;
    const uint8_t *mask = nullptr;
    float *part = nullptr;      // [workgroup][kMaxExperts]: sums of p
    int32_t *cpart = nullptr;   // [workgroup][kMaxExperts]: counts
    float *zpart = nullptr;     // [workgroup]: sum of lse^2
    int32_t *npart = nullptr;   // [workgroup]: tokens
    float *loss = nullptr;
    int32_t *counts = nullptr;  // [E + 1]
    const float *d_loss = nullptr, *add = nullptr;
    float *out = nullptr;
    int T = 0, E = 0, K = 0, blocks = 0, four = 0;
};

// Reductions over the L lanes (a power of two up to 16) that hold a token.
template <int L, typename F>
__device__ __forceinline__ float over_lanes(float v, F op) {
    if constexpr (L > 1) v = op(v, dpp_f32<0xB1>(v));    // quad_perm [1,0,3,2]
    if constexpr (L > 2) v = op(v, dpp_f32<0x4E>(v));    // quad_perm [2,3,0,1]
    if constexpr (L > 4) v = op(v, dpp_f32<0x141>(v));   // row_half_mirror
    if constexpr (L > 8) v = op(v, dpp_f32<0x140>(v));   // row_mirror
    return v;
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
    return over_lanes<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
    return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

// Four logits of token t, from expert e on; NaN and what lies past the last
// expert are -inf.
__device__ __forceinline__ void load_logits(const BalArgs &a, int t, int e, bool in, float (&l)[4]) {
    const float *p = a.logits + (size_t)t * a.E + e;
    if (a.four && in && e < a.E) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = in && e + i < a.E ? p[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;
}

// Softmax of a token's logits in place, its log-sum, with the hardware's exp2, log2 and
// reciprocal (a unit or two in the last place each; the difference to the largest is
// multiplied once): the forward pass's time is its instructions.  Whether it counts: the mask
// leaves it and a logit above the lowest finite value.
template <int L>
__device__ __forceinline__ bool soft(float (&l)[4], bool in, float &lse) {
    const float m = lanes_max<L>(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])));
    in = in && m > -FLT_MAX;
    // (equal to the largest: 1, an infinite one too)
#pragma unroll
    for (int i = 0; i < 4; ++i) l[i] = l[i] == m ? 1.f : __builtin_amdgcn_exp2f((l[i] - m) * 1.44269504f);
    const float s = lanes_sum<L>((l[0] + l[1]) + (l[2] + l[3]));
    const float r = in ? __builtin_amdgcn_rcpf(s) : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) l[i] = in ? l[i] * r : 0.f;
    lse = in ? m + __builtin_amdgcn_logf(s) * 0.693147181f : 0.f;
    return in;
}

// Sum over the lanes l, l + L, l + 2 L, ... of the wave, in every one of them.
template <int L>
__device__ __forceinline__ float over_tokens(float v) {
#pragma unroll
    for (int d = L; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

}  // namespace

// loss from the sums of p and of lse^2 (lane e: expert e's; all lanes: z) and the
// counts, by one wave.
__device__ __forceinline__ void finish_loss(const BalArgs &a, int lane, double p, double z, int count, int n) {
    const double nn = n > 0 ? (double)n : 1.0;
    double f = lane < a.E ? (double)count / ((double)a.K * nn) * (p / nn) : 0.0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) f += __shfl_xor(f, d);
    if (lane == 0) {
        a.loss[0] = (float)(a.E * f);
        a.loss[1] = (float)(z / nn);
        a.counts[a.E] = n;
    }
    if (lane < a.E) a.counts[lane] = count;
}

// A wave takes 64 / L tokens at once, U rounds of them with their loads on their way
// together (one after another, 200001 tokens of 64 experts 29 us; this 19, with the
// hardware's exp2 and log2 14).
template <int L>
__global__ __launch_bounds__(kBalThreads) void balance_kernel(BalArgs a) {
    constexpr int G = 64 / L, U = 2, KL = (kMaxTopK + L - 1) / L;  // choices of a token a lane
    __shared__ int cnt[kMaxExperts + 1];
    __shared__ float sum[kBalWaves][4 * L + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sub = lane & (L - 1), tok = lane / L;
    for (int i = tid; i < kMaxExperts + 1; i += kBalThreads) cnt[i] = 0;
    __syncthreads();
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, z = 0.f;
    int n = 0;
    const int step = a.blocks * kBalWaves * G;
    // (whole waves stay in the loop: a token's lanes exchange their maxima)
    for (int t0 = (blockIdx.x * kBalWaves + wave) * G; t0 < a.T; t0 += U * step) {
        float l[U][4], lse[U];
        int e[U][KL];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * step + tok;
            in[u] = t < a.T;
            const int tt = in[u] ? t : 0;
            if (a.mask) in[u] = in[u] && a.mask[tt] != 0;
            load_logits(a, tt, sub * 4, in[u], l[u]);
#pragma unroll
            for (int k = 0; k < KL; ++k) {
                const bool have = in[u] && sub + k * L < a.K;
                e[u][k] = have ? a.idx[(size_t)tt * a.K + sub + k * L] : -1;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            in[u] = soft<L>(l[u], in[u], lse[u]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += l[u][i];
            z += lse[u] * lse[u];
            n += in[u] ? 1 : 0;
#pragma unroll
            for (int k = 0; k < KL; ++k)
                if (in[u] && e[u][k] >= 0 && e[u][k] < a.E) atomicAdd(&cnt[e[u][k]], 1);  // (in LDS: the order does not matter)
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = over_tokens<L>(acc[i]);
    z = over_tokens<L>(z);
    if (sub == 0 && n) atomicAdd(&cnt[kMaxExperts], n);
    if (lane < L) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[wave][4 * lane + i] = acc[i];
        if (lane == 0) sum[wave][4 * L] = z;
    }
    __syncthreads();
    if (wave > 0) return;
    float p = 0.f;
    z = 0.f;
#pragma unroll
    for (int w = 0; w < kBalWaves; ++w) {
        p += lane < 4 * L ? sum[w][lane] : 0.f;
        z += sum[w][4 * L];
    }
    if (a.blocks == 1) {
        finish_loss(a, lane, p, z, cnt[lane], cnt[kMaxExperts]);
        return;
    }
    a.part[blockIdx.x * kMaxExperts + lane] = p;
    a.cpart[blockIdx.x * kMaxExperts + lane] = cnt[lane];
    if (lane == 0) {
        a.zpart[blockIdx.x] = z;
        a.npart[blockIdx.x] = cnt[kMaxExperts];
    }
}

// The workgroups' sums (256 at most): a wave takes every 16th of them, all its loads
// on their way together, then wave 0 the waves'.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalArgs a) {
    constexpr int N = kMaxBalBlocks / 16;
    __shared__ double s_p[16][64];
    __shared__ int s_c[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float v[N];
    int w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int b = min(wave + 16 * i, a.blocks - 1);
        v[i] = a.part[b * kMaxExperts + lane];
        w[i] = a.cpart[b * kMaxExperts + lane];
    }
    double z = 0.0;
    int n = 0;
    if (wave == 0) {
        float zv[kMaxBalBlocks / 64];
        int nv[kMaxBalBlocks / 64];
#pragma unroll
        for (int i = 0; i < kMaxBalBlocks / 64; ++i) {
            const int b = min(64 * i + lane, a.blocks - 1);
            zv[i] = a.zpart[b];
            nv[i] = a.npart[b];
        }
#pragma unroll
        for (int i = 0; i < kMaxBalBlocks / 64; ++i) {
            z += 64 * i + lane < a.blocks ? (double)zv[i] : 0.0;
            n += 64 * i + lane < a.blocks ? nv[i] : 0;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            z += __shfl_xor(z, d);
            n += __shfl_xor(n, d);
        }
    }
    double p = 0.0;
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p += wave + 16 * i < a.blocks ? (double)v[i] : 0.0;
        c += wave + 16 * i < a.blocks ? w[i] : 0;
    }
    s_p[wave][lane] = p;
    s_c[wave][lane] = c;
    __syncthreads();
    if (wave > 0) return;
    p = 0.0;
    c = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        p += s_p[i][lane];
        c += s_c[i][lane];
    }
    finish_loss(a, lane, p, z, c, n);
}

template <int L>
__global__ __launch_bounds__(kGradThreads) void balance_grad_kernel(BalArgs a) {
    constexpr int G = 64 / L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane & (L - 1), tok = lane / L, e = sub * 4;
    const int n = a.counts[a.E];
    const float rn = n > 0 ? 1.f / (float)n : 0.f;
    const float d0 = a.d_loss[0] * (float)a.E * rn, d1 = a.d_loss[1] * 2.f * rn;
    const float kn = n > 0 ? 1.f / ((float)a.K * (float)n) : 0.f;
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = e + i < a.E ? (float)a.counts[e + i] * kn : 0.f;
    const int step = gridDim.x * kGradWaves * G;
    for (int t0 = (blockIdx.x * kGradWaves + wave) * G; t0 < a.T; t0 += step) {
        const int t = t0 + tok;
        const bool have = t < a.T;
        bool in = have;
        if (a.mask) in = in && a.mask[in ? t : 0] != 0;
        float l[4], lse;
        load_logits(a, t, e, in, l);
        in = soft<L>(l, in, lse);
        const float dot = lanes_sum<L>((f[0] * l[0] + f[1] * l[1]) + (f[2] * l[2] + f[3] * l[3]));
        // (no z gradient: an infinite log-sum leaves nothing)
        const float zt = d1 != 0.f ? d1 * lse : 0.f;
        if (!have) continue;
        float d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = in ? l[i] * (d0 * (f[i] - dot) + zt) : 0.f;
        const size_t at = (size_t)t * a.E + e;
        if (a.four) {
            if (e >= a.E) continue;
            f32x4 o = {d[0], d[1], d[2], d[3]};
            if (a.add) o += *reinterpret_cast<const f32x4 *>(a.add + at);
            *reinterpret_cast<f32x4 *>(a.out + at) = o;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e + i < a.E) a.out[at + i] = (a.add ? a.add[at + i] : 0.f) + d[i];
        }
    }
}

namespace {

// Lanes that hold a token's logits.
int lanes_of(int E) {
    int L = 1;
    while (4 * L < E) L *= 2;
    return L;
}

// Workgroups: one takes up to 4 rounds (1024 tokens of 16 experts; another launch adds up
// several ones' sums); above that one a unit.
int balance_blocks(int T, int E) {
    const int round = kBalThreads / lanes_of(E);
    return T <= 4 * round ? 1 : std::min(ceil_div(T, round), kMaxBalBlocks);
}

size_t balance_ws_bytes(int T, int E, int K) {
    if (check_route_dims(T, E, K) != TS_OK) return 0;
    const int b = balance_blocks(T, E);
    return b == 1 ? 0 : align_up256((size_t)b * (kMaxExperts + 1) * 8);
}

template <typename F>
void by_lanes(int E, F f) {
    switch (lanes_of(E)) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 8: return f(std::integral_constant<int, 8>{});
        default: return f(std::integral_constant<int, 16>{});
    }
}

}  // namespace

}  // namespace ts

extern "C" {

size_t ts_moe_balance_workspace_bytes(int tokens, int n_experts, int top_k) {
    return ts::balance_ws_bytes(tokens, n_experts, top_k);
}

ts_status ts_moe_balance(const float *logits, const int32_t *topk_idx, const uint8_t *mask, int tokens, int n_experts,
                         int top_k, float *loss, int32_t *counts, void *ws, size_t ws_bytes, void *stream) {
    ts_status s = ts::check_route_dims(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if ((tokens > 0 && (!logits || !topk_idx)) || !loss || !counts) return TS_ERR_NULL;
    if (!ts::aligned4(logits) || !ts::aligned4(topk_idx) || !ts::aligned4(loss) || !ts::aligned4(counts))
        return TS_ERR_ALIGN;
    ts::BalArgs a;
    a.logits = logits;
    a.idx = topk_idx;
    a.mask = mask;
    a.loss = loss;
    a.counts = counts;
    a.T = tokens;
    a.E = n_experts;
    a.K = top_k;
    a.four = n_experts % 4 == 0 && ts::aligned16(logits);
    a.blocks = ts::balance_blocks(tokens, n_experts);
    if (a.blocks > 1) {
        if (!ws || ws_bytes < ts::balance_ws_bytes(tokens, n_experts, top_k)) return TS_ERR_WORKSPACE;
        if (!ts::aligned16(ws)) return TS_ERR_ALIGN;
        a.part = static_cast<float *>(ws);
        a.cpart = reinterpret_cast<int32_t *>(a.part + (size_t)a.blocks * ts::kMaxExperts);
        a.zpart = reinterpret_cast<float *>(a.cpart + (size_t)a.blocks * ts::kMaxExperts);
        a.npart = reinterpret_cast<int32_t *>(a.zpart + a.blocks);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    ts::by_lanes(n_experts, [&](auto l) {
        ts::launch<ts::BalArgs>("moe_balance", ts::balance_kernel<l>, dim3(a.blocks), dim3(ts::kBalThreads), st, a);
    });
    s = ts::check_launch("moe_balance");
    if (s != TS_OK || a.blocks == 1) return s;
    ts::launch<ts::BalArgs>("moe_balance_sum", ts::balance_finish_kernel, dim3(1), dim3(1024), st, a);
    return ts::check_launch("moe_balance_sum");
}

ts_status ts_moe_balance_grad(const float *logits, const int32_t *counts, const float *d_loss, const uint8_t *mask,
                              const float *add, int tokens, int n_experts, int top_k, float *d_logits, void *stream) {
    ts_status s = ts::check_route_dims(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if (tokens == 0) return TS_OK;
    if (!logits || !counts || !d_loss || !d_logits) return TS_ERR_NULL;
    if (!ts::aligned4(logits) || !ts::aligned4(counts) || !ts::aligned4(d_loss) || !ts::aligned4(add) ||
        !ts::aligned4(d_logits))
        return TS_ERR_ALIGN;
    ts::BalArgs a;
    a.logits = logits;
    a.counts = const_cast<int32_t *>(counts);  // (read)
    a.d_loss = d_loss;
    a.mask = mask;
    a.add = add;
    a.out = d_logits;
    a.T = tokens;
    a.E = n_experts;
    a.K = top_k;
    a.four = n_experts % 4 == 0 && ts::aligned16(logits) && ts::aligned16(d_logits) && ts::aligned16(add);
    const int round = ts::kGradThreads / ts::lanes_of(n_experts);
    const int grid = std::min(ts::ceil_div(tokens, round), 256 * 8);
    ts::by_lanes(n_experts, [&](auto l) {
        ts::launch<ts::BalArgs>("moe_balance_grad", ts::balance_grad_kernel<l>, dim3(grid), dim3(ts::kGradThreads),
                                static_cast<hipStream_t>(stream), a);
    });
    return ts::check_launch("moe_balance_grad");
}

}  // extern "C"
