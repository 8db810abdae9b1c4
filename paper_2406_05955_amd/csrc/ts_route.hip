// Routing of the MoE layer on any number of tokens: top-k with the softmax of
// the chosen logits, the stable order of (token, slot) pairs by expert, the
// combine of the experts' rows, and the gradients of both.
//
// All of it is bytes and latency.  One workgroup routes and sorts a small call
// in one launch.  A large one takes two: every workgroup routes its tokens and
// counts its pairs per expert; then every workgroup adds up the counts before
// its own and places its pairs.  16384 tokens, top 6 of 64: 9.2 + 4.7 us, the first
// bound by the top-k's instructions (a wave per token; four tokens' chains side by
// side), the rest launches (4 us each); 1 token 4.0 us.  No atomics on memory: the order is the pairs'
// own, the same on every run.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ts_gmm.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

namespace {

constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;

struct RouteArgs {
    const float *logits = nullptr;      // null: topk_idx is given
    const int32_t *idx_in = nullptr;
    int32_t *idx = nullptr;
    float *w = nullptr;
    int32_t *offsets = nullptr, *row_token = nullptr, *pair_row = nullptr;  // null: routing only
    int32_t *counts = nullptr;          // [workgroup][kMaxExperts]
    int T = 0, E = 0, K = 0, tpb = 0, blocks = 0;
};

// Order of logits as unsigned integers: larger is greater, NaN below
// everything, as -inf (lanes past the last expert: 0, below both).
__device__ __forceinline__ uint32_t logit_key(float v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x007fffffu;  // the key of -inf
    // -0 equals 0
    const uint32_t z = u == 0x80000000u ? 0u : u;
    return z & 0x80000000u ? ~z : z | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
    v = dpp_umax<0xB1>(v);
    v = dpp_umax<0x4E>(v);
    v = dpp_umax<0x124>(v);
    v = dpp_umax<0x128>(v);
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return max(max(a, b), max(c, d));
}

// U tokens by one wave, lane e holding expert e's logits: K times the largest
// that is left (ties: the lowest lane), then their softmax; the tokens' chains
// run side by side.  A token with nothing but -inf (or NaN) chooses the lowest
// experts, with weights of zero.  Lane k returns choice k and its weight.
template <int U>
__device__ __forceinline__ void route_tokens(const RouteArgs &a, const float (&logit)[U], int lane, int (&my_idx)[U],
                                             float (&my_w)[U]) {
    uint32_t key[U], my_key[U];
    float m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        key[u] = lane < a.E ? logit_key(logit[u]) : 0u;
        my_key[u] = 0x007fffffu;
        my_idx[u] = 0;
    }
    for (int k = 0; k < a.K; ++k) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t top = wave_umax(key[u]);
            const int who = __ffsll((unsigned long long)__ballot(key[u] == top)) - 1;
            if (k == 0) m[u] = key_logit(top);
            my_idx[u] = lane == k ? who : my_idx[u];
            my_key[u] = lane == k ? top : my_key[u];
            key[u] = lane == who ? 0u : key[u];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float l = key_logit(my_key[u]);
        // equal to the largest: 1 (inf - inf is no number)
        const float e = lane < a.K && m[u] > -INFINITY ? (l == m[u] ? 1.f : expf(l - m[u])) : 0.f;
        const float sum = wave_sum(e);
        my_w[u] = sum > 0.f ? e / sum : 0.f;
    }
}

// Places pairs [p0, p1) of this workgroup, whose expert e's first row is
// base[e] (lane e): waves take consecutive runs, count them, add up the counts
// of the waves before, then place 64 pairs at a time, each behind the lower
// lanes of its expert.
__device__ __forceinline__ void place_pairs(const RouteArgs &a, const int32_t *idx, int p0, int p1, int base,
                                            int (*cnt)[kMaxExperts], int wave, int lane) {
    const int per = ((p1 - p0 + kRouteWaves - 1) / kRouteWaves + 63) / 64 * 64;
    const int w0 = min(p0 + wave * per, p1), w1 = min(w0 + per, p1);
    cnt[wave][lane] = 0;
    __syncthreads();
    for (int p = w0 + lane; p < w1; p += 64) {
        const int e = idx[p];
        if (e >= 0 && e < a.E) atomicAdd(&cnt[wave][e], 1);  // (counts in LDS: the order does not matter)
    }
    __syncthreads();
    int at = base;
    for (int w = 0; w < wave; ++w) at += cnt[w][lane];
    for (int p = w0; p < w1; p += 64) {
        const int q = p + lane;
        const int e = q < w1 ? idx[q] : -1;
        const bool in = e >= 0 && e < a.E;
        // lanes whose pair has this lane's expert, and those that have expert `lane`
        uint64_t same = __ballot(in), mine = same;
#pragma unroll
        for (int bit = 0; bit < 6; ++bit) {
            const uint64_t set = __ballot(in && ((e >> bit) & 1));
            same &= (e >> bit) & 1 ? set : ~set;
            mine &= (lane >> bit) & 1 ? set : ~set;
        }
        const int row = __shfl(at, in ? e : 0) + lane_prefix(same, lane);
        if (in) a.row_token[row] = q / a.K;
        if (q < w1) a.pair_row[q] = in ? row : -1;
        at += __popcll(mine);
    }
}

}  // namespace

// The whole of a small call.
__global__ __launch_bounds__(kRouteThreads) void route_one(RouteArgs a) {
    __shared__ int cnt[kRouteWaves][kMaxExperts];
    __shared__ int s_idx[kRouteOneMax];
    __shared__ int total[kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pairs = a.T * a.K;
    if (a.logits) {
        for (int t = wave; t < a.T; t += kRouteWaves) {
            const float l[1] = {lane < a.E ? a.logits[(size_t)t * a.E + lane] : 0.f};
            int i[1];
            float w[1];
            route_tokens<1>(a, l, lane, i, w);
            if (lane < a.K) {
                a.idx[t * a.K + lane] = i[0];
                a.w[t * a.K + lane] = w[0];
                s_idx[t * a.K + lane] = i[0];
            }
        }
    } else {
        for (int p = tid; p < pairs; p += kRouteThreads) s_idx[p] = a.idx_in[p];
    }
    if (!a.offsets) return;
    if (tid < kMaxExperts) total[tid] = 0;
    __syncthreads();
    for (int p = tid; p < pairs; p += kRouteThreads)
        if (s_idx[p] >= 0 && s_idx[p] < a.E) atomicAdd(&total[s_idx[p]], 1);
    __syncthreads();
    const int mine = total[lane], scan = wave_scan<false>(mine);
    if (wave == 0) {
        if (lane == 0) a.offsets[0] = 0;
        if (lane < a.E) a.offsets[lane + 1] = scan;
    }
    place_pairs(a, s_idx, 0, pairs, scan - mine, cnt, wave, lane);
}

// First launch of a large call: routes this workgroup's tokens and counts its
// pairs per expert.
__global__ __launch_bounds__(kRouteThreads) void route_count(RouteArgs a) {
    __shared__ int total[kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = min(blockIdx.x * a.tpb, (unsigned)a.T), t1 = min(t0 + a.tpb, a.T);
    if (tid < kMaxExperts) total[tid] = 0;
    __syncthreads();
    if (a.logits) {
        constexpr int U = 4;
        for (int t = t0 + wave; t < t1; t += U * kRouteWaves) {
            float l[U], w[U];
            int i[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int tt = t + u * kRouteWaves;
                l[u] = tt < t1 && lane < a.E ? a.logits[(size_t)tt * a.E + lane] : 0.f;
            }
            route_tokens<U>(a, l, lane, i, w);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int tt = t + u * kRouteWaves;
                if (tt < t1 && lane < a.K) {
                    a.idx[(size_t)tt * a.K + lane] = i[u];
                    a.w[(size_t)tt * a.K + lane] = w[u];
                    atomicAdd(&total[i[u]], 1);  // (in LDS: the order does not matter)
                }
            }
        }
    } else {
        for (int p = t0 * a.K + tid; p < t1 * a.K; p += kRouteThreads) {
            const int e = a.idx_in[p];
            if (e >= 0 && e < a.E) atomicAdd(&total[e], 1);
        }
    }
    if (!a.offsets) return;
    __syncthreads();
    if (tid < kMaxExperts) a.counts[blockIdx.x * kMaxExperts + tid] = total[tid];
}

// Second launch: offsets, and the rows of this workgroup's pairs.
__global__ __launch_bounds__(kRouteThreads) void route_place(RouteArgs a) {
    __shared__ int cnt[kRouteWaves][kMaxExperts];
    __shared__ int all[kRouteWaves][kMaxExperts], before[kRouteWaves][kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int blk = blockIdx.x;
    const int t0 = min(blk * a.tpb, a.T), t1 = min(t0 + a.tpb, a.T);
    int n = 0, m = 0;
#pragma unroll 8
    for (int b = wave; b < a.blocks; b += kRouteWaves) {
        const int c = a.counts[b * kMaxExperts + lane];
        n += c;
        m += b < blk ? c : 0;
    }
    all[wave][lane] = n;
    before[wave][lane] = m;
    __syncthreads();
    int mine = 0, prior = 0;
#pragma unroll
    for (int w = 0; w < kRouteWaves; ++w) {
        mine += all[w][lane];
        prior += before[w][lane];
    }
    const int scan = wave_scan<false>(mine);
    if (blk == 0 && wave == 0) {
        if (lane == 0) a.offsets[0] = 0;
        if (lane < a.E) a.offsets[lane + 1] = scan;
    }
    place_pairs(a, a.logits ? a.idx : a.idx_in, t0 * a.K, t1 * a.K, scan - mine + prior, cnt, wave, lane);
}

// d_logits[t] = w_k (d_w_k - sum_j w_j d_w_j) at the chosen experts, 0
// elsewhere.  A lane writes V neighbouring elements; its token's K choices come
// from cache, all of them at once.  An expert listed twice takes both terms.
template <int V>
__global__ __launch_bounds__(256) void route_grad_kernel(const int32_t *idx, const float *w, const float *dw,
                                                         float *dl, int T, int E, int K) {
    const int per = E / V;
    const long long n = (long long)T * per, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int t = (int)(i / per), e = (int)(i - (long long)t * per) * V;
        int c[kMaxTopK];
        float p[kMaxTopK], d[kMaxTopK];
#pragma unroll
        for (int k = 0; k < kMaxTopK; ++k) {
            const size_t at = (size_t)t * K + min(k, K - 1);
            c[k] = k < K ? idx[at] : -1;
            p[k] = k < K ? w[at] : 0.f;
            d[k] = k < K ? dw[at] : 0.f;
        }
        float dot = 0.f, v[V] = {};
#pragma unroll
        for (int k = 0; k < kMaxTopK; ++k) dot += p[k] * d[k];
#pragma unroll
        for (int k = 0; k < kMaxTopK; ++k)
#pragma unroll
            for (int u = 0; u < V; ++u) v[u] += c[k] == e + u ? p[k] * (d[k] - dot) : 0.f;
        if constexpr (V == 4) *reinterpret_cast<f32x4 *>(dl + (size_t)t * E + e) = f32x4{v[0], v[1], v[2], v[3]};
        else dl[(size_t)t * E + e] = v[0];
    }
}

// out[t] = sum of w y over the token's rows.  A lane takes 8 columns of a token:
// bytes, 8192 tokens of 2 rows x 4096 bf16 31 us = 6.5 TB/s.
template <typename Y, typename O>
__global__ __launch_bounds__(256) void combine_kernel(const Y *y, const int32_t *pair_row, const float *w, O *out,
                                                      int T, int K, int H, int rows) {
    constexpr int CE = 8;  // values per lane: one 16-byte chunk of bf16, two of fp32
    const int per = H / CE + (H % CE ? 1 : 0);
    const long long n = (long long)T * per, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int t = (int)(i / per), c = (int)(i - (long long)t * per) * CE;
        float acc[CE] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const bool second = c + 4 < H;  // (fp32 rows of 4 more values)
        for (int k = 0; k < K; ++k) {
            const int r = pair_row[(size_t)t * K + k];
            if (r < 0 || r >= rows) continue;
            const float f = w ? w[(size_t)t * K + k] : 1.f;
            float v[CE] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const Y *p = y + (size_t)r * H + c;
            if constexpr (sizeof(Y) == 4) {
                unpack<float>(ld_cached(p), v);
                if (second) unpack<float>(ld_cached(p + 4), v + 4);
            } else {
                unpack<uint16_t>(ld_cached(p), v);
            }
#pragma unroll
            for (int e = 0; e < CE; ++e) acc[e] += f * v[e];
        }
        store4(out, sizeof(O) == 4, (size_t)t * H + c, f32x4{acc[0], acc[1], acc[2], acc[3]});
        if (second) store4(out, sizeof(O) == 4, (size_t)t * H + c + 4, f32x4{acc[4], acc[5], acc[6], acc[7]});
    }
}

// One token per workgroup: d_y[row] = w d_out[t] for its rows, d_w = their
// products with d_out[t], which is read once: 8192 tokens as above 54 us, 6.2 TB/s.
template <typename Y, typename O>
__global__ __launch_bounds__(256) void combine_grad_kernel(const O *d_out, const Y *y, const int32_t *pair_row,
                                                           const float *w, Y *d_y, float *d_w, int K, int H,
                                                           int rows) {
    constexpr int CE = 8;
    __shared__ float red[4][kMaxTopK];
    const int t = blockIdx.x, tid = threadIdx.x;
    float dot[kMaxTopK] = {};
    int row[kMaxTopK];
    float f[kMaxTopK];
#pragma unroll
    for (int k = 0; k < kMaxTopK; ++k) {
        const int r = k < K ? pair_row[(size_t)t * K + k] : -1;
        row[k] = r < rows ? r : -1;
        f[k] = k < K ? w[(size_t)t * K + k] : 0.f;
    }
    auto load = [&](const auto *p, bool second, float *v) {
        if constexpr (sizeof(*p) == 4) {
            unpack<float>(ld_cached(p), v);
            if (second) unpack<float>(ld_cached(p + 4), v + 4);
        } else {
            unpack<uint16_t>(ld_cached(p), v);
        }
    };
    for (int c = tid * CE; c < H; c += 256 * CE) {
        const bool second = c + 4 < H;
        float d[CE] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        load(d_out + (size_t)t * H + c, second, d);
#pragma unroll
        for (int k = 0; k < kMaxTopK; ++k) {
            if (row[k] < 0) continue;
            float v[CE] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const size_t at = (size_t)row[k] * H + c;
            load(y + at, second, v);
#pragma unroll
            for (int e = 0; e < CE; ++e) dot[k] += d[e] * v[e];
            store4(d_y, sizeof(Y) == 4, at, f32x4{f[k] * d[0], f[k] * d[1], f[k] * d[2], f[k] * d[3]});
            if (second)
                store4(d_y, sizeof(Y) == 4, at + 4, f32x4{f[k] * d[4], f[k] * d[5], f[k] * d[6], f[k] * d[7]});
        }
    }
#pragma unroll
    for (int k = 0; k < kMaxTopK; ++k) {
        if (k >= K) break;
        const float s = wave_sum(dot[k]);
        if ((tid & 63) == 0) red[tid >> 6][k] = s;
    }
    __syncthreads();
    if (tid < K) d_w[(size_t)t * K + tid] = (red[0][tid] + red[1][tid]) + (red[2][tid] + red[3][tid]);
}

namespace {

ts_status run_route(RouteArgs a, void *ws, size_t ws_bytes, hipStream_t st) {
    a.tpb = route_tokens_per_block(a.T, a.K);
    if (a.tpb == 0) {
        launch<RouteArgs>("moe_route", route_one, dim3(1), dim3(kRouteThreads), st, a);
        return check_launch("moe_route");
    }
    a.blocks = ceil_div(a.T, a.tpb);
    if (a.offsets) {
        if (!ws || ws_bytes < route_ws_bytes(a.T, a.E, a.K)) return TS_ERR_WORKSPACE;
        if (!aligned16(ws)) return TS_ERR_ALIGN;
        a.counts = static_cast<int32_t *>(ws);
    }
    launch<RouteArgs>("moe_route", route_count, dim3(a.blocks), dim3(kRouteThreads), st, a);
    ts_status s = check_launch("moe_route");
    if (s != TS_OK || !a.offsets) return s;
    launch<RouteArgs>("moe_place", route_place, dim3(a.blocks), dim3(kRouteThreads), st, a);
    return check_launch("moe_place");
}

ts_status check_maps(const int32_t *offsets, const int32_t *row_token, const int32_t *pair_row) {
    if (!aligned4(offsets) || !aligned4(row_token) || !aligned4(pair_row)) return TS_ERR_ALIGN;
    return TS_OK;
}

ts_status check_combine(int tokens, int top_k, int hidden, int rows, ts_dtype ydtype, ts_dtype odtype) {
    if (!type_ok(ydtype) || !type_ok(odtype)) return TS_ERR_DTYPE;
    const int q = ydtype == TS_BF16 || odtype == TS_BF16 ? 8 : 4;
    if (tokens < 0 || top_k < 1 || top_k > kMaxTopK || (long long)tokens * top_k > kMaxRows || rows < 0 ||
        rows > kMaxRows || hidden < q || hidden > kMaxDim || hidden % q != 0)
        return TS_ERR_SHAPE;
    return TS_OK;
}

template <typename F>
ts_status by_types(ts_dtype y, ts_dtype o, F f) {
    if (y == TS_F32) return o == TS_F32 ? f((float *)nullptr, (float *)nullptr) : f((float *)nullptr, (uint16_t *)nullptr);
    return o == TS_F32 ? f((uint16_t *)nullptr, (float *)nullptr) : f((uint16_t *)nullptr, (uint16_t *)nullptr);
}

}  // namespace

}  // namespace ts

extern "C" {

size_t ts_moe_route_workspace_bytes(int tokens, int n_experts, int top_k) {
    return ts::route_ws_bytes(tokens, n_experts, top_k);
}

ts_status ts_moe_route(const float *logits, int tokens, int n_experts, int top_k, int32_t *topk_idx, float *topk_w,
                       int32_t *offsets, int32_t *row_token, int32_t *pair_row, void *ws, size_t ws_bytes,
                       void *stream) {
    ts_status s = ts::check_route_dims(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if (tokens > 0 && (!logits || !topk_idx || !topk_w)) return TS_ERR_NULL;
    if ((offsets || row_token || pair_row) && (!offsets || (tokens > 0 && (!row_token || !pair_row))))
        return TS_ERR_NULL;
    if (!ts::aligned4(logits) || !ts::aligned4(topk_idx) || !ts::aligned4(topk_w)) return TS_ERR_ALIGN;
    s = ts::check_maps(offsets, row_token, pair_row);
    if (s != TS_OK) return s;
    if (tokens == 0 && !offsets) return TS_OK;
    ts::RouteArgs a;
    a.logits = logits;
    a.idx = topk_idx;
    a.w = topk_w;
    a.offsets = offsets;
    a.row_token = row_token;
    a.pair_row = pair_row;
    a.T = tokens;
    a.E = n_experts;
    a.K = top_k;
    return ts::run_route(a, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

ts_status ts_moe_group(const int32_t *topk_idx, int tokens, int n_experts, int top_k, int32_t *offsets,
                       int32_t *row_token, int32_t *pair_row, void *ws, size_t ws_bytes, void *stream) {
    ts_status s = ts::check_route_dims(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if (!offsets || (tokens > 0 && (!topk_idx || !row_token || !pair_row))) return TS_ERR_NULL;
    if (!ts::aligned4(topk_idx)) return TS_ERR_ALIGN;
    s = ts::check_maps(offsets, row_token, pair_row);
    if (s != TS_OK) return s;
    ts::RouteArgs a;
    a.idx_in = topk_idx;
    a.offsets = offsets;
    a.row_token = row_token;
    a.pair_row = pair_row;
    a.T = tokens;
    a.E = n_experts;
    a.K = top_k;
    return ts::run_route(a, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

ts_status ts_moe_route_grad(const int32_t *topk_idx, const float *topk_w, const float *d_w, int tokens, int n_experts,
                            int top_k, float *d_logits, void *stream) {
    ts_status s = ts::check_route_dims(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if (tokens == 0) return TS_OK;
    if (!topk_idx || !topk_w || !d_w || !d_logits) return TS_ERR_NULL;
    if (!ts::aligned4(topk_idx) || !ts::aligned4(topk_w) || !ts::aligned4(d_w) || !ts::aligned4(d_logits))
        return TS_ERR_ALIGN;
    const bool four = n_experts % 4 == 0 && ts::aligned16(d_logits);
    const long long n = (long long)tokens * (four ? n_experts / 4 : n_experts);
    const unsigned grid = (unsigned)std::min<long long>((n + 255) / 256, 256 * 16);
    ts::launch<const int32_t *, const float *, const float *, float *, int, int, int>(
        "moe_route_grad", four ? ts::route_grad_kernel<4> : ts::route_grad_kernel<1>, dim3(grid), dim3(256),
        static_cast<hipStream_t>(stream), topk_idx, topk_w, d_w, d_logits, tokens, n_experts, top_k);
    return ts::check_launch("moe_route_grad");
}

ts_status ts_moe_combine(const void *y, ts_dtype ydtype, const int32_t *pair_row, const float *w, int tokens,
                         int top_k, int hidden, int rows, void *out, ts_dtype odtype, void *stream) {
    ts_status s = ts::check_combine(tokens, top_k, hidden, rows, ydtype, odtype);
    if (s != TS_OK) return s;
    if (tokens == 0) return TS_OK;
    if ((rows > 0 && !y) || !pair_row || !out) return TS_ERR_NULL;
    if (!ts::aligned16(y) || !ts::aligned16(out) || !ts::aligned4(pair_row) || !ts::aligned4(w)) return TS_ERR_ALIGN;
    const long long n = (long long)tokens * ts::ceil_div(hidden, 8);
    const unsigned grid = (unsigned)std::min<long long>((n + 255) / 256, 256 * 64);
    return ts::by_types(ydtype, odtype, [&](auto *yp, auto *op) {
        using Y = std::remove_pointer_t<decltype(yp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        ts::launch<const Y *, const int32_t *, const float *, O *, int, int, int, int>(
            "moe_combine", ts::combine_kernel<Y, O>, dim3(grid), dim3(256), static_cast<hipStream_t>(stream),
            static_cast<const Y *>(y), pair_row, w, static_cast<O *>(out), tokens, top_k, hidden, rows);
        return ts::check_launch("moe_combine");
    });
}

ts_status ts_moe_combine_grad(const void *d_out, ts_dtype odtype, const void *y, ts_dtype ydtype,
                              const int32_t *pair_row, const float *w, int tokens, int top_k, int hidden, int rows,
                              void *d_y, float *d_w, void *stream) {
    ts_status s = ts::check_combine(tokens, top_k, hidden, rows, ydtype, odtype);
    if (s != TS_OK) return s;
    if (tokens == 0) return TS_OK;
    if (!d_out || (rows > 0 && (!y || !d_y)) || !pair_row || !w || !d_w) return TS_ERR_NULL;
    if (!ts::aligned16(d_out) || !ts::aligned16(y) || !ts::aligned16(d_y) || !ts::aligned4(pair_row) ||
        !ts::aligned4(w) || !ts::aligned4(d_w))
        return TS_ERR_ALIGN;
    return ts::by_types(ydtype, odtype, [&](auto *yp, auto *op) {
        using Y = std::remove_pointer_t<decltype(yp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        ts::launch<const O *, const Y *, const int32_t *, const float *, Y *, float *, int, int, int>(
            "moe_combine_grad", ts::combine_grad_kernel<Y, O>, dim3(tokens), dim3(256),
            static_cast<hipStream_t>(stream), static_cast<const O *>(d_out), static_cast<const Y *>(y), pair_row, w,
            static_cast<Y *>(d_y), d_w, top_k, hidden, rows);
        return ts::check_launch("moe_combine_grad");
    });
}

}  // extern "C"
