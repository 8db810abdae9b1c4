// Low-rank adapters of many requests beside a shared projection:
//   y[r] = x[r] W^T + s_a (x[r] A_a^T) B_a^T,  a = adapter of r's segment (or none)
// and the same in front of dReLU for gate and up.
//
// Two launches.  adapter_rows computes t = s_a x A_a^T, `rank` values a row (a
// few ranks, a long contraction).  The product then contracts t with B behind x with
// W, in the same accumulators (gmm_tiled's adapter steps): y is written once and nothing is
// read twice.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ts_gmm.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

namespace {

struct AdaptRowsArgs {
    const char *x = nullptr, *a[2] = {nullptr, nullptr};
    const float *scale = nullptr;
    const int32_t *offsets = nullptr, *adapter = nullptr;
    char *t = nullptr;
    int32_t *ids = nullptr;
    int rows = 0, segs = 0, adapters = 0, rank = 0, ranks = 0, parts = 1, k = 0;  // ranks: of both matrices
};

// Segment s's rows in pieces of Q: its first piece has the number offsets[s] / Q +
// s, which no other segment's piece has (a segment's pieces are at most its rows / Q
// + 1), so the pieces need no count of those before.  This finds the last s whose
// first piece is not behind piece `p`: 64 probes a round.
template <int Q>
__device__ __forceinline__ int segment_of(const AdaptRowsArgs &a, int p, int lane) {
    auto first = [&](int s) { return min(max(a.offsets[s], 0), a.rows) / Q + s; };
    int lo = 0, hi = a.segs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, s = lo + lane * step;
        const bool ok = s < hi && first(min(s, hi - 1)) <= p;
        const int n = max(__popcll(__ballot(ok)), 1);
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

}  // namespace

// t of up to 16 RT rows of a segment and 16 NR ranks; W waves share the contraction,
// their sums are added in a fixed order.
template <GmmKind KIND, int RT, int NR, int W>
__global__ __launch_bounds__(64 * W) void adapter_rows(AdaptRowsArgs a) {
    constexpr int SZ = GmmElem<KIND>::SZ, KS = 64 / SZ, CE = 16 / SZ, Q = 16 * RT;
    constexpr int U = RT * NR == 1 ? 8 : RT * NR <= 8 ? 4 : 2;  // steps whose loads are on their way together
    __shared__ f32x4 red[W][RT * NR][64];
    const int lane = threadIdx.x & 63, lm = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int seg = __builtin_amdgcn_readfirstlane(segment_of<Q>(a, blockIdx.x, lane));
    const int b = min(max(a.offsets[seg], 0), a.rows), e = min(max(a.offsets[seg + 1], 0), a.rows);
    const int piece = (int)blockIdx.x - (b / Q + seg);
    if (piece < 0 || b + (long long)piece * Q >= e) return;
    const int r0 = b + piece * Q, r1 = min(r0 + Q, e);
    const int id = a.adapter[seg];
    const bool none = id < 0 || id >= a.adapters;
    if (blockIdx.y == 0 && (int)threadIdx.x < r1 - r0) a.ids[r0 + threadIdx.x] = none ? -1 : id;
    if (none) return;

    const size_t row_bytes = (size_t)a.k * SZ;
    const char *ar[NR], *xr[RT];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const int r = min(((int)blockIdx.y * NR + f) * 16 + lm, a.ranks - 1);
        const bool second = r >= a.rank;
        ar[f] = a.a[second] + ((size_t)id * a.rank + (second ? r - a.rank : r)) * row_bytes;
    }
#pragma unroll
    for (int j = 0; j < RT; ++j) xr[j] = a.x + (size_t)min(r0 + j * 16 + lm, r1 - 1) * row_bytes;
    const int steps = (a.k + KS - 1) / KS, per = (steps + W - 1) / W;
    const int s0 = wave * per, s1 = min(s0 + per, steps);
    f32x4 acc[NR][RT] = {};
    for (int s = s0; s < s1; s += U) {
        u32x4 af[U][NR], xf[U][RT];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + u) * KS + lq * CE;
            in[u] = s + u < s1 && k < a.k;
            const size_t at = (size_t)min(k, a.k - CE) * SZ;
#pragma unroll
            for (int f = 0; f < NR; ++f) af[u][f] = ld_cached(ar[f] + at);
#pragma unroll
            for (int j = 0; j < RT; ++j) xf[u][j] = ld_cached(xr[j] + at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int f = 0; f < NR; ++f) af[u][f] = in[u] ? af[u][f] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < RT; ++j) xf[u][j] = in[u] ? xf[u][j] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int f = 0; f < NR; ++f)
#pragma unroll
                for (int j = 0; j < RT; ++j) acc[f][j] = mma<KIND>(af[u][f], xf[u][j], acc[f][j]);
        }
    }
#pragma unroll
    for (int f = 0; f < NR; ++f)
#pragma unroll
        for (int j = 0; j < RT; ++j) red[wave][f * RT + j][lane] = acc[f][j];
    __syncthreads();
    const float scale = a.scale ? a.scale[id] : 1.f;
    for (int i = wave; i < NR * RT; i += W) {
        f32x4 v = red[0][i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) v += red[w][i][lane];
        v *= scale;
        // lane (lm, lq): ranks 4 lq ... of row lm
        const int row = r0 + i % RT * 16 + lm, r = ((int)blockIdx.y * NR + i / RT) * 16 + 4 * lq;
        if (row >= r1 || r >= a.ranks) continue;
        const size_t at = (size_t)row * a.ranks * a.parts + r;
        store4(a.t, KIND == kGmmF32, at, v);
        if (KIND == kGmmBf16 && a.parts == 2) {
            // what the first rounding left (nothing of what has no remainder)
            f32x4 rest;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float hi = (float)(__bf16)v[c];
                rest[c] = fabsf(hi) < INFINITY ? v[c] - hi : 0.f;
            }
            store4(a.t, 0, at + a.ranks, rest);
        }
    }
}

namespace {

constexpr int kMaxRank = 128;

// The ranks' intermediate: bf16 operands hold t in one bf16 where the output is
// rounded to bf16 as well, and in two (16 significant bits) where it is fp32: one
// rounding of t is 2^-9 of the adapter's share.
int adapt_parts(ts_dtype dtype, ts_dtype odtype) { return dtype == TS_BF16 && odtype == TS_F32 ? 2 : 1; }

size_t adapt_t_bytes(int rows, int rank, int products, ts_dtype dtype, ts_dtype odtype) {
    return align_up256((size_t)rows * rank * products * adapt_parts(dtype, odtype) * (dtype == TS_F32 ? 4 : 2));
}

bool adapt_dims_ok(int rows, int rank, ts_dtype dtype) {
    return rows >= 0 && rows <= kMaxRows && rank >= quantum(dtype) && rank <= kMaxRank && rank % quantum(dtype) == 0;
}

size_t adapt_ws_bytes(int rows, int rank, int products, ts_dtype dtype, ts_dtype odtype) {
    if (!type_ok(dtype) || !type_ok(odtype) || products < 1 || products > 2 || !adapt_dims_ok(rows, rank, dtype)) return 0;
    return adapt_t_bytes(rows, rank, products, dtype, odtype) + align_up256((size_t)rows * 4);
}

struct AdaptCall {
    const void *x, *w[2], *a[2], *b[2];
    const float *scale;
    const int32_t *offsets, *adapter;
    ts_dtype dtype, odtype;
    int w_kn, products, rows, segments, adapters, rank, n, k;
    void *out, *ws;
    size_t ws_bytes;
    hipStream_t stream;
};

template <GmmKind KIND, int RT, int NR, int W>
ts_status run_rows(const AdaptRowsArgs &r, hipStream_t st) {
    const long long pieces = (long long)r.rows / (16 * RT) + r.segs;
    const int tall = ceil_div(r.ranks, 16 * NR);
    if (pieces * tall * 64 * W >= (1LL << 32)) return TS_ERR_UNSUPPORTED;
    launch<AdaptRowsArgs>("adapter_rows", adapter_rows<KIND, RT, NR, W>, dim3((unsigned)pieces, tall), dim3(64 * W), st, r);
    return check_launch("adapter_rows");
}

template <GmmKind KIND>
ts_status run_adapt(const AdaptCall &c) {
    AdaptRowsArgs r;
    r.x = static_cast<const char *>(c.x);
    for (int i = 0; i < c.products; ++i) r.a[i] = static_cast<const char *>(c.a[i]);
    r.scale = c.scale;
    r.offsets = c.offsets;
    r.adapter = c.adapter;
    r.t = static_cast<char *>(c.ws);
    r.ids = reinterpret_cast<int32_t *>(r.t + adapt_t_bytes(c.rows, c.rank, c.products, c.dtype, c.odtype));
    r.rows = c.rows;
    r.segs = c.segments;
    r.adapters = c.adapters;
    r.rank = c.rank;
    r.ranks = c.rank * c.products;
    r.parts = adapt_parts(c.dtype, c.odtype);
    r.k = c.k;
    ts_status s;
    if (c.rows < 16LL * c.segments) s = run_rows<KIND, 1, 1, 16>(r, c.stream);
    else if (r.ranks <= 16) s = run_rows<KIND, 4, 1, 8>(r, c.stream);
    else s = run_rows<KIND, 4, 4, 4>(r, c.stream);
    if (s != TS_OK) return s;

    GmmAdaptArgs a;
    a.x[0] = static_cast<const char *>(c.x);
    for (int i = 0; i < c.products; ++i) {
        a.w[i] = static_cast<const char *>(c.w[i]);
        a.b[i] = static_cast<const char *>(c.b[i]);
    }
    a.offsets = c.offsets;
    a.rows = a.src_rows = c.rows;
    a.n = c.n;
    a.k = c.k;
    a.out = c.out;
    a.out_f32 = c.odtype == TS_F32;
    a.t = r.t;
    a.ids = r.ids;
    a.segs = c.segments;
    a.adapters = c.adapters;
    a.rank = c.rank;
    a.parts = r.parts;
    if (c.products == 2) return run_fwd<KIND, kDreluAdapt, false>("adapter_drelu", a, c.stream);
    return c.w_kn ? run_fwd<KIND, kFwdAdapt, true>("adapter_mm", a, c.stream)
                  : run_fwd<KIND, kFwdAdapt, false>("adapter_mm", a, c.stream);
}

ts_status adapt(const AdaptCall &c) {
    if (!type_ok(c.dtype) || !type_ok(c.odtype)) return TS_ERR_DTYPE;
    ts_status s = check_group_dims(c.rows, 1, c.n, c.k, quantum(c.dtype));
    if (s != TS_OK) return s;
    if (!adapt_dims_ok(c.rows, c.rank, c.dtype) || c.segments < 0 || c.segments > kMaxRows || c.adapters < 1 ||
        c.adapters > kMaxRows)
        return TS_ERR_SHAPE;
    if (c.rows == 0 || c.segments == 0) return TS_OK;
    if (!c.x || !c.offsets || !c.adapter || !c.out) return TS_ERR_NULL;
    if (!aligned16(c.x) || !aligned4(c.offsets) || !aligned4(c.adapter) || !aligned4(c.scale) || !aligned16(c.out))
        return TS_ERR_ALIGN;
    for (int i = 0; i < c.products; ++i) {
        if (!c.w[i] || !c.a[i] || !c.b[i]) return TS_ERR_NULL;
        if (!aligned16(c.w[i]) || !aligned16(c.a[i]) || !aligned16(c.b[i])) return TS_ERR_ALIGN;
    }
    if (!c.ws || c.ws_bytes < adapt_ws_bytes(c.rows, c.rank, c.products, c.dtype, c.odtype)) return TS_ERR_WORKSPACE;
    if (!aligned16(c.ws)) return TS_ERR_ALIGN;
    return c.dtype == TS_BF16 ? run_adapt<kGmmBf16>(c) : run_adapt<kGmmF32>(c);
}

}  // namespace

}  // namespace ts

extern "C" {

size_t ts_adapter_workspace_bytes(int rows, int rank, int products, ts_dtype dtype, ts_dtype odtype) {
    return ts::adapt_ws_bytes(rows, rank, products, dtype, odtype);
}

ts_status ts_adapter_mm(const void *x, const void *w, const void *a, const void *b, const float *scale, ts_dtype dtype,
                        int w_kn, const int32_t *offsets, const int32_t *adapter, int rows, int segments,
                        int n_adapters, int rank, int n, int k, void *out, ts_dtype odtype, void *ws, size_t ws_bytes,
                        void *stream) {
    return ts::adapt({x, {w, nullptr}, {a, nullptr}, {b, nullptr}, scale, offsets, adapter, dtype, odtype, w_kn, 1, rows,
                      segments, n_adapters, rank, n, k, out, ws, ws_bytes, static_cast<hipStream_t>(stream)});
}

ts_status ts_adapter_drelu(const void *x, const void *w_gate, const void *w_up, const void *a_gate, const void *b_gate,
                           const void *a_up, const void *b_up, const float *scale, ts_dtype dtype,
                           const int32_t *offsets, const int32_t *adapter, int rows, int segments, int n_adapters,
                           int rank, int n, int k, void *c, ts_dtype odtype, void *ws, size_t ws_bytes, void *stream) {
    return ts::adapt({x, {w_gate, w_up}, {a_gate, a_up}, {b_gate, b_up}, scale, offsets, adapter, dtype, odtype, 0, 2,
                      rows, segments, n_adapters, rank, n, k, c, ws, ws_bytes, static_cast<hipStream_t>(stream)});
}

}  // extern "C"
