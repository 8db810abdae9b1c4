// Gate + up products whose activations are kept in 8 bits (ts_keep.h), the
// backward product that reads them, and their values.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ts_gmm.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

// V columns of a row a lane (n is a multiple of V; they share an exponent byte).
template <int V>
__global__ __launch_bounds__(256) void drelu_unpack_kernel(const uint8_t *codes, const uint16_t *exps, uint16_t *gate,
                                                           uint16_t *up, int rows, int n) {
    const int per = n / V, eb = (n + kKeepBlock - 1) / kKeepBlock;
    const long long total = (long long)rows * per, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const int r = (int)(i / per), c = (int)(i - (long long)r * per) * V;
        const size_t at = (size_t)r * n + c;
        const uint32_t e = exps[(size_t)r * eb + c / kKeepBlock];
        uint2 q[V / 4];
        if constexpr (V == 8) {
            const u32x4 v = ld_stream(codes + 2 * at);
            q[0] = uint2{v.x, v.y};
            q[1] = uint2{v.z, v.w};
        } else {
            q[0] = *reinterpret_cast<const uint2 *>(codes + 2 * at);
        }
        uint32_t g[V / 2], u[V / 2];
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            float gv[4], uv[4];
            bool go[4], uo[4];
            keep_values4(q[h], e, gv, uv, go, uo);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                gv[v] = go[v] ? gv[v] : 0.f;
                uv[v] = uo[v] ? uv[v] : 0.f;
            }
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                // exact: the low halves are zeros
                g[2 * h + v] = __float_as_uint(gv[2 * v]) >> 16 | __float_as_uint(gv[2 * v + 1]);
                u[2 * h + v] = __float_as_uint(uv[2 * v]) >> 16 | __float_as_uint(uv[2 * v + 1]);
            }
        }
        if constexpr (V == 8) {
            *reinterpret_cast<u32x4 *>(gate + at) = u32x4{g[0], g[1], g[2], g[3]};
            *reinterpret_cast<u32x4 *>(up + at) = u32x4{u[0], u[1], u[2], u[3]};
        } else {
            *reinterpret_cast<uint2 *>(gate + at) = uint2{g[0], g[1]};
            *reinterpret_cast<uint2 *>(up + at) = uint2{u[0], u[1]};
        }
    }
}

namespace {

ts_status check_kept(const void *codes, const void *exps) {
    if (!codes || !exps) return TS_ERR_NULL;
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(exps) % 2 != 0) return TS_ERR_ALIGN;
    return TS_OK;
}

void fill(GmmKeepArgs *a, const void *x, const void *w, const int32_t *row_src, const int32_t *offsets, int rows,
          int src_rows, int groups, int n, int k, ts_dtype odtype) {
    a->x[0] = static_cast<const char *>(x);
    a->w[0] = static_cast<const char *>(w);
    a->row_src = row_src;
    a->offsets = offsets;
    a->rows = rows;
    a->src_rows = src_rows;
    a->groups = groups;
    a->n = n;
    a->k = k;
    a->out_f32 = odtype == TS_F32;
}

}  // namespace

}  // namespace ts

extern "C" {

ts_status ts_grouped_drelu_pack(const void *x, const void *w_gate, const void *w_up, ts_dtype dtype,
                                const int32_t *row_src, const int32_t *offsets, int rows, int src_rows, int n_groups,
                                int n, int k, void *c, void *codes, void *exps, ts_dtype odtype, void *stream) {
    bool empty;
    ts_status s = ts::check_fwd(x, w_gate, dtype, odtype, row_src, offsets, rows, src_rows, n_groups, n, k, c, &empty);
    if (s != TS_OK || empty) return s;
    if (!w_up) return TS_ERR_NULL;
    if (!ts::aligned16(w_up)) return TS_ERR_ALIGN;
    s = ts::check_kept(codes, exps);
    if (s != TS_OK) return s;
    ts::GmmKeepArgs a;
    ts::fill(&a, x, w_gate, row_src, offsets, rows, src_rows, n_groups, n, k, odtype);
    a.w[1] = static_cast<const char *>(w_up);
    a.out = c;
    a.codes = static_cast<uint8_t *>(codes);
    a.exps = static_cast<uint8_t *>(exps);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == TS_BF16 ? ts::run_fwd<ts::kGmmBf16, ts::kDreluPack, false>("grouped_drelu_pack", a, st)
                            : ts::run_fwd<ts::kGmmF32, ts::kDreluPack, false>("grouped_drelu_pack", a, st);
}

ts_status ts_grouped_drelu_grad(const void *d_y, const void *w, ts_dtype dtype, const int32_t *row_src,
                                const int32_t *offsets, int rows, int src_rows, int n_groups, int n, int k,
                                const void *codes, const void *exps, void *d_gate, void *d_up, void *c,
                                ts_dtype odtype, void *stream) {
    bool empty;
    ts_status s = ts::check_fwd(d_y, w, dtype, odtype, row_src, offsets, rows, src_rows, n_groups, n, k, d_gate, &empty);
    if (s != TS_OK || empty) return s;
    if (!d_up) return TS_ERR_NULL;
    if (!ts::aligned16(d_up) || !ts::aligned16(c)) return TS_ERR_ALIGN;
    s = ts::check_kept(codes, exps);
    if (s != TS_OK) return s;
    ts::GmmKeepArgs a;
    ts::fill(&a, d_y, w, row_src, offsets, rows, src_rows, n_groups, n, k, odtype);
    a.codes = static_cast<uint8_t *>(const_cast<void *>(codes));  // (read)
    a.exps = static_cast<uint8_t *>(const_cast<void *>(exps));
    a.gate = d_gate;
    a.up = d_up;
    a.out = c;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == TS_BF16 ? ts::run_fwd<ts::kGmmBf16, ts::kDreluGrad, false>("grouped_drelu_grad", a, st)
                            : ts::run_fwd<ts::kGmmF32, ts::kDreluGrad, false>("grouped_drelu_grad", a, st);
}

ts_status ts_drelu_unpack(const void *codes, const void *exps, int rows, int n, void *gate, void *up, void *stream) {
    if (rows < 0 || rows > ts::kMaxRows || n < 4 || n > ts::kMaxDim || n % 4 != 0) return TS_ERR_SHAPE;
    if (rows == 0) return TS_OK;
    ts_status s = ts::check_kept(codes, exps);
    if (s != TS_OK) return s;
    if (!gate || !up) return TS_ERR_NULL;
    if (!ts::aligned16(gate) || !ts::aligned16(up)) return TS_ERR_ALIGN;
    const bool eight = n % 8 == 0;
    const long long chunks = (long long)rows * (n / (eight ? 8 : 4));
    const unsigned grid = (unsigned)std::min<long long>((chunks + 255) / 256, 256 * 64);
    ts::launch<const uint8_t *, const uint16_t *, uint16_t *, uint16_t *, int, int>(
        "drelu_unpack", eight ? ts::drelu_unpack_kernel<8> : ts::drelu_unpack_kernel<4>, dim3(grid), dim3(256),
        static_cast<hipStream_t>(stream), static_cast<const uint8_t *>(codes), static_cast<const uint16_t *>(exps),
        static_cast<uint16_t *>(gate), static_cast<uint16_t *>(up), rows, n);
    return ts::check_launch("drelu_unpack");
}

}  // extern "C"
