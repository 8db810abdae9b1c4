// Products grouped by expert with ragged sizes, bf16 and fp32: forward, with
// dReLU in the epilogue, and the weights' gradient; dReLU's own gradient.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ts_gmm.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

namespace {

// Weight gradients: short contractions (a group's rows) over a large output, 1.9
// GB in fp32 at 8 x 14336 x 4096.  6002 rows of 8 groups 0.95 ms (0.74 PFLOP/s),
// of it 0.29 the stores (6.5 TB/s) and 0.16 the tiles' starts; groups of 6144 rows
// 1.2 PFLOP/s.  128 x 128 tiles take half as long again, 256 x 128 a fifth more.
// Outputs of as many elements as 256 of the large tile's take it (bf16; counted in
// elements: of n or k below 256 most of such a tile is empty).  One workgroup contracts
// all of a group's rows: few tiles with many rows are one long chain of steps (n 8 to
// 64, k 4096, one group of 16384 rows, 32 workgroups: bf16 0.18 to 0.23 ms, fp32 1.1).
template <GmmKind KIND>
ts_status run_grad_w(const GmmArgs &a, hipStream_t st) {
    if (gmm_wide<KIND>(a)) return run_tiled<KIND, kGradW, true, 128, 128, 2, 2, 2, 2, 1, true>("grouped_mm_dw", a, st);
    if constexpr (KIND == kGmmBf16)
        if ((long long)a.n * a.k * a.groups >= 256LL * 65536)
            return run_tiled<KIND, kGradW, true, 256, 256, 2, 4, 3, 2>("grouped_mm_dw", a, st);
    return run_tiled<KIND, kGradW, true, 128, 128, 2, 2, 2, 2>("grouped_mm_dw", a, st);
}

}  // namespace

// d_gate = d_c up, d_up = d_c gate where gate > 0 and up > 0, otherwise 0.
// One pass, 16 bytes of each tensor a lane: 6002 x 14336 bf16 160 us, 5.4 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void drelu_grad_kernel(const u32x4 *gate, const u32x4 *up, const u32x4 *dc,
                                                         u32x4 *dgate, u32x4 *dup, long long chunks) {
    constexpr int CE = WTraits<T>::CE;
    const long long step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += step) {
        float g[CE], u[CE], d[CE];
        unpack<T>(ld_stream(gate + i), g);
        unpack<T>(ld_stream(up + i), u);
        unpack<T>(ld_stream(dc + i), d);
#pragma unroll
        for (int e = 0; e < CE; e += 4) {
            f32x4 a, b;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const bool on = g[e + v] > 0.f && u[e + v] > 0.f;
                a[v] = on ? d[e + v] * u[e + v] : 0.f;
                b[v] = on ? d[e + v] * g[e + v] : 0.f;
            }
            store4(dgate, CE == 4, (size_t)i * CE + e, a);
            store4(dup, CE == 4, (size_t)i * CE + e, b);
        }
    }
}

}  // namespace ts

namespace {

int quantum(ts_dtype d) { return d == TS_F32 ? 4 : 8; }

// Checks that the forward products share; TS_OK with *empty set: nothing to do.
ts_status check_fwd(const void *x, const void *w, ts_dtype dtype, ts_dtype odtype, const int32_t *row_src,
                    const int32_t *offsets, int rows, int src_rows, int groups, int n, int k, const void *out,
                    bool *empty) {
    *empty = false;
    if (!ts::type_ok(dtype) || !ts::type_ok(odtype)) return TS_ERR_DTYPE;
    ts_status s = ts::check_group_dims(rows, groups, n, k, quantum(dtype));
    if (s != TS_OK) return s;
    if (!offsets && groups != 1) return TS_ERR_NULL;
    if (src_rows < 0 || src_rows > ts::kMaxRows || (rows > 0 && src_rows < 1) || (!row_src && src_rows < rows))
        return TS_ERR_SHAPE;
    if (rows == 0) {
        *empty = true;
        return TS_OK;
    }
    if (!x || !w || !out) return TS_ERR_NULL;
    if (!ts::aligned16(x) || !ts::aligned16(w) || !ts::aligned16(out) || !ts::aligned4(row_src) ||
        !ts::aligned4(offsets))
        return TS_ERR_ALIGN;
    return TS_OK;
}

}  // namespace

extern "C" {

ts_status ts_grouped_mm(const void *x, const void *w, const void *x2, const void *w2, ts_dtype dtype, int w_kn,
                        const int32_t *row_src, const int32_t *offsets, int rows, int src_rows, int n_groups, int n,
                        int k, void *out, ts_dtype odtype, void *stream) {
    bool empty;
    ts_status s = check_fwd(x, w, dtype, odtype, row_src, offsets, rows, src_rows, n_groups, n, k, out, &empty);
    if (s != TS_OK) return s;
    if ((x2 == nullptr) != (w2 == nullptr)) return TS_ERR_NULL;
    if (!ts::aligned16(x2) || !ts::aligned16(w2)) return TS_ERR_ALIGN;
    if (empty) return TS_OK;
    ts::GmmArgs a;
    a.x[0] = static_cast<const char *>(x);
    a.x[1] = static_cast<const char *>(x2);
    a.w[0] = static_cast<const char *>(w);
    a.w[1] = static_cast<const char *>(w2);
    a.pairs = x2 ? 2 : 1;
    a.row_src = row_src;
    a.offsets = offsets;
    a.rows = rows;
    a.src_rows = src_rows;
    a.groups = n_groups;
    a.n = n;
    a.k = k;
    a.out = out;
    a.out_f32 = odtype == TS_F32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == TS_BF16)
        return w_kn ? ts::run_fwd<ts::kGmmBf16, ts::kFwd, true>("grouped_mm", a, st)
                    : ts::run_fwd<ts::kGmmBf16, ts::kFwd, false>("grouped_mm", a, st);
    return w_kn ? ts::run_fwd<ts::kGmmF32, ts::kFwd, true>("grouped_mm", a, st)
                : ts::run_fwd<ts::kGmmF32, ts::kFwd, false>("grouped_mm", a, st);
}

ts_status ts_grouped_drelu(const void *x, const void *w_gate, const void *w_up, ts_dtype dtype,
                           const int32_t *row_src, const int32_t *offsets, int rows, int src_rows, int n_groups,
                           int n, int k, void *c, void *gate, void *up, ts_dtype odtype, void *stream) {
    bool empty;
    ts_status s = check_fwd(x, w_gate, dtype, odtype, row_src, offsets, rows, src_rows, n_groups, n, k, c, &empty);
    if (s != TS_OK) return s;
    if ((gate == nullptr) != (up == nullptr)) return TS_ERR_NULL;
    if (!ts::aligned16(w_up) || !ts::aligned16(gate) || !ts::aligned16(up)) return TS_ERR_ALIGN;
    if (empty) return TS_OK;
    if (!w_up) return TS_ERR_NULL;
    ts::GmmArgs a;
    a.x[0] = static_cast<const char *>(x);
    a.w[0] = static_cast<const char *>(w_gate);
    a.w[1] = static_cast<const char *>(w_up);
    a.row_src = row_src;
    a.offsets = offsets;
    a.rows = rows;
    a.src_rows = src_rows;
    a.groups = n_groups;
    a.n = n;
    a.k = k;
    a.out = c;
    a.gate = gate;
    a.up = up;
    a.out_f32 = odtype == TS_F32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == TS_BF16 ? ts::run_fwd<ts::kGmmBf16, ts::kDrelu, false>("grouped_drelu", a, st)
                            : ts::run_fwd<ts::kGmmF32, ts::kDrelu, false>("grouped_drelu", a, st);
}

ts_status ts_grouped_mm_dw(const void *d_y, const void *x, ts_dtype dtype, const int32_t *row_src,
                           const int32_t *offsets, int rows, int src_rows, int n_groups, int n, int k, void *d_w,
                           ts_dtype odtype, void *stream) {
    bool empty;
    ts_status s = check_fwd(x, d_y, dtype, odtype, row_src, offsets, rows, src_rows, n_groups, n, k, d_w, &empty);
    if (s != TS_OK) return s;
    if (!d_w) return TS_ERR_NULL;
    if (!ts::aligned16(d_w) || !ts::aligned4(offsets)) return TS_ERR_ALIGN;  // (read without rows, too)
    ts::GmmArgs a;
    a.w[0] = static_cast<const char *>(x);
    a.x[0] = static_cast<const char *>(d_y);
    a.row_src = row_src;
    a.offsets = offsets;
    a.rows = rows;  // 0: every group is empty and its gradient zero
    a.src_rows = src_rows;
    a.groups = n_groups;
    a.n = n;
    a.k = k;
    a.out = d_w;
    a.out_f32 = odtype == TS_F32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == TS_BF16 ? ts::run_grad_w<ts::kGmmBf16>(a, st) : ts::run_grad_w<ts::kGmmF32>(a, st);
}

ts_status ts_drelu_grad(const void *gate, const void *up, const void *d_c, ts_dtype dtype, int rows, int n,
                        void *d_gate, void *d_up, void *stream) {
    if (!ts::type_ok(dtype)) return TS_ERR_DTYPE;
    if (rows < 0 || rows > ts::kMaxRows || n < quantum(dtype) || n > ts::kMaxDim || n % quantum(dtype) != 0)
        return TS_ERR_SHAPE;
    if (rows == 0) return TS_OK;
    if (!gate || !up || !d_c || !d_gate || !d_up) return TS_ERR_NULL;
    for (const void *p : {gate, up, d_c, (const void *)d_gate, (const void *)d_up})
        if (!ts::aligned16(p)) return TS_ERR_ALIGN;
    const long long chunks = (long long)rows * (n / quantum(dtype));
    const unsigned grid = (unsigned)std::min<long long>((chunks + 255) / 256, 256 * 64);
    using ts::u32x4;
    auto go = [&](auto kernel) {
        ts::launch<const u32x4 *, const u32x4 *, const u32x4 *, u32x4 *, u32x4 *, long long>(
            "drelu_grad", kernel, dim3(grid), dim3(256), static_cast<hipStream_t>(stream),
            static_cast<const u32x4 *>(gate), static_cast<const u32x4 *>(up), static_cast<const u32x4 *>(d_c),
            static_cast<u32x4 *>(d_gate), static_cast<u32x4 *>(d_up), chunks);
        return ts::check_launch("drelu_grad");
    };
    return dtype == TS_F32 ? go(ts::drelu_grad_kernel<float>) : go(ts::drelu_grad_kernel<uint16_t>);
}

}  // extern "C"
