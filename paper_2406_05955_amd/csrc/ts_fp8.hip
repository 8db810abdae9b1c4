// 8-bit floating point (OCP e4m3) with an fp32 scale for each block of 128
// values of a row, and each 128 x 128 tile of a weight matrix: the quantisers
// and the products.
//   amax = max(|block|, 2^-100), scale = amax / 448, code = e4m3(448 x / amax)
// 448 is the largest e4m3 value.  The quotient is correctly rounded to 32
// bits before its rounding to e4m3: with bf16 inputs no code depends on it.
// A block with an infinity has an infinite scale and NaN codes; a NaN makes
// its own code NaN.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ts_gmm.h"
#include "ts_plan.h"
#include "ts_runtime.h"
#include "turbosparse.h"

namespace ts {

namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kAmaxMin = 0x1p-100f;

// Values x mul are divided by d: 448 / amax, both times 2^-40 where 448 x
// could leave the fp32 range.
struct QuantDiv {
    float mul, d, r;
    __device__ __forceinline__ explicit QuantDiv(float amax) {
        const float pre = amax > 0x1p100f ? 0x1p-40f : 1.f;
        mul = kE4m3Max * pre;
        d = amax * pre;
        r = 1.f / d;
    }
    // The correctly rounded quotient from the correctly rounded reciprocal:
    // one residual step.
    __device__ __forceinline__ float operator()(float x) const {
        const float n = x * mul;
        const float q = n * r;
        const float rem = __builtin_fmaf(-q, d, n);
        return __builtin_fmaf(rem, r, q);
    }
};

// Four fp32 values to four e4m3 codes (hardware conversion, to nearest even).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    return (uint32_t)v;
}

__device__ __forceinline__ float max_abs(float m, float v) { return fmaxf(m, fabsf(v)); }

}  // namespace

// Rows: 8 values per lane, 16 lanes per block of 128.  Bytes: 8192 x 4096 bf16 22
// us, 4.6 TB/s; a few rows are one launch, 4 us.
template <typename T>
__global__ __launch_bounds__(256) void fp8_quant_kernel(const T *x, uint8_t *q, float *s, int rows, int cols) {
    const int kb = (cols + kScaleBlock - 1) / kScaleBlock;
    const int lane16 = threadIdx.x & 15;
    const long long blocks = (long long)rows * kb, step = (long long)gridDim.x * 16;
    // (whole waves stay in the loop: a block's lanes exchange their maxima)
    for (long long b0 = (long long)blockIdx.x * 16; b0 < blocks; b0 += step) {
        const long long blk = b0 + (threadIdx.x >> 4);
        const bool in = blk < blocks;
        const int row = in ? (int)(blk / kb) : 0, b = in ? (int)(blk % kb) : 0;
        const int c0 = b * kScaleBlock + lane16 * 8;
        const bool ok = in && c0 < cols;  // cols is a multiple of 16: all 8 or none
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (ok) {
            const T *p = x + (size_t)row * cols + c0;
            if constexpr (sizeof(T) == 4) {
                unpack<float>(ld_cached(p), v);
                unpack<float>(ld_cached(p + 4), v + 4);
            } else {
                unpack<uint16_t>(ld_cached(p), v);
            }
        }
        float amax = kAmaxMin;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max_abs(amax, v[i]);
        amax = fmaxf(amax, dpp_f32<0xB1>(amax));
        amax = fmaxf(amax, dpp_f32<0x4E>(amax));
        amax = fmaxf(amax, dpp_f32<0x124>(amax));
        amax = fmaxf(amax, dpp_f32<0x128>(amax));
        if (ok) {
            const QuantDiv div(amax);
            uint2 o;
            o.x = codes4(div(v[0]), div(v[1]), div(v[2]), div(v[3]));
            o.y = codes4(div(v[4]), div(v[5]), div(v[6]), div(v[7]));
            *reinterpret_cast<uint2 *>(q + (size_t)row * cols + c0) = o;
        }
        if (in && lane16 == 0) s[blk] = amax / kE4m3Max;
    }
}

// Weights: one 128 x 128 tile per workgroup; KN: the matrix is stored [k][n]
// and leaves as [n][k] (laid out once, read by every later product).
template <typename T, bool KN>
__global__ __launch_bounds__(256) void fp8_quant_weights_kernel(const T *w, uint8_t *q, float *s, int n, int k) {
    __shared__ float red[4];
    __shared__ float tile[KN ? 128 : 1][KN ? 132 : 1];
    const int nb = (n + 127) / 128, kb = (k + 127) / 128;
    const int bk = blockIdx.x % kb, bn = blockIdx.x / kb % nb;
    const size_t g = blockIdx.x / kb / nb;
    const T *m = w + g * (size_t)n * k;
    const int srows = KN ? k : n, scols = KN ? n : k;  // as stored
    const int r0 = (KN ? bk : bn) * 128, c0 = (KN ? bn : bk) * 128;
    const int tc = (threadIdx.x & 15) * 8, tr = threadIdx.x >> 4;
    float v[8][8];
    float amax = kAmaxMin;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = r0 + tr + 16 * j, c = c0 + tc;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
        if (r < srows && c < scols) {
            const T *p = m + (size_t)r * scols + c;
            if constexpr (sizeof(T) == 4) {
                unpack<float>(ld_cached(p), v[j]);
                unpack<float>(ld_cached(p + 4), v[j] + 4);
            } else {
                unpack<uint16_t>(ld_cached(p), v[j]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_abs(amax, v[j][e]);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    if constexpr (KN) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[tr + 16 * j][tc + e] = v[j][e];
    }
    __syncthreads();
    amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const QuantDiv div(amax);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int rn = tr + 16 * j;  // row n of the tile as it leaves
        if constexpr (KN) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = tile[tc + e][rn];
        }
        const int on = bn * 128 + rn, ok = bk * 128 + tc;
        if (on < n && ok < k) {
            uint2 o;
            o.x = codes4(div(v[j][0]), div(v[j][1]), div(v[j][2]), div(v[j][3]));
            o.y = codes4(div(v[j][4]), div(v[j][5]), div(v[j][6]), div(v[j][7]));
            *reinterpret_cast<uint2 *>(q + g * (size_t)n * k + (size_t)on * k + ok) = o;
        }
    }
    if (threadIdx.x == 0) s[(g * nb + bn) * kb + bk] = amax / kE4m3Max;
}

namespace {

ts_status fp8_args(GmmArgs *a, const void *x, const float *x_scale, const void *w, const float *w_scale,
                   const int32_t *row_src, const int32_t *offsets, int rows, int src_rows, int groups, int n, int k,
                   void *out, ts_dtype odtype) {
    if (!type_ok(odtype)) return TS_ERR_DTYPE;
    ts_status s = check_group_dims(rows, groups, n, k, 16);
    if (s != TS_OK) return s;
    if (!offsets && groups != 1) return TS_ERR_NULL;
    if (src_rows < 0 || src_rows > kMaxRows || (rows > 0 && src_rows < 1) || (!row_src && src_rows < rows))
        return TS_ERR_SHAPE;
    if (rows > 0) {
        if (!x || !x_scale || !w || !w_scale || !out) return TS_ERR_NULL;
        if (!aligned16(x) || !aligned16(w) || !aligned16(out) || !aligned4(x_scale) || !aligned4(w_scale) ||
            !aligned4(row_src) || !aligned4(offsets))
            return TS_ERR_ALIGN;
    }
    a->x[0] = static_cast<const char *>(x);
    a->xs = x_scale;
    a->w[0] = static_cast<const char *>(w);
    a->ws[0] = w_scale;
    a->row_src = row_src;
    a->offsets = offsets;
    a->rows = rows;
    a->src_rows = src_rows;
    a->groups = groups;
    a->n = n;
    a->k = k;
    a->out = out;
    a->out_f32 = odtype == TS_F32;
    return TS_OK;
}

ts_status check_quant(const void *x, ts_dtype dtype, const void *q, const void *scale) {
    if (!x || !q || !scale) return TS_ERR_NULL;
    if (!aligned16(x) || !aligned16(q) || !aligned4(scale)) return TS_ERR_ALIGN;
    return TS_OK;
}

}  // namespace

}  // namespace ts

extern "C" {

ts_status ts_fp8_quant(const void *x, ts_dtype dtype, int rows, int cols, void *q, float *scale, void *stream) {
    if (!ts::type_ok(dtype)) return TS_ERR_DTYPE;
    if (rows < 0 || rows > ts::kMaxRows || cols < 16 || cols > ts::kMaxDim || cols % 16 != 0) return TS_ERR_SHAPE;
    if (rows == 0) return TS_OK;
    ts_status s = ts::check_quant(x, dtype, q, scale);
    if (s != TS_OK) return s;
    const long long blocks = (long long)rows * ts::ceil_div(cols, ts::kScaleBlock);
    const long long grid = std::min<long long>((blocks + 15) / 16, 1 << 20);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == TS_F32)
        ts::launch<const float *, uint8_t *, float *, int, int>("fp8_quant", ts::fp8_quant_kernel<float>,
            dim3((unsigned)grid), dim3(256), st, static_cast<const float *>(x), static_cast<uint8_t *>(q), scale, rows,
            cols);
    else
        ts::launch<const uint16_t *, uint8_t *, float *, int, int>("fp8_quant", ts::fp8_quant_kernel<uint16_t>,
            dim3((unsigned)grid), dim3(256), st, static_cast<const uint16_t *>(x), static_cast<uint8_t *>(q), scale,
            rows, cols);
    return ts::check_launch("fp8_quant");
}

ts_status ts_fp8_quant_weights(const void *w, ts_dtype dtype, int w_kn, int n_groups, int n, int k, void *q,
                               float *scale, void *stream) {
    if (!ts::type_ok(dtype)) return TS_ERR_DTYPE;
    ts_status s = ts::check_group_dims(1, n_groups, n, k, 16);
    if (s != TS_OK) return s;
    s = ts::check_quant(w, dtype, q, scale);
    if (s != TS_OK) return s;
    const long long grid = (long long)n_groups * ts::ceil_div(n, 128) * ts::ceil_div(k, 128);
    if (grid * 256 >= (1LL << 32)) return TS_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto kernel, auto *p) {
        ts::launch<decltype(p), uint8_t *, float *, int, int>("fp8_quant_weights", kernel, dim3((unsigned)grid),
                                                              dim3(256), st, p, static_cast<uint8_t *>(q), scale, n, k);
        return ts::check_launch("fp8_quant_weights");
    };
    if (dtype == TS_F32) {
        const float *p = static_cast<const float *>(w);
        return w_kn ? go(ts::fp8_quant_weights_kernel<float, true>, p) : go(ts::fp8_quant_weights_kernel<float, false>, p);
    }
    const uint16_t *p = static_cast<const uint16_t *>(w);
    return w_kn ? go(ts::fp8_quant_weights_kernel<uint16_t, true>, p)
                : go(ts::fp8_quant_weights_kernel<uint16_t, false>, p);
}

ts_status ts_fp8_mm(const void *x, const float *x_scale, const void *w, const float *w_scale, const int32_t *row_src,
                    const int32_t *offsets, int rows, int src_rows, int n_groups, int n, int k, void *out,
                    ts_dtype odtype, void *stream) {
    ts::GmmArgs a;
    ts_status s = ts::fp8_args(&a, x, x_scale, w, w_scale, row_src, offsets, rows, src_rows, n_groups, n, k, out,
                               odtype);
    if (s != TS_OK || rows == 0) return s;
    return ts::run_fwd<ts::kGmmFp8, ts::kFwd, false>("fp8_mm", a, static_cast<hipStream_t>(stream));
}

ts_status ts_fp8_drelu(const void *x, const float *x_scale, const void *w_gate, const float *gate_scale,
                       const void *w_up, const float *up_scale, const int32_t *row_src, const int32_t *offsets,
                       int rows, int src_rows, int n_groups, int n, int k, void *c, ts_dtype odtype, void *stream) {
    ts::GmmArgs a;
    ts_status s = ts::fp8_args(&a, x, x_scale, w_gate, gate_scale, row_src, offsets, rows, src_rows, n_groups, n, k, c,
                               odtype);
    if (s != TS_OK || rows == 0) return s;
    if (!w_up || !up_scale) return TS_ERR_NULL;
    if (!ts::aligned16(w_up) || !ts::aligned4(up_scale)) return TS_ERR_ALIGN;
    a.w[1] = static_cast<const char *>(w_up);
    a.ws[1] = up_scale;
    return ts::run_fwd<ts::kGmmFp8, ts::kDrelu, false>("fp8_drelu", a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
