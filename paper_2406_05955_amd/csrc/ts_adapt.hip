// Low-rank adapters of many requests beside a shared projection:
//   y[r] = x[r] W^T + s_a (x[r] A_a^T) B_a^T,  a = adapter of r's segment (or none)
// and the same in front of dReLU for gate and up.
//
// adapter_rows computes t = s_a x A_a^T, `rank` values a row (a few ranks, a long
// contraction), and of each row tile of the product which adapters it meets.  The
// product then contracts t with B behind x with W, in the same accumulators
// (gmm_tiled's adapter steps): y is written once and nothing is read twice.  Few
// rows and columns with a long contraction share it among workgroups, whose sums
// a third launch adds in a fixed order.
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
    int32_t *slots = nullptr, *slot_ad = nullptr, *slot_count = nullptr;
    int rows = 0, segs = 0, adapters = 0, rank = 0, ranks = 0, parts = 1, k = 0;  // ranks: of both matrices
    int first = 0;                // workgroups of earlier launches
    int pieces = 0, per = 16;     // ranks of a workgroup
    int wr = 0, blocks = 0;       // rows of one of the product's waves, their number
};

// The segments as a wave looks them up: up to 64 are held, one a lane, by loads on their
// way together (probing memory for 9 to 32 segments, each probe waits for the last:
// adapter_rows 2 us longer); more are probed where they are.
struct Segments {
    const AdaptRowsArgs &a;
    int first = 0, behind = 0, adapter = 0;  // lane s: segment s's
    bool held, ordered = true;               // (ordered: of held ones)
    __device__ __forceinline__ int clamped(int s) const { return min(max(a.offsets[s], 0), a.rows); }
    __device__ __forceinline__ Segments(const AdaptRowsArgs &args, int lane) : a(args), held(args.segs <= 64) {
        if (held) {
            first = clamped(min(lane, a.segs - 1));
            behind = clamped(min(lane, a.segs - 1) + 1);
            adapter = a.adapter[min(lane, a.segs - 1)];
            ordered = !__any(first > behind);
        }
    }
    // Whether the offsets ascend, by all of a workgroup of THREADS.
    template <int THREADS>
    __device__ __forceinline__ bool all_ordered() const {
        if (held) return ordered;
        int bad = 0;
        for (int s = threadIdx.x; s < a.segs; s += THREADS) bad |= clamped(s) > clamped(s + 1);
        return !__syncthreads_or(bad);
    }
    // (s uniform)
    __device__ __forceinline__ int begin(int s) const { return held ? __builtin_amdgcn_readlane(first, s) : clamped(s); }
    __device__ __forceinline__ int end(int s) const { return held ? __builtin_amdgcn_readlane(behind, s) : clamped(s + 1); }
    __device__ __forceinline__ int id(int s) const { return held ? __builtin_amdgcn_readlane(adapter, s) : a.adapter[s]; }
    // Segment s's rows in pieces of Q: its first piece has the number offsets[s] / Q +
    // s, which no other segment's piece has (a segment's pieces are at most its rows / Q
    // + 1), so the pieces need no count of those before.  The last s whose first piece is
    // not behind piece `p`.
    template <int Q>
    __device__ __forceinline__ int of_piece(int p, int lane) const {
        if (held) return max(__popcll(__ballot(lane < a.segs && first / Q + lane <= p)), 1) - 1;
        int lo = 0, hi = a.segs;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64, s = lo + lane * step;
            const bool ok = s < hi && clamped(min(s, hi - 1)) / Q + min(s, hi - 1) <= p;
            const int n = max(__popcll(__ballot(ok)), 1);
            lo += (n - 1) * step;
            hi = min(hi, lo + step);
        }
        return lo;
    }
    // The adapter of each lane's row: that of the last segment that begins at or in
    // front of it.
    __device__ __forceinline__ int id_of_row(int row) const {
        int lo = 0, hi = a.segs;
        while (__any(hi - lo > 1)) {
            const int mid = (lo + hi) / 2, o = held ? __shfl(first, mid) : clamped(mid);
            if (hi - lo > 1) (o <= row ? lo : hi) = mid;
        }
        return held ? __shfl(adapter, lo) : a.adapter[lo];
    }
};

// Slots of the adapters of rows r0 ... of one of the product's waves (a.wr rows: lane
// l has row r0 + l), by one wave: a slot for each adapter, in the order of their
// first rows.  Runs of rows with one adapter are looked up one after another: prompts
// have few.  Offsets that descend anywhere leave all rows without an adapter: two
// segments may then have the same row, whose t is whichever's comes last, and nothing
// reads it.
__device__ __forceinline__ void wave_slots(const AdaptRowsArgs &a, const Segments &seg, bool ordered, int block, int lane) {
    const int b = seg.begin(0), e = seg.end(a.segs - 1);
    const int r0 = b + block * a.wr, row = r0 + lane;
    if (r0 >= e) return;
    int id = seg.id_of_row(row);
    if (!ordered || lane >= a.wr || row >= e || id < 0 || id >= a.adapters) id = -1;
    const int before = __shfl_up(id, 1);
    uint64_t starts = __ballot(id >= 0 && (lane == 0 || id != before));
    int list = -1, n = 0, slot = -1;
    while (starts) {
        const int at = __builtin_ctzll(starts);
        starts &= starts - 1;
        const int want = __builtin_amdgcn_readlane(id, at);
        const uint64_t same = __ballot(list == want);
        const int s = same ? __builtin_ctzll(same) : n++;
        if (lane == s) list = want;
        if (lane >= at) slot = s;
    }
    if (lane < a.wr) {
        a.slots[(size_t)block * a.wr + lane] = id >= 0 ? slot : -1;
        a.slot_ad[(size_t)block * a.wr + lane] = max(list, 0);
    }
    if (lane == 0) a.slot_count[block] = n;
}

// Where t stands of a row (counted from the first segment's) and rank; parts are 16
// a.rank behind one another.
template <GmmKind KIND>
__device__ __forceinline__ size_t t_at(const AdaptRowsArgs &a, int row, int r) {
    constexpr int CE = 16 / GmmElem<KIND>::SZ;
    const int room = adapt_room(a.parts), second = r >= a.rank;
    const size_t place = (size_t)(row / 16) * a.ranks * room + r + (second ? a.rank * (room - 1) : 0);
    return place / CE * CE * 16 + row % 16 * CE + place % CE;
}
// N neighbouring ranks (1 or 4, of one matrix).
template <GmmKind KIND, int N>
__device__ __forceinline__ void store_t(const AdaptRowsArgs &a, int row, int r, const float (&x)[N]) {
    size_t at = t_at<KIND>(a, row, r);
    if constexpr (KIND == kGmmF32) {
        float *const t = reinterpret_cast<float *>(a.t) + at;
        if constexpr (N == 4) *reinterpret_cast<f32x4 *>(t) = f32x4{x[0], x[1], x[2], x[3]};
        else *t = x[0];
    } else {
        typedef __bf16 b16xn __attribute__((ext_vector_type(N)));
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = x[i];
        // each part is what the ones before left (nothing of what has no remainder; of a value
        // that would round to infinity the first is the largest finite one)
        constexpr float most = 0x1.FEp127f;
        for (int p = 0; p < a.parts; ++p, at += 16 * a.rank) {
            b16xn hi;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool finite = fabsf(v[i]) < INFINITY;
                hi[i] = (__bf16)(finite ? fminf(fmaxf(v[i], -most), most) : v[i]);
                v[i] = finite ? v[i] - (float)hi[i] : 0.f;
            }
            *reinterpret_cast<b16xn *>(reinterpret_cast<__bf16 *>(a.t) + at) = hi;
        }
    }
}

}  // namespace

// t of up to 16 RT rows of a segment and 16 NR ranks; W waves share the contraction, U
// steps' loads of each on their way together; their sums are added in a fixed order.
template <GmmKind KIND, int RT, int NR, int W, int U>
__global__ __launch_bounds__(64 * W) void adapter_rows(AdaptRowsArgs a) {
    constexpr int SZ = GmmElem<KIND>::SZ, KS = 64 / SZ, CE = 16 / SZ, Q = 16 * RT;
    static_assert(RT > 1 || (NR == 1 && W == 16), "a single row: W / per waves a rank");
    __shared__ f32x4 red[W][RT * NR][64];
    const int lane = threadIdx.x & 63, lm = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Segments segments(a, lane);
    const int wg = a.first + (int)blockIdx.x;
    if (wg >= a.pieces) {
        if (blockIdx.y > 0) return;
        const bool ordered = segments.all_ordered<64 * W>();
        const int block = (wg - a.pieces) * W + wave;
        if (block < a.blocks) wave_slots(a, segments, ordered, block, lane);
        return;
    }
    if (!segments.ordered) return;
    const int seg = __builtin_amdgcn_readfirstlane(segments.of_piece<Q>(wg, lane));
    const int b = segments.begin(seg), e = segments.end(seg);
    const int piece = wg - (b / Q + seg);
    // (a segment in front of the first one's rows: offsets that descend)
    const int row0 = segments.begin(0);
    if (piece < 0 || b < row0 || b + (long long)piece * Q >= e) return;
    const int r0 = b + piece * Q, r1 = min(r0 + Q, e);
    const int id = segments.id(seg);
    if (id < 0 || id >= a.adapters) return;
    // ranks [k0, k1) (of both matrices, one behind the other)
    const int k0 = blockIdx.y * a.per, k1 = min(k0 + a.per, a.ranks);

    const size_t row_bytes = (size_t)a.k * SZ;
    const float scale = a.scale ? a.scale[id] : 1.f;
    if constexpr (RT == 1) {
        if (r1 - r0 == 1) {
            // A single row (a decoded token): W / a.per waves a rank, 1 KB of its A a load,
            // all of a wave's loads on their way together (as a matrix product, 16 rows x
            // 64 bytes a load and 1 of 16 columns used: k 14336 rank 16 15 us, this 8).
            constexpr int V = 8;
            float *const part = reinterpret_cast<float *>(red);
            const int g = W / a.per, r = k0 + wave / g, chunks = a.k / CE;
            float sum = 0.f;
            if (r < k1) {
                const bool second = r >= a.rank;
                const char *const pa = a.a[second] + ((size_t)id * a.rank + (second ? r - a.rank : r)) * row_bytes;
                const char *const px = a.x + (size_t)r0 * row_bytes;
                for (int c0 = wave % g * 64 + lane; c0 < chunks; c0 += V * g * 64) {
                    u32x4 va[V], vx[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const size_t at = (size_t)min(c0 + v * g * 64, chunks - 1) * 16;
                        va[v] = ld_cached(pa + at);
                        vx[v] = ld_cached(px + at);
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        using T = std::conditional_t<KIND == kGmmF32, float, uint16_t>;
                        float fa[CE], fx[CE];
                        unpack<T>(va[v], fa);
                        unpack<T>(vx[v], fx);
                        float dot = 0.f;
#pragma unroll
                        for (int i = 0; i < CE; ++i) dot += fa[i] * fx[i];
                        sum += c0 + v * g * 64 < chunks ? dot : 0.f;
                    }
                }
            }
            sum = wave_sum(sum);
            if (lane == 0) part[wave] = sum;
            __syncthreads();
            const int i = threadIdx.x, rr = k0 + i;
            if (i >= a.per || rr >= k1) return;
            float v = part[i * g];
            for (int w = 1; w < g; ++w) v += part[i * g + w];
            store_t<KIND, 1>(a, r0 - row0, rr, {v * scale});
            return;
        }
    }
    const char *ar[NR], *xr[RT];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const int r = min(k0 + f * 16 + lm, k1 - 1);
        const bool second = r >= a.rank;
        ar[f] = a.a[second] + ((size_t)id * a.rank + (second ? r - a.rank : r)) * row_bytes;
    }
#pragma unroll
    for (int j = 0; j < RT; ++j) xr[j] = a.x + (size_t)min(r0 + j * 16 + lm, r1 - 1) * row_bytes;
    const int steps = (a.k + KS - 1) / KS, per = (steps + W - 1) / W;
    const int s0 = wave * per, s1 = min(s0 + per, steps);
    f32x4 acc[NR][RT] = {};
    // (from another step on in each workgroup: rows of 2^n bytes lie in one channel of
    // the L2 at the same step)
    const int turns = (s1 - s0 + U - 1) / U, ahead = turns > 0 ? (int)((unsigned)wg + blockIdx.y) % turns : 0;
    for (int i = 0; i < turns; ++i) {
        const int s = s0 + (i + ahead < turns ? i + ahead : i + ahead - turns) * U;
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
    for (int i = wave; i < NR * RT; i += W) {
        f32x4 v = red[0][i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) v += red[w][i][lane];
        v *= scale;
        // lane (lm, lq): ranks 4 lq ... of row lm
        const int row = r0 + i % RT * 16 + lm, r = k0 + i / RT * 16 + 4 * lq;
        if (row >= r1 || r >= k1) continue;
        store_t<KIND, 4>(a, row - row0, r, {v[0], v[1], v[2], v[3]});
    }
}

// The sums of `split` workgroups a tile, in their order; dReLU behind gate's and
// up's.  Four columns a lane.
template <bool DRELU>
__global__ __launch_bounds__(256) void adapter_sum_kernel(GmmAdaptArgs a) {
    constexpr int both = DRELU ? 2 : 1;
    const int b = min(max(a.offsets[0], 0), a.rows), e = min(max(a.offsets[a.segs], 0), a.rows);
    const long long per = a.n / 4, total = (e - b) * per, step = (long long)gridDim.x * 256;
    const size_t part = (size_t)a.rows * both * a.n;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const size_t q = b + i / per, p = i % per * 4;
        const float *s = a.sums + q * both * a.n + p;
        f32x4 v[both];
#pragma unroll
        for (int h = 0; h < both; ++h) {
            v[h] = *reinterpret_cast<const f32x4 *>(s + (size_t)h * a.n);
#pragma unroll 4
            for (int k = 1; k < a.split; ++k) v[h] += *reinterpret_cast<const f32x4 *>(s + k * part + (size_t)h * a.n);
        }
        if constexpr (DRELU) {
#pragma unroll
            for (int c = 0; c < 4; ++c) v[0][c] = drelu1(v[0][c], v[1][c]);
        }
        store4(a.out, a.out_f32, q * a.n + p, v[0]);
    }
}

namespace {

// The ranks' intermediate: fp32 sums, which beside bf16 operands are held in bf16 parts of
// 8 bits: all 24 in three where the output is fp32, 16 in two where it is bf16 (a
// rounding of t to 8 bits, 2^-9 of the adapter's share, is what the output's own is: 0.0020
// from the result in 64 bits where 16 bits leave 0.0017, the output's rounding).
int adapt_parts(ts_dtype dtype, ts_dtype odtype) { return dtype == TS_F32 ? 1 : odtype == TS_F32 ? 3 : 2; }

size_t adapt_t_bytes(int rows, int rank, int products, ts_dtype dtype, ts_dtype odtype) {
    return align_up256((size_t)ceil_div(rows, 16) * 16 * rank * products * adapt_room(adapt_parts(dtype, odtype)) * (dtype == TS_F32 ? 4 : 2));
}

bool adapt_dims_ok(int rows, int rank, ts_dtype dtype) {
    return rows >= 0 && rows <= kMaxRows && rank >= quantum(dtype) && rank <= kMaxRank && rank % quantum(dtype) == 0;
}

struct AdaptPlan {
    GmmTileId tile;
    int split;
    size_t t, slots, sums;  // bytes
    size_t all() const { return t + slots + sums; }
};

AdaptPlan adapt_plan(int rows, int rank, int products, bool w_kn, int n, int k, ts_dtype dtype, ts_dtype odtype) {
    AdaptPlan p;
    const bool drelu = products == 2;
    const GmmKind kind = dtype == TS_F32 ? kGmmF32 : kGmmBf16;
    const int esz = dtype == TS_F32 ? 4 : 2;
    const bool wide = (unsigned long long)rows * k * esz >= (1ull << 32);
    p.tile = kTile128x128;
    p.split = 1;
    if (!wide && rows > 0) adapt_tile(kind, drelu, w_kn, rows, n, k, &p.tile, &p.split);
    p.t = adapt_t_bytes(rows, rank, products, dtype, odtype);
    const size_t wr = wave_rows(p.tile), blocks = ceil_div(rows, (int)wr);
    p.slots = align_up256(blocks * (wr + wr + 1) * 4);
    p.sums = p.split > 1 ? align_up256((size_t)p.split * rows * products * n * 4) : 0;
    return p;
}

size_t adapt_ws_bytes(int rows, int rank, int products, bool w_kn, int n, int k, ts_dtype dtype, ts_dtype odtype) {
    if (!type_ok(dtype) || !type_ok(odtype) || products < 1 || products > 2 || !adapt_dims_ok(rows, rank, dtype) ||
        check_group_dims(rows, 1, n, k, quantum(dtype)) != TS_OK)
        return 0;
    return adapt_plan(rows, rank, products, w_kn, n, k, dtype, odtype).all();
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

template <GmmKind KIND, int RT, int NR, int W, int RU>
ts_status run_rows(AdaptRowsArgs r, hipStream_t st) {
    const long long pieces = (long long)r.rows / (16 * RT) + r.segs;
    // few pieces: fewer ranks a workgroup, whose A comes through one unit's loads (us, 16
    // / 8 / 4 ranks: k 14336, 1 row x 16 ranks 9.8 / 6.4 / 6.5, 32 rows of as many requests
    // 11.7 / 7.3 / 6.2, x 32 11.2 / 7.9 / 10.0; 256 rows of one request, 128 ranks 32 / 49
    // / 65; a row each of 32 requests x 128 ranks 26 / 25 / 24)
    r.per = 16 * NR;
    while (NR == 1 && r.per > 4 && pieces * ceil_div(r.ranks, r.per) < 128) r.per /= 2;
    const int tall = ceil_div(r.ranks, r.per);
    // (a launch takes less than 2^32 threads)
    const long long wide = pieces + ceil_div(r.blocks, W), most = ((1LL << 32) - 1) / (64 * W * tall);
    r.pieces = (int)pieces;
    for (long long first = 0; first < wide; first += most) {
        r.first = (int)first;
        launch<AdaptRowsArgs>("adapter_rows", adapter_rows<KIND, RT, NR, W, RU>,
                              dim3((unsigned)std::min(most, wide - first), tall), dim3(64 * W), st, r);
        const ts_status s = check_launch("adapter_rows");
        if (s != TS_OK) return s;
    }
    return TS_OK;
}

// Rows x ranks of a workgroup, by how much there is to do.  16 x 16 reads a row once for
// every 16 ranks and a rank's A once for every 16 rows; 32 x 64 and 64 x 64 read less
// and leave units idle, or lanes where there are fewer ranks or shorter segments.  us,
// 16 x 16 / 32 x 64 / 64 x 64: bf16, k 4096, 40 segments: 2048 rows x 16 ranks 12 / 18
// / 22, 8192 x 16 27 / 29 / 26; 1024 x 64 19 / 23 / 27, 2048 x 64 (2^17) 28 / 25 / 30,
// 6001 x 64 61 / 25 / 33, 8192 x 64 (2^19) 77 / 47 / 33, 16384 x 256 547 / 218 / 189; in
// 750 segments of 8 rows 6001 x 32 55 / 44 / 53, x 256 390 / 218 / 271, in 2048 of one
// row 2048 x 64 146 / 135 / 177, and of k 14336 370 / 517 / 531.  fp32, whose matrix
// instructions take eight times as long: 2048 x 64 55 / 56 / 104, 6001 x 128 213 / 120 /
// 200, 16384 x 256 1024 / 529 / 556.  Over 1400 calls (512 to 40000 rows, 1 segment to
// one a row, 8 to 256 ranks) 4% above each one's best.
template <GmmKind KIND>
ts_status run_ranks(const AdaptRowsArgs &r, hipStream_t st) {
    const long long each = (long long)r.rows * r.ranks;
    if (r.ranks <= 16 || each < 1 << 17 || r.rows < 8LL * r.segs) return run_rows<KIND, 1, 1, 16, 8>(r, st);
    if constexpr (KIND == kGmmBf16)
        if (each >= 1 << 19 && r.rows >= 32LL * r.segs) return run_rows<KIND, 4, 4, 8, 2>(r, st);
    return run_rows<KIND, 2, 4, 8, 2>(r, st);
}

template <GmmKind KIND>
ts_status run_adapt(const AdaptCall &c) {
    const AdaptPlan plan = adapt_plan(c.rows, c.rank, c.products, c.w_kn != 0, c.n, c.k, c.dtype, c.odtype);
    GmmAdaptArgs a;
    a.tile = plan.tile;
    a.split = plan.split;
    AdaptRowsArgs r;
    r.x = static_cast<const char *>(c.x);
    for (int i = 0; i < c.products; ++i) r.a[i] = static_cast<const char *>(c.a[i]);
    r.scale = c.scale;
    r.offsets = c.offsets;
    r.adapter = c.adapter;
    r.t = static_cast<char *>(c.ws);
    r.wr = wave_rows(plan.tile);
    r.blocks = ceil_div(c.rows, r.wr);
    r.slots = reinterpret_cast<int32_t *>(r.t + plan.t);
    r.slot_ad = r.slots + (size_t)r.blocks * r.wr;
    r.slot_count = r.slot_ad + (size_t)r.blocks * r.wr;
    r.rows = c.rows;
    r.segs = c.segments;
    r.adapters = c.adapters;
    r.rank = c.rank;
    r.ranks = c.rank * c.products;
    r.parts = adapt_parts(c.dtype, c.odtype);
    r.k = c.k;
    ts_status s = run_ranks<KIND>(r, c.stream);
    if (s != TS_OK) return s;

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
    a.slots = r.slots;
    a.slot_ad = r.slot_ad;
    a.slot_count = r.slot_count;
    a.sums = reinterpret_cast<float *>(r.t + plan.t + plan.slots);
    a.segs = c.segments;
    a.rank = c.rank;
    a.parts = r.parts;
    if (c.products == 2) s = run_fwd<KIND, kDreluAdapt, false>("adapter_drelu", a, c.stream);
    else if (c.w_kn) s = run_fwd<KIND, kFwdAdapt, true>("adapter_mm", a, c.stream);
    else s = run_fwd<KIND, kFwdAdapt, false>("adapter_mm", a, c.stream);
    if (s != TS_OK || a.split == 1) return s;
    const unsigned grid = (unsigned)std::min<long long>(((long long)c.rows * (c.n / 4) + 255) / 256, 256 * 16);
    launch<GmmAdaptArgs>("adapter_sum", c.products == 2 ? adapter_sum_kernel<true> : adapter_sum_kernel<false>, dim3(grid),
                         dim3(256), c.stream, a);
    return check_launch("adapter_sum");
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
    if (!c.ws || c.ws_bytes < adapt_ws_bytes(c.rows, c.rank, c.products, c.w_kn != 0, c.n, c.k, c.dtype, c.odtype)) return TS_ERR_WORKSPACE;
    if (!aligned16(c.ws)) return TS_ERR_ALIGN;
    return c.dtype == TS_BF16 ? run_adapt<kGmmBf16>(c) : run_adapt<kGmmF32>(c);
}

}  // namespace

}  // namespace ts

extern "C" {

size_t ts_adapter_workspace_bytes(int rows, int rank, int products, int w_kn, int n, int k, ts_dtype dtype,
                                  ts_dtype odtype) {
    return ts::adapt_ws_bytes(rows, rank, products, w_kn != 0, n, k, dtype, odtype);
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
