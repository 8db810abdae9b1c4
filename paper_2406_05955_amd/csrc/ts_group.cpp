// Host-side checks of the grouped operators (no HIP headers; see ts_group.h).
#include "ts_group.h"

#include <algorithm>
#include <cmath>

#include "ts_plan.h"

namespace ts {

bool type_ok(ts_dtype d) { return d == TS_F32 || d == TS_BF16; }

// `quantum`: elements in 16 bytes; rows of n and of k elements are whole
// 16-byte chunks, and a weight matrix is below 4 GB.
ts_status check_group_dims(int rows, int groups, int n, int k, int quantum) {
    if (rows < 0 || rows > kMaxRows || groups < 1 || groups > kMaxGroups) return TS_ERR_SHAPE;
    if (n < quantum || k < quantum || n > kMaxDim || k > kMaxDim) return TS_ERR_SHAPE;
    if (n % quantum != 0 || k % quantum != 0) return TS_ERR_SHAPE;
    if ((unsigned long long)n * (unsigned long long)k * (16u / (unsigned)quantum) >= (1ull << 32)) return TS_ERR_SHAPE;
    return TS_OK;
}

ts_status check_route_dims(int tokens, int n_experts, int top_k) {
    if (n_experts < 1 || n_experts > kMaxExperts || top_k < 1 || top_k > kMaxTopK || top_k > n_experts)
        return TS_ERR_SHAPE;
    if (tokens < 0 || (long long)tokens * top_k > kMaxRows) return TS_ERR_SHAPE;
    return TS_OK;
}

// At most 256 workgroups, one per unit: each adds up all their counts (64 KB)
// for itself.  At least 64 tokens, four a wave.
int route_tokens_per_block(int tokens, int top_k) {
    if ((long long)tokens * top_k <= kRouteOneMax) return 0;
    return std::max(64, ceil_div(ceil_div(tokens, 256), 16) * 16);
}

size_t route_ws_bytes(int tokens, int n_experts, int top_k) {
    if (check_route_dims(tokens, n_experts, top_k) != TS_OK) return 0;
    const int tpb = route_tokens_per_block(tokens, top_k);
    if (tpb == 0) return 0;
    return align_up256((size_t)ceil_div(tokens, tpb) * kMaxExperts * sizeof(int32_t));
}

// The tile whose time is least by a simple count, in cycles: a step (128 bytes
// of contraction) takes its matrix instructions at half their peak, or its
// operands at 20 bytes a cycle and unit (what a unit draws with all units busy),
// or a round trip of 2000 cycles shared by the stages ahead and the contraction
// groups; the tiles run in rounds of 256 units.  Groups are taken as spread evenly
// over their sizes (half a tile over); a second pair's steps are not counted.
// Us, 64x32 / 64x64 / 128x64 / 128x128 / 256x128 / 256x256: down bf16 4096 x 14336 1 token 39 / 41 /
// 67 / 131 / 142 / 236, 32 tokens 181 / 172 / 153 / 232 / 192 / 322, 512 tokens 503
// / 391 / 310 / 305 / 243 / 292; one fp8 layer 4096 x 4096 100 rows 9.5 / 11 / 24 /
// 32 / 31 / 47, 2000 rows 97 / 80 / 61 / 52 / 42 / 66; 2048 x 8192 400 rows 26 / 19
// / 41 / 68 / 58 / 106.  32 x 32 / 64 x 32: plain products of few tiles and a long
// contraction, where its three contraction groups and twice the workgroups share the
// round trips: fp32 672 x 2832, 42 rows of 4 groups 18 / 30; bf16 672 x 5456, 1 token
// 11 / 15, 1024 x 4096, 100 rows 9.4 / 12; fp8 4096 x 8192, 1 row 12 / 16, 100 rows
// of 4096 x 4096 15 / 11.
GmmTileId pick_tile(GmmKind kind, bool drelu, int groups, int rows, int n, int k) {
    const int esz = kind == kGmmF32 ? 4 : kind == kGmmFp8 ? 1 : 2;
    const int used = std::max(1, std::min(groups, rows));
    const double mean = (double)rows / used;
    const double steps = (double)ceil_div(k * esz, 128);
    GmmTileId best = kTile128x64;
    double least = 0.0;
    for (int i = 0; i < kTiles; ++i) {
        const GmmTileSize &t = kTileSize[i];
        // (fp32: matrix instructions are all of the time, larger tiles gain nothing;
        // 64 x 64 had no call where it was the best)
        if (kind == kGmmF32 && (t.p == 256 || i == kTile64x64)) continue;
        if (drelu && i == kTile32x32) continue;  // (16 rows of gate and of up a wave)
        const double row_tiles = groups == 1 ? ceil_div(rows, t.q) : used * std::max(1.0, mean / t.q + 0.5);
        const double tiles = ceil_div(n, drelu ? t.p / 2 : t.p) * row_tiles;
        const double matrix = (double)t.p * t.q / (kind == kGmmF32 ? 2.0 : 16.0);
        const double step = std::max(matrix, (t.p + t.q) * 128 / 20.0);
        const double trip = 2000.0 / (t.stages - 1) / t.kw, start = 250.0 * (t.kw + 1);
        const int per_unit = tiles_per_unit(kind, i);
        double cycles;
        if (kind == kGmmF32) {
            // a unit's matrix cores take its tiles one after another; a step's
            // barrier and first reads are another 100 cycles of theirs (many tiles of
            // 32 x 32, 64 x 32, 128 x 64: 986, 896, 880 us at 2048 x 4096, 6000 rows)
            const double each = tiles / 256 < 8 ? std::ceil(tiles / 256) : tiles / 256 + 0.5;
            const double together = std::min<double>(per_unit, each);
            cycles = each * (steps * std::max(step + 100, trip / together) + start / together);
        } else {
            const double together = std::min<double>(per_unit, std::max(1.0, tiles / 256));
            const double r = tiles / (256.0 * per_unit);
            const double rounds = r < 4 ? std::ceil(r) : r + 0.5;
            cycles = rounds * (steps * std::max(together * step, trip) + start);
            // (from the second a unit on its operands, twice those of 64 x 32, are what it waits for:
            // bf16 688 x 5456, 300 rows of 8 groups 32 us, 64 x 32 21)
            if (i == kTile32x32 && tiles > 256) continue;
        }
        if (least == 0.0 || cycles < least) {
            least = cycles;
            best = (GmmTileId)i;
        }
    }
    return best;
}

}  // namespace ts
