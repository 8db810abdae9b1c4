// Operators of the MoE layer on any number of tokens: routing and row maps,
// products grouped by expert, block-scaled fp8 products, the combine.  This
// header holds what the host side shares: limits, checks (ts_group.cpp, no HIP
// headers) and the arguments of the grouped products.
#pragma once

#include <cstddef>
#include <cstdint>

#include "turbosparse.h"

namespace ts {

constexpr int kMaxRows = 1 << 23;   // tokens, rows and (token, slot) pairs of one call
constexpr int kMaxDim = 1 << 17;    // n and k of a grouped product
constexpr int kMaxGroups = 64;      // as the MoE entry points: one lane per group
constexpr int kScaleBlock = 128;    // values (rows: 128; weights: 128 x 128) per fp8 scale

constexpr int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Element kinds of a grouped product's operands.
enum GmmKind { kGmmBf16 = 0, kGmmF32 = 1, kGmmFp8 = 2 };

// Arguments of the grouped products.  "P" is the dimension contiguous in the
// output, "Q" the other one.  Forward: P = n, Q = the group's rows, contraction
// over k.  Weight gradient: P = k, Q = n, contraction over the group's rows.
struct GmmArgs {
    const char *w[2] = {nullptr, nullptr};  // weights; second pair's, or gate and up
    const char *x[2] = {nullptr, nullptr};  // rows; second pair's.  Weight gradient: x[0] = dy, w[0] = x
    const float *ws[2] = {nullptr, nullptr};
    const float *xs = nullptr;              // fp8 scales
    const int32_t *row_src = nullptr;
    const int32_t *offsets = nullptr;
    int rows = 0, src_rows = 0, groups = 1, n = 0, k = 0;
    int pairs = 1;
    void *out = nullptr, *gate = nullptr, *up = nullptr;
    int out_f32 = 0;
};

// With dReLU's activations in 8 bits (ts_keep.h): written behind gate and up
// (out: Combined), or read behind the gradient of Combined (gate, up: their
// gradients; out: Combined or null).
struct GmmKeepArgs : GmmArgs {
    uint8_t *codes = nullptr;  // [rows][n][2]
    uint8_t *exps = nullptr;   // [rows][ceil(n / 16)][2]
};

// Tiles of the forward products: columns (dReLU: of gate and up together) x
// rows, workgroups of it that a compute unit holds, stages, contraction groups.
// (equal costs: the first)
enum GmmTileId { kTile256x256 = 0, kTile128x128, kTile128x64, kTile64x32, kTile256x128, kTile64x64, kTile32x32, kTiles };
struct GmmTileSize {
    int p, q, per_unit, stages, kw;
};
constexpr GmmTileSize kTileSize[kTiles] = {{256, 256, 1, 2, 1}, {128, 128, 2, 2, 1}, {128, 64, 2, 3, 1},
                                           {64, 32, 2, 3, 2},   {256, 128, 1, 3, 1}, {64, 64, 1, 4, 2},
                                           {32, 32, 2, 3, 3}};
// (fp8 32 x 32: with its scales more than half of LDS)
constexpr int tiles_per_unit(GmmKind kind, int t) {
    return kind == kGmmFp8 && t == kTile32x32 ? 1 : kTileSize[t].per_unit;
}
// Adapters beside one group's product (ts_adapt.hip).  offsets: the segments'.
// Of the rows of each wave of the product: the rows' slots (-1: no adapter), the
// slots' adapters, how many slots.
struct GmmAdaptArgs : GmmArgs {
    // scale x A^T: [rows / 16][gate, up][room of parts][ranks' 16 bytes][16 rows][16 bytes],
    // the rows from the first segment's on: what a wave loads of a part is 1 KB in a row
    const char *t = nullptr;
    const int32_t *slots = nullptr, *slot_ad = nullptr, *slot_count = nullptr;
    const char *b[2] = {nullptr, nullptr};
    float *sums = nullptr;    // [split][rows][gate, up][n]
    int segs = 0, rank = 0, parts = 1, split = 1;
    GmmTileId tile = kTile128x64;
};
constexpr int kMaxRank = 128;
// Places that a row's parts of t take (a power of two: its lines begin alike).
constexpr int adapt_room(int parts) { return parts == 3 ? 4 : parts; }
// Rows of a wave of each tile.
constexpr int wave_rows(GmmTileId t) { return t == kTile64x32 || t == kTile32x32 ? 16 : t == kTile64x64 ? 32 : 64; }
void adapt_tile(GmmKind kind, bool drelu, bool w_kn, int rows, int n, int k, GmmTileId *tile, int *split);
GmmTileId pick_tile(GmmKind kind, bool drelu, int groups, int rows, int n, int k);

ts_status check_group_dims(int rows, int groups, int n, int k, int quantum);
bool type_ok(ts_dtype d);
constexpr int quantum(ts_dtype d) { return d == TS_F32 ? 4 : 8; }  // elements in 16 bytes
// Checks that the forward products share; TS_OK with *empty set: nothing to do.
ts_status check_fwd(const void *x, const void *w, ts_dtype dtype, ts_dtype odtype, const int32_t *row_src,
                    const int32_t *offsets, int rows, int src_rows, int groups, int n, int k, const void *out,
                    bool *empty);
ts_status check_route_dims(int tokens, int n_experts, int top_k);

// Row maps: tokens per workgroup of the two-launch form (0: one workgroup
// does it all) and its workspace.
constexpr int kRouteOneMax = 1024;  // (token, slot) pairs that one workgroup takes
int route_tokens_per_block(int tokens, int top_k);
size_t route_ws_bytes(int tokens, int n_experts, int top_k);

}  // namespace ts
