// Host side of the grouped operators (ts_group.cpp): the tile choice, the
// routing launch shapes and workspace, the size checks, over a grid of sizes.
// With an argument it prints the tile's number for each line "kind drelu groups
// rows n k" that it reads.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "ts_group.h"
#include "ts_plan.h"

#define CHECK(c)                                             \
    do {                                                     \
        if (!(c)) {                                          \
            std::printf("line %d: %s\n", __LINE__, #c);      \
            return 1;                                        \
        }                                                    \
    } while (0)

int main(int argc, char **) {
    using namespace ts;
    if (argc > 1) {
        int kind, drelu, groups, rows, n, k;
        while (std::scanf("%d %d %d %d %d %d", &kind, &drelu, &groups, &rows, &n, &k) == 6)
            std::printf("%d\n", (int)pick_tile((GmmKind)kind, drelu != 0, groups, rows, n, k));
        return 0;
    }
    const int sizes[] = {1, 2, 7, 8, 16, 63, 64, 65, 128, 300, 1000, 1024, 4096, 14336, 131072};
    for (int kind = 0; kind < 3; ++kind)
        for (int drelu = 0; drelu < 2; ++drelu)
            for (int g : {1, 2, 8, 64})
                for (int rows : {1, 2, 63, 64, 1000, 16384, kMaxRows})
                    for (int n : sizes)
                        for (int k : sizes) {
                            const GmmTileId t = pick_tile((GmmKind)kind, drelu != 0, g, rows, n, k);
                            CHECK(t >= 0 && t < kTiles);
                            // fp32 has no tile of 256 and no 64 x 64
                            CHECK(kind != kGmmF32 || (kTileSize[t].p < 256 && t != kTile64x64));
                            // 32 x 32 is too narrow for gate and up side by side
                            CHECK(!drelu || t != kTile32x32);
                        }
    for (int k = 1; k <= kMaxTopK; ++k)
        for (int t : {0, 1, 2, 127, 128, 129, 512, 1024, 1025, 5000, 65536, 1000000, kMaxRows / 8}) {
            const int per = route_tokens_per_block(t, k);
            if (per == 0) {
                CHECK((long long)t * k <= kRouteOneMax && route_ws_bytes(t, 8, k) == 0);
                continue;
            }
            const int blocks = ceil_div(t, per);
            CHECK(per % 16 == 0 && blocks >= 1 && blocks <= 256 && (long long)blocks * per >= t);
            CHECK(route_ws_bytes(t, 64, k) >= (size_t)blocks * kMaxExperts * 4);
        }
    CHECK(route_ws_bytes(-1, 8, 2) == 0 && route_ws_bytes(5000, 8, 9) == 0);
    CHECK(check_group_dims(0, 1, 8, 8, 8) == TS_OK && check_group_dims(kMaxRows, 64, kMaxDim, 8, 8) == TS_OK);
    CHECK(check_group_dims(kMaxRows + 1, 1, 8, 8, 8) == TS_ERR_SHAPE && check_group_dims(1, 1, 8, 4, 8) == TS_ERR_SHAPE);
    // a weight matrix of 4 GB: 16-bit 2^31 elements, 8-bit 2^32, fp32 2^30
    CHECK(check_group_dims(1, 1, 1 << 16, 1 << 15, 8) == TS_ERR_SHAPE);
    CHECK(check_group_dims(1, 1, 1 << 16, (1 << 15) - 8, 8) == TS_OK);
    CHECK(check_group_dims(1, 1, 1 << 16, 1 << 16, 16) == TS_ERR_SHAPE);
    CHECK(check_group_dims(1, 1, 1 << 16, (1 << 16) - 16, 16) == TS_OK);
    CHECK(check_group_dims(1, 1, 1 << 15, 1 << 15, 4) == TS_ERR_SHAPE);
    std::printf("ok\n");
    return 0;
}
