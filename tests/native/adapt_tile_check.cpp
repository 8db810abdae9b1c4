// The tile and split that adapt_tile chooses: over a grid of sizes they are ones that
// exist; with an argument it prints both for each line "kind drelu w_kn rows n k"
// that it reads.
#include <cstdio>
#include <initializer_list>

#include "ts_group.h"

#define CHECK(c)                                             \
    do {                                                     \
        if (!(c)) {                                          \
            std::printf("line %d: %s\n", __LINE__, #c);      \
            return 1;                                        \
        }                                                    \
    } while (0)

int main(int argc, char **) {
    using namespace ts;
    GmmTileId t;
    int split;
    if (argc > 1) {
        int kind, drelu, w_kn, rows, n, k;
        while (std::scanf("%d %d %d %d %d %d", &kind, &drelu, &w_kn, &rows, &n, &k) == 6) {
            adapt_tile((GmmKind)kind, drelu != 0, w_kn != 0, rows, n, k, &t, &split);
            std::printf("%d %d\n", (int)t, split);
        }
        return 0;
    }
    for (int kind = 0; kind < 2; ++kind)
        for (int mode = 0; mode < 3; ++mode)
            for (int rows : {1, 2, 16, 63, 64, 65, 300, 1000, 16384, kMaxRows})
                for (int n : {8, 72, 128, 1000, 4096, 14336, kMaxDim})
                    for (int k : {8, 72, 128, 1000, 4096, 14336, kMaxDim}) {
                        adapt_tile((GmmKind)kind, mode == 2, mode == 1, rows, n, k, &t, &split);
                        CHECK(t >= 0 && t < kTiles && split >= 1 && split <= 16);
                        CHECK(kind != kGmmF32 || (kTileSize[t].p < 256 && t != kTile64x64));
                        CHECK(kind != kGmmBf16 || t != kTile128x128);
                        CHECK(mode != 2 || t != kTile32x32);
                        // every workgroup of a split has blocks to contract
                        CHECK(split == 1 || ceil_div(k * (kind ? 4 : 2), 128) / split >= 4);
                        // a wave's rows divide a tile's
                        CHECK(kTileSize[t].q % wave_rows(t) == 0);
                    }
    std::printf("ok\n");
    return 0;
}
