// The tile table against LDS: as many workgroups as it says that a compute unit
// holds fit its 160 KB, counted here from the tiles' sizes.
#include <cstdio>

#include "ts_group.h"

int main() {
    using namespace ts;
    int bad = 0;
    for (int kind = 0; kind < 3; ++kind)
        for (int t = 0; t < kTiles; ++t) {
            const GmmTileSize &s = kTileSize[t];
            if (s.p == 256) continue;  // (one a unit in any case)
            // four waves a contraction group; a step of both operands, 128 bytes a
            // row, and with fp8 4 bytes a thread of scales
            const int step = (s.p + s.q) * 128 + (kind == kGmmFp8 ? 256 * 4 : 0);
            const int bytes = s.kw * s.stages * step;
            const int held = tiles_per_unit((GmmKind)kind, t);
            if (held < 1 || held * bytes > 160 * 1024) {
                std::printf("kind %d tile %d: %d of %d bytes\n", kind, t, held, bytes);
                ++bad;
            }
        }
    if (!bad) std::printf("ok\n");
    return bad != 0;
}
