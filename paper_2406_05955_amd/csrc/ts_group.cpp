// Host-side checks of the grouped operators (no HIP headers; see ts_group.h).
#include "ts_group.h"

#include <algorithm>

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

// At most 256 workgroups, of at least 256 tokens: each adds up all their
// counts (64 KB) for itself.
int route_tokens_per_block(int tokens, int top_k) {
    if ((long long)tokens * top_k <= kRouteOneMax) return 0;
    return std::max(256, ceil_div(ceil_div(tokens, 256), 64) * 64);
}

size_t route_ws_bytes(int tokens, int n_experts, int top_k) {
    if (check_route_dims(tokens, n_experts, top_k) != TS_OK) return 0;
    const int tpb = route_tokens_per_block(tokens, top_k);
    if (tpb == 0) return 256;
    return align_up256((size_t)ceil_div(tokens, tpb) * kMaxExperts * sizeof(int32_t));
}

}  // namespace ts
