// Tiles of 256 columns on codes: instances of the four-wave kernel (ffn_wide.h) whose operands are codes.
#include "ffn_wide.h"

namespace moe {

int launch_i8_wide(const I8GemmArgs& first, const I8GemmArgs* second, int tile_rows, int epi, hipStream_t s) {
    if (first.G <= 0 || first.max_rows <= 0) return MOE_OK;
    if (first.K % 32 || first.N % 8 || (second && (second->K != first.K || second->N != first.N))) return MOE_ERR_INVALID_ARG;
    I8GemmArgs a = first, b = second ? *second : first;
    if (second && b.max_rows > 128 && a.max_rows <= 128) std::swap(a, b);      // the full tiles first
    // weights that one row tile reads once and that do not stay in the Infinity Cache (wide_policy in ffn_wide.hip has the figures)
    auto streams = [](const I8GemmArgs& x) { return (long long)x.G * x.K * x.N * 2 > (128ll << 20); };
    a.stream = streams(a);
    b.stream = streams(b);
    const I8GemmArgs* pb = second ? &b : nullptr;
    int policy = WIDE_CACHED;
    if (a.stream && a.max_rows <= tile_rows && (!pb || (b.stream && b.max_rows <= tile_rows))) policy = WIDE_STREAMED;
    else if (tile_rows == 256 && (a.stream || (pb && b.stream))) policy = WIDE_BY_GROUP;
    switch (epi) {
        case EPI_STORE: return launch_wide_epi<EPI_STORE>(a, pb, tile_rows, policy, s);
        case EPI_GELU: return launch_wide_epi<EPI_GELU>(a, pb, tile_rows, policy, s);
        case EPI_SCATTER: return second ? MOE_ERR_INVALID_ARG : launch_wide_epi<EPI_SCATTER>(a, pb, tile_rows, policy, s);
        default: return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace moe
