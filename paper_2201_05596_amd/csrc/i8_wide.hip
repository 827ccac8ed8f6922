// Tiles of 256 columns on codes: instances of the four-wave kernel (ffn_wide.h) whose operands are codes.
#include "ffn_wide.h"

namespace moe {

template <int EPI> static int launch_i8_epi(const I8GemmArgs& a, const I8GemmArgs* b, int policy, hipStream_t s) {
    return a.K % kChunk ? launch_wide_r<256, EPI, true>(a, b, policy, s) : launch_wide_r<256, EPI, false>(a, b, policy, s);
}

// Against tiles of 128 rows with three work-groups per compute unit (i8_tile.hip), which hide a tile's epilogue and stores and deal finer
// pieces, but load half as many bytes more per product.  us here / there: 16384 rows, N = 4096, K = 512 / 1024 / 2048 / 4096 / 8192: 69 / 53, 92 / 77,
// 134 / 127, 230 / 242, 435 / 516; with one tile for each compute unit (4096 rows) 19 / 18, 24 / 24, 34 / 37, 55 / 65, 99 / 123; fewer than 160
// tiles of 256 rows leave compute units idle (4096 rows, N = 1024, K = 1024: 17.4 / 10.6; 1024 rows, N = 2048, K = 4096: 42 / 26); 64 experts of up to 200
// rows, 1024 x 4096 and back 78 + 64 / 91 + 90; of up to 128 rows the same; 16 of up to 512 rows, 2048 x 8192: 139 / 149; of groups with more rows, whose
// weights many row tiles share: 8 experts of up to 1024 rows, 2048 x 8192: 117 / 98; a dense branch of 8192 tokens with 32 experts of up to 320 rows,
// 1024 x 4096: 134 / 101, back 95 / 97.
bool i8_wide_faster(const I8GemmArgs& a, const I8GemmArgs* b) {
    auto tiles = [](const I8GemmArgs& x) { return (long long)few_groups(x) * ((x.max_rows + 255) / 256) * ((x.N + kWideCols - 1) / kWideCols); };
    const int most = b && b->max_rows > a.max_rows ? b->max_rows : a.max_rows;
    if (most <= 128 || tiles(a) + (b ? tiles(*b) : 0) < 160) return false;
    auto high = [&](const I8GemmArgs& x) { return x.max_rows >= 1024 ? tiles(x) : 0; };
    return !(a.K <= 1024 && high(a) + (b ? high(*b) : 0) >= 512);        // (pairs of codes)
}

int launch_i8_wide(const I8GemmArgs& first, const I8GemmArgs* second, int epi, hipStream_t s) {
    if (first.G <= 0 || first.max_rows <= 0) return MOE_OK;
    if (first.K % 32 || first.N % 8 || (second && (second->K != first.K || second->N != first.N))) return MOE_ERR_INVALID_ARG;
    I8GemmArgs a = first, b = second ? *second : first;
    // weights that one row tile reads once and that do not stay in the Infinity Cache (wide_policy in ffn_wide.hip has the figures)
    auto streams = [](const I8GemmArgs& x) { return (long long)x.G * x.K * x.N * 2 > (128ll << 20); };
    a.stream = streams(a);
    b.stream = streams(b);
    const I8GemmArgs* pb = second ? &b : nullptr;
    const int policy = a.stream && a.max_rows <= 256 && (!pb || (b.stream && b.max_rows <= 256)) ? WIDE_STREAMED
                       : a.stream || (pb && b.stream)                                           ? WIDE_BY_GROUP
                                                                                                : WIDE_CACHED;
    switch (epi) {
        case EPI_STORE: return launch_i8_epi<EPI_STORE>(a, pb, policy, s);
        case EPI_GELU: return launch_i8_epi<EPI_GELU>(a, pb, policy, s);
        case EPI_SCATTER: return second ? MOE_ERR_INVALID_ARG : launch_i8_epi<EPI_SCATTER>(a, pb, policy, s);
        default: return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace moe
