// Tiles of 256 columns on codes: instances of the four-wave kernel (ffn_wide.h) whose operands are codes.
#include "ffn_wide.h"

namespace moe {

template <int EPI> static int launch_i8_epi(const I8GemmArgs& a, const I8GemmArgs* b, int policy, hipStream_t s) {
    return a.K % kChunk ? launch_wide_r<256, EPI, true>(a, b, policy, s) : launch_wide_r<256, EPI, false>(a, b, policy, s);
}

// Against tiles of 128 rows with three work-groups per compute unit (i8_tile.hip), which hide a tile's epilogue and stores and deal finer pieces, but load
// half as many bytes more per product.  What either takes in us, from products of 1536 to 32768 rows, N = 2048 to 8192, k = 512 to 16384 bytes: a round
// of 256 tiles here 7.5 + k / 102, there 1.9 + k / 165 (of groups 2.2 + k / 161) with 4 once, and alone on the chip 6 + k / 98.  Here / there, N = 4096: 16384 rows with k = 512 / 1024 /
// 2048 / 4096 53 / 43, 73 / 67, 116 / 122, 208 / 235; 8192 rows 28 / 26, 39 / 37, 61 / 66, 106 / 124; 4608 rows, 288 tiles, 25 / 17, 35 / 26, 54 / 45, 91 / 83;
// 2560 rows 14 / 14, 20 / 20, 30 / 32, 51 / 56.  Fewer tiles leave compute units idle that tiles of 64 rows reach (4096 rows, N = 1024, k = 2048: 17 / 11).
// Rows of groups, by their room: 32 experts of up to 256 rows, 2048 / 8192 260 / 332 for both products, 16 of up to 512 246 / 301, 64 of up to 200 rows,
// 1024 / 4096 155 / 198; 24 of up to 400 rows, 1024 / 2048 78 / 73, as said here 68; a dense branch of 8192 tokens with 32 experts of up to 320 rows, 1024 / 4096, the layer 293 / 262 (with results in bf16).  Without
// a gate's order nobody knows how much of the room is filled: tiles of 256 rows that are part empty cost less, 0.85 of a round here (24 experts of 0 to 512 rows,
// 8192 -> 2048: 174 / 195, 20 of 0 to 400, 4096 -> 2048: 87 / 103).  With a short k and 768 rows of room or more finer pieces are better
// (8 experts of 0 to 1024, 2048 -> 8192: 117 / 97, 16 of 0 to 1000, 1024 -> 4096: 85 / 65).
bool i8_wide_faster(const I8GemmArgs& a, const I8GemmArgs* b) {
    auto tiles = [&](int rows) {
        auto of = [&](const I8GemmArgs& x) { return (long long)few_groups(x) * ((x.max_rows + rows - 1) / rows); };
        return (of(a) + (b ? of(*b) : 0)) * ((a.N + kWideCols - 1) / kWideCols);
    };
    const int most = b && b->max_rows > a.max_rows ? b->max_rows : a.max_rows;
    const long long wide = tiles(256), rounds = (tiles(128) + 255) / 256;
    const double k = 2.0 * a.K;
    if (most <= 128 || wide < (k >= 4096 ? 112 : 160)) return false;
    if (a.G > 1 && !b && a.max_rows >= 768 && k <= 2048 && wide >= 512) return false;
    const double there = a.G == 1 && !b ? 1.9 + k / 165 : 2.2 + k / 161;
    const double filled = a.G > 1 && !a.order ? 0.85 : 1;
    return filled * ((wide + 255) / 256) * (7.5 + k / 102) <= (rounds == 1 ? 6 + k / 98 : 4 + rounds * there);
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
