// Attention of several new tokens per sequence over its cached positions and, through a bit mask, over each other.
//   out[b, i, h] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q . k_j - m),  c = log2(e) / sqrt(DH),     over what token i sees
// The rows of one key/value head -- drafted tokens times the query heads that share it -- form the columns of a matrix product:
// scores K Q^T in tiles of 16 positions x 16 rows, then O^T += V^T P^T, with one pass over the positions and a running maximum
// and sum per row.  The first product's result is laid out as the second one's operand has to be, so probabilities stay in
// their lanes; keys go from memory into operand order by the choice of addresses, values by a transposition in registers.
#pragma once

#include "cache_kind.h"

namespace moe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;              // positions per step of a wave; one word of a row's mask
constexpr float kLowest = -3.40282347e38f;

struct TreePlan {                      // how the host sets a call up
    int mt, wr;                        // 16-row tiles per wave, waves with rows of their own (the other factor of 4 splits positions)
    int groups;                        // work-groups
    int row_blocks;                    // blocks of 16 mt wr rows per key/value head, at most
    size_t partial_bytes;
};

// ---- the share of a work-group ----------------------------------------------------------------------------------
// A sequence has G x (blocks of ROWS rows) items of `tiles` steps each: ceil(len / 32) over the cache, ceil(count / 32) over the
// drafted tokens.  All items' steps in a row are cut into equal shares, so that work-groups take as long as each other whatever
// the lengths are; an item that lies in several shares is merged from its parts by tree_merge_kernel.
struct Sequence {
    int len, count, cached, tiles;     // cached: steps over the cache
    long long items;
};
__device__ __forceinline__ Sequence sequence(const TreeArgs& a, int b, int ROWS) {
    Sequence s;
    s.len = min(max(a.lens[b], 0), a.max_len);
    s.count = a.counts ? min(max(a.counts[b], 0), a.N) : a.N;
    s.cached = (s.len + kTile - 1) / kTile;
    s.tiles = s.cached + (s.count + kTile - 1) / kTile;
    s.items = (long long)a.G * ((s.count * (a.H / a.G) + ROWS - 1) / ROWS);
    return s;
}

// The drafted tokens j0 .. j0 + 31 that token `tok` sees, a bit each
__device__ __forceinline__ uint32_t seen_word(const TreeArgs& a, const Sequence& s, int b, int tok, int j0) {
    const int i = tok - j0, left = s.count - j0;
    const uint32_t w = a.tree ? (uint32_t)a.tree[((long long)b * a.N + tok) * ((a.N + 31) / 32) + j0 / 32]
                              : i < 0 ? 0u : i >= 31 ? ~0u : (2u << i) - 1;           // a chain: up to its own
    return left < 32 ? w & ((1u << left) - 1) : w;
}
__device__ __forceinline__ bool sees_anything(const TreeArgs& a, const Sequence& s, int b, int tok) {
    for (int j = 0; j < s.count; j += 32)
        if (seen_word(a, s, b, tok, j)) return true;
    return s.len > 0;
}

struct TreeParts {                     // workspace: parts of items that lie in several shares
    float* o;                          // [slot][ROWS][DH]
    float* ml;                         // [slot][ROWS][2]: maximum, sum
    int groups;
};

struct Shares { long long total, size; };

// Sum and maximum over 256 threads; sh: 8 words of LDS
__device__ __forceinline__ void block_sum_max(long long& sum, int& most, long long* sh, int tid) {
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) {
        sum += __shfl_xor(sum, x);
        most = max(most, __shfl_xor(most, x));
    }
    if (tid % kWave == 0) { sh[tid / kWave] = sum; sh[4 + tid / kWave] = most; }
    __syncthreads();
    sum = sh[0] + sh[1] + sh[2] + sh[3];
    most = max(max((int)sh[4], (int)sh[5]), max((int)sh[6], (int)sh[7]));
    __syncthreads();
}

// least: steps below which a share is not worth a work-group of its own (an item that is shorter is not cut)
__device__ __forceinline__ Shares shares(const TreeArgs& a, int ROWS, int groups, int wp, long long* sh, int tid) {
    long long total = 0;
    int most = 0;
    for (int b = tid; b < a.n_seq; b += 256) {
        const Sequence s = sequence(a, b, ROWS);
        total += s.items * s.tiles;
        if (s.items) most = max(most, s.tiles);
    }
    block_sum_max(total, most, sh, tid);
    Shares r;
    r.total = total;
    r.size = (total + groups - 1) / groups;
    if (r.size > wp) r.size = (r.size + wp - 1) / wp * wp;
    r.size = max(r.size, (long long)min(most, 4 * wp));
    r.size = max(r.size, 1ll);
    return r;
}

// Where share `w` puts its part of an item that is not all its own: its first part, or the last one
__device__ __forceinline__ size_t partial_slot(long long w, bool first) { return 2 * (size_t)w + (first ? 0 : 1); }

}  // namespace moe
