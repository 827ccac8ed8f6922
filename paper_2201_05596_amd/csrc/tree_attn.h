// Attention of several new tokens per sequence over its cached positions and, through a bit mask, over each other.
//   out[b, i, h] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q . k_j - m),  c = log2(e) / sqrt(DH),     over what token i sees
// The rows of one key/value head -- drafted tokens times the query heads that share it -- form the columns of a matrix product:
// scores K Q^T in tiles of 16 positions x 16 rows, then O^T += V^T P^T, with one pass over the positions and a running maximum
// and sum per row.  The first product's result is laid out as the second one's operand has to be, so probabilities stay in
// their lanes; keys go from memory into operand order by the choice of addresses, values by a transposition in registers.
// Up to 16 rows per key/value head, in bf16 up to 64, the reading of the cache bounds it; beyond that the issue of instructions: with
// 128 rows on 8 bits the matrix unit is busy for 0.35 of the time, the vector unit (softmax, change of order, conversion) for 0.46
// and its exponentials on top of that, with two waves per SIMD to overlap them.  us without the merge (5 to 11): 64 sequences of 64
// to 2040 positions, 16 heads of 128 in bf16, 8 tokens each: 98 (5.7 TB/s); 128 of 1 to 4095, 8 heads in 8 bits, 4 rows each: 96
// (5.8 TB/s); 64 of 4096, 8 heads in 4 bits, 16 rows each: 59 (4.8 TB/s); 16 of 2000 to 16001, 8 heads in 8 bits, 128 rows each: 104
// (580 TFLOP/s); 8 of 3000 to 8100, 4 heads in bf16, 512 rows each: 65 (570 TFLOP/s).
// (The times of the rules below are from before scores were subtracted ahead of the factor c, which takes 1 to 2 % beyond 16 rows.)
#pragma once

#include "cache_kind.h"

namespace moe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;              // positions per step of a wave; one word of a row's mask
constexpr int kComputeUnits = 256;
// Work-groups of the main kernel that a compute unit takes at once, which is also how many shares there are for it; the kernel is built
// for so many.  Two have enough of the cache on its way, and a third only adds ends of items (64 sequences of 64 to 2040 positions, 16
// heads of 128 in bf16: 102 us with 512 shares, 118 with 768), unless a wave's tile is small and its own: 4096 positions in 4 bits
// 128 / 111 us, heads of 64 in 8 bits 117 / 103, in 4 bits 77 / 69.
constexpr int groups_per_unit(int kind, int head_dim, int wr) {
    const int bits = kind == MOE_CACHE_BF16 ? 16 : kind == MOE_CACHE_FP8 ? 8 : 4;
    return wr == 1 && 2 * kTile * head_dim * bits / 8 <= 4096 ? 3 : 2;
}
constexpr int kMaxGroups = 3 * kComputeUnits;
// What an item's beginning and end take, in steps.  us of the kernel with 0 / 4 / 8 / 12: 64 sequences of 50 to 1024 positions, 16
// heads of 128 in bf16 136 / 107 / 102 / 105; 64 of 100 to 8192, 8 heads in 8 bits 132 / 120 / 107 / 105
constexpr int kItemSteps = 8;
// Steps of a wave below which an item is not cut: smaller shares end sooner, but leave more to merge.  us of both kernels with
// 1 / 2 / 4 / 8, one sequence of 8 heads of 128 in 8 bits: 256 positions 14 / 15 / 11 / 11, 2048 19 / 21 / 19 / 23, 16384
// 28 / 29 / 31 / 42; four of 16384 23 / 23 / 25 / 30
constexpr int kLeastSteps = 4;
constexpr float kLowest = -3.40282347e38f;
__device__ __forceinline__ float score_factor(int head_dim) { return 1.44269504f * rsqrtf((float)head_dim); }     // c above

struct TreePlan {                      // how the host sets a call up
    int mt, wr;                        // 16-row tiles per wave; waves with rows of their own, the other factor of 4 splits positions
    int groups;                        // work-groups, a multiple of 8
    int row_blocks;                    // blocks of 16 mt wr rows per key/value head, at most
    size_t partial_bytes, ml_bytes;
};

// Quotient of values that are the same in every lane.  Divisions (and clamps) are done by the vector unit; what depends on them
// has to come back into scalar registers, or every load through a window becomes a loop over the lanes' different windows.
__device__ __forceinline__ int quotient(int a, int b) { return __builtin_amdgcn_readfirstlane(a / b); }

// ---- the share of a work-group ----------------------------------------------------------------------------------
// A sequence has G x (blocks of ROWS rows) items of `tiles` steps each: ceil(len / 32) over the cache, ceil(count / 32) over the
// drafted tokens; an item's beginning and end count as kItemSteps more, ahead of its own.  All items' steps in a row are cut into
// equal shares, so that work-groups take as long as each other whatever the lengths are; an item that lies in several shares is
// merged from its parts by tree_merge_kernel.  The host refuses shapes with 2^30 steps.
struct Sequence {
    int len, count, cached, tiles;     // cached: steps over the cache
    int blocks, items;                 // blocks of rows per key/value head
    __device__ __forceinline__ int item_steps() const { return tiles + kItemSteps; }
};
// SAME: b is the same in every lane, and so is what is read (which the compiler does not know)
template <bool SAME> __device__ __forceinline__ Sequence sequence(const TreeArgs& a, int b, int ROWS) {
    Sequence s;
    s.len = a.lens[b];
    s.count = a.counts ? a.counts[b] : a.N;
    s.len = min(max(s.len, 0), a.max_len);
    s.count = min(max(s.count, 0), a.N);
    if (SAME) { s.len = __builtin_amdgcn_readfirstlane(s.len); s.count = __builtin_amdgcn_readfirstlane(s.count); }
    s.cached = (s.len + kTile - 1) / kTile;
    s.tiles = s.cached + (s.count + kTile - 1) / kTile;
    s.blocks = (s.count * a.R + ROWS - 1) / ROWS;
    s.items = a.G * s.blocks;
    return s;
}

struct TreeParts {                     // workspace: parts of items that lie in several shares
    float* o;                          // [slot][ROWS][DH]
    float* ml;                         // [slot][ROWS][2]: maximum, sum
    int4* split;                       // per share: the item that begins and does not end in it: sequence (-1: none), item, last share, slot
    int groups;
};
// where share `w` puts its part of an item that is not all its own: its first part, or the last one
__device__ __forceinline__ size_t partial_slot(int w, bool first) { return 2 * (size_t)w + (first ? 0 : 1); }

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

struct Share {
    int begin, end, size;              // steps of all items in a row; size: of a whole share
    int b, off;                        // the sequence that holds step `begin`, and that step in it
};

// The share of work-group `w`, by each wave.  wp: positions are split over so many waves.
__device__ __forceinline__ Share share_of(const TreeArgs& a, int ROWS, int groups, int wp, int w, int lane) {
    auto steps = [&](int b, int& tiles) {
        const Sequence s = sequence<false>(a, min(b, a.n_seq - 1), ROWS);
        tiles = b < a.n_seq && s.items ? s.item_steps() : 0;
        return s.items * tiles;
    };
    int tiles, most, mine = steps(lane, most), total = mine;
    for (int b = lane + kWave; b < a.n_seq; b += kWave) {
        total += steps(b, tiles);
        most = max(most, tiles);
    }
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) {
        total += __shfl_xor(total, x);
        most = max(most, __shfl_xor(most, x));
    }
    total = __builtin_amdgcn_readfirstlane(total);
    most = __builtin_amdgcn_readfirstlane(most);
    Share r;
    r.size = quotient(total + groups - 1, groups);
    if (r.size > wp) r.size = (r.size + wp - 1) / wp * wp;
    r.size = max(r.size, max(1, min(most, kLeastSteps * wp + kItemSteps)));     // shorter items are not cut
    r.begin = (int)min((long long)w * r.size, (long long)total);
    r.end = min(r.begin + r.size, total);
    r.b = r.off = 0;
    if (r.begin >= r.end) return r;
    for (int base = 0, b0 = 0;; b0 += kWave) {
        if (b0) mine = steps(b0 + lane, tiles);
        int sum = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) { const int v = __shfl_up(sum, d); sum += lane >= d ? v : 0; }
        const uint64_t behind = __ballot(r.begin < base + sum);        // the sequences that end behind it
        if (behind) {
            const int l = __ffsll((unsigned long long)behind) - 1;
            r.b = b0 + l;
            r.off = r.begin - base - __builtin_amdgcn_readlane(sum - mine, l);
            return r;
        }
        base += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
}

}  // namespace moe
