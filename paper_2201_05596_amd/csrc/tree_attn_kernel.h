// The kernel of tree_attn.h; instances are spread over several files.
#pragma once

#include "tree_attn.h"

namespace moe {

// ---- one tile of the cache in registers, as loaded ---------------------------------------------------------------
// Keys: lane (r = lane % 16, g = lane / 16) holds row r of each half tile, the elements that operand word group g takes.
// Values: lane (c, g) holds elements c * DH / 16 .. of the rows 4 g .. 4 g + 3 of each half tile.
template <int KIND, int DH> struct Layout {
    static constexpr int bits = CacheKind<KIND>::bits;
    static constexpr int row = DH * bits / 8;                     // bytes per position
    static constexpr int srow = KIND == MOE_CACHE_BF16 ? 0 : DH / kScaleBlock;
    static constexpr int kload = DH / 4 * bits / 8 >= 16 ? 16 : DH / 4 * bits / 8;     // bytes per key load
    static constexpr int nk = DH / 4 * bits / 8 / kload;          // key loads per row
    static constexpr int vload = DH / 16 * bits / 8;              // bytes per value load
    // first of the 8 dimensions that word group g takes in step s of the products over the head dimension
    static __device__ __forceinline__ int dim(int s, int g) {
        constexpr int run = kload * 8 / bits;                     // consecutive elements of a lane
        return (s * 8 / run) * 4 * run + g * run + (s * 8) % run;
    }
};

// Memory from p on, of which `bytes` may be read (the same in every lane): loads behind them give 0, by lane and by scalar offset alike
typedef __amdgpu_buffer_rsrc_t Window;
__device__ __forceinline__ Window window(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}
// AUX: 2 for bytes that nobody reads again, which need not stay in the caches
template <int BYTES, int AUX = 0> __device__ __forceinline__ void load_raw(Window p, int at, int plus, uint32_t (&w)[(BYTES + 3) / 4]) {
    if constexpr (BYTES == 16) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b128(p, at, plus, AUX);
        w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3];
    } else if constexpr (BYTES == 8) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(p, at, plus, AUX);
        w[0] = v[0]; w[1] = v[1];
    } else if constexpr (BYTES == 4) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b32(p, at, plus, AUX);
    } else {
        w[0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(p, at, plus, AUX);
    }
}

// 16 HALVES positions.  ONCE: each is read by one work-group only, and the cache as a whole is too large to be there still when the
// next call reads it
template <int KIND, int DH, int HALVES, bool ONCE> struct CacheTile {
    typedef Layout<KIND, DH> L;
    static constexpr int AUX = ONCE ? 2 : 0;
    static constexpr int kw = L::kload / 4, vw = (L::vload + 3) / 4;
    uint32_t k[HALVES][L::nk][kw];
    uint32_t v[4 * HALVES][vw];
    uint32_t ks[HALVES], vs[4 * HALVES];                          // scale bytes of the rows

    // kc, kx, vc, vx: the positions that are there
    __device__ __forceinline__ void load_keys(Window kc, Window kx, int lane) {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < HALVES; ++t) {
#pragma unroll
            for (int n = 0; n < L::nk; ++n) load_raw<L::kload, AUX>(kc, r * L::row + g * L::kload, t * 16 * L::row + n * 4 * L::kload, k[t][n]);
            if constexpr (KIND != MOE_CACHE_BF16) {
                uint32_t w[1];
                load_raw<L::srow>(kx, r * L::srow, t * 16 * L::srow, w);
                ks[t] = w[0];
            }
        }
    }
    __device__ __forceinline__ void load_values(Window vc, Window vx, int lane) {
        const int c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int j = 0; j < 4 * HALVES; ++j) {
            const int at = (j >> 2) * 16 + (j & 3);
            load_raw<L::vload, AUX>(vc, g * 4 * L::row + c * L::vload, at * L::row, v[j]);
            if constexpr (KIND != MOE_CACHE_BF16) vs[j] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(vx, g * 4 * L::srow + c * L::srow / 16, at * L::srow, 0);
        }
    }

    // step s of the product over the head dimension: 8 elements of row r of half t
    __device__ __forceinline__ uint4 key(int t, int s, int lane) const {
        if constexpr (KIND == MOE_CACHE_BF16) {
            return make_uint4(k[t][s][0], k[t][s][1], k[t][s][2], k[t][s][3]);
        } else {
            const int g = lane >> 4;
            constexpr int run = L::kload * 8 / L::bits;
            const int block = L::dim(s, 0) / kScaleBlock + g * run / kScaleBlock;
            const float f = scale_value((ks[t] >> (8 * block)) & 0xffu);
            if constexpr (KIND == MOE_CACHE_FP8) {
                const uint32_t a = k[t][s / 2][s % 2 * 2], b = k[t][s / 2][s % 2 * 2 + 1];
                return make_uint4(fp8_pair<false>(a, f), fp8_pair<true>(a, f), fp8_pair<false>(b, f), fp8_pair<true>(b, f));
            } else {
                const uint32_t a = k[t][0][s];
                return make_uint4(fp4_pair<0>(a, f), fp4_pair<1>(a, f), fp4_pair<2>(a, f), fp4_pair<3>(a, f));
            }
        }
    }
    // elements 2 i and 2 i + 1 of the lane's DH / 16 of row j, in bf16
    __device__ __forceinline__ uint32_t value(int j, int i) const {
        if constexpr (KIND == MOE_CACHE_BF16) return v[j][i];
        const float f = scale_value(vs[j]);
        if constexpr (KIND == MOE_CACHE_FP8) return i & 1 ? fp8_pair<true>(v[j][i / 2], f) : fp8_pair<false>(v[j][i / 2], f);
        return i == 0 ? fp4_pair<0>(v[j][0], f) : i == 1 ? fp4_pair<1>(v[j][0], f) : i == 2 ? fp4_pair<2>(v[j][0], f) : fp4_pair<3>(v[j][0], f);
    }
};

// pairs: two elements of N positions each -> their words of the operand of V^T for the first (HIGH: the second) of them
template <bool HIGH, int N> __device__ __forceinline__ void gather(const uint32_t (&pairs)[N], uint32_t (&w)[N / 2]) {
#pragma unroll
    for (int j = 0; j < N / 2; ++j) w[j] = __builtin_amdgcn_perm(pairs[2 * j + 1], pairs[2 * j], HIGH ? 0x07060302u : 0x05040100u);
}
template <bool HIGH> __device__ __forceinline__ uint4 gather(const uint32_t (&pairs)[8]) {
    uint32_t w[4];
    gather<HIGH, 8>(pairs, w);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// the same number, worked out anew from here on: what depends on it takes no registers elsewhere
__device__ __forceinline__ int anew(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ f32x4 mfma(const uint4& a, const uint4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// over the four lanes that hold a row
__device__ __forceinline__ float row_sum(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }
__device__ __forceinline__ float row_max(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }

template <int DH, int MT> struct Rows {          // a wave's rows: lane (n, g) holds row n of every 16, elements (4 g + i) DH / 16 + q in o[.][q][i]
    f32x4 o[MT][DH / 16];
    float l[MT];                                 // sums of the lane's own positions
    float m[MT];                                 // maximum score
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            m[t] = kLowest;
            l[t] = 0.f;
#pragma unroll
            for (int q = 0; q < DH / 16; ++q) o[t][q] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
};

// The maximum moves only when a score exceeds it by 2^8: until then probabilities are at most 2^8, which sums in 32 bits and
// bf16's range take, and neither the rows' lanes nor the sums have to be touched.  ahead: 8 / c.
template <int DH, int MT> __device__ __forceinline__ void raise_maximum(Rows<DH, MT>& r, const f32x4 (&s)[MT][2], float c, float ahead) {
    bool grows = false;
    float top[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        top[t] = s[t][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top[t] = fmaxf(top[t], s[t][i / 4][i % 4]);
        grows |= top[t] > r.m[t] + ahead;
    }
    if (__any(grows)) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const float m = fmaxf(r.m[t], row_max(top[t])), f = __builtin_amdgcn_exp2f((r.m[t] - m) * c);
            r.m[t] = m;
            r.l[t] *= f;
#pragma unroll
            for (int q = 0; q < DH / 16; ++q) r.o[t][q] *= f;
        }
    }
}
// A tile's scores -> probabilities, as the second product's operands.  Scores are subtracted before the factor c: of c s - c m, with
// c m rounded, what rounding leaves grows with the scores, beyond exp2's range from 2^34 on.  Rounded to bf16 probabilities add as
// much to the result's error as its own rounding does (1.3 to 1.4 times the error without); PARTS = 2 keeps what is left in a second
// number, for a product more.
template <int DH, int MT, int PARTS>
__device__ __forceinline__ void probabilities(Rows<DH, MT>& r, const f32x4 (&s)[MT][2], float c, uint4 (&out)[MT][PARTS]) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        float p[8];
        uint32_t w[PARTS][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f((s[t][i / 4][i % 4] - r.m[t]) * c);
        r.l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
        for (int n = 0; n < PARTS; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[n][i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
                p[2 * i] -= __uint_as_float(w[n][i] << 16);
                p[2 * i + 1] -= __uint_as_float(w[n][i] & 0xffff0000u);
            }
            out[t][n] = make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]);
        }
    }
}
template <int PARTS> __device__ __forceinline__ f32x4 add_values(const uint4& v, const uint4 (&p)[PARTS], f32x4 o) {
#pragma unroll
    for (int n = PARTS - 1; n >= 0; --n) o = mfma(v, p[n], o);
    return o;
}

// bits of the row's 32 positions that it sees: the others have no score
__device__ __forceinline__ void mask_scores(f32x4 (&s)[2], uint32_t seen, int g) {
    seen >>= 4 * g;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(seen & (1u << (i / 4 * 16 + i % 4)))) s[i / 4][i % 4] = -INFINITY;
}

// Nothing of it may be in scratch memory, which build.py and the tests look at.  A version under work kept a share's bookkeeping there
// (`split`, `Piece`) and got it back wrong; that version is gone and the cause was not found.  (Where an earlier one spilled `split`, its
// assembly stores the record with all lanes active and loads it in lane 0 alone, as it should, and its results were right.)  Scalars
// beyond the registers for them are in lanes of one vector register, which nothing else writes.
template <int KIND, int DH, int MT, int WR>
__global__ __launch_bounds__(256, groups_per_unit(KIND, DH, WR)) void tree_attn_kernel(const TreeArgs a, const TreeParts parts) {
    typedef Layout<KIND, DH> L;
    constexpr int WP = 4 / WR, QT = 16 * MT, ROWS = QT * WR, KS = DH / 32, NF = DH / 16, OS = DH + 4, FRAGS = 2 * KS + NF;
    // Numbers per probability.  Beyond 32 rows per key/value head a second one takes time that nothing hides.  us with one / two: 16 x 32
    // tokens on 8 bits 117 / 137, 2 x 16 on 4 bits 102 / 124, 8 x 64 in bf16 77 / 86; up to 32 rows (16 x 8 on 4096 positions, 8 key/value
    // heads) in bf16 54.5 / 54.9, 8 bits 39.2 / 40.3, 4 bits 32.3 / 34.0.  Error against 64 bits (relative, over all elements): 0.0023 /
    // 0.0017, which is what rounding the result leaves.
    constexpr int PARTS = MT == 1 ? 2 : 1;
    constexpr bool SHARED = WR > 1;                   // a tile is in operand order in LDS, for all waves; else in its own wave's registers
    extern __shared__ uint4 lds16[];                  // SHARED: [2 rounds][2 tiles][FRAGS][64]; WP > 1, behind the steps: [4][QT][OS] and [4][QT][2] floats
    float* lds = reinterpret_cast<float*>(lds16);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WP, wp = wave % WP, n = lane & 15, g4 = lane >> 4;
    const int R = a.R;
    const float c = score_factor(DH), ahead = 8.f / c;

    // consecutive shares on one XCD: they read the same keys and values where an item's rows take several blocks
    const int w = (blockIdx.x % 8) * (parts.groups / 8) + blockIdx.x / 8;
    const Share share = share_of(a, ROWS, parts.groups, WP, w, lane);
    const int begin = share.begin, end = share.end;
    int4 split = make_int4(-1, 0, 0, 0);
    if (begin >= end) {
        if (tid == 0) parts.split[w] = split;
        return;
    }
    struct Piece {                                    // a share's part of an item
        Sequence s;
        int b, off, t0, steps, g, row0, cached;       // off: the step behind it in the sequence
        bool first;                                   // it begins where the share does
        const uint8_t *kc, *vc, *kx, *vx;
    };
    // from p.s, p.b and p.off on, with `left` steps in the share; p.steps: 0 if there is none
    auto piece = [&](Piece& p, int& left) {
        p.steps = 0;
        int item, ahead;
        for (;; left -= ahead, p.off += ahead) {      // parts of an item's beginning alone are none
            if (left <= 0) { left = 0; p.cached = p.t0 = 0; return; }
            while (p.off >= p.s.items * p.s.item_steps()) { p.off = 0; p.s = sequence<true>(a, ++p.b, ROWS); }
            item = quotient(p.off, p.s.item_steps());
            const int at = p.off - item * p.s.item_steps();
            p.t0 = max(at - kItemSteps, 0);
            ahead = min(max(kItemSteps - at, 0), left);
            if (left > ahead) break;
        }
        p.first = left == end - begin;
        left -= ahead;
        p.off += ahead;
        p.steps = min(p.s.tiles - p.t0, left);
        left -= p.steps;
        p.off += p.steps;
        p.g = quotient(item, p.s.blocks);
        p.row0 = (item - p.g * p.s.blocks) * ROWS + wr * QT;
        p.cached = min(p.t0 + p.steps, p.s.cached);
        const long long head = ((long long)p.b * a.G + p.g) * a.max_len;
        p.kc = static_cast<const uint8_t*>(a.k_cache) + head * L::row;
        p.vc = static_cast<const uint8_t*>(a.v_cache) + head * L::row;
        p.kx = KIND == MOE_CACHE_BF16 ? nullptr : a.k_scale + head * L::srow;
        p.vx = KIND == MOE_CACHE_BF16 ? nullptr : a.v_scale + head * L::srow;
        // the share that holds the item's last step: as many steps behind this part as are left of it
        if (p.t0 == 0 && p.steps < p.s.tiles)
            split = make_int4(p.b, item, w + quotient(p.s.tiles - p.steps + share.size - 1, share.size), (int)partial_slot(w, p.first));
    };
    // Keys and values of the next step are loaded into the registers that a step is done with; behind the last step nothing is
    // read (an empty window), so that loads are no branches and their waits are counted
    constexpr int HALVES = SHARED ? 1 : 2;
    // Blocks of rows read the same positions again (WR = 4).  us with loads that leave traces in the caches and without: 64 sequences
    // of 64 to 2040 positions, 16 heads in bf16 112 / 102, 128 of 1 to 4095 in 8 bits 109 / 101; four blocks of 128 rows 76 / 84.  (A
    // call on the cache of the call before it, with nothing between, can be slower without: 134 MB in 8 bits 27 / 31; in a model the
    // other layers' caches and weights pass in between.)
    typedef CacheTile<KIND, DH, HALVES, WR != 4> Tile;
    Tile tile, later;                  // SHARED: of two rounds
    // the 16 HALVES positions from `at` half tiles on
    auto there = [&](const Piece& p, const uint8_t* from, int at, int row) {
        return window(from + (long long)at * (16 * row), at < 2 * p.cached ? max(min(p.s.len - at * 16, 16 * HALVES), 0) * row : 0);
    };
    auto load_keys = [&](const Piece& p, Tile& x, int at) { x.load_keys(there(p, p.kc, at, L::row), there(p, p.kx, at, L::srow), lane); };
    auto load_values = [&](const Piece& p, Tile& x, int at) { x.load_values(there(p, p.vc, at, L::row), there(p, p.vx, at, L::srow), lane); };
    auto load_first = [&](const Piece& p) {
        if constexpr (SHARED) {
            load_keys(p, tile, 2 * p.t0 + wave);
            load_values(p, tile, 2 * p.t0 + wave);
        } else {
            load_keys(p, tile, 2 * (p.t0 + wp));
            load_values(p, tile, 2 * (p.t0 + wp));
        }
    };

    Piece next;
    next.b = share.b;
    next.off = share.off;
    next.s = sequence<true>(a, next.b, ROWS);
    int left_steps = end - begin;
    piece(next, left_steps);
    load_first(next);
    while (next.steps) {
        const Piece now = next;
        const Sequence& s = now.s;
        const int b = now.b, g = now.g, row0 = now.row0, t0 = now.t0, steps = now.steps, cached = now.cached, rows = s.count * R;
        // queries, in the order that the cache's elements come in
        uint4 q[MT][KS];
        int token[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int row = min(row0 + t * 16 + n, rows - 1);
            token[t] = row / R;
            const uint16_t* src = a.q + ((long long)b * a.N + token[t]) * a.q_stride + (g * R + row - token[t] * R) * DH;
#pragma unroll
            for (int i = 0; i < KS; ++i) q[t][i] = *reinterpret_cast<const uint4*>(src + L::dim(i, g4));
        }
        Rows<DH, MT> r;
        r.clear();

        // The drafted tokens, dealt to the waves that split positions, come first: their loads are on their way together with the
        // queries' and the first keys'.
        for (int t = max(t0, s.cached) + wp; t < t0 + steps; t += WP) {
            const int j0 = (t - s.cached) * kTile, left = s.count - j0, lane = anew(tid) & 63, n = lane & 15, g4 = lane >> 4;
            const Window kd = window(a.k + ((long long)b * a.N + j0) * a.k_stride + g * DH, (int)((min(left, kTile) - 1) * a.k_stride + DH) * 2);
            const Window vd = window(a.v + ((long long)b * a.N + j0) * a.v_stride + g * DH, (int)((min(left, kTile) - 1) * a.v_stride + DH) * 2);
            f32x4 sc[MT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    uint32_t w4[4];
                    load_raw<16>(kd, (h * 16 + n) * (int)a.k_stride * 2 + L::dim(0, g4) * 2, L::dim(i, 0) * 2, w4);
                    const uint4 k = make_uint4(w4[0], w4[1], w4[2], w4[3]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) sc[m][h] = mfma(k, q[m][i], i ? sc[m][h] : f32x4{0.f, 0.f, 0.f, 0.f});
                }
            __builtin_amdgcn_sched_barrier(0);         // the keys' registers are the values'
            uint32_t rowsv[8][DH / 32];
            uint32_t largest = 0;                      // magnitude bits of the values: infinities and NaN from 0x7f80 on
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                load_raw<DH / 8>(vd, ((j >> 2) * 16 + g4 * 4 + (j & 3)) * (int)a.v_stride * 2 + n * (DH / 8), 0, rowsv[j]);
#pragma unroll
                for (int i = 0; i < DH / 32; ++i) largest = max(largest, max(rowsv[j][i] & 0x7fffu, (rowsv[j][i] >> 16) & 0x7fffu));
            }
            uint4 p[MT][PARTS];
            uint32_t seen[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                seen[m] = seen_word(a, s, b, token[m], j0);
                mask_scores(sc[m], seen[m], g4);
            }
            raise_maximum<DH, MT>(r, sc, c, ahead);
            probabilities<DH, MT, PARTS>(r, sc, c, p);
            auto operand = [&](int f) {
                uint32_t pairs[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) pairs[j] = rowsv[j][f / 2];
                return f % 2 ? gather<true>(pairs) : gather<false>(pairs);
            };
            if (__any(largest >= 0x7f80u)) {
                // Infinities and NaN among the values are for the rows that see them, products with 0 would give them to all: added
                // here, a position at a time, and 0 in the product
#pragma unroll 1
                for (int j = 0; j < min(left, kTile); ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[DH / 32];
                        load_raw<DH / 8>(vd, j * (int)a.v_stride * 2 + (g4 * 4 + i) * (DH / 8), 0, w);
#pragma unroll
                        for (int f = 0; f < NF; ++f) {
                            const float e = __uint_as_float(f & 1 ? w[f / 2] & 0xffff0000u : w[f / 2] << 16);
                            const float add = fabsf(e) < INFINITY ? 0.f : e;
#pragma unroll
                            for (int m = 0; m < MT; ++m) r.o[m][f][i] += seen[m] >> j & 1u ? add : 0.f;
                        }
                    }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < DH / 32; ++i) {
                        if ((rowsv[j][i] & 0x7f80u) == 0x7f80u) rowsv[j][i] &= 0xffff0000u;
                        if ((rowsv[j][i] & 0x7f800000u) == 0x7f800000u) rowsv[j][i] &= 0xffffu;
                    }
            }
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const uint4 v = operand(f);
#pragma unroll
                for (int m = 0; m < MT; ++m) r.o[m][f] = add_values<PARTS>(v, p[m], r.o[m][f]);
            }
        }

        if constexpr (SHARED) {
            // A round is two tiles, of which every wave brings 16 positions into operand order; while one round is multiplied the
            // next one is written beside it and the one after that is on its way from memory.
            auto write = [&](const Tile& x, int buffer) {
                uint4* to = lds16 + (buffer * 2 + wave / 2) * FRAGS * 64 + lane;
#pragma unroll
                for (int i = 0; i < KS; ++i) to[(wave % 2 * KS + i) * 64] = x.key(0, i, lane);
                uint2* to8 = reinterpret_cast<uint2*>(to + 2 * KS * 64) + wave % 2;
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    uint32_t pairs[4], w[2];
#pragma unroll
                    for (int j = 0; j < 4; ++j) pairs[j] = x.value(j, f / 2);
                    gather<false, 4>(pairs, w);
                    to8[f * 128] = make_uint2(w[0], w[1]);
                    gather<true, 4>(pairs, w);
                    to8[(f + 1) * 128] = make_uint2(w[0], w[1]);
                }
            };
            // the round of tiles `first` and first + 1 in `buffer`; x: the next round's part
            auto round = [&](int first, int buffer, Tile& x) {
                constexpr int half = NF / 2;
                constexpr bool EARLY = KIND != MOE_CACHE_BF16;         // registers: two rounds in flight take 64 in bf16
#pragma unroll
                for (int u = wp; u < 2; u += WP) {
                    const uint4* from = lds16 + (buffer * 2 + u) * FRAGS * 64 + lane;
                    uint4 k0[KS], k1[KS], v0[half], v1[half];
                    f32x4 sc[MT][2];
#pragma unroll
                    for (int i = 0; i < KS; ++i) k0[i] = from[i * 64];
                    if (EARLY) {
#pragma unroll
                        for (int i = 0; i < KS; ++i) k1[i] = from[(KS + i) * 64];
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < KS; ++i)
#pragma unroll
                        for (int m = 0; m < MT; ++m) sc[m][0] = mfma(k0[i], q[m][i], i ? sc[m][0] : f32x4{0.f, 0.f, 0.f, 0.f});
                    if (!EARLY) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int i = 0; i < KS; ++i) k1[i] = from[(KS + i) * 64];
                    }
#pragma unroll
                    for (int f = 0; f < half; ++f) v0[f] = from[(2 * KS + f) * 64];
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < KS; ++i)
#pragma unroll
                        for (int m = 0; m < MT; ++m) sc[m][1] = mfma(k1[i], q[m][i], i ? sc[m][1] : f32x4{0.f, 0.f, 0.f, 0.f});
                    const int left = first + u < cached ? s.len - (first + u) * kTile : 0;      // 0: the last round's second tile is none
                    if (left < kTile) {
#pragma unroll
                        for (int m = 0; m < MT; ++m) mask_scores(sc[m], (1u << left) - 1, g4);
                    }
                    raise_maximum<DH, MT>(r, sc, c, ahead);
                    uint4 p[MT][PARTS];
                    probabilities<DH, MT, PARTS>(r, sc, c, p);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int f = 0; f < half; ++f) v1[f] = from[(2 * KS + half + f) * 64];
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int f = 0; f < half; ++f)
#pragma unroll
                        for (int m = 0; m < MT; ++m) r.o[m][f] = add_values<PARTS>(v0[f], p[m], r.o[m][f]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int f = 0; f < half; ++f)
#pragma unroll
                        for (int m = 0; m < MT; ++m) r.o[m][half + f] = add_values<PARTS>(v1[f], p[m], r.o[m][half + f]);
                    if (u == wp) write(x, buffer ^ 1);         // in the shadow of the products
                    __builtin_amdgcn_sched_barrier(0);
                    if (u == wp) {
                        load_keys(now, x, 2 * first + 12 + wave);
                        load_values(now, x, 2 * first + 12 + wave);
                    }
                }
                lds_barrier();
            };
            if (t0 < cached) {
                load_keys(now, later, 2 * t0 + 4 + wave);
                load_values(now, later, 2 * t0 + 4 + wave);
                write(tile, 0);
                load_keys(now, tile, 2 * t0 + 8 + wave);
                load_values(now, tile, 2 * t0 + 8 + wave);
                lds_barrier();
                for (int first = t0; first < cached; first += 4) {
                    round(first, 0, later);
                    if (first + 2 < cached) round(first + 2, 1, tile);
                }
                lds_barrier();
            }
        } else {
            for (int t = t0 + wp; t < cached; t += WP) {
                const int left = s.len - t * kTile;
                f32x4 sc[MT][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        const uint4 k = tile.key(h, i, lane);
#pragma unroll
                        for (int m = 0; m < MT; ++m) sc[m][h] = mfma(k, q[m][i], i ? sc[m][h] : f32x4{0.f, 0.f, 0.f, 0.f});
                    }
                load_keys(now, tile, 2 * (t + WP));
                if (left < kTile) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) mask_scores(sc[m], (1u << left) - 1, g4);
                }
                uint4 p[MT][PARTS];
                raise_maximum<DH, MT>(r, sc, c, ahead);
                probabilities<DH, MT, PARTS>(r, sc, c, p);
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    uint32_t pairs[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) pairs[j] = tile.value(j, f / 2);
                    const uint4 lo = gather<false>(pairs), hi = gather<true>(pairs);
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        r.o[m][f] = add_values<PARTS>(lo, p[m], r.o[m][f]);
                        r.o[m][f + 1] = add_values<PARTS>(hi, p[m], r.o[m][f + 1]);
                    }
                }
                load_values(now, tile, 2 * (t + WP));
            }
        }
        // the next part's first keys and values are on their way while this one's rows are finished
        piece(next, left_steps);
        load_first(next);

        // ---- the rows' results: to out if the item is all this share's, else into its part
        const int lane = anew(tid) & 63, n = lane & 15, g4 = lane >> 4;
        const bool whole = steps == s.tiles;
        const size_t slot = partial_slot(w, now.first);
        auto put = [&](int row, int first, const float* v, int count, float m, float l) {      // elements first.. of a row of the block
            if (row >= rows) return;
            const int local = row % ROWS;
            if (whole) {
                const int tok = row / R;
                const float f = 1.f / l, none = l == 0.f && sees_anything(a, s, b, tok) ? __uint_as_float(0x7fc00000u) : 0.f;
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (2 * i < count) o[i] = l == 0.f ? pack_bf16x2(none, none) : pack_bf16x2(v[2 * i] * f, v[2 * i + 1] * f);
                uint16_t* dst = a.out + ((long long)b * a.N + tok) * a.out_stride + (g * R + row - tok * R) * DH + first;
                if (count == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
                else *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
            } else {
                float* dst = parts.o + (slot * ROWS + local) * DH + first;
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    if (i < count) *reinterpret_cast<float4*>(dst + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                if (first == 0) *reinterpret_cast<float2*>(parts.ml + (slot * ROWS + local) * 2) = make_float2(m, l);
            }
        };
        if constexpr (WP == 1) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float l = row_sum(r.l[m]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[8];
#pragma unroll
                    for (int f = 0; f < NF; ++f) v[f] = r.o[m][f][i];
                    put(row0 + m * 16 + n, (g4 * 4 + i) * NF, v, NF, r.m[m], l);
                }
            }
        } else {
            float* ml = lds + 4 * QT * OS;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float l = row_sum(r.l[m]);
                float* o = lds + (wave * QT + m * 16 + n) * OS;
                if (g4 == 0) { ml[(wave * QT + m * 16 + n) * 2] = r.m[m]; ml[(wave * QT + m * 16 + n) * 2 + 1] = l; }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int f = 0; f < NF; f += 4)
                        *reinterpret_cast<float4*>(o + (g4 * 4 + i) * NF + f) = make_float4(r.o[m][f][i], r.o[m][f + 1][i], r.o[m][f + 2][i], r.o[m][f + 3][i]);
            }
            lds_barrier();
            for (int e = tid; e < ROWS * 16; e += 256) {           // 16 pieces of NF elements per row
                const int row = e / 16, first = e % 16 * NF, set = row / QT;
                float M = kLowest, l = 0.f, v[8] = {};
#pragma unroll
                for (int i = 0; i < WP; ++i) M = fmaxf(M, ml[((set * WP + i) * QT + row % QT) * 2]);
#pragma unroll
                for (int i = 0; i < WP; ++i) {
                    const int at = (set * WP + i) * QT + row % QT;
                    const float f = __builtin_amdgcn_exp2f((ml[at * 2] - M) * c);
                    l += ml[at * 2 + 1] * f;
#pragma unroll
                    for (int j = 0; j < NF; ++j) v[j] += lds[at * OS + first + j] * f;
                }
                put(row0 - wr * QT + row, first, v, NF, M, l);
            }
            lds_barrier();
        }
    }
    if (tid == 0) parts.split[w] = split;
}

template <int KIND, int DH, int MT, int WR> int launch_tree_instance(const TreeArgs& a, const TreeParts& parts, hipStream_t s) {
    static OncePerDevice asked;
    constexpr int tiles = WR > 1 ? 4 * (DH / 32 * 2 + DH / 16) * 1024 : 0, merge = WR < 4 ? 4 * 16 * MT * (DH + 4 + 2) * (int)sizeof(float) : 0;
    const int lds = tiles > merge ? tiles : merge;
    const int rc = ask_lds(reinterpret_cast<const void*>(&tree_attn_kernel<KIND, DH, MT, WR>), lds, asked);
    if (rc != MOE_OK) return rc;
    hipLaunchKernelGGL((tree_attn_kernel<KIND, DH, MT, WR>), dim3((unsigned)parts.groups), dim3(256), lds, s, a, parts);
    return MOE_OK;
}

template <int KIND> int launch_tree_kind(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s) {
#define MOE_TREE(DH) \
    (wr == 1 ? launch_tree_instance<KIND, DH, 1, 1>(a, p, s) : mt == 1 ? launch_tree_instance<KIND, DH, 1, 2>(a, p, s) \
     : wr == 2 ? launch_tree_instance<KIND, DH, 2, 2>(a, p, s) : launch_tree_instance<KIND, DH, 2, 4>(a, p, s))
    const int rc = head_dim == 128 ? MOE_TREE(128) : MOE_TREE(64);
#undef MOE_TREE
    return rc != MOE_OK ? rc : hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
