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
    static constexpr int per = 128 / bits;                        // elements in 16 bytes
    static constexpr int kload = DH / 4 * bits / 8 >= 16 ? 16 : DH / 4 * bits / 8;     // bytes per key load
    static constexpr int nk = DH / 4 * bits / 8 / kload;          // key loads per row
    static constexpr int vload = DH / 16 * bits / 8;              // bytes per value load
    // first of the 8 dimensions that word group g takes in step s of the products over the head dimension
    static __device__ __forceinline__ int dim(int s, int g) {
        constexpr int run = kload * 8 / bits;                     // consecutive elements of a lane
        return (s * 8 / run) * 4 * run + g * run + (s * 8) % run;
    }
};

template <int BYTES> __device__ __forceinline__ void load_raw(const uint8_t* p, uint32_t (&w)[(BYTES + 3) / 4]) {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    if constexpr (BYTES == 16) {
        const u4 v = *reinterpret_cast<const u4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (BYTES == 8) {
        const u2 v = *reinterpret_cast<const u2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
}

template <int KIND, int DH> struct CacheTile {
    typedef Layout<KIND, DH> L;
    static constexpr int kw = L::kload / 4, vw = (L::vload + 3) / 4;
    uint32_t k[2][L::nk][kw];
    uint32_t v[8][vw];
    uint32_t ks[2], vs[8];                                        // scale bytes of the rows

    // whole: all 32 positions are there; else `left` of them (at least one): the others read the last one and are not used
    __device__ __forceinline__ void load(const uint8_t* kc, const uint8_t* vc, const uint8_t* kx, const uint8_t* vx, int left, int lane) {
        const int r = lane & 15, g = lane >> 4;
        const bool whole = left >= kTile;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int p = whole ? t * 16 + r : min(t * 16 + r, left - 1);
#pragma unroll
            for (int n = 0; n < L::nk; ++n) load_raw<L::kload>(kc + p * L::row + n * 4 * L::kload + g * L::kload, k[t][n]);
            if constexpr (KIND != MOE_CACHE_BF16) {
                if constexpr (L::srow == 4) ks[t] = *reinterpret_cast<const uint32_t*>(kx + p * 4);
                else ks[t] = *reinterpret_cast<const uint16_t*>(kx + p * 2);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = (j >> 2) * 16 + g * 4 + (j & 3), p = whole ? at : min(at, left - 1);
            load_raw<L::vload>(vc + p * L::row + r * L::vload, v[j]);
            if constexpr (KIND != MOE_CACHE_BF16) vs[j] = vx[p * L::srow + r * L::srow / 16];
        }
    }

    // step s of the product over the head dimension: 8 elements of row r of half tile t
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
    // the row's DH / 16 elements in bf16; `there`: 0 where the position is none
    __device__ __forceinline__ void value(int j, bool there, uint32_t (&o)[DH / 32]) const {
        const uint32_t none = there ? ~0u : 0u;
        if constexpr (KIND == MOE_CACHE_BF16) {
#pragma unroll
            for (int i = 0; i < DH / 32; ++i) o[i] = v[j][i] & none;
        } else {
            const float f = scale_value(vs[j]);
            if constexpr (KIND == MOE_CACHE_FP8) {
#pragma unroll
                for (int i = 0; i < DH / 64; ++i) { o[2 * i] = fp8_pair<false>(v[j][i], f) & none; o[2 * i + 1] = fp8_pair<true>(v[j][i], f) & none; }
            } else {
                o[0] = fp4_pair<0>(v[j][0], f) & none;
                o[1] = fp4_pair<1>(v[j][0], f) & none;
                if constexpr (DH == 128) { o[2] = fp4_pair<2>(v[j][0], f) & none; o[3] = fp4_pair<3>(v[j][0], f) & none; }
            }
        }
    }
};

// rows[8][DH / 32]: DH / 16 elements of eight positions -> operands of V^T: fragment q is element q of each
template <int DH> __device__ __forceinline__ void transpose(const uint32_t (&rows)[8][DH / 32], uint4 (&f)[DH / 16]) {
#pragma unroll
    for (int q = 0; q < DH / 16; ++q) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)      // low or high halves of two positions' words
            w[j] = __builtin_amdgcn_perm(rows[2 * j + 1][q / 2], rows[2 * j][q / 2], q & 1 ? 0x07060302u : 0x05040100u);
        f[q] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ f32x4 mfma(const uint4& a, const uint4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// over the four lanes that hold a row
__device__ __forceinline__ float row_max(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float row_sum(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

template <int DH, int MT> struct Rows {          // a wave's rows: lane (n, g) holds row n of every 16, elements (4 g + i) DH / 16 + q in o[.][q][i]
    f32x4 o[MT][DH / 16];
    float m[MT], l[MT];                          // l: of the lane's own positions
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

// A tile's scores -> probabilities (as the second product's operand).  seen: bits of the row's 32 positions, only with MASKED.
// The maximum moves only when a score exceeds it by 2^8: until then probabilities are at most 2^8, which sums in 32 bits and
// bf16's range take, and neither the rows' lanes nor the sums have to be touched.
template <int DH, int MT, bool MASKED>
__device__ __forceinline__ uint4 probabilities(Rows<DH, MT>& r, int t, f32x4 (&s)[2], float c, uint32_t seen, int g) {
    float x[8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = s[i / 4][i % 4] * c;
        if (MASKED && !(seen >> ((i / 4) * 16 + g * 4 + i % 4) & 1u)) x[i] = -INFINITY;
        top = fmaxf(top, x[i]);
    }
    if (__any(top > r.m[t] + 8.f)) {
        const float m = fmaxf(r.m[t], row_max(top)), f = __builtin_amdgcn_exp2f(r.m[t] - m);
        r.m[t] = m;
        r.l[t] *= f;
#pragma unroll
        for (int q = 0; q < DH / 16; ++q) r.o[t][q] *= f;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(x[i] - r.m[t]);
        r.l[t] += p[i];
    }
    return make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
}

template <int KIND, int DH, int MT, int WR>
__global__ __launch_bounds__(256) void tree_attn_kernel(const TreeArgs a, const TreeParts parts) {
    typedef Layout<KIND, DH> L;
    constexpr int WP = 4 / WR, QT = 16 * MT, ROWS = QT * WR, KS = DH / 32, NF = DH / 16, OS = DH + 4;
    __shared__ long long sh[8];
    __shared__ long long found[2];
    extern __shared__ float lds[];                    // WP > 1: [4][QT][OS] and [4][QT][2]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WP, wp = wave % WP, n = lane & 15, g4 = lane >> 4;
    const int R = a.H / a.G;
    const float c = 1.44269504f * rsqrtf((float)DH);

    const Shares share = shares(a, ROWS, parts.groups, WP, sh, tid);
    // consecutive shares on one XCD: they read the same keys and values where an item's rows take several blocks
    const long long w = (blockIdx.x % 8) * (long long)(parts.groups / 8) + blockIdx.x / 8;
    long long x = w * share.size;
    const long long end = min(x + share.size, share.total), begin = x;
    if (x >= end) return;

    // the sequence that holds step x
    int b = 0;
    long long off = 0;                                // step x in the sequence
    {
        long long base = 0;
        for (int b0 = 0;; b0 += 256) {
            long long mine = 0;
            if (b0 + tid < a.n_seq) { const Sequence s = sequence(a, b0 + tid, ROWS); mine = s.items * s.tiles; }
            long long sum = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) { const long long v = __shfl_up(sum, d); if (lane >= d) sum += v; }
            if (lane == 63) sh[tid >> 6] = sum;
            __syncthreads();
            for (int i = 0; i < (tid >> 6); ++i) sum += sh[i];
            const long long all = sh[0] + sh[1] + sh[2] + sh[3];
            if (x < base + all) {
                if (x >= base + sum - mine && x < base + sum) { found[0] = b0 + tid; found[1] = base + sum - mine; }
                __syncthreads();
                b = __builtin_amdgcn_readfirstlane((int)found[0]);
                off = x - found[1];
                break;
            }
            base += all;
            __syncthreads();
        }
    }

    Sequence s = sequence(a, b, ROWS);
    while (x < end) {
        while (off >= s.items * s.tiles) { off = 0; s = sequence(a, ++b, ROWS); }
        const int item = (int)(off / s.tiles), t0 = (int)(off - (long long)item * s.tiles);
        const int steps = (int)min((long long)(s.tiles - t0), end - x);
        const int blocks = (int)(s.items / a.G), g = item / blocks, row0 = (item - g * blocks) * ROWS + wr * QT;
        const int rows = s.count * R;

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

        const long long head = ((long long)b * a.G + g) * a.max_len;
        const uint8_t* kc = static_cast<const uint8_t*>(a.k_cache) + head * L::row;
        const uint8_t* vc = static_cast<const uint8_t*>(a.v_cache) + head * L::row;
        const uint8_t* kx = KIND == MOE_CACHE_BF16 ? nullptr : a.k_scale + head * L::srow;
        const uint8_t* vx = KIND == MOE_CACHE_BF16 ? nullptr : a.v_scale + head * L::srow;
        const int cached = min(t0 + steps, s.cached);
        int t = t0 + wp;
        CacheTile<KIND, DH> next;
        auto load = [&](int at) {
            const long long p = (long long)at * kTile;
            next.load(kc + p * L::row, vc + p * L::row, kx + p * L::srow, vx + p * L::srow, s.len - (int)p, lane);
        };
        if (t < cached) load(t);
        for (; t < cached; t += WP) {
            const CacheTile<KIND, DH> tile = next;
            if (t + WP < cached) load(t + WP);
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
            uint32_t rowsv[8][DH / 32];
            uint4 vt[NF];
#pragma unroll
            for (int j = 0; j < 8; ++j) tile.value(j, (j >> 2) * 16 + g4 * 4 + (j & 3) < left, rowsv[j]);
            transpose<DH>(rowsv, vt);
            uint4 p[MT];
            if (left >= kTile) {
#pragma unroll
                for (int m = 0; m < MT; ++m) p[m] = probabilities<DH, MT, false>(r, m, sc[m], c, 0, g4);
            } else {
#pragma unroll
                for (int m = 0; m < MT; ++m) p[m] = probabilities<DH, MT, true>(r, m, sc[m], c, (1u << left) - 1, g4);
            }
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int m = 0; m < MT; ++m) r.o[m][f] = mfma(vt[f], p[m], r.o[m][f]);
        }
        // the drafted tokens
        for (; t < t0 + steps; t += WP) {
            const int j0 = (t - s.cached) * kTile, left = s.count - j0;
            const uint16_t* kd = a.k + ((long long)b * a.N + j0) * a.k_stride + g * DH;
            const uint16_t* vd = a.v + ((long long)b * a.N + j0) * a.v_stride + g * DH;
            f32x4 sc[MT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* row = kd + min(h * 16 + n, left - 1) * a.k_stride;
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const uint4 k = *reinterpret_cast<const uint4*>(row + L::dim(i, g4));
#pragma unroll
                    for (int m = 0; m < MT; ++m) sc[m][h] = mfma(k, q[m][i], i ? sc[m][h] : f32x4{0.f, 0.f, 0.f, 0.f});
                }
            }
            uint32_t rowsv[8][DH / 32];
            uint4 vt[NF];
            bool odd = false;                          // infinities and NaN among the values
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = (j >> 2) * 16 + g4 * 4 + (j & 3);
                load_raw<DH / 8>(reinterpret_cast<const uint8_t*>(vd + min(at, left - 1) * a.v_stride + n * (DH / 16)), rowsv[j]);
#pragma unroll
                for (int i = 0; i < DH / 32; ++i) {
                    rowsv[j][i] = at < left ? rowsv[j][i] : 0u;
                    odd = odd || (rowsv[j][i] & 0x7f80u) == 0x7f80u || (rowsv[j][i] & 0x7f800000u) == 0x7f800000u;
                }
            }
            transpose<DH>(rowsv, vt);
            uint4 p[MT];
            uint32_t seen[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                seen[m] = seen_word(a, s, b, token[m], j0);
                p[m] = probabilities<DH, MT, true>(r, m, sc[m], c, seen[m], g4);
            }
            if (__any(odd)) {
                // Such a value is for the rows that see it: products with 0 would give it to all.  It counts as an infinity of either
                // sign, NaN as both, in products of their own with the masks; the values proper have 0 in its place.
                const uint32_t one = 0x3f80u;
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    uint32_t up[4], down[4], w4[4] = {vt[f].x, vt[f].y, vt[f].z, vt[f].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        up[i] = down[i] = 0;
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
                            const uint32_t e = (w4[i] >> h) & 0xffffu;
                            if ((e & 0x7f80u) != 0x7f80u) continue;
                            if ((e & 0x7fu) || !(e & 0x8000u)) up[i] |= one << h;
                            if ((e & 0x7fu) || (e & 0x8000u)) down[i] |= one << h;
                            w4[i] &= ~(0xffffu << h);
                        }
                    }
                    vt[f] = make_uint4(w4[0], w4[1], w4[2], w4[3]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint32_t v4[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t two = seen[m] >> ((i / 2) * 16 + g4 * 4 + (i % 2) * 2);
                            v4[i] = (two & 1u ? one : 0u) | (two & 2u ? one << 16 : 0u);
                        }
                        const uint4 vis = make_uint4(v4[0], v4[1], v4[2], v4[3]);
                        const f32x4 zero{0.f, 0.f, 0.f, 0.f};
                        const f32x4 ups = mfma(make_uint4(up[0], up[1], up[2], up[3]), vis, zero);
                        const f32x4 downs = mfma(make_uint4(down[0], down[1], down[2], down[3]), vis, zero);
#pragma unroll
                        for (int i = 0; i < 4; ++i) r.o[m][f][i] += (ups[i] > 0.f ? INFINITY : 0.f) + (downs[i] > 0.f ? -INFINITY : 0.f);
                    }
                }
            }
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int m = 0; m < MT; ++m) r.o[m][f] = mfma(vt[f], p[m], r.o[m][f]);
        }

        // ---- the rows' results: to out if the item is all this share's, else into its part
        const bool whole = steps == s.tiles;
        const size_t slot = partial_slot(w, x == begin);
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
            __syncthreads();
            for (int e = tid; e < ROWS * 16; e += 256) {           // 16 pieces of NF elements per row
                const int row = e / 16, first = e % 16 * NF, set = row / QT;
                float M = kLowest, l = 0.f, v[8] = {};
#pragma unroll
                for (int i = 0; i < WP; ++i) M = fmaxf(M, ml[((set * WP + i) * QT + row % QT) * 2]);
#pragma unroll
                for (int i = 0; i < WP; ++i) {
                    const int at = (set * WP + i) * QT + row % QT;
                    const float f = __builtin_amdgcn_exp2f(ml[at * 2] - M);
                    l += ml[at * 2 + 1] * f;
#pragma unroll
                    for (int j = 0; j < NF; ++j) v[j] += lds[at * OS + first + j] * f;
                }
                put(row0 - wr * QT + row, first, v, NF, M, l);
            }
            __syncthreads();
        }
        x += steps;
        off += steps;
    }
}

template <int KIND, int DH, int MT, int WR> int launch_tree_instance(const TreeArgs& a, const TreeParts& parts, hipStream_t s) {
    static OncePerDevice asked;
    const int lds = WR == 4 ? 0 : 4 * 16 * MT * (DH + 4 + 2) * (int)sizeof(float);
    const int rc = ask_lds(reinterpret_cast<const void*>(&tree_attn_kernel<KIND, DH, MT, WR>), lds, asked);
    if (rc != MOE_OK) return rc;
    hipLaunchKernelGGL((tree_attn_kernel<KIND, DH, MT, WR>), dim3((unsigned)parts.groups), dim3(256), lds, s, a, parts);
    return MOE_OK;
}

template <int KIND> int launch_tree_kind(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s) {
#define MOE_TREE(DH) \
    (mt == 1 ? launch_tree_instance<KIND, DH, 1, 1>(a, p, s) : mt == 2 && wr == 1 ? launch_tree_instance<KIND, DH, 2, 1>(a, p, s) \
     : mt == 2 ? launch_tree_instance<KIND, DH, 2, 2>(a, p, s) : wr == 2 ? launch_tree_instance<KIND, DH, 4, 2>(a, p, s) \
                                                                         : launch_tree_instance<KIND, DH, 4, 4>(a, p, s))
    const int rc = head_dim == 128 ? MOE_TREE(128) : MOE_TREE(64);
#undef MOE_TREE
    return rc != MOE_OK ? rc : hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
