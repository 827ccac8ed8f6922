// A tile of a product of codes with few rows (i8.h): a work-group of NW waves owns 16 NF columns and up to 16 MSMAX rows of a group, its waves
// split K between them.  Operands come straight from memory into registers, kFAhead blocks of 64 k ahead; the NW partial tiles are
// added up through LDS.  As the bf16 products of few rows have it (ffn_rows.hip).
#pragma once

#include <type_traits>

#include "i8.h"

namespace moe {

constexpr int kFAhead = 4;              // k-blocks in flight per wave (even: a lane's pair of blocks stays together)

// codes of 16 bf16 values
__device__ __forceinline__ bf16x8_t codes16(const uint4 lo, const uint4 hi, float inv) {
    float f[8], g[8];
    unpack_bias8(lo, f);
    unpack_bias8(hi, g);
    uint32_t c[16];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        c[q] = i8_code_bits(f[q], inv);
        c[8 + q] = i8_code_bits(g[q], inv);
    }
    return __builtin_bit_cast(bf16x8_t, make_uint4(i8_pack4(c[0], c[1], c[2], c[3]), i8_pack4(c[4], c[5], c[6], c[7]),
                                                   i8_pack4(c[8], c[9], c[10], c[11]), i8_pack4(c[12], c[13], c[14], c[15])));
}

// columns of thread tid's part of a finished row, and the tile's number of them
template <int NF> __device__ __forceinline__ int few_column(int nt, int tid) { return nt * NF / 8 * 128 + nt * NF % 8 + (tid & 15) * 8; }
template <int NF> __host__ __device__ __forceinline__ int few_tiles(int N) { return (N + 127) / 128 * (8 / NF); }
template <int NW, int MSMAX> constexpr int few_subs() { return MSMAX > 1 ? NW / 4 : 1; }   // 16-row sub-tiles that one pass of the reduction finishes
template <int NW, int MSMAX, int NF> constexpr int few_lds_ints() { return NW * few_subs<NW, MSMAX>() * 16 * 16 * NF; }

// Tile nt, rows m0.. of group g.  part: few_lds_ints() ints of LDS.  finish(row, column, here, v): called by all threads of the work-group for
// NF finished columns of a row of the group; `here`: the row and the columns exist.  Weights are asked for before the rows are known.
// BF16: A in bf16 with a_max, whose codes each wave makes for its blocks as it needs them.
template <int NW, int MSMAX, int NF, bool BF16, class Finish>
__device__ __forceinline__ void few_tile(const I8GemmArgs& a, int g, int nt, int m0, int* part, Finish finish) {
    constexpr int SUBS = few_subs<NW, MSMAX>(), COLS = 16 * NF;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, kg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nkb = a.K / 32, p_ng = (a.N + 127) / 128;          // K counts pairs of codes, in whole blocks
    // wave w: blocks 2w, 2w + 1, 2w + 2 NW, ...
    const int whole = nkb / (2 * NW), rest = nkb - whole * 2 * NW;
    const int mine = __builtin_amdgcn_readfirstlane(whole * 2 + max(0, min(2, rest - 2 * w)));
    auto block_of = [&](int i) { return (i >> 1) * (2 * NW) + w * 2 + (i & 1); };
    const uint16_t* B = a.B + (((size_t)g * nkb * p_ng + nt * NF / 8) * 8 + nt * NF % 8) * 512 + lane * 8;
    i32x4_t bf[kFAhead][NF];
    auto load_b = [&](i32x4_t (&b)[NF], int i) {
        const uint16_t* p = B + (size_t)block_of(i) * p_ng * 4096;
#pragma unroll
        for (int j = 0; j < NF; ++j) b[j] = __builtin_bit_cast(i32x4_t, load_stream16(p + j * 512));
    };
    // rows past the end repeat an earlier one or take row 0 (a map's -1): multiplied, never stored
    const int rows = a.rows ? min(a.rows[g], a.max_rows) : a.fixed_rows;
    long long a_row[MSMAX];
#pragma unroll
    for (int ms = 0; ms < MSMAX; ++ms) {
        const int r = min(m0 + ms * 16 + c, a.max_rows - 1);
        a_row[ms] = a.row_map ? (long long)max(a.row_map[(size_t)g * a.map_stride + r], 0) : (long long)g * a.a_group_stride + r;
    }
#pragma unroll
    for (int s = 0; s < kFAhead; ++s)
        if (s < mine) load_b(bf[s], s);
    const int nrows = min(MSMAX * 16, rows - m0);

    auto run = [&](auto ms_count) {
        constexpr int MS = decltype(ms_count)::value;
        constexpr int PASSES = (MS + SUBS - 1) / SUBS;
        const uint16_t* a_src[MS];
        float inv[MS];
#pragma unroll
        for (int ms = 0; ms < MS; ++ms) {
            a_src[ms] = a.A + (size_t)a_row[ms] * a.lda + kg * (BF16 ? 16 : 8);
            inv[ms] = 0.f;
            if constexpr (BF16) inv[ms] = i8_inverse(a.a_max[a_row[ms]]);
        }
        uint4 av[kFAhead][MS][BF16 ? 2 : 1];
        auto load_a = [&](uint4 (&v)[MS][BF16 ? 2 : 1], int i) {
            const int kb = block_of(i);
#pragma unroll
            for (int ms = 0; ms < MS; ++ms) {
                const uint4* p = reinterpret_cast<const uint4*>(a_src[ms] + kb * (BF16 ? 64 : 32));
                v[ms][0] = p[0];
                if constexpr (BF16) v[ms][1] = p[1];
            }
        };
#pragma unroll
        for (int s = 0; s < kFAhead; ++s)
            if (s < mine) load_a(av[s], s);

        // this thread's part of the epilogue: row (tid / 16) of every pass, NF columns
        const int fr = tid >> 4, fc = tid & 15;
        const int n_fin = few_column<NF>(nt, tid);
        const bool fin = fr < SUBS * 16 && n_fin < a.N;
        float row_scale[PASSES], bias[NF], col_scale[NF];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = m0 + min(p * SUBS * 16 + fr, nrows - 1);
            const long long ar = a.row_map ? (long long)a.row_map[(size_t)g * a.map_stride + r] : (long long)g * a.a_group_stride + r;
            if constexpr (BF16) row_scale[p] = i8_scale(a.a_max[ar]);
            else row_scale[p] = a.a_scale[ar];
        }
        load_bias<NF>(a, g, min(n_fin, a.N - NF), bias);
#pragma unroll
        for (int f = 0; f < NF; ++f) col_scale[f] = a.b_scale[(size_t)g * a.N + min(n_fin, a.N - NF) + f];

        i32x4_t acc[MS][NF];
#pragma unroll
        for (int ms = 0; ms < MS; ++ms)
#pragma unroll
            for (int i = 0; i < NF; ++i) acc[ms][i] = i32x4_t{0, 0, 0, 0};
        auto multiply = [&](int s) {
#pragma unroll
            for (int ms = 0; ms < MS; ++ms) {
                i32x4_t v;
                if constexpr (BF16) v = __builtin_bit_cast(i32x4_t, codes16(av[s][ms][0], av[s][ms][1], inv[ms]));
                else v = __builtin_bit_cast(i32x4_t, av[s][ms][0]);
#pragma unroll
                for (int f = 0; f < NF; ++f) acc[ms][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, bf[s][f], acc[ms][f], 0, 0, 0);
            }
        };
        int i = 0;
        for (; i + 2 * kFAhead <= mine; i += kFAhead) {          // whole rounds that a whole round follows
#pragma unroll
            for (int s = 0; s < kFAhead; ++s) {
                multiply(s);
                __builtin_amdgcn_sched_barrier(0);
                load_a(av[s], i + s + kFAhead);
                load_b(bf[s], i + s + kFAhead);
                __builtin_amdgcn_sched_barrier(0);               // the refill stays here, kFAhead blocks before its use
            }
        }
        // what is on its way, and behind it what is left: fewer than kFAhead blocks
#pragma unroll
        for (int s = 0; s < kFAhead; ++s) {
            if (i + s < mine) multiply(s);
            if (i + s + kFAhead < mine) {
                load_a(av[s], i + s + kFAhead);
                load_b(bf[s], i + s + kFAhead);
            }
        }
#pragma unroll
        for (int s = 0; s < kFAhead - 1; ++s)
            if (i + s + kFAhead < mine) multiply(s);

#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            if (p > 0) lds_barrier();                            // the previous pass has been read
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                if (p * SUBS + u >= MS) break;
#pragma unroll
                for (int r = 0; r < 4; ++r)                      // D: rows 4 (lane / 16) + r, column lane % 16
#pragma unroll
                    for (int f = 0; f < NF; ++f) part[(w * SUBS * 16 + u * 16 + kg * 4 + r) * COLS + c * NF + f] = acc[p * SUBS + u][f][r];
            }
            lds_barrier();
            const int rl = p * SUBS * 16 + fr;
            const bool here = fin && rl < nrows && rl < MS * 16;
            float v[NF];
#pragma unroll
            for (int f = 0; f < NF; ++f) v[f] = 0.f;
            if (here) {
                int sum[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f) sum[f] = 0;
#pragma unroll
                for (int s = 0; s < NW; ++s)
#pragma unroll
                    for (int f = 0; f < NF; ++f) sum[f] += part[(s * SUBS * 16 + fr) * COLS + fc * NF + f];
#pragma unroll
                for (int f = 0; f < NF; ++f) v[f] = i8_value(sum[f], row_scale[p] * col_scale[f], bias[f]);
            }
            finish(m0 + rl, n_fin, here, v);
        }
    };
    if (nrows <= 0) return;
    if (MSMAX == 1 || nrows <= 16) run(std::integral_constant<int, 1>());
    else if (MSMAX == 2 || nrows <= 32) run(std::integral_constant<int, MSMAX < 2 ? MSMAX : 2>());
    else run(std::integral_constant<int, MSMAX>());
}

// NF values of a row in bf16, rounded: packed, and the bit pattern of their largest magnitude
template <int NF> __device__ __forceinline__ uint32_t few_pack(const float (&v)[NF], typename Bf16Vec<NF>::type& packed) {
    uint32_t o[(NF + 1) / 2], most = 0;
#pragma unroll
    for (int q = 0; q < (NF + 1) / 2; ++q) {
        o[q] = pack_bf16x2(v[2 * q], NF > 1 ? v[(2 * q + 1) % NF] : 0.f);
        most = max(most, (o[q] << 16) & 0x7fffffffu);
        if (NF > 1) most = max(most, o[q] & 0x7fff0000u);
    }
    __builtin_memcpy(&packed, o, sizeof packed);
    return most;
}
// the largest of a row's 16 threads
__device__ __forceinline__ uint32_t row_max_bits(uint32_t m) {
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
    return m;
}

}  // namespace moe
