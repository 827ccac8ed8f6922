// Grouped products of codes with few rows per group (i8.h): a decode step's experts, a projection of a few tokens.  Bound by the
// read of the weights, and with few of them by how many compute units share it.  As the bf16 products of few rows have it
// (ffn_rows.hip): a work-group of eight waves owns 16 NF columns, its waves split K between them, operands come straight from
// memory into registers kAhead blocks of 64 k ahead, and the eight partial tiles are added up through LDS.
// Rows of a second product come in bf16 with their largest magnitudes, which the first one's work-groups raised as they wrote
// them; each wave makes the codes of its blocks as it needs them: no launch and no trip through memory for codes.
#include <type_traits>

#include "i8.h"

namespace moe {

namespace {

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

// NW waves, NF 16-column fragments per work-group, at most 16 MSMAX rows per tile; BF16: rows in bf16 with a_max
template <int NW, int MSMAX, int NF, int EPI, bool BF16>
__global__ __launch_bounds__(NW * 64) void i8_few_kernel(const I8GemmArgs a0, const I8GemmArgs a1, const int split,
                                                         const int n_tiles, const int m_tiles0, const int m_tiles1) {
    constexpr int SUBS = MSMAX > 1 ? NW / 4 : 1;                 // 16-row sub-tiles that one pass of the reduction finishes
    constexpr int COLS = 16 * NF;
    __shared__ __attribute__((aligned(16))) int part[NW][SUBS * 16][COLS];

    const bool second = (int)blockIdx.x >= split;                // two products may share a launch (same K and N)
    const I8GemmArgs& a = second ? a1 : a0;
    const int block = second ? (int)blockIdx.x - split : (int)blockIdx.x, m_tiles = second ? m_tiles1 : m_tiles0;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, kg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nt = block % n_tiles, mt = block / n_tiles % m_tiles, slot = block / n_tiles / m_tiles;
    // groups with rows come first in the order, and it says how many they are: the weights are asked for before the rows are known
    const int g = __builtin_amdgcn_readfirstlane(a.order ? a.order[slot] : slot);
    const bool live = a.order ? slot < (a.order[a.G] >> 1) : !a.rows || a.rows[g] > 0;
    const int m0 = mt * MSMAX * 16;

    // tokens that no expert kept have no other writer (top-1 combine): the work-group's first one is looked up here
    bool zero_first = false;
    if (EPI == EPI_SCATTER && a.zero_slot_idx) zero_first = (int)blockIdx.x < a.T && a.zero_slot_idx[blockIdx.x] < 0;

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

    auto run = [&](auto ms_count, int nrows, const long long (&a_row)[MSMAX]) {
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
        const int n_fin = nt * NF / 8 * 128 + nt * NF % 8 + fc * 8;
        const bool fin = fr < SUBS * 16 && n_fin < a.N;
        int tok[PASSES];
        float gw[PASSES], row_scale[PASSES], bias[NF], col_scale[NF];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = m0 + min(p * SUBS * 16 + fr, nrows - 1);
            const long long ar = a.row_map ? (long long)a.row_map[(size_t)g * a.map_stride + r] : (long long)g * a.a_group_stride + r;
            tok[p] = 0;
            gw[p] = 1.f;
            if (EPI == EPI_SCATTER) scatter_lookup(a, g, r, tok[p], gw[p]);
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
                    for (int f = 0; f < NF; ++f) part[w][u * 16 + kg * 4 + r][c * NF + f] = acc[p * SUBS + u][f][r];
            }
            lds_barrier();
            const int rl = p * SUBS * 16 + fr;
            const bool here = fin && rl < nrows && rl < MS * 16;
            uint32_t most = 0;
            if (here) {
                int sum[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f) sum[f] = 0;
#pragma unroll
                for (int s = 0; s < NW; ++s)
#pragma unroll
                    for (int f = 0; f < NF; ++f) sum[f] += part[s][fr][fc * NF + f];
                float v[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f) v[f] = i8_value(sum[f], row_scale[p] * col_scale[f], bias[f]);
                if constexpr (EPI == EPI_SCATTER) {
                    finish_row<EPI, NF, true>(a, g, m0 + rl, 0, n_fin, v, tok[p], gw[p]);
                } else {
                    if (EPI == EPI_GELU) {
#pragma unroll
                        for (int f = 0; f < NF; ++f) v[f] = gelu_tanh(v[f]);
                    }
                    const size_t at = (size_t)((long long)g * a.o_group_stride + m0 + rl) * a.ldo + n_fin;
                    if (a.out32) {
                        float* o = reinterpret_cast<float*>(a.out) + at;
#pragma unroll
                        for (int f = 0; f < NF; ++f) o[f] = v[f];
                    } else {
                        uint32_t o[(NF + 1) / 2];
#pragma unroll
                        for (int q = 0; q < (NF + 1) / 2; ++q) {
                            o[q] = pack_bf16x2(v[2 * q], NF > 1 ? v[(2 * q + 1) % NF] : 0.f);
                            most = max(most, (o[q] << 16) & 0x7fffffffu);
                            if (NF > 1) most = max(most, o[q] & 0x7fff0000u);
                        }
                        typedef typename Bf16Vec<NF>::type Vec;
                        Vec ov;
                        __builtin_memcpy(&ov, o, sizeof ov);
                        *reinterpret_cast<Vec*>(a.out + at) = ov;
                    }
                }
            }
            if constexpr (EPI == EPI_GELU) {                     // the row's 16 threads
                if (a.out_max) {
#pragma unroll
                    for (int s = 1; s < 16; s <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
                    if (fc == 0 && rl < nrows && rl < MS * 16 && fr < SUBS * 16) atomicMax(a.out_max + (long long)g * a.o_group_stride + m0 + rl, most);
                }
            }
        }
    };
    if (live) {
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
        if (nrows > 0) {
            if (MSMAX == 1 || nrows <= 16) run(std::integral_constant<int, 1>(), nrows, a_row);
            else if (MSMAX == 2 || nrows <= 32) run(std::integral_constant<int, MSMAX < 2 ? MSMAX : 2>(), nrows, a_row);
            else run(std::integral_constant<int, MSMAX>(), nrows, a_row);
        }
    }
    if (EPI == EPI_SCATTER && a.zero_slot_idx) {
        for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
            if (t != (int)blockIdx.x ? a.zero_slot_idx[t] < 0 : zero_first) {
                uint4* o = reinterpret_cast<uint4*>(a.out + (size_t)t * a.N);
                for (int i = tid; i < a.N / 8; i += NW * 64) o[i] = make_uint4(0, 0, 0, 0);
            }
        }
    }
}

template <int NW, int MSMAX, int NF, int EPI, bool BF16> int launch_few(const I8GemmArgs& a, const I8GemmArgs* b, hipStream_t s) {
    const int n_tiles = (a.N + 127) / 128 * (8 / NF);
    const int m0 = (a.max_rows + MSMAX * 16 - 1) / (MSMAX * 16), m1 = b ? (b->max_rows + MSMAX * 16 - 1) / (MSMAX * 16) : 1;
    const long long blocks_a = (long long)few_groups(a) * m0 * n_tiles, blocks_b = b ? (long long)few_groups(*b) * m1 * n_tiles : 0;
    if (blocks_a + blocks_b >= (1ll << 32) / (NW * 64)) return MOE_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((i8_few_kernel<NW, MSMAX, NF, EPI, BF16>), dim3((unsigned)(blocks_a + blocks_b)), dim3(NW * 64), 0, s, a,
                       b ? *b : a, (int)blocks_a, n_tiles, m0, m1);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
template <int NF, int EPI, bool BF16> int launch_few_rows(const I8GemmArgs& a, const I8GemmArgs* b, hipStream_t s) {
    const int most = b && b->max_rows > a.max_rows ? b->max_rows : a.max_rows;
    if (most <= 16) {
        // a K of few blocks: four waves (up to two blocks for each of eight)
        return a.K <= 512 ? launch_few<4, 1, NF, EPI, BF16>(a, b, s) : launch_few<8, 1, NF, EPI, BF16>(a, b, s);
    }
    if constexpr (NF <= 2) {                                     // (with 64 columns more registers than there are)
        if (most <= 32) return launch_few<8, 2, NF, EPI, BF16>(a, b, s);
        if constexpr (!BF16) return launch_few<8, 4, NF, EPI, false>(a, b, s);
    }
    return MOE_ERR_INVALID_ARG;
}
template <int EPI, bool BF16> int launch_few_columns(const I8GemmArgs& a, const I8GemmArgs* b, int NF, hipStream_t s) {
    switch (NF) {
        case 1: return launch_few_rows<1, EPI, BF16>(a, b, s);
        case 2: return launch_few_rows<2, EPI, BF16>(a, b, s);
        case 4: return launch_few_rows<4, EPI, BF16>(a, b, s);
        default: return launch_few_rows<8, EPI, BF16>(a, b, s);
    }
}

}  // namespace

// Columns of a work-group: the most that leave enough of them; 128 columns read the rows least often.  us per product: 64 experts of up
// to 16 rows, 2048 x 8192, with 16 / 32 / 64 / 128 columns 267 / 210 / 178 / 166; one row, 2048 x 6144, 5.9 / 4.2 / 6.4 with 16 / 32 / 64
// (384, 192, 96 work-groups).
static long long few_blocks(long long groups, int max_rows, int N, int nf) {
    return groups * (max_rows <= 32 ? 1 : (max_rows + 63) / 64) * ((N + 16 * nf - 1) / (16 * nf));
}
static int few_columns(long long groups, int max_rows, int N) {
    if (max_rows <= 16 && few_blocks(groups, max_rows, N, 8) >= 512) return 8;
    for (int nf = max_rows <= 16 ? 4 : 2; nf > 1; nf /= 2)
        if (few_blocks(groups, max_rows, N, nf) >= 160) return nf;
    return 1;
}

// Up to 32 rows a group, against tiles of 32 rows with h brought into codes by a launch between the products (4.4 us).  What decides is
// how many tiles of 256 columns the product with fewer columns has; with 256 of them a tile for each compute unit (64 experts of up to 16 rows, 1024 /
// 4096: 48 + 56 us here, 44 + 4 + 41 there; 50 experts of a decode step, 2048 / 8192: 138 + 142 and 128 + 4 + 128).
bool i8_few_faster(int groups, int max_rows, int d, int f) { return max_rows <= kI8FewRows && (long long)groups * (((d < f ? d : f) + 255) / 256) < 192; }
// One product of codes: 2048 x 6144 with 32 / 64 / 128 rows 7.2 / 9.6 / 15.1 us here, 64 / 128 rows in tiles 12.0 / 12.2.
bool i8_few_faster_alone(int rows, int N) { return rows <= 64 && N < 192 * 256; }

int launch_i8_few(const I8GemmArgs& a, const I8GemmArgs* b, int epi, hipStream_t s) {
    if (a.G <= 0 || a.max_rows <= 0) return MOE_OK;
    if (a.K % 32 || a.N % 8) return MOE_ERR_INVALID_ARG;
    if (b && (epi == EPI_SCATTER || b->K != a.K || b->N != a.N || (b->a_max != nullptr) != (a.a_max != nullptr))) return MOE_ERR_INVALID_ARG;
    const bool bf16 = a.a_max != nullptr;
    const int NF = few_columns(few_groups(a) + (b ? few_groups(*b) : 0), b && b->max_rows > a.max_rows ? b->max_rows : a.max_rows, a.N);
    switch (epi) {
        case EPI_STORE: return bf16 ? launch_few_columns<EPI_STORE, true>(a, b, NF, s) : launch_few_columns<EPI_STORE, false>(a, b, NF, s);
        case EPI_GELU: return bf16 ? MOE_ERR_INVALID_ARG : launch_few_columns<EPI_GELU, false>(a, b, NF, s);
        case EPI_SCATTER: return bf16 ? launch_few_columns<EPI_SCATTER, true>(a, b, NF, s) : MOE_ERR_INVALID_ARG;
        default: return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace moe
