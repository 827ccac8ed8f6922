// Grouped products of codes with few rows per group: a decode step's experts, a projection of a few tokens.  Bound by the read of the
// weights, and with few of them by how many compute units share it (i8_few.h).
// Rows of a second product come in bf16 with their largest magnitudes, which the first one's work-groups raised as they wrote
// them: no launch and no trip through memory for codes.
#include "i8_few.h"

namespace moe {

namespace {

// work-groups of a product, at least
long long few_blocks(long long groups, int max_rows, int N, int nf) {
    return groups * (max_rows <= 32 ? 1 : (max_rows + 63) / 64) * ((N + 16 * nf - 1) / (16 * nf));
}

// NW waves, NF 16-column fragments per work-group, at most 16 MSMAX rows per tile; BF16: rows in bf16 with a_max
template <int NW, int MSMAX, int NF, int EPI, bool BF16>
__global__ __launch_bounds__(NW * 64) void i8_few_kernel(const I8GemmArgs a, const int n_tiles, const int m_tiles) {
    __shared__ __attribute__((aligned(16))) int part[few_lds_ints<NW, MSMAX, NF>()];
    const int nt = blockIdx.x % n_tiles, mt = blockIdx.x / n_tiles % m_tiles;
    const int g = __builtin_amdgcn_readfirstlane((int)blockIdx.x / n_tiles / m_tiles);
    if (a.rows && a.rows[g] <= 0) return;
    few_tile<NW, MSMAX, NF, BF16>(a, g, nt, mt * MSMAX * 16, part, [&](int row, int n, bool here, float (&v)[NF]) {
        uint32_t most = 0;
        if (here) {
            if (EPI == EPI_GELU) {
#pragma unroll
                for (int f = 0; f < NF; ++f) v[f] = gelu_tanh(v[f]);
            }
            const size_t at = (size_t)((long long)g * a.o_group_stride + row) * a.ldo + n;
            if (a.out32) {
                float* o = reinterpret_cast<float*>(a.out) + at;
#pragma unroll
                for (int f = 0; f < NF; ++f) o[f] = v[f];
            } else {
                typename Bf16Vec<NF>::type o;
                most = few_pack<NF>(v, o);
                *reinterpret_cast<typename Bf16Vec<NF>::type*>(a.out + at) = o;
            }
        }
        if (EPI == EPI_GELU && a.out_max) {
            most = row_max_bits(most);
            if ((threadIdx.x & 15) == 0 && here) atomicMax(a.out_max + (long long)g * a.o_group_stride + row, most);
        }
    });
}

template <int NW, int MSMAX, int NF, int EPI, bool BF16> int launch_few(const I8GemmArgs& a, hipStream_t s) {
    const int n_tiles = few_tiles<NF>(a.N), m_tiles = (a.max_rows + MSMAX * 16 - 1) / (MSMAX * 16);
    const long long blocks = (long long)a.G * m_tiles * n_tiles;
    if (blocks >= (1ll << 32) / (NW * 64)) return MOE_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((i8_few_kernel<NW, MSMAX, NF, EPI, BF16>), dim3((unsigned)blocks), dim3(NW * 64), 0, s, a, n_tiles, m_tiles);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
template <int NF, int EPI, bool BF16> int launch_few_rows(const I8GemmArgs& a, hipStream_t s) {
    if (a.max_rows <= 16) {
        // Four waves on a K of few blocks (up to two for each of eight), and where there are work-groups enough, of which then three fit a compute unit
        // (FFN of 16 experts of up to 16 rows, 2048 / 8192: 100 -> 96 us; one row, 8192 x 2048, 128 work-groups: 6.5 with eight, 7.8 with four)
        const bool four = NF == 8 || a.K <= 512 || few_blocks(a.G, a.max_rows, a.N, NF) >= 512;      // (128 columns: there are 512)
        return four ? launch_few<4, 1, NF, EPI, BF16>(a, s) : launch_few<NF == 8 ? 4 : 8, 1, NF, EPI, BF16>(a, s);
    }
    if constexpr (NF <= 2) {                                     // (with 64 columns more registers than there are)
        if constexpr (!BF16) return a.max_rows <= 32 ? launch_few<8, 2, NF, EPI, false>(a, s) : launch_few<8, 4, NF, EPI, false>(a, s);
    }
    return MOE_ERR_INVALID_ARG;
}
template <int EPI, bool BF16> int launch_few_columns(const I8GemmArgs& a, int NF, hipStream_t s) {
    switch (NF) {
        case 1: return launch_few_rows<1, EPI, BF16>(a, s);
        case 2: return launch_few_rows<2, EPI, BF16>(a, s);
        case 4: return launch_few_rows<4, EPI, BF16>(a, s);
        default: if constexpr (EPI == EPI_GELU) return launch_few_rows<8, EPI, BF16>(a, s); else return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace

// Columns of a work-group: the most that leave enough of them; 128 columns read the rows least often.  us per product: 64 experts of up
// to 16 rows, 2048 x 8192, with 16 / 32 / 64 / 128 columns 267 / 210 / 178 / 166; one row, 2048 x 6144, 5.9 / 4.2 / 6.4 with 16 / 32 / 64
// (384, 192, 96 work-groups).  More than 32 rows: one work-group for each compute unit, with 16 columns if that is enough.
int few_columns(long long groups, int max_rows, int N) {
    if (max_rows <= 16 && few_blocks(groups, max_rows, N, 8) >= 512) return 8;
    if (max_rows > 32) return few_blocks(groups, max_rows, N, 1) > 256 ? 2 : 1;
    for (int nf = max_rows <= 16 ? 4 : 2; nf > 1; nf /= 2)
        if (few_blocks(groups, max_rows, N, nf) >= 160) return nf;
    return 1;
}

// Up to 16 rows a group, against tiles of 32 rows with h brought into codes by a launch between the products (4.4 us).  (With more rows a wave
// makes codes of two sub-tiles for each block, and takes longer: 16 experts of up to 17 / 32 rows, 1024 / 4096 57 / 67 us, that way 53 / 54.)  What decides is
// how many tiles of 256 columns the product with fewer columns has; with 256 of them a tile for each compute unit (64 experts of up to 16 rows, 1024 /
// 4096: 48 + 56 us here, 44 + 4 + 41 there; 50 experts of a decode step, 2048 / 8192: 138 + 142 and 128 + 4 + 128).
bool i8_few_faster(int groups, int max_rows, int d, int f) { return max_rows <= kI8FewRows && (long long)groups * (((d < f ? d : f) + 255) / 256) < 192; }
// One product of codes, where one work-group of 64 rows x 32 columns for each compute unit is enough: they share K among their waves, which tiles of 256
// columns do not.  us here / in tiles, N = 2048: 256 rows with K = 512 / 2048 / 8192 5.8 / 5.8, 8.6 / 12.2, 23.6 / 37.3, 384 rows (384 work-groups) 9.3 / 5.8,
// 15.1 / 12.4, 44 / 38.  (A long K is far from the read of its weights either way, about 3 us with K = 8192: every work-group
// reads all rows, and no two share a K.  Not built.)  Up to 64 rows the weights are read once: 2048 x 6144 with 32 / 64 rows 7.2 / 9.6, in tiles 12.0.
bool i8_few_faster_alone(const I8GemmArgs& a, int epi) {
    if (epi == EPI_SCATTER) return false;
    return few_blocks(a.G, a.max_rows, a.N, 2) <= 256 || (a.G == 1 && a.max_rows <= 64 && a.N < 192 * 256);
}

int launch_i8_few(const I8GemmArgs& a, int epi, hipStream_t s) {
    if (a.G <= 0 || a.max_rows <= 0) return MOE_OK;
    if (a.K % 32 || a.N % 8) return MOE_ERR_INVALID_ARG;
    const bool bf16 = a.a_max != nullptr;
    // (128 columns: first products of FFNs alone have as many work-groups where they come here at all)
    const int NF = std::min(few_columns(a.G, a.max_rows, a.N), epi == EPI_GELU ? 8 : 4);
    switch (epi) {
        case EPI_STORE: return bf16 ? launch_few_columns<EPI_STORE, true>(a, NF, s) : launch_few_columns<EPI_STORE, false>(a, NF, s);
        case EPI_GELU: return bf16 ? MOE_ERR_INVALID_ARG : launch_few_columns<EPI_GELU, false>(a, NF, s);
        default: return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace moe
