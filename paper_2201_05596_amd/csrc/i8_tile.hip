// Tiles of 128, 64 or 32 rows x 256 columns on codes (i8.h), two or three work-groups per compute unit: one's epilogue and stores run beside the
// others' matrix instructions.  The four-wave kernel of 256-row tiles (ffn_wide.h) has one work-group per unit, whose epilogue and
// stores nothing hides: on codes its main loop is half as long, and with a short K that is most of a tile's time.
//
// A wave owns every other 16-row sub-tile of 128 columns: 128 accumulator registers with 128 rows, operands of one 64-deep stage.  Stages go
// from memory straight to LDS; a stage's barrier also frees the slot that the stage before it left.  Two stages in the ring with 128 rows: then
// three work-groups fit, and what a short ring does not hide the others do (16384 rows, N = 4096, K = 512 / 1024 / 2048: 44 / 69 / 128 us, with
// three stages and two work-groups 51 / 77 / 136); three with fewer rows, where 32 rows take 18 KB of weights and rows for each stage and loads are all there is.
// Bound by what a compute unit takes in by direct loads (46 to 60 GB/s with 256 of them at work): 128 rows of codes of 16384 x 2048 x 4096 105 us
// = 2.6 PFLOP/s; 50 experts of a decode step, 2048 x 8192 with up to 16 rows, 128 us = 6.6 TB/s of codes.
#include "ffn_wide.h"

namespace moe {

namespace {

constexpr int kTileCols = 256, kTileThreads = 256;
// stages in the ring: with 128 rows two, for three work-groups per compute unit
constexpr int tile_stages(int rows) { return rows == 128 ? 2 : 3; }

// ROWS: 128, 64 or 32 rows of a tile; NT: weights with the non-temporal hint
template <int ROWS, int EPI, bool NT>
__global__ __launch_bounds__(kTileThreads, ROWS == 128 ? 3 : 2) void i8_tile_kernel(const I8GemmArgs a0, const I8GemmArgs a1, const int split) {
    constexpr int NS = tile_stages(ROWS), STAGE = 64 * (ROWS + kTileCols);               // bytes of a stage: activations, then weights
    static_assert((ROWS == 128 ? 3 : 2) * NS * STAGE <= 160 * 1024 && NS * STAGE >= 4 * 1280, "work-groups per compute unit; room for the epilogue's tables");
    const bool second = EPI != EPI_SCATTER && (int)blockIdx.x >= split;   // uniform over the work-group (a combine is a launch of its own)
    const I8GemmArgs& a = second ? a1 : a0;
    const int block = second ? (int)blockIdx.x - split : (int)blockIdx.x;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, kg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 1, wn = w & 1;

    const int n_tiles = (a.N + kTileCols - 1) / kTileCols;
    const int m_tiles = (a.max_rows + ROWS - 1) / ROWS;
    const TileId tile = tile_spread(a, n_tiles) ? tile_of_block_spread(a, n_tiles, m_tiles, block)
                                                : tile_of_block(a, n_tiles, m_tiles, block);
    const int g = tile.g, n0 = tile.nt * kTileCols, m0 = tile.inner * ROWS;
    if (EPI == EPI_SCATTER) zero_dropped_rows(a, tid, kTileThreads);
    if (!tile.live) return;
    const int rows = a.rows ? min(a.rows[g], a.max_rows) : a.fixed_rows;
    if (m0 >= rows) return;
    const int nrows = min(ROWS, rows - m0);

    auto run = [&](auto act_c) {
        constexpr int ACT = decltype(act_c)::value;              // sub-tiles of a wave: 32 ACT rows
        constexpr int NA = ACT / 2 > 0 ? ACT / 2 : 1, PER = NA + 4;      // direct loads of a wave and stage
        const int stages = a.K / 32;
        // activations: load i of wave w copies 64 bytes of 16 rows; slot lane % 4 of a row holds k-piece slot ^ (row / 4 % 4), with which 16
        // lanes next to each other, reading a piece of 16 rows, would meet every bank once.  The counter says that those which are served together do
        // not: 1.2 conflicts per LDS instruction with 128 rows (four of twelve reads are the rows'), 0.5 with 32
        int row[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) row[i] = m0 + min(((w * NA + i) % (2 * ACT)) * 16 + (lane >> 2), nrows - 1);   // past the end: the last valid one
        int s_row = m0 + min(tid, nrows - 1);
        if (a.row_map) {
            const int32_t* map = a.row_map + (size_t)g * a.map_stride;
#pragma unroll
            for (int i = 0; i < NA; ++i) row[i] = map[row[i]];
            s_row = map[s_row];
        }
        const size_t first = a.row_map ? (size_t)0 : (size_t)g * a.a_group_stride;
        const int n_mine = min(n0 + tid, a.N - 1);               // one row's scale, one column's scale and bias for each thread
        const float row_scale = a.a_scale[first + s_row], col_scale = a.b_scale[(size_t)g * a.N + n_mine];
        const float bias = a.bias ? bf16_to_f32(a.bias[(size_t)g * a.N + n_mine]) : 0.f;
        int token = 0;                                           // top-1 combine: a row's token and gate weight for each thread
        float gate = 0.f;
        if constexpr (EPI == EPI_SCATTER) scatter_lookup(a, g, m0 + min(tid, nrows - 1), token, gate);
        const uint16_t* a_src[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) a_src[i] = a.A + (first + row[i]) * a.lda + ((lane & 3) ^ (lane >> 4)) * 8;
        // weights: wave w copies fragments 4 w .. 4 w + 3 of the tile's sixteen
        const int p_ng = (a.N + 127) / 128, p_grp = min(n0 / 128 + w / 2, p_ng - 1);       // clamped group: loaded, never stored
        const size_t b_step = (size_t)p_ng * 4096;
        const uint16_t* b_src = a.B + ((size_t)g * stages * p_ng + p_grp) * 4096 + (w & 1) * 2048 + lane * 8;
        const uint32_t b_dst = __builtin_amdgcn_readfirstlane(lds0 + 64 * ROWS + w * 4096);
        auto fill = [&](int stage, uint32_t slot) {
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                set_m0<0>(__builtin_amdgcn_readfirstlane(lds0 + slot + ((w * NA + i) % (2 * ACT)) * 1024));
                dma16_at<0, false>(a_src[i] + (size_t)stage * 32);
            }
            const uint16_t* b = b_src + (size_t)stage * b_step;
            set_m0<0>(b_dst + slot);
            dma16_at<0, NT>(b);
            dma16_at<1024, NT>(b);
            dma16_at<2048, NT>(b);
            dma16_at<3 * 1024, NT>(b);
        };
        i32x4_t acc[ACT][8];
#pragma unroll
        for (int i = 0; i < ACT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
        const int a_lane = (wm * 16 + c) * 64 + (kg ^ (c >> 2)) * 16, b_lane = 64 * ROWS + wn * 8192 + lane * 16;
        auto multiply = [&](uint32_t slot) {
            i32x4_t af[ACT], bf[8];
#pragma unroll
            for (int i = 0; i < ACT; ++i) af[i] = *reinterpret_cast<const i32x4_t*>(lds + slot + a_lane + i * 2048);
#pragma unroll
            for (int j = 0; j < 8; ++j) bf[j] = *reinterpret_cast<const i32x4_t*>(lds + slot + b_lane + j * 1024);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < ACT; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(af[i], bf[j], acc[i][j], 0, 0, 0);
        };
        // Stage s: its loads and no others are waited for (a wave issues PER a stage, NS - 1 stages ahead, and loads complete in order);
        // behind the barrier every wave has them, and has read stage s - 1, whose slot stage s + NS - 1 takes.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) fill(min(s, stages - 1), s * STAGE);        // (past the end: the last one again, for the count)
        uint32_t rd = 0, wr = (NS - 1) * STAGE;
        for (int s = 0; s < stages; ++s) {
            wait_vmcnt_barrier<(NS - 2) * PER>();
            if (s + NS - 1 < stages) fill(s + NS - 1, wr);
            else if (s + 1 < stages) fill(stages - 1, wr);
            multiply(rd);
            rd = rd == (NS - 1) * STAGE ? 0 : rd + STAGE;
            wr = wr == (NS - 1) * STAGE ? 0 : wr + STAGE;
        }

        // ---- epilogue ----------------------------------------------------------------------------------------
        float* share = reinterpret_cast<float*>(lds);            // rows' scales, columns' scales, columns' biases, rows' gate weights and tokens
        wait_vmcnt_barrier<0>();                                 // the ring has been read
        share[tid] = row_scale;
        share[256 + tid] = col_scale;
        share[512 + tid] = bias;
        if constexpr (EPI == EPI_SCATTER) {
            share[768 + tid] = gate;
            share[1024 + tid] = __int_as_float(token);
        }
        __syncthreads();
        const int n_lane = n0 + wn * 128 + c * 8;
        if (n_lane >= a.N) return;
        float cs[8], b8[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = share[256 + wn * 128 + c * 8 + j];
            b8[j] = share[512 + wn * 128 + c * 8 + j];
        }
#pragma unroll
        for (int i = 0; i < ACT; ++i) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int rl = (2 * i + wm) * 16 + kg * 4 + r;   // D: rows 4 (lane / 16) + r, column lane % 16
                const float rs = share[rl];
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = i8_value(acc[i][j][r], rs * cs[j], b8[j]);
                if constexpr (EPI == EPI_GELU) gelu_tanh8(v);
                if (rl >= nrows) continue;
                if constexpr (EPI == EPI_SCATTER) {
                    finish_row<EPI, 8>(a, g, m0 + rl, 0, n_lane, v, __float_as_int(share[1024 + rl]), share[768 + rl]);
                } else {
                    const size_t at = ((size_t)g * a.o_group_stride + m0 + rl) * a.ldo + n_lane;
                    if (a.out32) {
                        float* o = reinterpret_cast<float*>(a.out) + at;
                        *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
                    } else {
                        const uint4 o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                        store_stream16(a.out + at, o);
                    }
                }
            }
        }
    };
    if (ROWS > 64 && nrows > 64) run(std::integral_constant<int, ROWS / 32>());
    else if (ROWS > 32 && nrows > 32) run(std::integral_constant<int, ROWS < 64 ? 1 : 2>());
    else run(std::integral_constant<int, 1>());
}

template <int ROWS, int EPI, bool NT> int launch_tile(const I8GemmArgs& a, const I8GemmArgs* b, hipStream_t s) {
    const int n_tiles = (a.N + kTileCols - 1) / kTileCols, bytes = tile_stages(ROWS) * 64 * (ROWS + kTileCols);
    const long long blocks_a = tile_grid_blocks(a, n_tiles, (a.max_rows + ROWS - 1) / ROWS);
    const long long blocks = blocks_a + (b ? tile_grid_blocks(*b, n_tiles, (b->max_rows + ROWS - 1) / ROWS) : 0);
    if (blocks >= 1ll << 24) return MOE_ERR_UNSUPPORTED;
    static OncePerDevice asked;
    const int rc = ask_lds(reinterpret_cast<const void*>(&i8_tile_kernel<ROWS, EPI, NT>), bytes, asked);
    if (rc != MOE_OK) return rc;
    hipLaunchKernelGGL((i8_tile_kernel<ROWS, EPI, NT>), dim3((unsigned)blocks), dim3(kTileThreads), bytes, s, a, b ? *b : a, (int)blocks_a);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
// Rows of a tile: as many as the groups have, fewer where the tiles would leave compute units without work
int tile_rows(const I8GemmArgs& a, const I8GemmArgs* b, int most) {
    auto tiles = [&](int rows) {
        auto of = [&](const I8GemmArgs& x) { return (long long)few_groups(x) * ((x.max_rows + rows - 1) / rows); };
        return (of(a) + (b ? of(*b) : 0)) * ((a.N + kTileCols - 1) / kTileCols);
    };
    if (most > 64 && tiles(128) >= 160) return 128;
    return most > 32 && tiles(64) >= 80 ? 64 : 32;
}
template <int EPI> int launch_tile_rows(const I8GemmArgs& a, const I8GemmArgs* b, hipStream_t s) {
    const int most = b && b->max_rows > a.max_rows ? b->max_rows : a.max_rows;
    const int rows = tile_rows(a, b, most);
    // weights that one row tile reads and that do not stay in the Infinity Cache
    auto streams = [&](const I8GemmArgs& x) { return (long long)x.G * x.K * x.N * 2 > (128ll << 20) && x.max_rows <= rows; };
    const bool nt = streams(a) && (!b || streams(*b));
#define MOE_TILE(ROWS) return nt ? launch_tile<ROWS, EPI, true>(a, b, s) : launch_tile<ROWS, EPI, false>(a, b, s)
    if (rows == 32) MOE_TILE(32);
    if (rows == 64) MOE_TILE(64);
    MOE_TILE(128);
#undef MOE_TILE
}

}  // namespace

int launch_i8_tile(const I8GemmArgs& a, const I8GemmArgs* b, int epi, hipStream_t s) {
    if (a.G <= 0 || a.max_rows <= 0) return MOE_OK;
    if (a.K % 32 || a.N % 8 || (b && (b->K != a.K || b->N != a.N))) return MOE_ERR_INVALID_ARG;
    switch (epi) {
        case EPI_STORE: return launch_tile_rows<EPI_STORE>(a, b, s);
        case EPI_GELU: return launch_tile_rows<EPI_GELU>(a, b, s);
        case EPI_SCATTER: return b ? MOE_ERR_INVALID_ARG : launch_tile_rows<EPI_SCATTER>(a, b, s);
        default: return MOE_ERR_INVALID_ARG;
    }
}

}  // namespace moe
