// The products of a whole MoE layer for few tokens in two launches (the gate is the third): the first products of all experts that have rows and
// of the dense branch, then their second products with the combine.  Bound by latency with a token or two, by the read of the weights
// with more (i8_few.h).
// The first launch takes the tokens in bf16 with their largest magnitudes, which the gate's launch finds on its way, and the second one h with those
// that the first one raises: no launch makes codes.  With the fewest tokens a work-group of the second one has its columns of every group.  Else
// the work-group that finishes a column tile's last group adds the groups' results up for every token, in 32 bits, and rounds once: nobody waits for
// anybody.  Its hand-over across the XCDs' separate L2s costs about 4 us: results are written with device-scope stores (through the L2), a work-group
// waits for its stores before it counts itself, and the last one acquires at device scope before its loads.  The counters are cleared by the
// gate's launch.
// One token, top-2 of 128 experts beside a dense branch, 1024 / 4096: 6.7 + 8.6 us behind a gate of 9.2, with a hand-over (eight waves) 6.7 + 11.2; as launches that
// bring x into codes, multiply, multiply and combine 4.2 + 6.3 + 6.0 + 4.1.  Tried: both products in one launch, work-groups taking tiles by ticket and
// those of the second product waiting for a flag of their group: 27.6 us (11 ns for each ticket, and every hand-over is a chain of stores, count, flag and loads across the L2s).
#include "i8_few.h"

namespace moe {

namespace {

// Four waves: a work-group is a chain of trips to memory, and of those with 130 registers a wave three fit a compute unit, with eight waves and more registers
// one (us for the layer: 16 tokens, top-2 of 64 experts beside a dense branch, 1024 / 4096 72 -> 61, 8 tokens, top-1 of 64, 2048 / 8192 67 -> 60).
constexpr int kTokenWaves = 4, kTokenThreads = kTokenWaves * 64;

// a work-group's tile: columns fastest; the dense branch comes first, then the experts with rows in the gate's order
struct TokenTile {
    int g, nt, groups;
    bool dense, live;
};
__device__ __forceinline__ TokenTile token_tile(const I8TokenArgs& t, int n_tiles) {
    const int group = blockIdx.x / n_tiles, dense = t.dense ? 1 : 0;
    TokenTile r;
    r.nt = blockIdx.x % n_tiles;
    r.dense = group < dense;
    const int expert = r.dense ? 0 : t.order[group - dense];
    const int live = t.order[t.E] >> 1;
    r.groups = __builtin_amdgcn_readfirstlane(dense + live);
    r.live = group < r.groups;
    r.g = __builtin_amdgcn_readfirstlane(expert);
    return r;
}

// XBF16: x in bf16 with the tokens' largest magnitudes, else codes with scales
template <int NF, bool XBF16>
__global__ __launch_bounds__(kTokenThreads) void i8_token_first_kernel(const I8TokenArgs t) {
    __shared__ __attribute__((aligned(16))) int part[few_lds_ints<kTokenWaves, 1, NF>()];
    const TokenTile tile = token_tile(t, few_tiles<NF>(t.experts.N));
    if (!tile.live) return;
    const I8GemmArgs& a = tile.dense ? t.dense_branch : t.experts;
    few_tile<kTokenWaves, 1, NF, XBF16>(a, tile.g, tile.nt, 0, part, [&](int row, int n, bool here, float (&v)[NF]) {
        uint32_t most = 0;
        const long long r = (long long)tile.g * a.o_group_stride + row;
        if (here) {
#pragma unroll
            for (int f = 0; f < NF; ++f) v[f] = gelu_tanh(v[f]);
            typename Bf16Vec<NF>::type o;
            most = few_pack<NF>(v, o);
            *reinterpret_cast<typename Bf16Vec<NF>::type*>(a.out + r * a.ldo + n) = o;
        }
        most = row_max_bits(most);
        if ((threadIdx.x & 15) == 0 && here) atomicMax(a.out_max + r, most);
    });
}

template <int NF>
__global__ __launch_bounds__(kTokenThreads) void i8_token_second_kernel(const I8TokenArgs t) {
    __shared__ __attribute__((aligned(16))) int part[few_lds_ints<kTokenWaves, 1, NF>()];
    __shared__ int shared_last;
    const int tid = threadIdx.x, N = t.experts.N;
    const TokenTile tile = token_tile(t, few_tiles<NF>(N));
    if (!tile.live) return;
    // where the results of token tid / 16 will be, in case that this is the last work-group
    struct Source { int slot, expert; float gate; };
    Source src[2];
    auto look_up = [&](int token) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = min(token, t.T - 1) * t.top_k + min(j, t.top_k - 1);
            src[j] = {t.slot_idx[at], t.expert_idx[at], t.gate_w[at]};
            if (j >= t.top_k) src[j].slot = -1;
        }
    };
    look_up(tid >> 4);
    const I8GemmArgs& a = tile.dense ? t.dense_branch : t.experts;
    few_tile<kTokenWaves, 1, NF, true>(a, tile.g, tile.nt, 0, part, [&](int row, int n, bool here, float (&v)[NF]) {
        if (!here) return;
        float* o = reinterpret_cast<float*>(a.out) + ((long long)tile.g * a.o_group_stride + row) * N + n;
#pragma unroll
        for (int f = 0; f < NF; ++f) __hip_atomic_store(o + f, v[f], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this thread's results have left the L2 ...
    __syncthreads();                                             // ... and every thread's of the work-group, before it is counted
    if (tid == 0) shared_last = __hip_atomic_fetch_add(t.done + tile.nt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)tile.groups - 1;
    __syncthreads();
    if (!shared_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");           // nothing read below comes from a stale cache line
    const float* ye = reinterpret_cast<const float*>(t.experts.out);
    const float* yd = reinterpret_cast<const float*>(t.dense_branch.out);
    const int n = few_column<NF>(tile.nt, tid);
    if (n >= N) return;
    for (int token = tid >> 4; token < t.T; token += kTokenThreads / 16) {
        if (token >= kTokenThreads / 16) look_up(token);
        float v[NF], y[2][NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) v[f] = t.dense ? yd[(size_t)token * N + n + f] : 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                y[j][f] = src[j].slot >= 0 ? ye[((size_t)src[j].expert * t.experts.o_group_stride + src[j].slot) * N + n + f] : 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int f = 0; f < NF; ++f) v[f] = src[j].slot >= 0 ? fmaf(src[j].gate, y[j][f], v[f]) : v[f];
        typename Bf16Vec<NF>::type o;
        few_pack<NF>(v, o);
        *reinterpret_cast<typename Bf16Vec<NF>::type*>(t.out + (size_t)token * N + n) = o;
    }
}

// The second products and the combine of the fewest tokens, without a hand-over: a work-group has 8 columns of every group, its waves split K.  h's
// rows become codes in LDS once, while the weights are on their way: kGatherAhead pairs of blocks of 64 k for each wave and group.  A pair is one operand:
// columns 0 .. 7 are the first block's and 8 .. 15 the same eight of the second, rows 0 .. 7 of the other operand the codes of a group's rows in the first
// block and 8 .. 15 those in the second, and of the results the two blocks' own quarters are taken.  A group has up to kGatherRows rows.
constexpr int kGatherWaves = 8, kGatherThreads = kGatherWaves * 64, kGatherGroups = 4, kGatherRows = 4, kGatherAhead = 4, kGatherPieces = 8, kGatherBytes = kGatherThreads * kGatherPieces * 8;
// places of a group's rows
__host__ __device__ __forceinline__ int gather_places(const I8TokenArgs& t) { return t.dense && t.T > t.experts.max_rows ? t.T : t.experts.max_rows; }
__global__ __launch_bounds__(kGatherThreads) void i8_token_gather_kernel(const I8TokenArgs t) {
    __shared__ __attribute__((aligned(16))) int8_t codes[kGatherBytes];                          // [group][row's place][K]
    __shared__ int part[kGatherWaves][kGatherGroups][kGatherRows][16];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, kg = lane >> 4, half = c >> 3;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int N = t.experts.N, nkb = t.experts.K / 32, bytes = t.experts.K * 2, p_ng = (N + 127) / 128, dense = t.dense ? 1 : 0;
    const int places = gather_places(t);
    const int ng = blockIdx.x >> 4, frag = blockIdx.x >> 1 & 7, col8 = (blockIdx.x & 1) * 8;     // columns 128 ng + frag + 8 (col8 .. col8 + 7)
    const int groups = __builtin_amdgcn_readfirstlane(dense + (t.order[t.E] >> 1));
    int g[kGatherGroups];
#pragma unroll
    for (int q = 0; q < kGatherGroups; ++q) g[q] = __builtin_amdgcn_readfirstlane(q < groups && q >= dense ? t.order[q - dense] : 0);

    // h: a thread's pieces of 8 values (places behind a group's rows repeat one of them or hold anything: nobody looks at what becomes of them)
    const int row_pieces = bytes / 8, pieces = groups * places * row_pieces;
    uint4 x[kGatherPieces];
    uint32_t most[kGatherPieces];
#pragma unroll
    for (int i = 0; i < kGatherPieces; ++i) {
        const int p = tid + i * kGatherThreads;
        if (p >= pieces) break;
        const int row = p / row_pieces, q = row / places, r = row % places;
        const bool d = q < dense;
        const long long at = d ? min(r, t.T - 1) : (long long)(q == 0 ? g[0] : q == 1 ? g[1] : q == 2 ? g[2] : g[3]) * t.experts.a_group_stride +
                                         min(r, (int)t.experts.a_group_stride - 1);
        x[i] = *reinterpret_cast<const uint4*>((d ? t.dense_branch.A : t.experts.A) + at * t.experts.lda + (p % row_pieces) * 8);
        most[i] = (d ? t.dense_branch.a_max : t.experts.a_max)[at];
    }
    // weights: wave w has pairs w, w + 8, ... (behind the last block: its own again, against zeros)
    const int pairs = (nkb + 1) / 2;
    auto load_pair = [&](const uint16_t* b, int pair) {
        return __builtin_bit_cast(i32x4_t, load_stream16(b + (size_t)min(2 * pair + half, nkb - 1) * p_ng * 4096));
    };
    const uint16_t* B[kGatherGroups];
    i32x4_t bf[kGatherGroups][kGatherAhead];
#pragma unroll
    for (int q = 0; q < kGatherGroups; ++q) {
        B[q] = (q < dense ? t.dense_branch.B : t.experts.B) + (((size_t)g[q] * nkb * p_ng + ng) * 8 + frag) * 512 + (kg * 16 + col8 + (c & 7)) * 8;
        if (q >= groups) continue;
#pragma unroll
        for (int s = 0; s < kGatherAhead; ++s)
            if (s * kGatherWaves + w < pairs) bf[q][s] = load_pair(B[q], s * kGatherWaves + w);
    }
    // what thread (token, column) needs for its result
    const int token = min(tid >> 3, t.T - 1), n = ng * 128 + frag + (col8 + (tid & 7)) * 8, nc = min(n, N - 1);
    float col_scale[kGatherGroups], bias[kGatherGroups], row_scale[3], gate[2];
    int slot[2], expert[2];
    if (w == 0) {
#pragma unroll
        for (int q = 0; q < kGatherGroups; ++q) {
            const I8GemmArgs& a = q < dense ? t.dense_branch : t.experts;
            col_scale[q] = a.b_scale[(size_t)g[q] * N + nc];
            bias[q] = a.bias ? bf16_to_f32(a.bias[(size_t)g[q] * N + nc]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = token * t.top_k + min(j, t.top_k - 1);
            slot[j] = j < t.top_k ? t.slot_idx[at] : -1;
            expert[j] = t.expert_idx[at];
            gate[j] = t.gate_w[at];
            row_scale[j] = i8_scale(t.experts.a_max[(long long)expert[j] * t.experts.a_group_stride + max(slot[j], 0)]);
        }
        row_scale[2] = dense ? i8_scale(t.dense_branch.a_max[token]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kGatherPieces; ++i) {
        const int p = tid + i * kGatherThreads;
        if (p >= pieces) break;
        float f[8];
        unpack_bias8(x[i], f);
        const float inv = i8_inverse(most[i]);
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = i8_code_bits(f[e], inv);
        *reinterpret_cast<uint2*>(codes + (size_t)p * 8) = make_uint2(i8_pack4(o[0], o[1], o[2], o[3]), i8_pack4(o[4], o[5], o[6], o[7]));
    }
    lds_barrier();
    i32x4_t acc[kGatherGroups];
#pragma unroll
    for (int q = 0; q < kGatherGroups; ++q) acc[q] = i32x4_t{0, 0, 0, 0};
    const int a_row = min(c & 7, places - 1);
    for (int first = 0; first < pairs; first += kGatherAhead * kGatherWaves) {
#pragma unroll
        for (int q = 0; q < kGatherGroups; ++q) {
            if (q >= groups) continue;
#pragma unroll
            for (int s = 0; s < kGatherAhead; ++s) {
                const int pair = first + s * kGatherWaves + w, next = pair + kGatherAhead * kGatherWaves, kb = 2 * pair + half;
                if (pair >= pairs) continue;
                i32x4_t a = *reinterpret_cast<const i32x4_t*>(codes + (size_t)(q * places + a_row) * bytes + min(kb, nkb - 1) * 64 + kg * 16);
                if (kb >= nkb) a = i32x4_t{0, 0, 0, 0};
                acc[q] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, bf[q][s], acc[q], 0, 0, 0);
                if (next < pairs) bf[q][s] = load_pair(B[q], next);
            }
        }
    }
    if (kg == half * 2)                                          // D: rows 4 (lane / 16) + r, column lane % 16
#pragma unroll
        for (int q = 0; q < kGatherGroups; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[w][q][r][c] = acc[q][r];
    lds_barrier();
    if (tid >= t.T * 8 || n >= N) return;                       // (within wave 0)
    auto result = [&](int q, int r, float scale) {
        int sum = 0;
#pragma unroll
        for (int s = 0; s < kGatherWaves; ++s) sum += part[s][q][r][tid & 7] + part[s][q][r][8 + (tid & 7)];
        const float cs = q == 0 ? col_scale[0] : q == 1 ? col_scale[1] : q == 2 ? col_scale[2] : col_scale[3];
        return i8_value(sum, scale * cs, q == 0 ? bias[0] : q == 1 ? bias[1] : q == 2 ? bias[2] : bias[3]);
    };
    float v = dense ? result(0, token, row_scale[2]) : 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (slot[j] < 0) continue;
        int q = dense;
#pragma unroll
        for (int i = 0; i < kGatherGroups; ++i)
            if (i >= dense && i < groups && g[i] == expert[j]) q = i;
        v = fmaf(gate[j], result(q, slot[j], row_scale[j]), v);
    }
    t.out[(size_t)token * N + n] = f32_to_bf16(v);
}
// Where h's rows are a thread's pieces, and a work-group's weights no more than 128 KB (a compute unit takes in 33 GB/s of them).  us with / without the
// hand-over, T / groups / K / N: 1 / 1 / 4096 / 1024 10.3 / 5.5; 1 / 3 / 4096 / 1024 11.2 / 8.6; 1 / 2 / 1024 / 4096 13.2 / 6.6; 1 / 1 and 1 / 2 and
// 1 / 3 / 8192 / 2048 16.2 / 8.5, 17.2 / 12.9, 16.2 / 17.6; 2 / 3 and 2 / 4 / 4096 / 1024 11.1 / 9.6, 11.6 / 11.2; 4 / 4 / 2048 / 512 8.4 / 8.7.
bool gather_faster(const I8TokenArgs& t) {
    const long long groups = t.experts.slots + (t.dense ? 1 : 0), bytes = groups * t.experts.K * 2;
    return t.T <= 4 && gather_places(t) <= kGatherRows && groups <= kGatherGroups && bytes <= 16384 && bytes * gather_places(t) <= kGatherBytes;
}

long long token_groups(const I8TokenArgs& t) { return t.experts.slots + (t.dense ? 1 : 0); }

template <int NF> int launch_token(const I8TokenArgs& t, bool second, hipStream_t s) {
    const long long blocks = token_groups(t) * few_tiles<NF>(t.experts.N);
    if (blocks >= (1ll << 32) / kTokenThreads) return MOE_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks), threads(kTokenThreads);
    if (second) hipLaunchKernelGGL((i8_token_second_kernel<NF>), grid, threads, 0, s, t);
    else if (t.experts.a_max) hipLaunchKernelGGL((i8_token_first_kernel<NF, true>), grid, threads, 0, s, t);
    else hipLaunchKernelGGL((i8_token_first_kernel<NF, false>), grid, threads, 0, s, t);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace

// Against the products and what is between them as launches of their own.  us here / there, 1024 / 4096: 16 tokens, top-1 of 64 experts beside a dense branch
// 44 / 68 (20 tokens, whose rows in it are two sub-tiles, 75 / 70); without one 16 / 32 / 48 / 64 tokens 42 / 55, 55 / 63, 68 / 70, 81 / 79; top-1 of 32, 64 / 128 /
// 256 tokens 67 / 78, 78 / 83, 90 / 86; top-2 of 128, 16 / 32 60 / 73, 91 / 91.  512 / 2048, top-2 of 64, 64 / 128 tokens 46 / 50, 60 / 57.  2048 / 8192, top-2 of
// 16, 16 / 64 / 128 101 / 118, 116 / 126, 122 / 128 (room for 16 rows 134 / 130); room for 32 rows loses (8 experts, 64 tokens 51 / 45).
bool i8_token_faster(int T, int touched, int max_rows, int d, int f, bool dense) {
    return i8_few_faster(touched, max_rows, d, f) && (T <= kI8FewRows || (!dense && T <= (std::min(d, f) >= 1024 ? kI8TokenRows : 64)));
}

int launch_i8_token(const I8TokenArgs& t, bool second, hipStream_t s) {
    const I8GemmArgs& a = t.experts;
    if (!t.order || a.slots < 1 || a.slots > t.E || a.max_rows > kI8FewRows || (t.dense && t.T > kI8FewRows) || a.K % 32 || a.N % 8 || t.top_k > 2)
        return MOE_ERR_INVALID_ARG;
    if (second && gather_faster(t)) {
        hipLaunchKernelGGL(i8_token_gather_kernel, dim3((unsigned)(few_tiles<1>(a.N) * 2)), dim3(kGatherThreads), 0, s, t);
        return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
    }
    const int nf = std::min(few_columns(token_groups(t), kI8FewRows, a.N), 4);
    return nf == 1 ? launch_token<1>(t, second, s) : nf == 2 ? launch_token<2>(t, second, s) : launch_token<4>(t, second, s);
}

}  // namespace moe
