// The products of a whole MoE layer for few tokens in two launches (the gate is the third): the first products of all experts that have rows and
// of the dense branch, then their second products with the combine.  Bound by latency with a token or two, by the read of the weights
// with more (i8_few.h).
// The first launch takes the tokens in bf16 with their largest magnitudes, which the gate's launch finds on its way, and the second one h with those
// that the first one raises: no launch makes codes.  The work-group that finishes a column tile's last group adds the groups' results up for every
// token, in 32 bits, and rounds once: nobody waits for anybody.
// Hand-over across the XCDs' separate L2s: results are written with device-scope stores (through the L2), a work-group waits for its stores before
// it counts itself, and the last one acquires at device scope before its loads.  The counters are cleared by the gate's launch.
// One token, top-2 of 128 experts beside a dense branch, 1024 / 4096: 6.7 + 11.2 us behind a gate of 9.2, 26.4 for the call; as launches that bring x
// into codes, multiply, multiply and combine 4.2 + 6.3 + 6.0 + 4.1, 27.6 for the call.  16 tokens, top-2 of 64 experts beside one: 33 + 32 us
// (212 MB of codes: 3.2 TB/s).  Tried: both products in one launch, work-groups taking tiles by ticket and those of the second product waiting for
// a flag of their group: 27.6 us (11 ns for each ticket, and every hand-over is a chain of stores, count, flag and loads across
// the L2s of about 4 us, as long as a launch).
#include "i8_few.h"

namespace moe {

namespace {

constexpr int kTokenWaves = 8, kTokenThreads = kTokenWaves * 64;

// a work-group's tile: columns fastest; the dense branch's row tiles come first, then the experts with rows in the gate's order
struct TokenTile {
    int g, nt, m0, groups;
    bool dense, live;
};
template <int MSMAX> __device__ __forceinline__ TokenTile token_tile(const I8TokenArgs& t, int n_tiles) {
    const int group = blockIdx.x / n_tiles, dense = t.dense ? (t.T + 16 * MSMAX - 1) / (16 * MSMAX) : 0;
    TokenTile r;
    r.nt = blockIdx.x % n_tiles;
    r.dense = group < dense;
    const int expert = r.dense ? 0 : t.order[group - dense];
    const int live = t.order[t.E] >> 1;
    r.groups = __builtin_amdgcn_readfirstlane(dense + live);
    r.live = group < r.groups;
    r.g = __builtin_amdgcn_readfirstlane(expert);
    r.m0 = r.dense ? group * 16 * MSMAX : 0;
    return r;
}

// XBF16: x in bf16 with the tokens' largest magnitudes, else codes with scales
template <int MSMAX, int NF, bool XBF16>
__global__ __launch_bounds__(kTokenThreads) void i8_token_first_kernel(const I8TokenArgs t) {
    __shared__ __attribute__((aligned(16))) int part[few_lds_ints<kTokenWaves, MSMAX, NF>()];
    const TokenTile tile = token_tile<MSMAX>(t, few_tiles<NF>(t.experts.N));
    if (!tile.live) return;
    const I8GemmArgs& a = tile.dense ? t.dense_branch : t.experts;
    few_tile<kTokenWaves, MSMAX, NF, XBF16>(a, tile.g, tile.nt, tile.m0, part, [&](int row, int n, bool here, float (&v)[NF]) {
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

template <int MSMAX, int NF>
__global__ __launch_bounds__(kTokenThreads) void i8_token_second_kernel(const I8TokenArgs t) {
    __shared__ __attribute__((aligned(16))) int part[few_lds_ints<kTokenWaves, MSMAX, NF>()];
    __shared__ int shared_last;
    const int tid = threadIdx.x, N = t.experts.N;
    const TokenTile tile = token_tile<MSMAX>(t, few_tiles<NF>(N));
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
    few_tile<kTokenWaves, MSMAX, NF, true>(a, tile.g, tile.nt, tile.m0, part, [&](int row, int n, bool here, float (&v)[NF]) {
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

template <int MSMAX> long long token_groups(const I8TokenArgs& t) { return t.experts.slots + (t.dense ? (t.T + 16 * MSMAX - 1) / (16 * MSMAX) : 0); }

template <int MSMAX, int NF> int launch_token(const I8TokenArgs& t, bool second, hipStream_t s) {
    const long long blocks = token_groups<MSMAX>(t) * few_tiles<NF>(t.experts.N);
    if (blocks >= (1ll << 32) / kTokenThreads) return MOE_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks), threads(kTokenThreads);
    if (second) hipLaunchKernelGGL((i8_token_second_kernel<MSMAX, NF>), grid, threads, 0, s, t);
    else if (t.experts.a_max) hipLaunchKernelGGL((i8_token_first_kernel<MSMAX, NF, true>), grid, threads, 0, s, t);
    else hipLaunchKernelGGL((i8_token_first_kernel<MSMAX, NF, false>), grid, threads, 0, s, t);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace

int launch_i8_token(const I8TokenArgs& t, bool second, hipStream_t s) {
    const I8GemmArgs& a = t.experts;
    if (!t.order || a.slots < 1 || a.slots > t.E || a.max_rows > kI8FewRows || a.K % 32 || a.N % 8 || t.top_k > 2) return MOE_ERR_INVALID_ARG;
    const int most = t.dense && t.T > a.max_rows ? std::min(t.T, kI8FewRows) : a.max_rows;
    const int nf = few_columns(most <= 16 ? token_groups<1>(t) : token_groups<2>(t), most, a.N);
    if (most > 16) return nf == 1 ? launch_token<2, 1>(t, second, s) : launch_token<2, 2>(t, second, s);
    return nf == 1 ? launch_token<1, 1>(t, second, s) : nf == 2 ? launch_token<1, 2>(t, second, s) : launch_token<1, 4>(t, second, s);
}

}  // namespace moe
