// Attention for drafted tokens: the choice of an instance, its workspace, and the merge of items that lie in several shares.
#include <algorithm>

#include "tree_attn.h"

namespace moe {

int launch_tree_bf16(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);
int launch_tree_fp8(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);
int launch_tree_fp4(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);

// out of the parts of every item that lies in more than one share; the share in which it begins says which.  A work-group takes
// 16 rows of one share's item; 16 threads share a row (DH / 16 elements each), SETS such groups take every so many parts and are
// added up in LDS.
template <int DH, int SETS>
__global__ __launch_bounds__(256 * SETS) void tree_merge_kernel(const TreeArgs a, const TreeParts parts, int ROWS) {
    constexpr int NF = DH / 16;
    __shared__ float ml[SETS][16][2], o[SETS][16][16][NF];
    const int R = a.R, tid = threadIdx.x;
    const float c = score_factor(DH);
    int w0 = blockIdx.x;
    if constexpr (SETS > 1) {                                 // few items: the blockIdx.x-th share that has one, not a work-group for each
        __shared__ int some[4 * SETS], found;
        const bool here = tid < parts.groups && parts.split[tid].x >= 0;
        const uint64_t m = __ballot(here);
        if (tid % kWave == 0) some[tid / kWave] = __popcll(m);
        if (tid == 0) found = -1;
        __syncthreads();
        int before = __popcll(m & ((1ull << (tid % kWave)) - 1));
        for (int i = 0; i < tid / kWave; ++i) before += some[i];
        if (here && before == (int)blockIdx.x) found = tid;
        __syncthreads();
        w0 = found;
        if (w0 < 0) return;
    }
    const int4 split = parts.split[w0];
    if (split.x < 0) return;
    const int b = split.x, w1 = split.z;
    const Sequence s = sequence<true>(a, b, ROWS);
    const int g = split.y / s.blocks, block = split.y - g * s.blocks, rows = s.count * R, row0 = block * ROWS + blockIdx.y * 16;
    if (row0 >= rows) return;
    const int piece = tid % 16, local = tid / 16 % 16, set = tid / 256;
    const int row = row0 + local, in_block = blockIdx.y * 16 + local;
    float M = kLowest, L = 0.f, v[NF] = {};
    for (int w = w0 + set; w <= w1; w += 4 * SETS) {          // four parts' loads at once; behind the last: the last, with no weight
        float2 x[4];
        float e[4][NF], m = M;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int wu = min(w + u * SETS, w1);
            const size_t at = (wu > w0 ? partial_slot(wu, true) : (size_t)split.w) * ROWS + in_block;
            x[u] = *reinterpret_cast<const float2*>(parts.ml + at * 2);
#pragma unroll
            for (int i = 0; i < NF; i += 4) *reinterpret_cast<float4*>(e[u] + i) = *reinterpret_cast<const float4*>(parts.o + at * DH + piece * NF + i);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) m = w + u * SETS <= w1 ? fmaxf(m, x[u].x) : m;
        const float f = __builtin_amdgcn_exp2f((M - m) * c);
        M = m;
        L *= f;
#pragma unroll
        for (int i = 0; i < NF; ++i) v[i] *= f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (w + u * SETS > w1) break;
            const float h = __builtin_amdgcn_exp2f((x[u].x - m) * c);
            L += x[u].y * h;
#pragma unroll
            for (int i = 0; i < NF; ++i) v[i] += e[u][i] * h;
        }
    }
    if constexpr (SETS > 1) {
        if (piece == 0) { ml[set][local][0] = M; ml[set][local][1] = L; }
#pragma unroll
        for (int i = 0; i < NF; ++i) o[set][local][piece][i] = v[i];
        __syncthreads();
        if (set) return;
        const float own = M;
        for (int i = 1; i < SETS; ++i) M = fmaxf(M, ml[i][local][0]);
        float f = __builtin_amdgcn_exp2f((own - M) * c);
        L *= f;
#pragma unroll
        for (int j = 0; j < NF; ++j) v[j] *= f;
        for (int i = 1; i < SETS; ++i) {
            f = __builtin_amdgcn_exp2f((ml[i][local][0] - M) * c);
            L += ml[i][local][1] * f;
#pragma unroll
            for (int j = 0; j < NF; ++j) v[j] += o[i][local][piece][j] * f;
        }
    }
    if (row >= rows) return;
    const int tok = row / R;
    float none = 0.f;                                         // a row of sum 0: 0 if it sees nothing, NaN if all its scores are -inf
    if (L == 0.f && sees_anything(a, s, b, tok)) none = __uint_as_float(0x7fc00000u);
    const float f = 1.f / L;
    uint32_t w[NF / 2];
#pragma unroll
    for (int i = 0; i < NF / 2; ++i) w[i] = L == 0.f ? pack_bf16x2(none, none) : pack_bf16x2(v[2 * i] * f, v[2 * i + 1] * f);
    uint16_t* dst = a.out + ((long long)b * a.N + tok) * a.out_stride + (g * R + row - tok * R) * DH + piece * NF;
    if constexpr (DH == 128) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
}

static TreePlan tree_plan(int R, int N, int head_dim, int kind) {
    const int rows = N * R;                                   // at most, per key/value head
    TreePlan p;
    // Up to 16 rows the four waves split the positions, each with the tiles in its own registers; beyond, waves that take rows of
    // their own share the tiles in LDS, 16 rows each while the cache's reading takes the time, else 32.  us for 16 sequences of
    // 4096 positions, 8 key/value heads of 128, in 8 bits and in bf16, with rows x the waves that have their own:
    //                  16 x 1      16 x 2      32 x 2      32 x 4
    //      16 rows    31 / 48     37 / 49     40 / 50     50 / 50
    //      32 rows    50 / 88     38 / 50     41 / 52     49 / 51
    //      64 rows    82 / 145    61 / 87     43 / 55     50 / 54
    //     128 rows   153 / 268   102 / 157    69 / 93     55 / 68
    p.mt = rows <= 32 ? 1 : 2;
    p.wr = rows <= 16 ? 1 : rows <= 64 ? 2 : 4;
    p.groups = groups_per_unit(kind, head_dim, p.wr) * kComputeUnits;
    const int block = 16 * p.mt * p.wr;
    p.row_blocks = (rows + block - 1) / block;
    p.partial_bytes = (size_t)2 * p.groups * block * head_dim * sizeof(float);
    p.ml_bytes = (size_t)2 * p.groups * block * 2 * sizeof(float);
    return p;
}
size_t tree_attn_ws_bytes(const moe_cache_shape_t* c, int n_draft) {
    const TreePlan p = tree_plan(c->n_heads / c->n_kv_heads, n_draft, c->head_dim, c->kind);
    return p.partial_bytes + p.ml_bytes + (size_t)p.groups * sizeof(int4);
}
// steps of all items together, at most
long long tree_attn_steps(const moe_cache_shape_t* c, int n_draft) {
    const TreePlan p = tree_plan(c->n_heads / c->n_kv_heads, n_draft, c->head_dim, c->kind);
    return (long long)c->n_seq * c->n_kv_heads * p.row_blocks * ((c->max_len + kTile - 1) / kTile + (n_draft + kTile - 1) / kTile + kItemSteps);
}

int launch_tree_attn(const TreeArgs& a, int kind, int head_dim, void* ws, hipStream_t s) {
    const TreePlan p = tree_plan(a.R, a.N, head_dim, kind);
    char* at = static_cast<char*>(ws);
    const TreeParts parts{reinterpret_cast<float*>(at), reinterpret_cast<float*>(at + p.partial_bytes),
                          reinterpret_cast<int4*>(at + p.partial_bytes + p.ml_bytes), p.groups};
    const int rc = kind == MOE_CACHE_BF16 ? launch_tree_bf16(a, parts, head_dim, p.mt, p.wr, s)
                   : kind == MOE_CACHE_FP8 ? launch_tree_fp8(a, parts, head_dim, p.mt, p.wr, s) : launch_tree_fp4(a, parts, head_dim, p.mt, p.wr, s);
    if (rc != MOE_OK) return rc;
    const int block = 16 * p.mt * p.wr;
    const long long items = (long long)a.n_seq * a.G * p.row_blocks;
    const bool few = items * 8 <= p.groups;                   // items, which then have many parts each
    const dim3 grid((unsigned)(few ? items : p.groups), (unsigned)(std::min(block, a.N * a.R + 15) / 16));
    static_assert(kMaxGroups <= 1024, "a thread per share");
#define MOE_MERGE(DH) \
    do { \
        if (few) hipLaunchKernelGGL((tree_merge_kernel<DH, 4>), grid, dim3(1024), 0, s, a, parts, block); \
        else hipLaunchKernelGGL((tree_merge_kernel<DH, 1>), grid, dim3(256), 0, s, a, parts, block); \
    } while (0)
    if (head_dim == 128) MOE_MERGE(128);
    else MOE_MERGE(64);
#undef MOE_MERGE
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
