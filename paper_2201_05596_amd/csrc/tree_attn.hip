// Attention for drafted tokens: the choice of an instance, its workspace, and the merge of items that lie in several shares.
#include <algorithm>

#include "tree_attn.h"

namespace moe {

int launch_tree_bf16(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);
int launch_tree_fp8(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);
int launch_tree_fp4(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s);

// out of the parts of every item that lies in more than one share.  A work-group takes `per` rows of an item; 16 threads share
// a row (DH / 16 elements each), the other factor of 256 takes every so many parts and is added up in LDS.
template <int DH>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a, const TreeParts parts, int ROWS, int wp, int per, int blocks_per_head) {
    constexpr int NF = DH / 16;
    __shared__ long long sh[8];
    __shared__ float ml[16][16][2], o[16][16][NF];            // [part set][row] and, per thread, its sums
    const int tid = threadIdx.x, R = a.H / a.G;
    const int chunks = ROWS / per;
    const Shares share = shares(a, ROWS, parts.groups, wp, sh, tid);
    for (long long bx = blockIdx.x; bx < (long long)a.n_seq * a.G * blocks_per_head * chunks; bx += gridDim.x) {
    const int chunk = (int)(bx % chunks), block = (int)(bx / chunks % blocks_per_head), g = (int)(bx / chunks / blocks_per_head % a.G);
    const int b = (int)(bx / chunks / blocks_per_head / a.G);
    const Sequence s = sequence(a, b, ROWS);
    const int rows = s.count * R, row0 = block * ROWS + chunk * per;
    if (row0 >= rows) continue;
    long long before = 0;                                     // steps of the sequences before b
    int unused = 0;
    for (int i = tid; i < b; i += 256) { const Sequence t = sequence(a, i, ROWS); before += t.items * t.tiles; }
    block_sum_max(before, unused, sh, tid);
    const long long first = before + ((long long)g * (s.items / a.G) + block) * s.tiles, last = first + s.tiles - 1;
    const long long w0 = first / share.size, w1 = last / share.size;
    if (w0 == w1) continue;
    const int piece = tid % 16, local = tid / 16 % per, set = tid / 16 / per, sets = 16 / per;
    const int row = row0 + local, in_block = chunk * per + local;
    float M = kLowest, L = 0.f, v[NF] = {};
    for (long long w = w0 + set; w <= w1; w += sets) {
        const size_t at = partial_slot(w, w > w0 || first == w0 * share.size) * ROWS + in_block;
        const float2 x = *reinterpret_cast<const float2*>(parts.ml + at * 2);
        float e[NF];
#pragma unroll
        for (int i = 0; i < NF; i += 4) *reinterpret_cast<float4*>(e + i) = *reinterpret_cast<const float4*>(parts.o + at * DH + piece * NF + i);
        const float m = fmaxf(M, x.x), f = __builtin_amdgcn_exp2f(M - m), h = __builtin_amdgcn_exp2f(x.x - m);
        M = m;
        L = L * f + x.y * h;
#pragma unroll
        for (int i = 0; i < NF; ++i) v[i] = v[i] * f + e[i] * h;
    }
    if (sets > 1) {
        if (piece == 0) { ml[set][local][0] = M; ml[set][local][1] = L; }
#pragma unroll
        for (int i = 0; i < NF; ++i) o[tid / 16][piece][i] = v[i];
        __syncthreads();
        const float own = M;
        for (int i = 1; i < sets; ++i) M = fmaxf(M, ml[i][local][0]);
        float f = __builtin_amdgcn_exp2f(own - M);
        L *= f;
#pragma unroll
        for (int j = 0; j < NF; ++j) v[j] *= f;
        for (int i = 1; i < sets; ++i) {
            f = __builtin_amdgcn_exp2f(ml[i][local][0] - M);
            L += ml[i][local][1] * f;
#pragma unroll
            for (int j = 0; j < NF; ++j) v[j] += o[i * per + local][piece][j] * f;
        }
    }
    if (set || row >= rows) continue;
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
}

static TreePlan tree_plan(int n_seq, int G, int R, int N, int head_dim) {
    const int rows = N * R;                                   // at most, per key/value head
    TreePlan p;
    p.mt = rows <= 16 ? 1 : rows <= 64 ? 2 : 4;
    p.wr = rows <= 32 ? 1 : rows <= 128 ? 2 : 4;
    p.groups = p.mt == 1 ? 768 : p.mt == 2 ? 512 : 256;
    const int block = 16 * p.mt * p.wr;
    p.row_blocks = (rows + block - 1) / block;
    p.partial_bytes = (size_t)2 * p.groups * block * head_dim * sizeof(float);
    return p;
}
size_t tree_attn_ws_bytes(const moe_cache_shape_t* c, int n_draft) {
    const TreePlan p = tree_plan(c->n_seq, c->n_kv_heads, c->n_heads / c->n_kv_heads, n_draft, c->head_dim);
    return p.partial_bytes + (size_t)2 * p.groups * 16 * p.mt * p.wr * 2 * sizeof(float);
}

int launch_tree_attn(const TreeArgs& a, int kind, int head_dim, void* ws, hipStream_t s) {
    const TreePlan p = tree_plan(a.n_seq, a.G, a.H / a.G, a.N, head_dim);
    const TreeParts parts{static_cast<float*>(ws), reinterpret_cast<float*>(static_cast<char*>(ws) + p.partial_bytes), p.groups};
    const int rc = kind == MOE_CACHE_BF16 ? launch_tree_bf16(a, parts, head_dim, p.mt, p.wr, s)
                   : kind == MOE_CACHE_FP8 ? launch_tree_fp8(a, parts, head_dim, p.mt, p.wr, s) : launch_tree_fp4(a, parts, head_dim, p.mt, p.wr, s);
    if (rc != MOE_OK) return rc;
    const int block = 16 * p.mt * p.wr;
    const long long items = (long long)a.n_seq * a.G * p.row_blocks;
    const int per = items <= 32 ? 1 : items <= 128 ? 4 : 16;  // few items: many parts each
    const unsigned grid = (unsigned)std::min(items * (block / per), 8192ll);
    if (head_dim == 128) hipLaunchKernelGGL((tree_merge_kernel<128>), dim3(grid), dim3(256), 0, s, a, parts, block, 4 / p.wr, per, p.row_blocks);
    else hipLaunchKernelGGL((tree_merge_kernel<64>), dim3(grid), dim3(256), 0, s, a, parts, block, 4 / p.wr, per, p.row_blocks);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
