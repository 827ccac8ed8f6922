// Attention of several new tokens per sequence over its cached positions and, through a bit mask, over each other.
//   out[b, i, h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(q . k_j / sqrt(DH) - max)     over what token i sees
// One wave per row and head: 64 positions at a time, a score per lane, then DH / 64 dimensions of the values per lane.
#include "cache_kind.h"

namespace moe {

template <int KIND, int DH>
__device__ __forceinline__ float cached_element(const void* cache, const uint8_t* scale, long long row, int i) {
    if constexpr (KIND == MOE_CACHE_BF16) {
        return bf16_to_f32(static_cast<const uint16_t*>(cache)[row * DH + i]);
    } else {
        const float s = scale_value(scale[row * (DH / kScaleBlock) + i / kScaleBlock]);
        uint32_t pair;
        if constexpr (KIND == MOE_CACHE_FP8) pair = fp8_pair<false>(static_cast<const uint8_t*>(cache)[row * DH + i], s);
        else pair = fp4_pair<0>((uint32_t)static_cast<const uint8_t*>(cache)[row * (DH / 2) + i / 2] >> (4 * (i & 1)), s);
        return __uint_as_float(pair << 16);
    }
}

template <int KIND, int DH>
__global__ __launch_bounds__(64) void tree_attn_kernel(const TreeArgs a) {
    __shared__ float q[DH], p_sh[64];
    const int lane = threadIdx.x, h = blockIdx.x % a.H, row = blockIdx.x / a.H, b = row / a.N, i = row % a.N, g = h / (a.H / a.G);
    const int len = min(max(a.lens[b], 0), a.max_len), count = a.counts ? min(max(a.counts[b], 0), a.N) : a.N;
    if (i >= count) return;
    for (int d = lane; d < DH; d += 64) q[d] = bf16_to_f32(a.q[row * a.q_stride + h * DH + d]) * rsqrtf((float)DH);
    __syncthreads();
    const long long base = ((long long)b * a.G + g) * a.max_len;
    float m = -INFINITY, l = 0.f, o[DH / 64] = {};
    for (int j0 = 0; j0 < len + count; j0 += 64) {
        const int j = j0 + lane, t = j - len;                  // cached position j, or drafted token t
        bool sees = j < len + count;
        if (sees && t >= 0) sees = a.tree ? a.tree[(size_t)row * ((a.N + 31) / 32) + t / 32] >> (t % 32) & 1 : t <= i;
        float s = -INFINITY;
        if (sees) {
            s = 0.f;
            for (int d = 0; d < DH; ++d)
                s = fmaf(q[d], t >= 0 ? bf16_to_f32(a.k[(b * (long long)a.N + t) * a.k_stride + g * DH + d])
                                      : cached_element<KIND, DH>(a.k_cache, a.k_scale, base + j, d), s);
        }
        float mn = s;
        for (int x = 32; x >= 1; x >>= 1) mn = fmaxf(mn, __shfl_xor(mn, x));
        mn = fmaxf(m, mn);
        const float zero = mn == -INFINITY ? 0.f : mn, c = expf(m - zero), p = sees ? expf(s - zero) : 0.f;
        __syncthreads();
        p_sh[lane] = p;
        __syncthreads();
        const uint64_t seen = __ballot(sees);
        l *= c;
        for (int e = 0; e < DH / 64; ++e) o[e] *= c;
        for (int n = 0; n < 64; ++n) {
            if (!(seen >> n & 1)) continue;
            l += p_sh[n];
            const int tn = j0 + n - len;
            for (int e = 0; e < DH / 64; ++e)
                o[e] = fmaf(p_sh[n], tn >= 0 ? bf16_to_f32(a.v[(b * (long long)a.N + tn) * a.v_stride + g * DH + e * 64 + lane])
                                             : cached_element<KIND, DH>(a.v_cache, a.v_scale, base + j0 + n, e * 64 + lane), o[e]);
        }
        m = mn;
    }
    bool any = len > 0;
    for (int t = 0; !any && t < count; ++t) any = a.tree ? a.tree[(size_t)row * ((a.N + 31) / 32) + t / 32] >> (t % 32) & 1 : t <= i;
    for (int e = 0; e < DH / 64; ++e) a.out[row * a.out_stride + h * DH + e * 64 + lane] = any ? f32_to_bf16(o[e] / l) : 0;
}

size_t tree_attn_ws_bytes(const moe_cache_shape_t*, int) { return 256; }

int launch_tree_attn(const TreeArgs& a, int kind, int head_dim, void*, hipStream_t s) {
    const dim3 grid((unsigned)(a.n_seq * a.N * a.H));
#define MOE_TREE(KIND) \
    do { \
        if (head_dim == 128) hipLaunchKernelGGL((tree_attn_kernel<KIND, 128>), grid, dim3(64), 0, s, a); \
        else hipLaunchKernelGGL((tree_attn_kernel<KIND, 64>), grid, dim3(64), 0, s, a); \
    } while (0)
    if (kind == MOE_CACHE_BF16) MOE_TREE(MOE_CACHE_BF16);
    else if (kind == MOE_CACHE_FP8) MOE_TREE(MOE_CACHE_FP8);
    else MOE_TREE(MOE_CACHE_FP4);
#undef MOE_TREE
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
