// Rows of keys and values into the caches, quantised as they are written, and back.
// Bound by traffic.  A unit of work is 8 elements: 16 bytes of a row, and 16, 8 or 4 bytes of the cache.  A work-group takes
// some rows of one head's keys or values: rows that follow each other in a sequence (a prefill, a prefix) are consecutive in
// the cache, and so are their scales.
#include "cache_kind.h"

namespace moe {

struct CacheRows {
    const void* rows[2];       // keys, values: [n_rows, G * DH] bf16
    long long stride[2];
    void* cache[2];            // [n_seq, G, max_len, DH] elements
    uint8_t* scale[2];         // [n_seq, G, max_len, DH / 32]
    const int32_t* seq;
    const int32_t* pos;
    int n_rows, n_seq, G, max_len;
};

// place of a row's position in the caches, in rows of DH elements; -1: outside
__device__ __forceinline__ long long cache_row(const CacheRows& a, int r, int g) {
    if (r >= a.n_rows) return -1;
    const int b = a.seq[r], p = a.pos[r];
    if ((unsigned)b >= (unsigned)a.n_seq || (unsigned)p >= (unsigned)a.max_len) return -1;
    return ((long long)b * a.G + g) * a.max_len + p;
}

constexpr int kCacheRows = 32;                               // rows per work-group

template <int KIND, int DH>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8;                               // pieces per row
    const int tid = threadIdx.x, g = blockIdx.y >> 1, which = blockIdx.y & 1, piece = tid % PPR;
    const uint16_t* rows = static_cast<const uint16_t*>(a.rows[which]);
    uint8_t* cache = static_cast<uint8_t*>(a.cache[which]);
    for (int r = blockIdx.x * kCacheRows + tid / PPR; r < (int)(blockIdx.x + 1) * kCacheRows; r += 256 / PPR) {
        const long long at = cache_row(a, r, g);
        uint4 w = make_uint4(0, 0, 0, 0);
        if (at >= 0) w = *reinterpret_cast<const uint4*>(rows + r * a.stride[which] + g * DH + piece * 8);
        if constexpr (KIND == MOE_CACHE_BF16) {
            if (at >= 0) *reinterpret_cast<uint4*>(cache + (at * DH + piece * 8) * 2) = w;
        } else {
            uint32_t v[4] = {w.x, w.y, w.z, w.w};
            uint32_t top = 0;                                 // magnitudes of bf16 numbers are ordered as their bits are
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, max(v[i] & 0x7fffu, (v[i] >> 16) & 0x7fffu));
            top = max(top, (uint32_t)__shfl_xor((int)top, 1));
            top = max(top, (uint32_t)__shfl_xor((int)top, 2));         // the four lanes of a block
            if (top > kLargest<KIND> && top < 0x7f80u) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = (v[i] & 0x80008000u) | min(v[i] & 0x7fffu, kLargest<KIND>) | min((v[i] >> 16) & 0x7fffu, kLargest<KIND>) << 16;
                top = kLargest<KIND>;
            }
            const uint32_t byte = scale_byte<KIND>(top);
            const float scale = scale_value(byte);
            uint32_t code[2] = {0, 0};
            if (byte != 255) {
                typedef short s16x2 __attribute__((ext_vector_type(2)));
                bf16x2_vec x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(bf16x2_vec, v[i]);
                if constexpr (KIND == MOE_CACHE_FP8) {
                    s16x2 c = {0, 0};
                    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, x[0], scale, false);
                    code[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, x[1], scale, true));
                    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, x[2], scale, false);
                    code[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, x[3], scale, true));
                } else {
                    uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, x[0], scale, 0);
                    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, x[1], scale, 1);
                    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, x[2], scale, 2);
                    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, x[3], scale, 3);
                }
            }
            if (at >= 0) {
                if constexpr (KIND == MOE_CACHE_FP8) *reinterpret_cast<uint2*>(cache + at * DH + piece * 8) = make_uint2(code[0], code[1]);
                else *reinterpret_cast<uint32_t*>(cache + at * (DH / 2) + piece * 4) = code[0];
            }
            // the row's scale bytes by one lane
            constexpr int blocks = DH / kScaleBlock;
            uint32_t bytes = 0;
            const int first = (threadIdx.x & 63) - piece;
#pragma unroll
            for (int j = 0; j < blocks; ++j) bytes |= (uint32_t)__shfl((int)byte, first + 4 * j) << (8 * j);
            if (at >= 0 && piece == 0) {
                if constexpr (blocks == 4) *reinterpret_cast<uint32_t*>(a.scale[which] + at * 4) = bytes;
                else *reinterpret_cast<uint16_t*>(a.scale[which] + at * 2) = (uint16_t)bytes;
            }
        }
    }
}

template <int KIND, int DH>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8;
    const int tid = threadIdx.x, g = blockIdx.y >> 1, which = blockIdx.y & 1, piece = tid % PPR;
    uint16_t* rows = static_cast<uint16_t*>(const_cast<void*>(a.rows[which]));
    const uint8_t* cache = static_cast<const uint8_t*>(a.cache[which]);
    for (int r = blockIdx.x * kCacheRows + tid / PPR; r < (int)(blockIdx.x + 1) * kCacheRows; r += 256 / PPR) {
        const long long at = cache_row(a, r, g);
        if (at < 0) continue;
        uint4 w;
        if constexpr (KIND == MOE_CACHE_BF16) {
            w = *reinterpret_cast<const uint4*>(cache + (at * DH + piece * 8) * 2);
        } else {
            const float scale = scale_value(a.scale[which][at * (DH / kScaleBlock) + piece / 4]);
            if constexpr (KIND == MOE_CACHE_FP8) {
                const uint2 c = *reinterpret_cast<const uint2*>(cache + at * DH + piece * 8);
                w = make_uint4(fp8_pair<false>(c.x, scale), fp8_pair<true>(c.x, scale), fp8_pair<false>(c.y, scale), fp8_pair<true>(c.y, scale));
            } else {
                const uint32_t c = *reinterpret_cast<const uint32_t*>(cache + at * (DH / 2) + piece * 4);
                w = make_uint4(fp4_pair<0>(c, scale), fp4_pair<1>(c, scale), fp4_pair<2>(c, scale), fp4_pair<3>(c, scale));
            }
        }
        *reinterpret_cast<uint4*>(rows + r * a.stride[which] + g * DH + piece * 8) = w;
    }
}

static CacheRows cache_rows(const moe_cache_shape_t* c, int n_rows, const void* k, long long ks, const void* v, long long vs, const int32_t* seq,
                     const int32_t* pos, const void* kc, const void* vc, const uint8_t* kx, const uint8_t* vx) {
    return CacheRows{{k, v}, {ks, vs}, {const_cast<void*>(kc), const_cast<void*>(vc)}, {const_cast<uint8_t*>(kx), const_cast<uint8_t*>(vx)},
                     seq, pos, n_rows, c->n_seq, c->n_kv_heads, c->max_len};
}

#define MOE_CACHE_LAUNCH(KERNEL) \
    do { \
        const dim3 grid((unsigned)((n_rows + kCacheRows - 1) / kCacheRows), (unsigned)(2 * c->n_kv_heads)); \
        if (c->kind == MOE_CACHE_BF16) { \
            if (c->head_dim == 128) hipLaunchKernelGGL((KERNEL<MOE_CACHE_BF16, 128>), grid, dim3(256), 0, s, a); \
            else hipLaunchKernelGGL((KERNEL<MOE_CACHE_BF16, 64>), grid, dim3(256), 0, s, a); \
        } else if (c->kind == MOE_CACHE_FP8) { \
            if (c->head_dim == 128) hipLaunchKernelGGL((KERNEL<MOE_CACHE_FP8, 128>), grid, dim3(256), 0, s, a); \
            else hipLaunchKernelGGL((KERNEL<MOE_CACHE_FP8, 64>), grid, dim3(256), 0, s, a); \
        } else { \
            if (c->head_dim == 128) hipLaunchKernelGGL((KERNEL<MOE_CACHE_FP4, 128>), grid, dim3(256), 0, s, a); \
            else hipLaunchKernelGGL((KERNEL<MOE_CACHE_FP4, 64>), grid, dim3(256), 0, s, a); \
        } \
    } while (0)

int launch_cache_write(const moe_cache_shape_t* c, int n_rows, const void* k, long long k_stride, const void* v, long long v_stride,
                       const int32_t* seq, const int32_t* pos, void* kc, void* vc, uint8_t* kx, uint8_t* vx, hipStream_t s) {
    const CacheRows a = cache_rows(c, n_rows, k, k_stride, v, v_stride, seq, pos, kc, vc, kx, vx);
    MOE_CACHE_LAUNCH(cache_write_kernel);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
int launch_cache_read(const moe_cache_shape_t* c, int n_rows, const void* kc, const void* vc, const uint8_t* kx, const uint8_t* vx,
                      const int32_t* seq, const int32_t* pos, void* k, long long k_stride, void* v, long long v_stride, hipStream_t s) {
    const CacheRows a = cache_rows(c, n_rows, k, k_stride, v, v_stride, seq, pos, kc, vc, kx, vx);
    MOE_CACHE_LAUNCH(cache_read_kernel);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
#undef MOE_CACHE_LAUNCH

}  // namespace moe
