// Rows of keys and values into the caches, quantised as they are written, and back.
// Bound by traffic.  A unit of work is 8 elements: 16 bytes of a row, and 16, 8 or 4 bytes of the cache.  A work-group takes
// some rows of one head's keys or values: rows that follow each other in a sequence (a prefill, a prefix) are consecutive in
// the cache, and so are their scales.  Reading 65536 positions of 8 heads of 128 from 8 bits takes 80 us, 5.1 TB/s, where a large
// copy reaches 5.2; writing 64000 such rows 94 us, 3.9 TB/s (rows of other heads lie between a head's, 256 bytes each).
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

// A thread has IT units of rows STEP apart, all their loads on the way before the first is used.
template <int KIND, int DH, int IT>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8, STEP = 256 / PPR;             // pieces per row, rows per round of the work-group
    const int tid = threadIdx.x, g = blockIdx.y >> 1, which = blockIdx.y & 1, piece = tid % PPR;
    const uint16_t* rows = static_cast<const uint16_t*>(a.rows[which]);
    uint8_t* cache = static_cast<uint8_t*>(a.cache[which]);
    long long at[IT];
    uint4 w[IT];
#pragma unroll
    for (int n = 0; n < IT; ++n) at[n] = cache_row(a, (blockIdx.x * IT + n) * STEP + tid / PPR, g);
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        const int r = (blockIdx.x * IT + n) * STEP + tid / PPR;
        w[n] = at[n] >= 0 ? *reinterpret_cast<const uint4*>(rows + r * a.stride[which] + g * DH + piece * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        if constexpr (KIND == MOE_CACHE_BF16) {
            if (at[n] >= 0) *reinterpret_cast<uint4*>(cache + (at[n] * DH + piece * 8) * 2) = w[n];
        } else {
            uint32_t v[4] = {w[n].x, w[n].y, w[n].z, w[n].w};
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
            if (at[n] >= 0) {
                if constexpr (KIND == MOE_CACHE_FP8) *reinterpret_cast<uint2*>(cache + at[n] * DH + piece * 8) = make_uint2(code[0], code[1]);
                else *reinterpret_cast<uint32_t*>(cache + at[n] * (DH / 2) + piece * 4) = code[0];
            }
            // the row's scale bytes by one lane
            constexpr int blocks = DH / kScaleBlock;
            uint32_t bytes = 0;
            const int first = (threadIdx.x & 63) - piece;
#pragma unroll
            for (int j = 0; j < blocks; ++j) bytes |= (uint32_t)__shfl((int)byte, first + 4 * j) << (8 * j);
            if (at[n] >= 0 && piece == 0) {
                if constexpr (blocks == 4) *reinterpret_cast<uint32_t*>(a.scale[which] + at[n] * 4) = bytes;
                else *reinterpret_cast<uint16_t*>(a.scale[which] + at[n] * 2) = (uint16_t)bytes;
            }
        }
    }
}

template <int KIND, int DH>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8;
    const int tid = threadIdx.x, g = blockIdx.y >> 1, which = blockIdx.y & 1, piece = tid % PPR, r = blockIdx.x * (256 / PPR) + tid / PPR;
    const uint8_t* cache = static_cast<const uint8_t*>(a.cache[which]);
    const long long at = cache_row(a, r, g);
    if (at < 0) return;
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
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(const_cast<void*>(a.rows[which])) + r * a.stride[which] + g * DH + piece * 8) = w;
}

static CacheRows cache_rows(const moe_cache_shape_t* c, int n_rows, const void* k, long long ks, const void* v, long long vs, const int32_t* seq,
                     const int32_t* pos, const void* kc, const void* vc, const uint8_t* kx, const uint8_t* vx) {
    return CacheRows{{k, v}, {ks, vs}, {const_cast<void*>(kc), const_cast<void*>(vc)}, {const_cast<uint8_t*>(kx), const_cast<uint8_t*>(vx)},
                     seq, pos, n_rows, c->n_seq, c->n_kv_heads, c->max_len};
}

static dim3 cache_grid(const CacheRows& a, int rows_per_block) {
    return dim3((unsigned)((a.n_rows + rows_per_block - 1) / rows_per_block), (unsigned)(2 * a.G));
}
template <int KIND, int DH> void write_rows(const CacheRows& a, hipStream_t s) {
    constexpr int step = 256 / (DH / 8);
    // Two units per thread hide more of the memory's latency where there are work-groups enough: 64000 rows of 8 heads of 128 to
    // 8 bits 105 / 94 us, of 64 to 4 bits 43 / 36, 8192 rows of 8 heads 11.1 / 10.4, but 64 rows 2.6 / 3.1; bf16 rows, which are only
    // moved, 103 / 103.
    if constexpr (KIND != MOE_CACHE_BF16) {
        if ((long long)a.n_rows * a.G * DH >= 1 << 23) {
            hipLaunchKernelGGL((cache_write_kernel<KIND, DH, 2>), cache_grid(a, 2 * step), dim3(256), 0, s, a);
            return;
        }
    }
    hipLaunchKernelGGL((cache_write_kernel<KIND, DH, 1>), cache_grid(a, step), dim3(256), 0, s, a);
}
template <int KIND, int DH> void read_rows(const CacheRows& a, hipStream_t s) {
    hipLaunchKernelGGL((cache_read_kernel<KIND, DH>), cache_grid(a, 256 / (DH / 8)), dim3(256), 0, s, a);
}

#define MOE_CACHE_ROWS(CALL) \
    do { \
        const bool wide = c->head_dim == 128; \
        if (c->kind == MOE_CACHE_BF16) wide ? CALL<MOE_CACHE_BF16, 128>(a, s) : CALL<MOE_CACHE_BF16, 64>(a, s); \
        else if (c->kind == MOE_CACHE_FP8) wide ? CALL<MOE_CACHE_FP8, 128>(a, s) : CALL<MOE_CACHE_FP8, 64>(a, s); \
        else wide ? CALL<MOE_CACHE_FP4, 128>(a, s) : CALL<MOE_CACHE_FP4, 64>(a, s); \
    } while (0)

int launch_cache_write(const moe_cache_shape_t* c, int n_rows, const void* k, long long k_stride, const void* v, long long v_stride,
                       const int32_t* seq, const int32_t* pos, void* kc, void* vc, uint8_t* kx, uint8_t* vx, hipStream_t s) {
    const CacheRows a = cache_rows(c, n_rows, k, k_stride, v, v_stride, seq, pos, kc, vc, kx, vx);
    MOE_CACHE_ROWS(write_rows);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
int launch_cache_read(const moe_cache_shape_t* c, int n_rows, const void* kc, const void* vc, const uint8_t* kx, const uint8_t* vx,
                      const int32_t* seq, const int32_t* pos, void* k, long long k_stride, void* v, long long v_stride, hipStream_t s) {
    const CacheRows a = cache_rows(c, n_rows, k, k_stride, v, v_stride, seq, pos, kc, vc, kx, vx);
    MOE_CACHE_ROWS(read_rows);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
#undef MOE_CACHE_ROWS

}  // namespace moe
