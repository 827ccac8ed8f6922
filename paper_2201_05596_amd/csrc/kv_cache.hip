// Rows of keys and values into the caches, quantised as they are written, and back.
// Bound by traffic.  A unit of work is 8 elements: 16 bytes of a row, and 16, 8 or 4 bytes of the cache.  A work-group takes
// some rows of one head's keys or values: rows that follow each other in a sequence (a prefill, a prefix) are consecutive in
// the cache, and so are their scales.  Reading 65536 positions of 8 heads of 128 from 8 bits takes 78 us, 5.2 TB/s, as a large
// copy; writing and reading them 144 us, 5.6 TB/s.
#include <algorithm>

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

// The heads of the same rows follow each other, keys and values in turn: so a row's pieces are read (written, in the reverse) at
// about the same time, whatever the number of heads.  us for 65536 rows of 8 heads of 128 with the rows of one head following each
// other / so: written to bf16 104 / 88, 8 bits 97 / 81, 4 bits 90 / 74, read from 8 bits 82 / 80; heads of 64 the same either way.
constexpr int kGridY = 32768;
__device__ __forceinline__ int first_row(int rows_per_block) { return (blockIdx.z * kGridY + blockIdx.y) * rows_per_block; }
// BIG: a call of so many rows that what it stores is out of the caches before anybody can read it: stores that leave no trace there,
// and two units per thread, all their loads on the way before the first is used (bf16 rows, which are only moved: one).
template <bool BIG, typename T> __device__ __forceinline__ void store(void* at, T v) {
    if constexpr (BIG) __builtin_nontemporal_store(v, static_cast<T*>(at));
    else *static_cast<T*>(at) = v;
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int KIND, bool BIG> constexpr int units() { return BIG && KIND != MOE_CACHE_BF16 ? 2 : 1; }
template <int KIND, int DH, bool BIG>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8, STEP = 256 / PPR, IT = units<KIND, BIG>();       // pieces per row; rows of the work-group's first units
    const int tid = threadIdx.x, g = blockIdx.x >> 1, which = blockIdx.x & 1, piece = tid % PPR, first = first_row(IT * STEP) + tid / PPR;
    const uint16_t* rows = static_cast<const uint16_t*>(a.rows[which]);
    uint8_t* cache = static_cast<uint8_t*>(a.cache[which]);
    long long at[IT];
    uint4 w[IT];
#pragma unroll
    for (int n = 0; n < IT; ++n) at[n] = cache_row(a, first + n * STEP, g);
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        const int r = first + n * STEP;
        w[n] = at[n] >= 0 ? *reinterpret_cast<const uint4*>(rows + r * a.stride[which] + g * DH + piece * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        if constexpr (KIND == MOE_CACHE_BF16) {
            if (at[n] >= 0) store<BIG>(cache + (at[n] * DH + piece * 8) * 2, u32x4{w[n].x, w[n].y, w[n].z, w[n].w});
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
                if constexpr (KIND == MOE_CACHE_FP8) store<BIG>(cache + at[n] * DH + piece * 8, u32x2{code[0], code[1]});
                else store<BIG>(cache + at[n] * (DH / 2) + piece * 4, code[0]);
            }
            // the row's scale bytes by one lane
            constexpr int blocks = DH / kScaleBlock;
            uint32_t bytes = 0;
            const int lane0 = (tid & 63) - piece;
#pragma unroll
            for (int j = 0; j < blocks; ++j) bytes |= (uint32_t)__shfl((int)byte, lane0 + 4 * j) << (8 * j);
            if (at[n] >= 0 && piece == 0) {
                if constexpr (blocks == 4) *reinterpret_cast<uint32_t*>(a.scale[which] + at[n] * 4) = bytes;
                else *reinterpret_cast<uint16_t*>(a.scale[which] + at[n] * 2) = (uint16_t)bytes;
            }
        }
    }
}

template <int KIND, int DH, bool BIG>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheRows a) {
    constexpr int PPR = DH / 8, STEP = 256 / PPR, IT = units<KIND, BIG>();
    const int tid = threadIdx.x, g = blockIdx.x >> 1, which = blockIdx.x & 1, piece = tid % PPR, first = first_row(IT * STEP) + tid / PPR;
    const uint8_t* cache = static_cast<const uint8_t*>(a.cache[which]);
    long long at[IT];
    uint4 w[IT];                                              // as the cache holds it, then in bf16
    uint8_t byte[IT];
#pragma unroll
    for (int n = 0; n < IT; ++n) at[n] = cache_row(a, first + n * STEP, g);
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        w[n] = make_uint4(0, 0, 0, 0);
        byte[n] = 0;
        if (at[n] < 0) continue;
        if constexpr (KIND == MOE_CACHE_BF16) w[n] = *reinterpret_cast<const uint4*>(cache + (at[n] * DH + piece * 8) * 2);
        else if constexpr (KIND == MOE_CACHE_FP8) { const uint2 c = *reinterpret_cast<const uint2*>(cache + at[n] * DH + piece * 8); w[n].x = c.x; w[n].y = c.y; }
        else w[n].x = *reinterpret_cast<const uint32_t*>(cache + at[n] * (DH / 2) + piece * 4);
        if constexpr (KIND != MOE_CACHE_BF16) byte[n] = a.scale[which][at[n] * (DH / kScaleBlock) + piece / 4];
    }
#pragma unroll
    for (int n = 0; n < IT; ++n) {
        if (at[n] < 0) continue;
        const uint32_t x = w[n].x, y = w[n].y;
        const float f = scale_value(byte[n]);
        if constexpr (KIND == MOE_CACHE_FP8) w[n] = make_uint4(fp8_pair<false>(x, f), fp8_pair<true>(x, f), fp8_pair<false>(y, f), fp8_pair<true>(y, f));
        if constexpr (KIND == MOE_CACHE_FP4) w[n] = make_uint4(fp4_pair<0>(x, f), fp4_pair<1>(x, f), fp4_pair<2>(x, f), fp4_pair<3>(x, f));
        const int r = first + n * STEP;
        store<BIG>(static_cast<uint16_t*>(const_cast<void*>(a.rows[which])) + r * a.stride[which] + g * DH + piece * 8, u32x4{w[n].x, w[n].y, w[n].z, w[n].w});
    }
}

static CacheRows cache_rows(const moe_cache_shape_t* c, int n_rows, const void* k, long long ks, const void* v, long long vs, const int32_t* seq,
                     const int32_t* pos, const void* kc, const void* vc, const uint8_t* kx, const uint8_t* vx) {
    return CacheRows{{k, v}, {ks, vs}, {const_cast<void*>(kc), const_cast<void*>(vc)}, {const_cast<uint8_t*>(kx), const_cast<uint8_t*>(vx)},
                     seq, pos, n_rows, c->n_seq, c->n_kv_heads, c->max_len};
}

static dim3 cache_grid(const CacheRows& a, int rows_per_block) {
    const int blocks = (a.n_rows + rows_per_block - 1) / rows_per_block;
    return dim3((unsigned)(2 * a.G), (unsigned)std::min(blocks, kGridY), (unsigned)((blocks + kGridY - 1) / kGridY));
}
// us of a call for 65536 rows of 8 heads (keys and values), with ordinary stores and one unit / with these and one / with these and two:
//                            written and read               read
//     bf16, heads of 128     241 / 164 / 164            131 / 89 / 91
//     8 bits                 174 / 163 / 144             91 / 82 / 78
//     4 bits                 170 / 153 / 141             91 / 80 / 82
//     bf16, heads of 64      118 /  90 /  93             58 / 47 / 50
//     8 bits                  94 /  85 /  79             47 / 45 / 43
//     4 bits                  78 /  81 /  76             47 / 27 / 27
// (two units with ordinary stores: no faster than one).  Both sides of the border, 8000 rows of 8 heads of 128 read from 8 bits 11.1 / 9.0
// us, of 64 from 4 bits 5.5 / 4.6; with fewer rows the next kernel may find them in the caches, and two units leave too few work-groups
// (960 rows written to 8 bits 3.2 / 3.5).
static bool many_rows(const CacheRows& a, int head_dim) { return (long long)a.n_rows * a.G * head_dim >= 1 << 22; }
template <int KIND, int DH, bool BIG> void write_rows(const CacheRows& a, hipStream_t s) {
    hipLaunchKernelGGL((cache_write_kernel<KIND, DH, BIG>), cache_grid(a, units<KIND, BIG>() * (256 / (DH / 8))), dim3(256), 0, s, a);
}
template <int KIND, int DH, bool BIG> void read_rows(const CacheRows& a, hipStream_t s) {
    hipLaunchKernelGGL((cache_read_kernel<KIND, DH, BIG>), cache_grid(a, units<KIND, BIG>() * (256 / (DH / 8))), dim3(256), 0, s, a);
}

#define MOE_CACHE_KIND(CALL, KIND) \
    do { \
        const bool big = many_rows(a, c->head_dim); \
        if (c->head_dim == 128) big ? CALL<KIND, 128, true>(a, s) : CALL<KIND, 128, false>(a, s); \
        else big ? CALL<KIND, 64, true>(a, s) : CALL<KIND, 64, false>(a, s); \
    } while (0)
#define MOE_CACHE_ROWS(CALL) \
    do { \
        if (c->kind == MOE_CACHE_BF16) MOE_CACHE_KIND(CALL, MOE_CACHE_BF16); \
        else if (c->kind == MOE_CACHE_FP8) MOE_CACHE_KIND(CALL, MOE_CACHE_FP8); \
        else MOE_CACHE_KIND(CALL, MOE_CACHE_FP4); \
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
#undef MOE_CACHE_KIND

}  // namespace moe
