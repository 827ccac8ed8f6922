// Rotary positions: pairs of a head's dimensions turned by the angle position * frequency.
//   (x, y) -> amplitude (x cos - y sin, y cos + x sin)
// Bound by the rows' traffic (each element read and written once): 16384 rows of 40 heads of 128 take 57 us, 5.9 TB/s (float: 120,
// 5.6), where a large copy reaches 5.2.  A work-group takes a few rows of all heads: their angles are the same in every head, so they
// are worked out once, into LDS.
#include "moe_internal.h"

namespace moe {

template <typename T, int V> struct Piece;                   // V elements as they lie in memory
template <> struct Piece<uint16_t, 8> {
    uint4 w;
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void put(const float (&f)[8]) {
        w = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
};
template <> struct Piece<uint16_t, 4> {
    uint2 w;
    __device__ __forceinline__ void get(float (&f)[4]) const {
        f[0] = __uint_as_float(w.x << 16); f[1] = __uint_as_float(w.x & 0xffff0000u);
        f[2] = __uint_as_float(w.y << 16); f[3] = __uint_as_float(w.y & 0xffff0000u);
    }
    __device__ __forceinline__ void put(const float (&f)[4]) { w = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])); }
};
template <> struct Piece<float, 4> {
    float4 w;
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w; }
    __device__ __forceinline__ void put(const float (&f)[4]) { w = make_float4(f[0], f[1], f[2], f[3]); }
};

struct RopeArgs {
    const void* x;
    void* out;
    const double* turns;
    const int32_t* pos;
    long long x_stride, out_stride;
    int n_rows, n_heads, head_dim, rot_dim, rows_per_block;
    float amplitude;
};

// BIG: stores of 16 bytes that leave no trace in the caches, for calls whose rows are out of them before anybody can read them
template <bool BIG, typename P> __device__ __forceinline__ void store(void* at, const P& p) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    if constexpr (BIG && sizeof(P) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, p), static_cast<u32x4*>(at));
    else *static_cast<P*>(at) = p;
}

// V elements per access.  A unit of work is, of one head of one row, two pieces whose elements are partners (HALF) or one piece
// of adjacent pairs; behind the units that turn come those that are passed on (COPY: out is not x).
template <typename T, int V, bool HALF, bool COPY, bool BIG>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
    extern __shared__ float2 turn[];                          // [rows_per_block][rot_dim / 2] cos, sin
    typedef Piece<T, V> P;
    const int tid = threadIdx.x, half = a.rot_dim / 2;
    const int row0 = blockIdx.x * a.rows_per_block, rows = min(a.rows_per_block, a.n_rows - row0);
    for (int i = tid; i < rows * half; i += 256) {
        const int r = i / half, f = i - r * half;
        // whole turns come off in 64 bits: the angle of a far position is as exact as that of a near one
        const double t = (double)a.pos[row0 + r] * a.turns[f];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        turn[i] = make_float2(a.amplitude * c, a.amplitude * s);
    }
    __syncthreads();
    const int turning = HALF ? half / V : a.rot_dim / V, units = turning + (COPY ? (a.head_dim - a.rot_dim) / V : 0);
    const T* xs = static_cast<const T*>(a.x);
    T* os = static_cast<T*>(a.out);
    const int per_row = a.n_heads * units;
    for (int i = tid; i < rows * per_row; i += 256) {
        const int r = i / per_row, u0 = i - r * per_row, h = u0 / units, u = u0 - h * units;
        if (a.pos[row0 + r] < 0) continue;
        const T* x = xs + (row0 + r) * a.x_stride + h * a.head_dim;
        T* o = os + (row0 + r) * a.out_stride + h * a.head_dim;
        if (COPY && u >= turning) {
            const int at = a.rot_dim + (u - turning) * V;
            store<BIG>(o + at, *reinterpret_cast<const P*>(x + at));
            continue;
        }
        P p = *reinterpret_cast<const P*>(x + u * V), q;
        float f[V], g[V];
        p.get(f);
        if (HALF) {
            q = *reinterpret_cast<const P*>(x + half + u * V);
            q.get(g);
            float y[V], z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float2 cs = turn[r * half + u * V + e];
                y[e] = f[e] * cs.x - g[e] * cs.y;
                z[e] = g[e] * cs.x + f[e] * cs.y;
            }
            p.put(y);
            q.put(z);
            store<BIG>(o + u * V, p);
            store<BIG>(o + half + u * V, q);
        } else {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                const float2 cs = turn[r * half + u * (V / 2) + e];
                g[2 * e] = f[2 * e] * cs.x - f[2 * e + 1] * cs.y;
                g[2 * e + 1] = f[2 * e + 1] * cs.x + f[2 * e] * cs.y;
            }
            p.put(g);
            store<BIG>(o + u * V, p);
        }
    }
}

int launch_rope(const moe_rope_t* rope, int n_rows, int n_heads, const void* x, long long x_stride, const double* turns,
                const int32_t* pos, void* out, long long out_stride, hipStream_t s) {
    RopeArgs a{x, out, turns, pos, x_stride, out_stride, n_rows, n_heads, rope->head_dim, rope->rot_dim, 1, rope->amplitude};
    // Rows of few pieces together, as long as there are work-groups enough: 16384 rows of one head of 64 10.4 / 4.1 us, of 4 of 128
    // 12.2 / 7.8; of 40 heads a row stays alone (61 us, two rows 63, four 67), except that 2^24 go two by two: a grid has fewer than
    // 2^32 threads.
    const long long pieces = (long long)n_heads * rope->head_dim / 8;
    const auto more = [&](int rows) { return n_rows / rows >= 1 << 24 || (rows < 16 && rows * pieces < 512 && n_rows / (2 * rows) >= 1024); };
    while (more(a.rows_per_block)) a.rows_per_block *= 2;
    const dim3 grid((unsigned)((n_rows + a.rows_per_block - 1) / a.rows_per_block));
    const size_t lds = (size_t)a.rows_per_block * (rope->rot_dim / 2) * sizeof(float2);
    const bool copy = out != x, half = rope->layout == MOE_ROPE_HALF;
    // 32 MB of bf16 are all the L2 caches: 4096 rows of 40 heads of 128 18.9 us with ordinary stores / 14.2, 16384 rows 62.0 / 57.5
    const bool big = (long long)n_rows * n_heads * rope->head_dim >= 1 << 24;
#define MOE_ROPE_SIZE(T, V, HALF, COPY) \
    do { \
        if (big) hipLaunchKernelGGL((rope_kernel<T, V, HALF, COPY, true>), grid, dim3(256), lds, s, a); \
        else hipLaunchKernelGGL((rope_kernel<T, V, HALF, COPY, false>), grid, dim3(256), lds, s, a); \
    } while (0)
#define MOE_ROPE(T, V) \
    do { \
        if (half && copy) MOE_ROPE_SIZE(T, V, true, true); \
        else if (half) MOE_ROPE_SIZE(T, V, true, false); \
        else if (copy) MOE_ROPE_SIZE(T, V, false, true); \
        else MOE_ROPE_SIZE(T, V, false, false); \
    } while (0)
    if (rope->dtype == MOE_F32) MOE_ROPE(float, 4);
    else if (half && rope->rot_dim % 16) MOE_ROPE(uint16_t, 4);        // a half that ends inside 16 bytes
    else MOE_ROPE(uint16_t, 8);
#undef MOE_ROPE
#undef MOE_ROPE_SIZE
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
