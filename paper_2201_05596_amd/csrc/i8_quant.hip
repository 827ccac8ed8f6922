// Rows and weights into 8 bits (i8.h), and codes into the order of the products.  Bound by traffic.
#include "i8.h"

namespace moe {

namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t m) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
    return m;
}

// 8 values in 32 bits, as loaded
template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void none() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack_bias8(v, f); }
};
template <> struct Piece<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void none() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};

// TPR threads (a wave or a work-group) hold a row of up to 8 NP TPR values from its one read to its codes.
template <typename T, int TPR, int NP>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void i8_rows_kernel(const I8RowsArgs a) {
    constexpr int PER = TPR < 256 ? 256 / TPR : 1;               // rows of a work-group
    __shared__ uint32_t part[TPR / kWave];
    const int tid = threadIdx.x % TPR;
    const long long r = (long long)blockIdx.x * PER + threadIdx.x / TPR;
    if (a.zero)
        for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < a.n_zero; i += (long long)gridDim.x * blockDim.x) a.zero[i] = 0;
    if (r >= a.n_rows || (a.rows && r % a.capacity >= a.rows[r / a.capacity])) return;   // the whole wave or work-group
    const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
    Piece<T> p[NP];
    const int pieces = a.cols / 8, padded = (a.cols + 63) / 64 * 8;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = tid + i * TPR;
        if (at < pieces) p[i].load(x + (size_t)at * 8);
        else p[i].none();
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        float f[8];
        p[i].get(f);
#pragma unroll
        for (int q = 0; q < 8; ++q) m = max(m, __float_as_uint(f[q]) & 0x7fffffffu);
    }
    m = wave_max_bits(m);
    if constexpr (TPR > kWave) {
        if (tid % kWave == 0) part[tid / kWave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / kWave; ++w) m = max(m, part[w]);
    }
    const float inv = i8_inverse(m);
    if (tid == 0) a.scale[r] = i8_scale(m);
    int8_t* out = a.codes + r * a.codes_stride;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = tid + i * TPR;
        float f[8];
        p[i].get(f);
        uint32_t c[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) c[q] = m < 0x7f800000u ? i8_code_bits(f[q], inv) : 0u;
        const u32x2_t o = {i8_pack4(c[0], c[1], c[2], c[3]), i8_pack4(c[4], c[5], c[6], c[7])};
        if (at < padded) *reinterpret_cast<u32x2_t*>(out + (size_t)at * 8) = o;      // zeros behind the row's end
    }
}

template <typename T, int TPR, int NP> int launch_rows_p(const I8RowsArgs& a, hipStream_t s) {
    constexpr int per = TPR < 256 ? 256 / TPR : 1;
    const long long blocks = ((long long)a.n_rows + per - 1) / per;
    hipLaunchKernelGGL((i8_rows_kernel<T, TPR, NP>), dim3((unsigned)blocks), dim3(TPR < 256 ? 256 : TPR), 0, s, a);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
template <typename T> int launch_rows_t(const I8RowsArgs& a, hipStream_t s) {
    const int p = (a.cols + 63) / 64 * 8;                        // pieces of a row
    if (a.n_rows >= 2048) {                                      // a wave per row
        if (p <= 64) return launch_rows_p<T, 64, 1>(a, s);
        if (p <= 128) return launch_rows_p<T, 64, 2>(a, s);
        if (p <= 256) return launch_rows_p<T, 64, 4>(a, s);
        if (p <= 512) return launch_rows_p<T, 64, 8>(a, s);
    }
    if (p <= 256) return launch_rows_p<T, 256, 1>(a, s);
    if (p <= 512) return launch_rows_p<T, 256, 2>(a, s);
    if (p <= 1024) return launch_rows_p<T, 256, 4>(a, s);
    if (p <= 2048) return launch_rows_p<T, 256, 8>(a, s);
    if (p <= 8192) return launch_rows_p<T, 1024, 8>(a, s);
    return launch_rows_p<T, 1024, 16>(a, s);
}

// 64 columns of a group, all of K, by a work-group of 1024 threads: 8 columns of one of 128 k-rows for each thread and round.
// Codes cross LDS: a thread's piece of the packed order is 16 k of one column.
constexpr int kWCols = 64, kWRows = 128, kWThreads = 1024, kWPitch = kWCols + 4;
static_assert(kWThreads == kWRows * kWCols / 8, "a thread per 8 columns of a row");

// QUANTISE: from bf16, with the columns' scales; else codes are there.  KEEP: rounds whose values stay in registers from the
// first pass (the columns' largest magnitudes) to the second; longer K is read again
template <bool QUANTISE, int KEEP>
__global__ __launch_bounds__(kWThreads) void i8_weights_kernel(const void* __restrict__ W, int8_t* __restrict__ packed,
                                                               float* __restrict__ scale, int K, int N, int tiles) {
    __shared__ uint32_t most[kWThreads / kWave][kWCols];
    __shared__ int8_t codes[kWRows][kWPitch];
    const int tid = threadIdx.x, kr = tid >> 3, cp = tid & 7;
    const long long g = blockIdx.x / tiles;
    const int n0 = (int)(blockIdx.x % tiles) * kWCols, n = n0 + cp * 8;
    const int KB = (K + 63) / 64, NG = (N + 127) / 128, rounds = (K + kWRows - 1) / kWRows;
    const uint16_t* wb = static_cast<const uint16_t*>(W) + (size_t)g * K * N + n;
    const int8_t* wc = static_cast<const int8_t*>(W) + (size_t)g * K * N + n;
    auto load = [&](int round) {
        const int k = round * kWRows + kr;
        return k < K && n < N ? *reinterpret_cast<const uint4*>(wb + (size_t)k * N) : make_uint4(0, 0, 0, 0);
    };
    uint4 held[KEEP > 0 ? KEEP : 1];
    float inv[8];
    bool dead[8];
    if constexpr (QUANTISE) {
        uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        auto see = [&](const uint4& v) {
            float f[8];
            unpack_bias8(v, f);
#pragma unroll
            for (int q = 0; q < 8; ++q) m[q] = max(m[q], __float_as_uint(f[q]) & 0x7fffffffu);
        };
        if constexpr (KEEP > 0) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) held[i] = load(i);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) see(held[i]);
        } else {
#pragma unroll 4
            for (int i = 0; i < rounds; ++i) see(load(i));
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
#pragma unroll
            for (int s = 8; s < 64; s <<= 1) m[q] = max(m[q], (uint32_t)__shfl_xor((int)m[q], s));
            if ((tid & 63) < 8) most[tid >> 6][cp * 8 + q] = m[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            uint32_t b = 0;
#pragma unroll
            for (int w = 0; w < kWThreads / kWave; ++w) b = max(b, most[w][cp * 8 + q]);
            inv[q] = i8_inverse(b);
            dead[q] = b >= 0x7f800000u;
            if (kr == 0 && n < N) scale[(size_t)g * N + n + q] = i8_scale(b);
        }
    }
    auto finish = [&](int round, const uint4& v) {
        u32x2_t o = {0, 0};
        const int k = round * kWRows + kr;
        if constexpr (QUANTISE) {
            float f[8];
            unpack_bias8(v, f);
            uint32_t c[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) c[q] = dead[q] ? 0u : i8_code_bits(f[q], inv[q]);
            o = u32x2_t{i8_pack4(c[0], c[1], c[2], c[3]), i8_pack4(c[4], c[5], c[6], c[7])};
        } else if (k < K && n < N) {
            o = *reinterpret_cast<const u32x2_t*>(wc + (size_t)k * N);
        }
        __syncthreads();                                         // the round before has been read
        *reinterpret_cast<uint32_t*>(&codes[kr][cp * 8]) = o.x;
        *reinterpret_cast<uint32_t*>(&codes[kr][cp * 8 + 4]) = o.y;
        __syncthreads();
        // half a piece per thread: k-block, k-group, half | fragment, column of eight
        const int half = tid & 1, c = (tid >> 1) & 7, kq = (tid >> 4) & 3, j = (tid >> 6) & 7, kb = tid >> 9;
        uint32_t b[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) b[q] = (uint8_t)codes[kb * 64 + kq * 16 + half * 8 + q][c * 8 + j];
        const int kbg = round * 2 + kb;
        if (kbg < KB) {
            const size_t at = ((((size_t)g * KB + kbg) * NG + n0 / 128) * 8 + j) * 64 + kq * 16 + n0 % 128 / 8 + c;
            *reinterpret_cast<u32x2_t*>(packed + at * 16 + half * 8) =
                u32x2_t{i8_pack4(b[0], b[1], b[2], b[3]), i8_pack4(b[4], b[5], b[6], b[7])};
        }
    };
    if constexpr (KEEP > 0) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (i < rounds) finish(i, held[i]);
    } else {
        for (int i = 0; i < rounds; ++i) finish(i, QUANTISE ? load(i) : make_uint4(0, 0, 0, 0));
    }
}

template <bool QUANTISE, int KEEP> int launch_weights_k(const void* W, void* packed, float* scale, int G, int K, int N, hipStream_t s) {
    const int tiles = (N + 127) / 128 * 2;                       // whole blocks of 128 columns, zeros behind N
    const long long blocks = (long long)G * tiles;
    if (blocks >= (1ll << 31)) return MOE_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((i8_weights_kernel<QUANTISE, KEEP>), dim3((unsigned)blocks), dim3(kWThreads), 0, s, W, static_cast<int8_t*>(packed), scale, K, N, tiles);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace

int launch_i8_rows(const I8RowsArgs& a, int dtype, hipStream_t s) {
    if (a.n_rows <= 0) return MOE_OK;
    return dtype == MOE_F32 ? launch_rows_t<float>(a, s) : launch_rows_t<uint16_t>(a, s);
}

int launch_i8_pack(const int8_t* codes, void* packed, int G, int K, int N, hipStream_t s) {
    return launch_weights_k<false, 0>(codes, packed, nullptr, G, K, N, s);
}

int launch_i8_weights(const uint16_t* W, void* packed, float* scale, int G, int K, int N, hipStream_t s) {
    if (K <= 4 * kWRows) return launch_weights_k<true, 4>(W, packed, scale, G, K, N, s);
    if (K <= 8 * kWRows) return launch_weights_k<true, 8>(W, packed, scale, G, K, N, s);
    if (K <= 16 * kWRows) return launch_weights_k<true, 16>(W, packed, scale, G, K, N, s);
    return launch_weights_k<true, 0>(W, packed, scale, G, K, N, s);
}

}  // namespace moe
