// Rows and weights into 8 bits (i8.h), and codes into the order of the products.  Bound by traffic: what is large passes the caches by
// (16384 rows of 4096, 201 MB read and written: 37.1 us through the caches, 32.7 = 6.1 TB/s past them; 33 MB 9.8 and 10.7).
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
    template <bool BIG> __device__ __forceinline__ void load(const uint16_t* p) { v = BIG ? load_stream16(p) : *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void none() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack_bias8(v, f); }
};
template <> struct Piece<float> {
    u32x4_t a, b;
    template <bool BIG> __device__ __forceinline__ void load(const float* p) {
        const u32x4_t* v = reinterpret_cast<const u32x4_t*>(p);
        a = BIG ? __builtin_nontemporal_load(v) : v[0];
        b = BIG ? __builtin_nontemporal_load(v + 1) : v[1];
    }
    __device__ __forceinline__ void none() { a = b = u32x4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f[q] = __uint_as_float(a[q]);
            f[4 + q] = __uint_as_float(b[q]);
        }
    }
};

template <typename T> __device__ __forceinline__ uint32_t piece_max_bits(const Piece<T>& p) {
    float f[8];
    p.get(f);
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) m = max(m, __float_as_uint(f[q]) & 0x7fffffffu);
    return m;
}
template <typename T> __device__ __forceinline__ u32x2_t piece_codes(const Piece<T>& p, uint32_t m, float inv) {
    float f[8];
    p.get(f);
    uint32_t c[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) c[q] = m < 0x7f800000u ? i8_code_bits(f[q], inv) : 0u;
    return u32x2_t{i8_pack4(c[0], c[1], c[2], c[3]), i8_pack4(c[4], c[5], c[6], c[7])};
}
template <bool BIG> __device__ __forceinline__ void store_codes(int8_t* to, const u32x2_t o) {
    if (BIG) __builtin_nontemporal_store(o, reinterpret_cast<u32x2_t*>(to));
    else *reinterpret_cast<u32x2_t*>(to) = o;
}

// TPR threads (a wave or a work-group) hold the first 8 NP TPR values of a row from their one read to their codes.  LONG: there are more, which are read
// again for their codes (rows of more than 65536 columns, whose float values do not fit a work-group's registers: 150 x 131072 24.5 us, 300 in bf16 28.9; held,
// partly in scratch memory, 37.8 and 40.4).
// BIG: rows and codes past the caches
template <typename T, int TPR, int NP, bool LONG, bool BIG>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void i8_rows_kernel(const I8RowsArgs a) {
    constexpr int PER = TPR < 256 ? 256 / TPR : 1;               // rows of a work-group
    __shared__ uint32_t part[TPR / kWave];
    const int tid = threadIdx.x % TPR;
    const long long r = a.first + (long long)blockIdx.x * PER + threadIdx.x / TPR;
    if (a.zero)
        for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < a.n_zero; i += (long long)gridDim.x * blockDim.x) a.zero[i] = 0;
    if (r >= a.n_rows || (r < a.n_grouped && r % a.capacity >= a.rows[r / a.capacity])) return;   // the whole wave or work-group
    const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
    Piece<T> p[NP];
    const int pieces = a.cols / 8, padded = (a.cols + 63) / 64 * 8;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = tid + i * TPR;
        if (at < pieces) p[i].template load<BIG>(x + (size_t)at * 8);
        else p[i].none();
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) m = max(m, piece_max_bits(p[i]));
    if constexpr (LONG)
        for (int at = tid + NP * TPR; at < pieces; at += TPR) {
            Piece<T> v;
            v.template load<false>(x + (size_t)at * 8);
            m = max(m, piece_max_bits(v));
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
        const u32x2_t o = piece_codes(p[i], m, inv);
        if (at < padded) store_codes<BIG>(out + (size_t)at * 8, o);                              // zeros behind the row's end
    }
    if constexpr (LONG)
        for (int at = tid + NP * TPR; at < padded; at += TPR) {
            Piece<T> v;
            v.none();
            if (at < pieces) v.template load<BIG>(x + (size_t)at * 8);
            store_codes<BIG>(out + (size_t)at * 8, piece_codes(v, m, inv));
        }
}

template <typename T, int TPR, int NP, bool LONG = false> int launch_rows_p(const I8RowsArgs& a, hipStream_t s) {
    constexpr int threads = TPR < 256 ? 256 : TPR, per = threads / TPR;
    constexpr int most = 1 << 21;                                // work-groups of a launch, whose threads are counted in 32 bits
    constexpr bool can_be_big = TPR != 256 || NP > 2;             // (a work-group for each of fewer than 2048 short rows: 32 MB)
    const bool big = (long long)a.n_rows * a.cols * (long long)sizeof(T) > (64ll << 20);
    I8RowsArgs part = a;
    for (long long first = 0; first < a.n_rows; first += (long long)most * per) {
        const dim3 blocks((unsigned)std::min<long long>(most, (a.n_rows - first + per - 1) / per));
        part.first = (int)first;
        if (big && can_be_big) hipLaunchKernelGGL((i8_rows_kernel<T, TPR, NP, LONG, can_be_big>), blocks, dim3(threads), 0, s, part);
        else hipLaunchKernelGGL((i8_rows_kernel<T, TPR, NP, LONG, false>), blocks, dim3(threads), 0, s, part);
        part.zero = nullptr;
    }
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
    return launch_rows_p<T, 1024, 8, true>(a, s);
}

// COLS columns of a group, all of K, by a work-group of THREADS: four consecutive k-rows of 8 columns for each thread and round, so that
// a thread has whole words of the packed order (4 k of a column).  They cross LDS once, which then holds a round's bytes in that order.
// QUANTISE: from bf16, with the columns' scales; else codes are there.  KEEP: rounds whose values stay in registers from the
// first pass (the columns' largest magnitudes) to the second; a longer K is read again, mostly from the Infinity Cache.
// LARGE: W's last reading and the result past the caches.
// 64 columns are whole cache lines of W; with 32 there are twice the work-groups, for a single matrix.  Neighbouring tiles, which then share
// lines, are eight work-groups apart: on the same XCD.  us with 32 / 64 columns: 1000 x 4000 9.0 / 10.2; 64 x 2048 x 8192 876 / 773, past the
// caches 928 / 692, without values in scratch memory 666 (3.2 GB: 4.8 TB/s; a thread for 8 columns of one row with the transposition byte by byte in LDS 1083); 16 x 8192 x 2048, read twice,
// 315 / 285, past the caches 346 / 244.
template <bool QUANTISE, int KEEP, int THREADS, int COLS, bool LARGE>
__global__ __launch_bounds__(THREADS, KEEP > 4 ? 2 : 4) void i8_weights_kernel(const void* __restrict__ W, int8_t* __restrict__ packed,
                                                             float* __restrict__ scale, int K, int N, int tiles, int all) {
    constexpr int OCTETS = COLS / 8;
    constexpr int ROWS = THREADS / OCTETS * 4, WAVES = THREADS / kWave;        // k-rows of a round: whole blocks of 64
    static_assert(ROWS % 64 == 0, "whole blocks");
    __shared__ uint32_t most[WAVES][COLS];
    __shared__ uint32_t words[ROWS * COLS / 4];                // [block][fragment][k-group][column of the fragment][4 k]
    const int tid = threadIdx.x, cp = tid % OCTETS, quad = tid / OCTETS;
    const int pair = blockIdx.x >> 4, tile = ((pair << 3) + (blockIdx.x & 7)) * 2 + (blockIdx.x >> 3 & 1);
    const long long g = tile / tiles;
    const int n0 = tile % tiles * COLS, n = n0 + cp * 8;
    if (tile >= all) return;
    const int KB = (K + 63) / 64, NG = (N + 127) / 128, rounds = (K + ROWS - 1) / ROWS;
    const uint16_t* wb = static_cast<const uint16_t*>(W) + (size_t)g * K * N + min(n, N - 8);
    const int8_t* wc = static_cast<const int8_t*>(W) + (size_t)g * K * N + n;
    // A thread's four rows of a round, and its eight columns, are there or not (K and N are multiples of 8); if not, others stand in, which the maxima do
    // not mind and whose codes are made zero: loads under a condition were waited for one by one.
    auto there = [&](int round) { return round * ROWS + quad * 4 < K && n < N; };
    auto load = [&](int round, uint4 (&v)[4], bool last) {       // last: nobody reads it again
        const uint16_t* p = wb + (size_t)min(round * ROWS + quad * 4, K - 4) * N;
#pragma unroll
        for (int i = 0; i < 4; ++i, p += N) v[i] = LARGE && last ? load_stream16(p) : *reinterpret_cast<const uint4*>(p);
    };
    uint4 held[KEEP > 0 ? KEEP : 1][4];
    float inv[8];
    if constexpr (QUANTISE) {
        uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        auto see = [&](const uint4 (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float f[8];
                unpack_bias8(v[i], f);
#pragma unroll
                for (int q = 0; q < 8; ++q) m[q] = max(m[q], __float_as_uint(f[q]) & 0x7fffffffu);
            }
        };
        if constexpr (KEEP > 0) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) load(i, held[i], true);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                see(held[i]);
#pragma unroll
                for (int q = 0; q < 8; ++q) asm volatile("" : "+v"(m[q]));       // all of a round's maxima here, not one column after the other,
            }
            // and the values as loaded: left to itself the compiler keeps what it unpacked for the maxima, more than there are registers
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(held[i][q].x), "+v"(held[i][q].y), "+v"(held[i][q].z), "+v"(held[i][q].w));
        } else {
            uint4 next[4];
            load(0, held[0], false);
            for (int i = 0; i < rounds; ++i) {
                load(i + 1, next, false);
                see(held[0]);
#pragma unroll
                for (int q = 0; q < 4; ++q) held[0][q] = next[q];
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
#pragma unroll
            for (int s = OCTETS; s < 64; s <<= 1) m[q] = max(m[q], (uint32_t)__shfl_xor((int)m[q], s));
            if ((tid & 63) < OCTETS) most[tid >> 6][cp * 8 + q] = m[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            uint32_t b = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) b = max(b, most[w][cp * 8 + q]);
            inv[q] = i8_inverse(b);
            if (quad == 0 && n < N) scale[(size_t)g * N + n + q] = i8_scale(b);
            if (b >= 0x7f800000u) inv[q] = __uint_as_float(0x7fc00000u);
        }
    }
    auto finish = [&](int round, const uint4 (&v)[4]) {
        uint32_t o[8];                                           // word q: column q's four codes
        if constexpr (QUANTISE) {
            float f[4][8];
            const uint32_t mask = there(round) ? ~0u : 0u;       // zeros behind K and N
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack_bias8(v[i], f[i]);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                o[q] = i8_pack4(i8_code_bits(f[0][q], inv[q]), i8_code_bits(f[1][q], inv[q]), i8_code_bits(f[2][q], inv[q]), i8_code_bits(f[3][q], inv[q]));
                if (inv[q] != inv[q]) o[q] = 0;                  // a column that is not all numbers
                o[q] &= mask;
            }
        } else {
            u32x2_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = round * ROWS + quad * 4 + i;
                r[i] = there(round) ? *reinterpret_cast<const u32x2_t*>(wc + (size_t)k * N) : u32x2_t{0, 0};
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int s = q & 3;
                auto word = [&](int i) { return (q < 4 ? r[i].x : r[i].y) >> (8 * s); };
                o[q] = i8_pack4(word(0), word(1), word(2), word(3));
            }
        }
        const int at = (((quad >> 4) * 8 * 4 + (quad >> 2 & 3)) * OCTETS + cp) * 4 + (quad & 3);
        if (round > 0) __syncthreads();                          // the round before has been read
#pragma unroll
        for (int q = 0; q < 8; ++q) words[at + q * (4 * OCTETS * 4)] = o[q];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {                            // a round's pieces of 16 bytes, two for each thread
            const int p = tid + i * THREADS, c = p % OCTETS, kq = p / OCTETS & 3, j = p / (4 * OCTETS) & 7, kb = round * (ROWS / 64) + p / (32 * OCTETS);
            if (kb < KB) {
                const size_t to = ((((size_t)g * KB + kb) * NG + n0 / 128) * 8 + j) * 64 + kq * 16 + n0 % 128 / 8 + c;
                const uint4 o = *reinterpret_cast<const uint4*>(words + p * 4);
                if (LARGE) store_stream16(packed + to * 16, o);
                else *reinterpret_cast<uint4*>(packed + to * 16) = o;
            }
        }
    };
    if constexpr (KEEP > 0) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (i < rounds) finish(i, held[i]);
    } else {
        if (QUANTISE) load(0, held[0], true);
        for (int i = 0; i < rounds; ++i) {
            uint4 next[4];
            if (QUANTISE) load(i + 1, next, true);
            finish(i, held[0]);
            if (QUANTISE) {
#pragma unroll
                for (int q = 0; q < 4; ++q) held[0][q] = next[q];
            }
        }
    }
}

template <bool QUANTISE, int KEEP, int THREADS, int COLS, bool LARGE> int launch_weights_k(const void* W, void* packed, float* scale, int G, int K, int N, hipStream_t s) {
    const int tiles = (N + 127) / 128 * (128 / COLS);         // whole blocks of 128 columns, zeros behind N
    const long long blocks = ((long long)G * tiles + 15) / 16 * 16;
    if (blocks * THREADS >= (1ll << 32)) return MOE_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((i8_weights_kernel<QUANTISE, KEEP, THREADS, COLS, LARGE>), dim3((unsigned)blocks), dim3(THREADS), 0, s, W, static_cast<int8_t*>(packed), scale,
                       K, N, tiles, G * tiles);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace

int launch_i8_rows(const I8RowsArgs& a, int dtype, hipStream_t s) {
    if (a.n_rows <= 0) return MOE_OK;
    return dtype == MOE_F32 ? launch_rows_t<float>(a, s) : launch_rows_t<uint16_t>(a, s);
}

int launch_i8_pack(const int8_t* codes, void* packed, int G, int K, int N, hipStream_t s) {
    if (K <= 128) return launch_weights_k<false, 0, 128, 32, false>(codes, packed, nullptr, G, K, N, s);
    return launch_weights_k<false, 0, 512, 32, false>(codes, packed, nullptr, G, K, N, s);
}

int launch_i8_weights(const uint16_t* W, void* packed, float* scale, int G, int K, int N, hipStream_t s) {
    if ((long long)G * K * N > (32ll << 20)) {
        if (K <= 128) return launch_weights_k<true, 1, 256, 64, true>(W, packed, scale, G, K, N, s);
        if (K <= 1024) return launch_weights_k<true, 4, 512, 64, true>(W, packed, scale, G, K, N, s);
        if (K <= 2048) return launch_weights_k<true, 8, 512, 64, true>(W, packed, scale, G, K, N, s);
        return launch_weights_k<true, 0, 1024, 64, true>(W, packed, scale, G, K, N, s);
    }
    if (K <= 64) return launch_weights_k<true, 1, 64, 32, false>(W, packed, scale, G, K, N, s);
    if (K <= 256) return launch_weights_k<true, 1, 256, 32, false>(W, packed, scale, G, K, N, s);
    if (K <= 1024) return launch_weights_k<true, 2, 512, 32, false>(W, packed, scale, G, K, N, s);
    if (K <= 4096) return launch_weights_k<true, 8, 512, 32, false>(W, packed, scale, G, K, N, s);
    return launch_weights_k<true, 0, 1024, 32, false>(W, packed, scale, G, K, N, s);
}

}  // namespace moe
