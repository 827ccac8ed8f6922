// Products in 8-bit integers: the numbers they are made of, and what their kernels share.
//
// A row of activations (a column of weights) with largest magnitude m is held as codes round(v r), ties to even, and a scale s:
//   M = max(m, 2^-100),  r = 127 / M,  s = M / 127   (each rounded to 32 bits)
// and a product is  acc (s_row s_col) + bias  with acc the exact sum of products of codes, an integer below 2^31 for up to
// kI8MaxK of them.  Integer sums do not depend on an order: every kernel gives the same bits, however it splits K.
// A row that holds an infinity or NaN has codes 0 and scale NaN: its results are NaN, no other row's are.
//
// Bytes: rows of codes are padded to a multiple of 64 (weights hold zeros there, so what the codes hold there has no part), and
// 16 codes of a row or column are a lane's operand of v_mfma_i32_16x16x64_i8.  That is, byte for byte, the layout of bf16
// operands of the 16x16x32 instruction with half as many k: pieces of 16 bytes, four k-groups of 16 lanes, fragments of 1 KB.
// For that reason the products count K in pairs of codes.
#pragma once

#include <algorithm>

#include "ffn_common.h"

namespace moe {

constexpr int kI8MaxK = 131072;             // 2^17 products of at most 128 * 127 stay below 2^31
constexpr float kI8Least = 0x1p-100f;       // smallest M
inline int i8_row_bytes(int K) { return (K + 63) / 64 * 64; }
inline size_t i8_weight_bytes(int G, int K, int N) { return (size_t)G * ((K + 63) / 64) * ((N + 127) / 128) * 8192; }

typedef int i32x4_t __attribute__((ext_vector_type(4)));

// r and s of a row whose largest magnitude has the bit pattern m (infinities and NaN compare above every number)
__device__ __forceinline__ float i8_inverse(uint32_t m) { return m >= 0x7f800000u ? 0.f : 127.0f / fmaxf(__uint_as_float(m), kI8Least); }
__device__ __forceinline__ float i8_scale(uint32_t m) { return m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(m), kI8Least) / 127.0f; }
// The code of v in the low byte: the multiply-add rounds v r once, to a whole number, ties to even (the sum is between 2^23 and 2^24)
__device__ __forceinline__ uint32_t i8_code_bits(float v, float r) { return __float_as_uint(fmaf(v, r, 12582912.0f)); }
__device__ __forceinline__ uint32_t i8_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// value of a finished sum
__device__ __forceinline__ float i8_value(int acc, float scale, float bias) { return fmaf((float)acc, scale, bias); }

// A grouped product as WsGemmArgs says (B packed, K in pairs of codes), and
struct I8GemmArgs : WsGemmArgs {
    long long lda, ldo;        // from row to row: of A in pairs of codes, of out in elements
    const float* a_scale;      // by A row, as row_map gives it
    const float* b_scale;      // [G, N]
    int32_t out32;             // results in 32 bits (EPI_STORE, EPI_GELU)
    // few rows: A is bf16 (lda in elements), not codes, and a_max holds the bit patterns of its rows' largest magnitudes
    const uint32_t* a_max;
    uint32_t* out_max;         // EPI_GELU: the same of the rows written, at most raised; or nullptr
};

// groups of a product that can have rows
inline int few_groups(const I8GemmArgs& a) { return a.order && a.slots > 0 && a.slots < a.G ? a.slots : a.G; }

// (i8_quant.hip) rows x [n_rows, cols] -> codes, scale.  Of the first n_grouped rows, row r counts if r % capacity < rows[r / capacity], others
// stay as they are.  zero: n_zero words that are cleared on the way, or nullptr.
struct I8RowsArgs {
    const void* x;
    long long x_stride, codes_stride;
    int8_t* codes;
    float* scale;
    const int32_t* rows;
    int capacity, n_grouped, n_rows, cols;
    uint32_t* zero;
    long long n_zero;
    int first;                 // the launcher's: first row of a launch
};
int launch_i8_rows(const I8RowsArgs& a, int dtype, hipStream_t s);
// (i8_quant.hip) codes of W [G, K, N] in the order of the products, a lane's 16 bytes being 16 consecutive k of a column: byte (k, n)
// of group g at ((((g KB + k / 64) NG + n / 128) 8 + n % 8) 64 + (k % 64 / 16) 16 + n % 128 / 8) 16 + k % 16, KB = ceil(K / 64), NG =
// ceil(N / 128)
int launch_i8_pack(const int8_t* codes, void* packed, int G, int K, int N, hipStream_t s);
int launch_i8_weights(const uint16_t* W, void* packed, float* scale, int G, int K, int N, hipStream_t s);
// (i8_few.hip) few rows, bound by the read of the weights; `order` is not looked at
int launch_i8_few(const I8GemmArgs& a, int epi, hipStream_t s);
constexpr int kI8FewRows = 16;                                   // of a group, where a product makes codes from bf16
int few_columns(long long groups, int max_rows, int N);          // 16-column fragments of a work-group
bool i8_few_faster(int groups, int max_rows, int d, int f);      // for both products of FFNs
bool i8_few_faster_alone(const I8GemmArgs& a, int epi);          // for one product of codes
// (i8_token.hip) both products and the combine of a layer whose experts have few rows: the first (with h's largest magnitudes) or the second ones
// (in 32 bits, into ye and the dense branch's rows, then combined into out)
struct I8TokenArgs {
    I8GemmArgs experts, dense_branch;
    int32_t dense, T, E, top_k;
    const int32_t* order;                                        // as the gate leaves it
    uint32_t* done;                                              // second: i8_token_tiles(d) counters, 0 before
    const int32_t *expert_idx, *slot_idx;
    const float* gate_w;
    uint16_t* out;
};
inline int i8_token_tiles(int N) { return (N + 127) / 128 * 8; } // column tiles of a second product, at most
int launch_i8_token(const I8TokenArgs& t, bool second, hipStream_t s);
constexpr int kI8TokenRows = 128;                                // tokens of such a layer, at most
bool i8_token_faster(int T, int touched, int max_rows, int d, int f, bool dense);
// (i8_tile.hip) tiles of up to 128 rows, two or three work-groups per compute unit
int launch_i8_tile(const I8GemmArgs& a, const I8GemmArgs* b, int epi, hipStream_t s);
// (i8_wide.hip) tiles of 256 rows
int launch_i8_wide(const I8GemmArgs& a, const I8GemmArgs* b, int epi, hipStream_t s);
bool i8_wide_faster(const I8GemmArgs& a, const I8GemmArgs* b);   // than tiles of 128 rows

}  // namespace moe
