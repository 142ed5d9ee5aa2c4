// Attention of a chunk of new rows over the cache in pages and over the chunk itself.
//
//   out_i = softmax_j(sm_scale * s_ij) v_j,  j over the sequence's cached rows and the chunk's rows up to i;
//   cached: s_ij = (H q_i) . khat_j, khat = scale * (code - zero) or a 16-bit row, and H (sum_j p_ij vhat_j) is the cached rows' share;
//   new:    s_ij = q_i . k_j, with k and v as they arrive (binary16).
//
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, in tiles of 32 x 32: a query is a column, i.e. a lane and the
// lane 32 further, so the softmax needs no exchange between lanes but for a raised reference, and the weights leave the score product
// in the very registers in which the value product takes them: a lane's scores are those of rows 4q + i and 16 + 4q + i of a block for two
// q, and the packed V words and the 16-bit V tiles pair the rows that way.  Nothing goes through LDS but decoded meta words and 16-bit
// keys and values that several wavefronts share (the chunk's V rows are transposed by the reads).
//   K codes enter the scaled 32x32x64 product as 4-bit floats without decoding (three instructions per 16 codes), against the query as
// kDigits balanced base-32 digits that 6-bit floats hold exactly: 5 * kDigits bits of the query's largest channel, at the price of
// kDigits / 4 of a 16-bit product.  What else a score holds comes from one more product, that the codes' products are added onto: per row
// zero-point, 1 / scale and log2(V scale) / scale, per column the query's sum, the reference and 1, all in bfloat16 terms that
// together hold the 32-bit numbers.  One multiplication by the row's scale is left.
//   V codes are masked in place, which leaves binary16 subnormals code * 4^ii * 2^-24 (ii: the row's place in its word): one
// instruction per two codes.  The V scale and 4^-ii ride in the exponent of the weight, the denominator takes the weight back by
// 4^ii / scale, and zero-points are summed with the rounded weights.
//   Weights are binary16 (half a step is 2^-12 to 2^-11 of a weight; up to eight rows in a tile have two that round apart), relative to a reference
// that keeps the largest between 2^7 and 2^15: a weight below 2^-21 of its row's largest loses bits, one below 2^-31 all of them.  Scores, references, sums and accumulators are 32-bit.
//   Rows of a unit (a sequence's tokens times the heads of a KV head) come in tiles of 16 or 32 whose four wavefronts share the rows and deal
// the keys among them, or of 256, 32 for each of eight wavefronts that look at the same keys (paged_tile_rows says which, and what it measured).
//   Tiles of 256 are bound by the issue of vector and matrix instructions together, which share a SIMD's time (measured: a 32x32 product keeps
// the vector unit for 15 of its 33 cycles, a 16x16 one for 12 of 19, a vector instruction takes 3 to 4, an exponential 9), and by the power that
// matrix instructions may take (the 17 products of a block alone, on random data, take 0.9 ms of what follows).  So every block is expanded once
// for all eight.  4 x 2048 rows of 32 heads over 8192 cached ones: 1.23-1.3 ms, 955-1010 TFLOP/s of what the formula takes (a 16-bit
// matrix product of 8192 x 8192 x 8192: 1268); first chunks of 4096, which LDS reads bind as much, 0.27-0.29 ms, 760-805.
//   Tiles of 16 and 32 read the cache with what their wavefronts have under way.  One row of 4 heads over 32768 rows of 128 units (G = 64):
// 94-99 us, 3.4-3.6 TB/s, where vector instructions take 62 % of the time and matrix instructions 26; one row over 2048 to 4096 rows of 512 units
// 35-37 us, 3.1 TB/s, 13 of it before the first block and behind the last: two wavefronts a SIMD, 43 and 14 %.  One row over 640 of 32 units: 8.2 us
// and 2.8 for the merge, a chain of memory round trips.
//
// Pages of 4-bit codes (BITS = 4) take the same way.  A key's nibbles, two masked words for eight of them, are the 8-bit floats code * 2^-9 as they
// lie (subnormals among them), at twice the price of a 4-bit product; tiles of 256, which expand a block once for all, repack them as 6-bit floats
// code / 8, at its price.  A value's nibbles are masked in place, two a byte: code * 16^(ii mod 2) * 2^-24.
//   One row over 2048 to 4096 rows of 512 units 42 us, 5.0 TB/s, of which 10 to 12 lie before the first block and behind the last (in between
// 6.2 TB/s); one of 7 heads over 32768 rows of 128 units (G = 64) 110-115 us, 5.3-5.5 TB/s; one over 640 rows of 32 units 7.8 and 2.9 for the merge.
// 4 x 2048 rows of 32 heads over 8192 cached ones: 1.30-1.44 ms, 860-950 TFLOP/s, 2.93 million cycles at 2.0 to 2.25 GHz (down to 1.8, a large
// product's, where launches follow each other for long); with two groups 1.61-1.74 ms, 710-770 TFLOP/s, 3.74 million cycles.
#pragma once
#include "akvq_device.h"
#include "akvq_kernels.h"

#include <type_traits>

namespace akvq {
namespace {

constexpr int kDigits = 4;  // 3 or 4
constexpr int kFewWaves = 4;   // of a workgroup that has few rows: they share them and deal the keys among them
constexpr int kManyWaves = 8;  // of a workgroup that has many: each has its own, and all look at the same keys
constexpr int kCus = 256;
constexpr int kStageBlocks = 4;  // blocks of code rows that such a workgroup expands at a time, two wavefronts for each
constexpr float kNoScore = -1.0e30f;   // score of a row that takes no part, reference of a column without scores
constexpr float kRaiseAt = 15.0f;      // a score may exceed the reference by this (2^15 is the largest weight) ...
constexpr float kRaiseTo = 7.0f;       // ... and then gets a reference this far below it
constexpr float kApartFactor = 1.0f + 1.5f / 4096, kApart = 5.2823399e-4f;  // half a step of binary16, 2^-12 to 2^-11 of a number, and its base-2 logarithm
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(32))) _Float16 f16x32;
typedef __attribute__((ext_vector_type(8))) unsigned int u32x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ float exp2_bare(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_bare(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {  // round to nearest even, one conversion instruction
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
}
// ... of a times s and b times t, one instruction each
__device__ __forceinline__ uint32_t scaled_f16x2(float a, float b, float s, float t) {
  const f16x2 x = {(_Float16)__builtin_fmaf(a, s, 0.0f), (_Float16)__builtin_fmaf(b, t, 0.0f)};
  return __builtin_bit_cast(uint32_t, x);
}
// The values of lanes l % 32 and l % 32 + 32, in every lane.
struct Halves { float lo, hi; };
__device__ __forceinline__ Halves halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// ... of lanes l and l ^ 16, the one whose bit 4 is clear first.
__device__ __forceinline__ Halves neighbours(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// The value of lane l ^ 8.
__device__ __forceinline__ float other_eight(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, true)); }  // row_ror:8
__device__ __forceinline__ float halves_max(float v) {
  const Halves h = halves(v);
  return fmaxf(h.lo, h.hi);
}
__device__ __forceinline__ float halves_sum(float v) {
  const Halves h = halves(v);
  return h.lo + h.hi;
}

// How a wavefront's lanes share a tile of W columns (queries).  A lane group (`q` of W = 16, `h` of W = 32) holds slots 8 at a time of a
// product's inner dimension, and four consecutive rows of a result at a time.
//   A block's rows in a lane's result registers: y[4a + i] is row 8a + 4h + i (W = 32), row 16a + 4q + i (W = 16).
//   The inner slots of the value product: step s takes, in eight slots, rows 4g + i and 16 + 4g + i of the block, pair by pair, where g is
// 2s + h (W = 32) or q (W = 16), i.e. y[4s + i] and y[4s + 8 + i], or y[i] and y[4 + i].
//   Channels: of the query, 8 at a time, chunks 2k + h (W = 32, k < 8) or 4k + q (k < 4); of the output o[j][4a + i], 32j + 8a + 4h + i or,
// o[j][i], 16j + 4q + i.
template <int W>
struct Tile;
template <>
struct Tile<32> {
  typedef f32x16 Acc;
  static constexpr int kBlocks = 4, kSteps = 2, kChunks = 8, kScores = 16;  // of output channels; of value products and of query chunks; scores a lane
  static __device__ __forceinline__ Acc zero() { return (Acc){0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Acc f16(u32x4 a, u32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc bf16(u32x4 a, u32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // rows: codes as 4-bit floats code / 2; columns: query digits as 6-bit floats, times 2^(byte DIGIT of scale - 127)
  template <int DIGIT>
  static __device__ __forceinline__ Acc codes(u32x4 rows, u32x6 d, uint32_t scale, Acc c) {
    const i32x8 a = {(int)rows[0], (int)rows[1], (int)rows[2], (int)rows[3], 0, 0, 0, 0};
    const i32x8 b = {(int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4], (int)d[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, 0, 127, DIGIT, (int)scale);  // E2M1, E2M3
  }
  // ... as 6-bit floats code / 8
  template <int DIGIT>
  static __device__ __forceinline__ Acc codes(u32x6 rows, u32x6 d, uint32_t scale, Acc c) {
    const i32x8 a = {(int)rows[0], (int)rows[1], (int)rows[2], (int)rows[3], (int)rows[4], (int)rows[5], 0, 0};
    const i32x8 b = {(int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4], (int)d[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 2, 2, 0, 129, DIGIT, (int)scale);  // E2M3, E2M3
  }
  // ... as 8-bit floats code * 2^-9
  template <int DIGIT>
  static __device__ __forceinline__ Acc codes(u32x8 rows, u32x6 d, uint32_t scale, Acc c) {
    const i32x8 b = {(int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4], (int)d[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(__builtin_bit_cast(i32x8, rows), b, c, 0, 2, 0, 135, DIGIT, (int)scale);  // E4M3, E2M3
  }
  static __device__ __forceinline__ float column_max(float v) { return halves_max(v); }
  static __device__ __forceinline__ float column_sum(float v) { return halves_sum(v); }
  static __device__ __forceinline__ int row(int a, int g) { return 8 * a + 4 * g; }          // of y[4a]; g: lane group
  static __device__ __forceinline__ int channel(int j, int a, int g) { return 32 * j + 8 * a + 4 * g; }
};
template <>
struct Tile<16> {
  typedef f32x4 Acc;
  static constexpr int kBlocks = 8, kSteps = 1, kChunks = 4, kScores = 8;
  static __device__ __forceinline__ Acc zero() { return (Acc){0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Acc f16(u32x4 a, u32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc bf16(u32x4 a, u32x4 b, Acc c) { return mfma_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c); }
  template <int DIGIT>
  static __device__ __forceinline__ Acc codes(u32x4 rows, u32x6 d, uint32_t scale, Acc c) {
    const i32x8 a = {(int)rows[0], (int)rows[1], (int)rows[2], (int)rows[3], 0, 0, 0, 0};
    const i32x8 b = {(int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4], (int)d[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 2, 0, 127, DIGIT, (int)scale);
  }
  template <int DIGIT>
  static __device__ __forceinline__ Acc codes(u32x8 rows, u32x6 d, uint32_t scale, Acc c) {
    const i32x8 b = {(int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4], (int)d[5], 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, rows), b, c, 0, 2, 0, 135, DIGIT, (int)scale);
  }
  static __device__ __forceinline__ float column_max(float v) {
    const Halves h = neighbours(v);
    return halves_max(fmaxf(h.lo, h.hi));
  }
  static __device__ __forceinline__ float column_sum(float v) {
    const Halves h = neighbours(v);
    return halves_sum(h.lo + h.hi);
  }
  static __device__ __forceinline__ int row(int a, int g) { return 16 * a + 4 * g; }
  static __device__ __forceinline__ int channel(int j, int, int g) { return 16 * j + 4 * g; }
};

template <int CTRL>
struct Dpp { static constexpr int value = CTRL; };

template <int N>
__device__ __forceinline__ void butterflies(float (&x)[N], int s) {
#pragma unroll
  for (int e = 0; e < N; ++e)
    if ((e & s) == 0) {
      const float a = x[e], b = x[e + s];
      x[e] = a + b;
      x[e + s] = a - b;
    }
}
// one level across lanes, lane ^ 32 or lane ^ 16: exact products, one rounding
template <int ACROSS, int N>
__device__ __forceinline__ void butterflies_across(float (&x)[N], int lane) {
  const float sign = (lane & ACROSS) ? -1.0f : 1.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const Halves h = ACROSS == 32 ? halves(x[e]) : neighbours(x[e]);
    x[e] = __builtin_fmaf(sign, h.hi, h.lo);
  }
}
// 128-point transform without its factor of an output column in the layout of Tile
template <int W, int N>
__device__ __forceinline__ void wht128_output(float (&x)[N], int lane) {
  butterflies(x, 1);
  butterflies(x, 2);
  if constexpr (W == 16) butterflies_across<16>(x, lane);
  butterflies_across<32>(x, lane);
#pragma unroll
  for (int s = 4; s < N; s *= 2) butterflies(x, s);
}
// The transform of query columns as they are loaded, x[8k + i] = channel i of chunk k: by products with the matrix's signs, which binary16
// holds exactly (a hundred instructions; butterflies between lanes and registers take three times as many).  Row r of an operand is
// output channel e(r), inner slot j of lane group g channel c(g, j) of a chunk; the sign is the parity of e & c, so what depends on the chunk's
// number alone is left to a four-point transform of the results.
__device__ __forceinline__ u32x4 sign_row(int r, uint32_t base, uint32_t upper) {  // parities with r % 4 (slots j % 4), and of j / 4 = 1
  const uint32_t w0 = 0x3C003C00u ^ base ^ ((r & 1) ? 0x80000000u : 0u), w1 = 0x3C003C00u ^ base ^ ((r & 1) ? 0x80000000u : 0u) ^ ((r & 2) ? 0x80008000u : 0u);
  return (u32x4){w0, w1, w0 ^ upper, w1 ^ upper};
}
constexpr uint32_t kMinus = 0x80008000u;
__device__ __forceinline__ void rotate_query_columns(const u32x4 (&raw)[4], float (&x)[32], int lane) {  // W = 16
  // e = 32m + 8 (r / 4) + 4 hi + r % 4, c = 32k + 8g + j
  const int r = lane & 15, g = lane >> 4;
  const uint32_t base = (__popc((r >> 2) & g) & 1) ? kMinus : 0u;
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
    const u32x4 a = sign_row(r, base, hi ? kMinus : 0u);
    f32x4 t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = Tile<16>::f16(a, raw[k], Tile<16>::zero());
    const f32x4 s0 = t[0] + t[1], d0 = t[0] - t[1], s1 = t[2] + t[3], d1 = t[2] - t[3];
    const f32x4 y[4] = {s0 + s1, d0 + d1, s0 - s1, d0 - d1};
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[8 * m + 4 * hi + i] = y[m][i];
  }
}
__device__ __forceinline__ void rotate_query_columns(const u32x4 (&raw)[8], float (&x)[64], int lane) {  // W = 32
  // row r = 8a + 4h + i of an operand: e = 32b + 16 (a / 2) + 8h + 4 (a % 2) + i; c = 16k + 8g + j
  const int r = lane & 31, g = lane >> 5;
  const uint32_t base = ((r >> 2) & g & 1) ? kMinus : 0u, upper = ((r >> 3) & 1) ? kMinus : 0u;
  const u32x4 a0 = sign_row(r, base, upper), a1 = sign_row(r, base ^ (((r >> 4) & 1) ? kMinus : 0u), upper);
  f32x16 t[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) t[k] = Tile<32>::f16(a1, raw[2 * k + 1], Tile<32>::f16(a0, raw[2 * k], Tile<32>::zero()));
  const f32x16 s0 = t[0] + t[1], d0 = t[0] - t[1], s1 = t[2] + t[3], d1 = t[2] - t[3];
  const f32x16 y[4] = {s0 + s1, d0 + d1, s0 - s1, d0 - d1};
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) x[16 * b + e] = y[b][e];
}

// A float as three bfloat16 terms (its 24 bits), in the upper halves.
struct Terms { float a, b, c; };
__device__ __forceinline__ Terms split_terms(float v) {
  Terms t;
  t.a = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
  const float r = v - t.a;
  t.b = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
  t.c = r - t.b;
  return t;
}
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// A code of row ii of four lies this many bits above the others of its byte, in the words of the values.
template <int BITS>
__device__ __forceinline__ int code_place(int ii) { return BITS == 2 ? 2 * ii : 4 * (ii & 1); }
// A lane's words of a block's keys or values: what the two codes' order makes of it is at load_codes.
template <int BITS>
struct RowWords { u32x4 w[BITS / 2]; };
__device__ __forceinline__ u32x2 nibbles(uint32_t w) { return (u32x2){w & 0x0F0F0F0Fu, (w >> 4) & 0x0F0F0F0Fu}; }

// What is decoded of a block's meta words, a row a lane, for all columns that look at the block.
template <int NG>
struct BlockMeta {
  // Row operands of the product that a score starts with, sixteen bfloat16 slots.  First eight: minus the zero-point (low byte and multiples of
  // 256, three times each: times the three terms of the query's sum), two terms of (log2(V scale) - code_place) / scale (times 1).  Second
  // eight: terms of 1 / scale (times those of minus the reference), the third term.  A row that takes no part has kNoScore for the
  // logarithm, a scale of 1 and nothing else.
  __attribute__((aligned(16))) uint16_t start[32][2][8];
  __attribute__((aligned(16))) uint16_t start2[NG == 2 ? 32 : 1][8];  // first eight of the second group's product: its zero-point
  __attribute__((aligned(16))) float k_scale[NG][32];
  __attribute__((aligned(16))) float v_rcp[32];                       // 2^code_place / V scale, the larger one where there are two (no part: 0)
  __attribute__((aligned(16))) float v_share[NG == 2 ? 2 : 1][32];    // V scale / the larger one
  __attribute__((aligned(16))) uint16_t v_zero[2][NG][32];            // binary16, in the weights' order: zero-point * 2^(code_place - 6), low part and multiples of 2048
};

template <int NG>
struct MetaWords { uint32_t w[NG]; };

// a load with the non-temporal hint, or without
template <bool ONCE, typename T>
__device__ __forceinline__ T read(const T *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}
template <int NG, bool ONCE = false>
__device__ __forceinline__ MetaWords<NG> load_meta(const uint32_t *at) {
  if constexpr (NG == 2) {
    const u32x2 w = read<ONCE>(reinterpret_cast<const u32x2 *>(at));
    return {{w[0], w[1]}};
  } else {
    return {{read<ONCE>(at)}};
  }
}
// Scales of 0, which only rows have that were never written, count as the smallest that binary16 holds: their reciprocal is needed.
constexpr float kLeastScale = 5.9604645e-8f;  // 2^-24
// A row's scales and zero-points; one that takes no part has a scale of 1 and nothing else
template <int NG>
struct RowMeta {
  float scale[NG], zero[NG], top, rcp;  // the larger scale and its reciprocal (no part: 0)
  bool part;
  __device__ __forceinline__ RowMeta(const MetaWords<NG> &m, bool there, bool value) {
    part = there && (m.w[0] & 0x8000u) == 0u;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      scale[g] = part ? fmaxf(half_bits_to_float(m.w[g] & 0x7FFFu), kLeastScale) : 1.0f;
      zero[g] = part ? (float)((int)m.w[g] >> 16) : 0.0f;
    }
    top = NG == 2 && value ? fmaxf(scale[0], scale[NG - 1]) : scale[0];  // (keys: the first group's)
    rcp = part ? __builtin_amdgcn_rcpf(top) : 0.0f;
  }
};
// What scores need of a key's row; v_log: base-2 logarithm of what its value is multiplied by
template <int NG, typename Meta>
__device__ __forceinline__ void decode_key(const RowMeta<NG> &k, float v_log, Meta &bm, int r) {
  const Terms inv = split_terms(k.rcp), log = split_terms(k.part ? v_log * k.rcp : kNoScore);
  const float zh = rintf(k.zero[0] * (1.0f / 256.0f)) * -256.0f, zl = -k.zero[0] - zh;
  u32x4 *to = reinterpret_cast<u32x4 *>(&bm.start[r][0][0]);
  to[0] = (u32x4){upper_halves(zl, zl), upper_halves(zl, zh), upper_halves(zh, zh), upper_halves(log.a, log.b)};
  to[1] = (u32x4){upper_halves(inv.a, inv.a), upper_halves(inv.a, inv.b), upper_halves(inv.b, inv.c), upper_halves(log.c, 0.0f)};
  if constexpr (NG == 2) {
    const float yh = rintf(k.zero[1] * (1.0f / 256.0f)) * -256.0f, yl = -k.zero[1] - yh;
    *reinterpret_cast<u32x4 *>(&bm.start2[r][0]) = (u32x4){upper_halves(yl, yl), upper_halves(yl, yh), upper_halves(yh, yh), 0u};
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) bm.k_scale[g][r] = k.part || g == 0 ? k.scale[g] : 0.0f;
}
// Where row r of a block lies among its weights: in pairs (r, r + 16)
__device__ __forceinline__ int weight_place(int r) { return 2 * (r & 15) + (r >> 4); }
// Two blocks' meta words for values that stay in their words, a row a lane.  Returns whether some zero-point takes more than 11 bits.
template <int NG, int BITS>
__device__ __forceinline__ bool decode_pair(const MetaWords<NG> &kw, const MetaWords<NG> &vw, bool there, BlockMeta<NG> (&pair)[2], int lane) {
  const int r = lane & 31, ii = r & 3, at = weight_place(r);
  BlockMeta<NG> &bm = pair[lane >> 5];
  const RowMeta<NG> v(vw, there, true), k(kw, there, false);
  const int place = code_place<BITS>(ii);
  decode_key(k, log2_bare(v.top) - (float)place, bm, r);
  bm.v_rcp[r] = v.rcp * (float)(1 << place);
  bool far = false;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    if constexpr (NG == 2) bm.v_share[g][r] = v.scale[g] * v.rcp;
    const float hi = rintf(v.zero[g] * (1.0f / 2048.0f)) * 2048.0f, f = (float)(1 << place) * (1.0f / 64.0f);
    bm.v_zero[0][g][at] = (uint16_t)float_to_half_bits_rne((v.zero[g] - hi) * f);
    bm.v_zero[1][g][at] = (uint16_t)float_to_half_bits_rne(hi * f);
    far = far || hi != 0.0f;
  }
  return __ballot(far) != 0ull;
}

// A block expanded for the wavefronts of a workgroup of many rows: operands as their lanes take them.
template <int NG, int BITS>
struct CodeBlock {
  __attribute__((aligned(16))) uint16_t start[32][2][8];              // as in BlockMeta
  __attribute__((aligned(16))) uint16_t start2[NG == 2 ? 32 : 1][8];
  __attribute__((aligned(16))) float k_scale[NG][32];
  // 1 / V scale, where there are two 1 / the larger one's power of two (4 bits: its double), which its weight is multiplied by (no part: 0)
  __attribute__((aligned(16))) float v_rcp[32];
  __attribute__((aligned(16))) u32x4 k[2][kWave];                     // [product][lane] codes as 4-bit floats; of 6-bit ones the first four words
  __attribute__((aligned(8))) u32x2 k_more[BITS == 4 ? 2 : 1][BITS == 4 ? kWave : 1];  // ... and the others
  // [step][channel block][lane] code - low part of the zero-point, binary16; of two groups of 2-bit codes times the share
  __attribute__((aligned(16))) u32x4 v[2][4][kWave];
  // where some zero-point has one: minus its multiple of 1024, in the weights' order; of two groups of 2-bit codes times the share, in two binary16 terms
  __attribute__((aligned(16))) uint16_t v_far[NG][NG][32];
  // of two groups of 4-bit codes: their scales times v_rcp (32 bits: a scale may be 2^-40 of the other, which no binary16 number holds)
  __attribute__((aligned(16))) float v_share[BITS == 4 ? NG : 1][BITS == 4 && NG == 2 ? 32 : 1];
};
// The power of two at or below a positive number: its logarithm and reciprocal (of 0: -127 and 2^127).
__device__ __forceinline__ float power_log(float x) { return (float)((int)(__float_as_uint(x) >> 23) - 127); }
__device__ __forceinline__ float power_rcp(float x) { return __uint_as_float(0x7F000000u - (__float_as_uint(x) & 0x7F800000u)); }
// A value's zero-point: a low part, -512 to 511, and a multiple of 1024.  The first of two rows' as binary16 numbers -1536 - low: those from -1024 to
// -2047 hold ten bits as they are.
__device__ __forceinline__ uint32_t less_zero_low(uint32_t meta0, uint32_t meta1) {
  return (__builtin_amdgcn_perm(meta1, meta0, 0x07060302u) & 0x03FF03FFu) ^ 0xE600E600u;
}
__device__ __forceinline__ int zero_high(uint32_t meta) { return (((int)meta >> 16) + 512) & ~1023; }

__device__ __forceinline__ void lds_barrier() {  // leaves loads from memory in flight
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Rows of 16 chunks of 16 bytes in LDS: chunk c of row r lies at place c ^ 2 (r % 8), so that eight rows' chunks of the same number fall
// on all banks, read whole (a key operand) or as the two chunks of a transposing read.
__device__ __forceinline__ int staged_at(int row, int chunk) { return row * kD + ((chunk ^ (2 * (row & 7))) << 3); }
constexpr int kStage = 64;  // rows of 16-bit keys and values that a workgroup of many rows holds in LDS at a time (two such stages)

template <int G, int W, bool MANY, int BITS>
struct PagedShared;
template <int G, int W, int BITS>
struct PagedShared<G, W, true, BITS> {
  union {  // code rows come first, then 16-bit rows
    struct {
      CodeBlock<kD / G, BITS> blocks[2][kStageBlocks];  // being worked on, and the next
      __attribute__((aligned(4))) uint8_t far[2][kStageBlocks];  // whether v_far is written
    };
    struct { __attribute__((aligned(16))) uint16_t k[2][kStage * kD], v[2][kStage * kD]; };
  };
};
template <int G, int BITS>
struct PagedShared<G, 16, false, BITS> {
  union {  // of every wavefront its own: a pair of blocks' meta words and the next one's, then its sums
    BlockMeta<kD / G> meta[2][2];
    __attribute__((aligned(16))) float o[16][kD + 4];
  } own[kFewWaves];
  union {  // one after the other; (sixteen rows of a unit are of one block of the chunk)
    uint32_t digits[1][kDigits][6][kWave];
    __attribute__((aligned(16))) uint16_t v[1][32 * kD];
    __attribute__((aligned(16))) float self[16][kD + 4];  // sums over the chunk's rows
  };
  float m[kFewWaves + 1][16], l[kFewWaves + 1][16];
};
template <int G, int BITS>
struct PagedShared<G, 32, false, BITS> {
  union {  // the sums of the wavefronts come last
    struct {
      struct { BlockMeta<kD / G> meta[2][2]; } own[kFewWaves];
      union {
        __attribute__((aligned(16))) uint16_t v[kFewWaves][32 * kD];
        uint32_t digits[2][kDigits][6][kWave];
      };
    };
    __attribute__((aligned(16))) float o[kFewWaves][32][kD + 4];
  };
  float m[kFewWaves][32], l[kFewWaves][32];
};

// EIGHT: no workgroup has more than eight rows (of a tile of 16): the two columns of each also share the digits of its query.
//   Three workgroups of a tile of 16 run on a CU (168 registers), two of those with two groups of 4-bit codes and more than eight rows (16 rows
// of 256 units over 8192: 71 us, three at a time and one block after the other 72).
template <int G, int W, bool MANY, int BITS, bool EIGHT = false>
__global__ __launch_bounds__(64 * (MANY ? kManyWaves : kFewWaves), W == 16 && !(BITS == 4 && G == 64 && !EIGHT) ? 3 : 2) void paged_attention_kernel(PagedAttentionArgs a) {
  static_assert(BITS == 2 || kDigits == 4);
  static_assert(!EIGHT || (W == 16 && BITS == 4));
  typedef Tile<W> T;
  typedef typename T::Acc Acc;
  constexpr int NG = kD / G, NW = MANY ? kManyWaves : kFewWaves, WK = MANY ? 1 : NW, kWide = W == 32;
  constexpr int NB = T::kBlocks, NS = T::kSteps, NC = T::kChunks, NY = T::kScores, NA = NY / 4;
  __shared__ PagedShared<G, W, MANY, BITS> sh;
  const PagedArgs &c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & (W - 1), g_lane = lane / W, n = lane & 15, p = kWide ? (lane >> 4) & 1 : 0;
  const int wk = MANY ? 0 : wave, wr = MANY ? wave : 0;
  const int R = a.Hq / c.Hkv, split = blockIdx.z;
  constexpr int kRows = (MANY ? NW : 1) * W;  // of a workgroup
  int b = blockIdx.x / c.Hkv, head = blockIdx.x % c.Hkv, tile = gridDim.y - 1 - blockIdx.y;  // the rows that see most first
  // Unequal sequences, where a CU gets few workgroups: which ones decides.  Where it holds one (many rows), the longest begin first; where it
  // holds two or three, the first on every CU go from long to short, the second from short to long.
  ChunkSpan s;
  const bool ordered = MANY ? c.B <= kWave : c.B <= kWave && gridDim.x > kCus && gridDim.y * gridDim.z == 1;
  // Few rows: the pages' numbers where two loads hold them all (lane l: of pages window + l and window + 64 + l), and the beginning of the list of
  // 16-bit rows: asked for with the lengths where these decide nothing
  const bool short_table = c.max_pages <= 2 * kWave;
  [[maybe_unused]] int window = 0, pages = 0, next_pages = 0;
  int entry = 0, listed = 0;
  auto ask_table = [&](int from) { return c.table[(size_t)b * c.max_pages + min(from + lane, c.max_pages - 1)]; };
  auto ask_lists = [&] {
    if (!MANY && short_table) {
      pages = ask_table(0);
      next_pages = ask_table(kWave);
    }
    const size_t unit = (size_t)b * c.Hkv + head;
    entry = c.sal_idx[unit * c.S_cap + lane];  // (S_cap >= 64)
    listed = c.sal_cnt[unit];
  };
  constexpr bool kEarlyLists = !MANY && BITS == 4;
  if (kEarlyLists && !ordered) ask_lists();
  if (ordered) {
    const int me = min(lane, c.B - 1);
    const ChunkSpan mine = chunk_span(c.seq_len[me], c.row_start[me], c.row_start[me + 1], c);
    const int tiles = lane >= c.B ? 0 : MANY ? (mine.rows * R + kRows - 1) / kRows : 1, keys = mine.len + mine.rows;
    int begin = 0;  // of this lane's sequence in that order, in tiles
    if constexpr (kEarlyLists) {  // one tile each: how many are longer, by keys that no two lanes share (lengths past 2^24 count alike)
      const int mine_key = lane < c.B ? min(keys, (1 << 24) - 1) * kWave + (kWave - 1 - lane) : -1;
      for (int x = 0; x < c.B; x += 8)
#pragma unroll
        for (int y = 0; y < 8; ++y) begin += __builtin_amdgcn_readlane(mine_key, x + y) > mine_key;
    } else {
      for (int x = 0; x < c.B; ++x) {
        const int other = __builtin_amdgcn_readlane(keys, x);
        if (other > keys || (other == keys && x < lane)) begin += __builtin_amdgcn_readlane(tiles, x);
      }
    }
    int at = blockIdx.y * c.B + b;
    if constexpr (!MANY) {
      const int turn = blockIdx.x / kCus, last = min((int)gridDim.x, 2 * kCus) - 1;
      const int place = turn == 1 ? last - (blockIdx.x - kCus) : blockIdx.x;
      at = place / c.Hkv;
      head = place - at * c.Hkv;
    }
    const uint64_t here = __ballot(at >= begin && at < begin + tiles);
    if (here == 0ull) return;  // whole workgroup
    b = __builtin_ctzll(here);
    tile = __builtin_amdgcn_readlane(begin + tiles, b) - 1 - at;
    s = {__builtin_amdgcn_readlane(mine.len, b), __builtin_amdgcn_readlane(mine.first, b), __builtin_amdgcn_readlane(mine.rows, b)};
  } else {
    s = chunk_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  }
  const int unit = b * c.Hkv + head;
  const int rows = s.rows * R;                                  // of this unit: token by token, the heads of the group
  const int wg_row = tile * kRows;                              // first row of the workgroup
  if (wg_row >= rows) return;                                   // whole workgroup
  const int row0 = wg_row + wr * W;                             // first row of the wavefront
  const bool idle = row0 >= rows;                               // (of a workgroup whose wavefronts have rows of their own)
  // Up to eight rows in a tile of 16 (a generated token of every sequence): each in two columns, whose weights are half a step of binary16
  // apart, so that their roundings differ and half as much is left in the sum of both: 1.1e-4 of a weight, 2.1e-4 of one column.  Outputs are off by
  // 2.4e-4 of their norm in place of 2.9e-4 (2.1e-4 is their own rounding), for 0.25 us of a call over 640 rows and 1 % of long ones.  (The
  // second column for what the first one's rounding drops would leave 2.1e-4, and takes 6 to 17 %.)
  const bool twice = EIGHT || (W == 16 && rows - wg_row <= 8);
  auto apart = [&] { return twice && (lane & 8) ? kApart : 0.0f; };
  const int my_row = min(row0 + (twice ? col & 7 : col), rows - 1), my_token = my_row / R;
  const float sm2 = a.sm_scale * kLog2e;

  const uint16_t *q_at = a.q + (s.first + my_token) * a.q_stride + (head * R + my_row - my_token * R) * kD + 8 * g_lane;
  // the query as it arrives: a chunk of eight channels for every k (read again by each kind of keys: kept, it would take 32 registers all along)
  auto load_query = [&](u32x4 (&raw)[NC]) {
#pragma unroll
    for (int k = 0; k < NC; ++k) raw[k] = *reinterpret_cast<const u32x4 *>(q_at + kD / NC * k);
  };
  // Few rows: what needs nothing but the sequence is asked for in front of the search for its 16-bit rows: the query, too
  const int32_t *table = c.table + (size_t)b * c.max_pages;
  if (!kEarlyLists || ordered) ask_lists();
  [[maybe_unused]] u32x4 early_query[NC];
  if constexpr (!MANY) load_query(early_query);

  // ---- the keys of this workgroup: blocks of 32 code rows, of 32 overlay slots, of 32 chunk rows, dealt to the splits as one list
  const int32_t *sidx = c.sal_idx + (size_t)unit * c.S_cap;
  int wide = min(max(listed, 0), c.S_cap);                      // overlay slots of cached rows (the list may be final for new rows, too)
  if (wide <= kWave) {
    wide = __popcll(__ballot(lane < wide && entry < s.len));
  } else {
    int base = 0, span = wide;                                  // entries below s.len: an ascending list, sampled
    while (span > 0) {
      const int step = (span + 63) >> 6;
      const int below = __popcll(__ballot(lane * step < span && sidx[min(base + lane * step, c.S_cap - 1)] < s.len));
      if (below == 0) break;
      base += (below - 1) * step + 1;                           // the last sample below is below
      span = min(step - 1, wide - base);
    }
    wide = base;
  }
  const int last_row = min(wg_row + kRows, rows) - 1;
  const int n_code = (s.len + 31) >> 5, n_wide = (wide + 31) >> 5, n_self = last_row / R / 32 + 1;
  // equal runs of the list, of a workgroup (many rows) or of a wavefront (few): a block of 16-bit rows counts as two of code rows
  const int parts = a.n_split * WK, wide_at = n_code, self_at = n_code + 2 * n_wide;
  const int run = (self_at + 2 * n_self) / parts, longer = self_at + 2 * n_self - run * parts;  // the first runs are longer by one
  auto run_start = [&](int part) { return run * part + min(part, longer); };
  const int run_begin = run_start(split * WK + wk), run_end = run_start(split * WK + wk + 1), group_begin = run_start(split * WK);
  const int code_begin = min(run_begin, n_code), code_end = min(run_end, n_code);
  const int wide_begin = min((max(run_begin - wide_at, 0) + 1) / 2, n_wide), wide_end = min((max(run_end - wide_at, 0) + 1) / 2, n_wide);
  const int self_begin = min((max(run_begin - self_at, 0) + 1) / 2, n_self), self_end = min((max(run_end - self_at, 0) + 1) / 2, n_self);

  Acc o[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) o[j] = T::zero();
  // per column: the reference that weights are relative to, from which excess over it it is raised (before the first score: any), and
  // this lane's share of the sum
  float m = 0.0f, limit = 0.5f * kNoScore, l = 0.0f;
  // the rotated query without its factor, which is returned; and times it, sm_scale * log2(e) in it: products with that are base-2 logits
  auto turned = [&](const u32x4 (&raw)[NC], float (&x)[8 * NC]) {
    float f = sm2;
    if (!a.q_rotated) {
      rotate_query_columns(raw, x, lane);
      f *= inv_sqrt128();
    } else {
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          x[8 * k + 2 * w] = half_bits_to_float(raw[k][w] & 0xFFFFu);
          x[8 * k + 2 * w + 1] = half_bits_to_float(raw[k][w] >> 16);
        }
    }
    return f;
  };
  auto rotated = [&](const u32x4 (&raw)[NC], float (&x)[8 * NC]) {
    const float f = turned(raw, x);
#pragma unroll
    for (int e = 0; e < 8 * NC; ++e) x[e] *= f;
  };
  // A block's scores relative to the reference (no part: far below).  The reference is raised, and what was summed against it rescaled
  // (`more`: the rest of it), only when a score exceeds it by kRaiseAt.
  auto raise = [&](auto &&more, auto &...y) {
    float top = kNoScore;
    auto top_of = [&](float (&x)[NY]) {
#pragma unroll
      for (int i = 0; i < NY; ++i) top = fmaxf(top, x[i]);
    };
    (top_of(y), ...);
    if (__builtin_expect(__ballot(top > limit) != 0ull, 0)) {
      float all = T::column_max(top);
      if (W == 16 && twice) all = fmaxf(all, other_eight(all));  // (one reference for both columns)
      float by = 0.0f;
      if (all > limit) {  // the lanes of a column agree
        const float to = rintf(m + all) - kRaiseTo;
        by = to - m;
        const float alpha = limit < 0.0f ? 0.0f : exp2_bare(-by);  // (there was nothing before the first score)
#pragma unroll
        for (int j = 0; j < NB; ++j) o[j] *= alpha;
        l *= alpha;
        m = to;
        limit = kRaiseAt;
        more(alpha);
      }
      auto lower = [&](float (&x)[NY]) {
#pragma unroll
        for (int i = 0; i < NY; ++i) x[i] -= by;
      };
      (lower(y), ...);
    }
  };
  auto weigh = [&](float (&y)[NY]) {  // ... and their weights
    raise([](float) {}, y);
#pragma unroll
    for (int i = 0; i < NY; ++i) y[i] = exp2_bare(y[i]);
  };

  // against 16-bit rows the query is two bfloat16 terms, 16 bits
  // tiles of 16: the wavefronts' sums over cached rows are merged before they are rotated back, once
  constexpr bool kMergeFirst = W == 16;
  u32x4 q_hi[NC], q_lo[NC];
  auto split_query = [&](const float (&x)[8 * NC]) {
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x0 = x[8 * k + 2 * i], x1 = x[8 * k + 2 * i + 1];
        const uint32_t hi = pack_bf16x2(x0, x1);
        q_hi[k][i] = hi;
        q_lo[k][i] = pack_bf16x2(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xFFFF0000u));
      }
  };

  // ================= code rows =================
  if (group_begin < n_code) {  // uniform over the workgroup
    // Query digits.  A lane's inner slots of a product are what ExpandF4 makes of two code words: slot v is word v / 16, field f = 2 (v % 8) +
    // (v / 8) % 2, channel 32 (2w + f / 8) + 8c + f % 8 of the words' chunk c, where W = 32: product 0 takes words w = 0 of chunks
    // c = h and 2 + h, product 1 their words w = 1 (a group each where there are two); W = 16: one product, words 0 and 1 of chunk q.
    constexpr int NP = kWide ? 2 : 1;
    float acc_z[NG];  // this lane's share of the sums of weight * zero-point / 64
#pragma unroll
    for (int g = 0; g < NG; ++g) acc_z[g] = 0.0f;

    const ExpandF4 ex4;
    struct Where { size_t row; int limit; };  // first row of a block in the pools; rows from `limit` on (of the sequence) take no part
    auto find = [&](int blk, int page) {
      const bool there = page >= 0 && page < c.n_pages;
      return Where{(((size_t)(there ? page : 0) * c.Hkv + head) << c.page_shift) + ((blk * 32) & ((1 << c.page_shift) - 1)), there ? s.len : 0};
    };
    // Two bits, W = 32: words 2p and 2p + 1 of chunks h and 2 + h (the other half of the lanes takes the other two); W = 16: all words of a chunk.
    // Four bits, W = 32: all words of chunks h and 2 + h in the block's half p; W = 16: of a chunk in both halves.  (Halves are rows of keys and
    // every other channel block of values.)
    typedef RowWords<BITS> Words;
    constexpr bool kOnce = EIGHT;  // one workgroup reads them: with the non-temporal hint
    auto load_codes = [&](const uint32_t *pool, const Where &at) {
      const uint32_t *blk = pool + at.row * (4 * BITS);
      Words words;
      if constexpr (BITS == 4) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
          words.w[x] = read<kOnce>(reinterpret_cast<const u32x4 *>(blk + (kWide ? 256 * p + (32 * x + 16 * g_lane + n) * 4 : 256 * x + 4 * lane)));
      } else if constexpr (kWide) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(blk + (16 * g_lane + n) * 4 + 2 * p), y = *reinterpret_cast<const u32x2 *>(blk + (32 + 16 * g_lane + n) * 4 + 2 * p);
        words.w[0] = (u32x4){x[0], x[1], y[0], y[1]};
      } else {
        words.w[0] = *reinterpret_cast<const u32x4 *>(blk + 4 * lane);
      }
      return words;
    };
    const int first = code_begin;
    // Few rows, bound by the stream: blocks in pairs, whose rows' meta words are decoded a row a lane.  Keys and values of the next pair are asked
    // for as soon as this one's are used up, meta words of the one after it in front of them, and the first ones in front of the query's
    // preparation.  The pages' numbers come 64 at a time, another 64 ahead: one a block, by a scalar load, would be waited for with the next
    // access to LDS.
    const int few_last = min(max(code_end, first + 1), n_code) - 1;  // (a wavefront without code rows asks for some block that there is)
    auto page_of = [&](int blk) { return (blk * 32) >> c.page_shift; };
    struct Pair { Where at[2]; };
    auto locate = [&](int blk) {  // in ascending order
      Pair p;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = min(blk + x, few_last), page = page_of(at);
        if (page - window >= kWave) {
          window += kWave;
          pages = next_pages;
          next_pages = ask_table(window + kWave);
        }
        p.at[x] = find(at, __builtin_amdgcn_readlane(pages, page - window));
        if (blk + x >= code_end) p.at[x].limit = 0;
      }
      return p;
    };
    MetaWords<NG> few_kw, few_vw;
    Words few_k[2], few_v[2];
    constexpr bool kOneValue = kWide && BITS == 4 && NG == 2;  // registers for one block's values: asked for a block ahead
    auto ask_meta = [&](const Pair &p) {
      const size_t row = ((lane < 32 ? p.at[0].row : p.at[1].row) + (lane & 31)) * NG;
      few_kw = load_meta<NG, kOnce>(c.k_meta + row);
      few_vw = load_meta<NG, kOnce>(c.v_meta + row);
    };
    auto row_there = [&](int blk, const Pair &p) { return (blk + (lane >> 5)) * 32 + (lane & 31) < (lane < 32 ? p.at[0].limit : p.at[1].limit); };
    Pair now = {}, next = {};
    if constexpr (!MANY) {
      if (!short_table) {
        window = page_of(min(first, few_last));
        pages = ask_table(window);
        next_pages = ask_table(window + kWave);
      }
      now = locate(first);
      ask_meta(now);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        few_k[x] = load_codes(c.k_codes, now.at[x]);
        if (x == 0 || !kOneValue) few_v[x] = load_codes(c.v_codes, now.at[x]);
      }
      next = locate(first + 2);
    }
    // EIGHT: product P takes digit P of a row in its first column and digit 2 + P in its second
    constexpr int ND = EIGHT ? kDigits / 2 : kDigits;
    u32x6 digits[NP][ND];
    // exponents of the digits, a byte a product.  8-bit rows of both groups meet in one product (W = 16): its other group's lanes get 2^-127
    constexpr int NU = BITS == 4 && !kWide ? NG : 1;
    uint32_t unit_exp[NU];
    u32x4 start[NG];  // column operands of the first product: terms of the query's sum, of minus the reference, ones
    auto start_slots = [&](float v, uint32_t ones) {
      const Terms x = split_terms(v);
      return (u32x4){upper_halves(x.a, x.b), upper_halves(x.c, x.a), upper_halves(x.b, g_lane == 1 ? x.a : x.c), ones};
    };
    {
      float x[8 * NC], mx = 0.0f, factor = 1.0f;
      auto prepare = [&](const u32x4 (&raw)[NC]) {
        if constexpr (BITS == 4) factor = turned(raw, x);
        else rotated(raw, x);
      };
      if constexpr (MANY) {
        u32x4 raw[NC];
        load_query(raw);
        prepare(raw);
      } else {
        prepare(early_query);
      }
#pragma unroll
      for (int e = 0; e < 8 * NC; ++e) mx = fmaxf(mx, fabsf(x[e]));
      mx = T::column_max(mx);
      if constexpr (BITS == 4) mx *= fabsf(factor);
      // integers of up to 5 kDigits - 1 bits and a sign in units of a power of two U, |x| < 2^(5 kDigits - 1) U
      const uint32_t e_biased = min(max(__float_as_uint(mx) >> 23, BITS == 4 ? 64u : 20u), 250u);  // mx < 2^(e_biased - 126)
      const float unit_inv = __uint_as_float((252u + 5u * kDigits - e_biased) << 23), u = 1.0f / unit_inv;
      float sum[2] = {0.0f, 0.0f};
      // digit k of n is the signed five-bit field k of ((n + b) ^ b), b = 16 in every lower digit
      constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer in the low bits
      constexpr int kHalf = kDigits == 4 ? 16 * (1 + 32 + 1024) : 16 * (1 + 32);
      int v[8 * NC];
      // (4 bits: the factor and the unit at once, queries below 2^-62 in units of 2^-82; no unit that is infinite meets a query of zeros)
      const float to_unit = BITS == 4 ? fminf(fmaxf(factor * unit_inv, -3.0e38f), 3.0e38f) : unit_inv;
#pragma unroll
      for (int e = 0; e < 8 * NC; ++e) {
        const float t = __builtin_fmaf(x[e], to_unit, kMagic);
        if constexpr (BITS == 2) sum[e / (4 * NC)] += t - kMagic;  // (the upper half of a lane's channels is the second group)
        v[e] = (__float_as_int(t) + (kHalf - 0x4B400000)) ^ kHalf;
      }
      auto make_digit = [&](int pr, int shift, int bits) {
        f32x16 dig[2];  // even and odd slots, as the packing conversion takes them
#pragma unroll
        for (int slot = 0; slot < 32; ++slot) {
          // (nibbles come out of their word even ones first as 8-bit floats, i and 4 + i side by side as 6-bit ones)
          const int f = BITS == 2 ? 2 * (slot & 7) + ((slot >> 3) & 1) : (slot & 8) + (MANY ? 4 * (slot & 1) + ((slot >> 1) & 3) : 2 * (slot & 3) + ((slot >> 2) & 1));
          const int word = slot >> 4;
          // W = 32: x[16 m + 8 s + i] with m = 2 pr + f / 8, s = word; W = 16: x[8 m + i] with m = 2 word + f / 8
          const int e = kWide ? 16 * (2 * pr + (f >> 3)) + 8 * word + (f & 7) : 8 * (2 * word + (f >> 3)) + (f & 7);
          dig[slot & 1][slot >> 1] = (float)(int)__builtin_amdgcn_sbfe(v[e], shift, bits);
        }
        const u32x6 made = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(dig[0], dig[1], 8.0f));
        // The conversion reads its operands while it already writes: they are kept past it, so that the result gets registers of its own.
        // (And one digit after the other: all of them at once take 128 registers.)
        asm volatile("" ::"v"(dig[0]), "v"(dig[1]), "v"(made) : "memory");
        return made;
      };
      constexpr int kTop = 5 * (kDigits - 1);
      if constexpr (MANY) {
#pragma unroll
        for (int pr = 0; pr < NP; ++pr)
#pragma unroll
          for (int d = 0; d < kDigits; ++d) digits[pr][d] = make_digit(pr, 5 * d, d == kDigits - 1 ? 32 - kTop : 5);
      } else {  // the wavefronts have the same rows: a digit each
        static_assert(kDigits <= kFewWaves);
#pragma unroll
        for (int pr = 0; pr < NP; ++pr) {
          const u32x6 made = make_digit(pr, 5 * wave, wave == kDigits - 1 ? 32 - kTop : 5);
#pragma unroll
          for (int i = 0; i < 6; ++i) sh.digits[pr][wave][i][lane] = made[i];
        }
        lds_barrier();
#pragma unroll
        for (int pr = 0; pr < NP; ++pr)
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 6; ++i) {
              // 8-bit rows: the product's inner slots 32L .. 32L + 31, which 6-bit digits of lane group L hold, lie in two lane groups of the rows,
              // sixteen in each: the lower or the upper half of their slots
              const int L = lane / W, from = kWide ? col + 32 * (i / 3) : col + 16 * (2 * (L & 1) + i / 3), word = i % 3 + 3 * (kWide ? L : L >> 1);
              digits[pr][d][i] = BITS == 2 ? sh.digits[pr][d][i][lane] : sh.digits[pr][EIGHT ? d + 2 * (col >> 3) : d][word][from];
            }
        lds_barrier();  // (what comes last lies where the digits were)
      }
      unit_exp[0] = (e_biased + 6u - 5u * kDigits) * 0x01010101u + 0x0F0A0500u;  // a byte a digit: each 32 times the one below
      if (EIGHT && col >= 8) unit_exp[0] >>= 16;
      if constexpr (NU == 2) {
        unit_exp[1] = g_lane >= 2 ? unit_exp[0] : 0u;
        unit_exp[0] = g_lane < 2 ? unit_exp[0] : 0u;
      }
      if constexpr (BITS == 4) {  // the sums of a group's channels: products with rows of ones, 2^-9 as 8-bit floats, 1 / 8 as 6-bit ones
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          Acc acc = T::zero();
#pragma unroll
          for (int pr = 0; pr < NP; ++pr) {
            if (NG == 2 && NP == 2 && pr != g) continue;
            auto add = [&](auto ones) {
              const uint32_t scale = unit_exp[NU == 2 ? g : 0];
              acc = T::template codes<0>(ones, digits[pr][0], scale, acc);
              acc = T::template codes<1>(ones, digits[pr][1], scale, acc);
              if constexpr (!EIGHT) {
                acc = T::template codes<2>(ones, digits[pr][2], scale, acc);
                acc = T::template codes<3>(ones, digits[pr][kDigits - 1], scale, acc);
              }
            };
            constexpr uint32_t kOne = 0x01010101u;
            if constexpr (MANY) add((u32x6){0x41041041u, 0x10410410u, 0x04104104u, 0x41041041u, 0x10410410u, 0x04104104u});
            else add((u32x8){kOne, kOne, kOne, kOne, kOne, kOne, kOne, kOne});
          }
          sum[g] = EIGHT ? acc[0] + other_eight(acc[0]) : acc[0];
        }
      } else {
        sum[0] = T::column_sum(NG == 2 ? sum[0] * u : sum[0] * u + sum[1] * u);
        if constexpr (NG == 2) sum[1] = T::column_sum(sum[1] * u);
      }
      // (EIGHT: in the first column, whose products the second one's are added to)
      const bool none = EIGHT && col >= 8;
      start[0] = start_slots(none ? 0.0f : g_lane == 0 ? sum[0] : g_lane == 1 && !EIGHT ? apart() : 0.0f, none ? 0u : g_lane == 0 ? 0x3F803F80u : g_lane == 1 ? 0x00003F80u : 0u);
      if constexpr (NG == 2) start[1] = start_slots(none || g_lane != 0 ? 0.0f : sum[1], 0u);
    }
    // scores of a block; codes(product): the row operand (W = 16: of the half that is being formed)
    auto scores = [&](const auto &bm, float (&y)[NY], auto &&codes) {
#pragma unroll
      for (int half = 0; half < (kWide ? 1 : 2); ++half) {
        const int row = kWide ? lane & 31 : 16 * half + n;  // of the row operands
        u32x4 first[NG];  // (lane groups without a slot to fill meet zeros in the column operand)
        first[0] = *reinterpret_cast<const u32x4 *>(&bm.start[row][g_lane & 1][0]);
        if constexpr (NG == 2) first[1] = *reinterpret_cast<const u32x4 *>(&bm.start2[row][0]);
        Acc acc[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) acc[g] = T::bf16(first[g], start[g], T::zero());
#pragma unroll
        for (int pr = 0; pr < (kWide ? 2 : NG); ++pr) {
          const int g = NG == 2 ? pr : 0, of = kWide ? pr : 0;
          const auto rows = codes(pr, half);
          const uint32_t scale = unit_exp[NU == 2 ? pr : 0];
          acc[g] = T::template codes<0>(rows, digits[of][0], scale, acc[g]);
          acc[g] = T::template codes<1>(rows, digits[of][1], scale, acc[g]);
          if constexpr (!EIGHT) {
            acc[g] = T::template codes<2>(rows, digits[of][2], scale, acc[g]);
            if constexpr (kDigits == 4) acc[g] = T::template codes<kDigits - 1>(rows, digits[of][kDigits - 1], scale, acc[g]);
          }
        }
        if constexpr (EIGHT) {
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[g][i] += other_eight(acc[g][i]);
        }
#pragma unroll
        for (int x = 0; x < (kWide ? 4 : 1); ++x) {
          const int at = kWide ? x : half;
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const f32x4 scale = *reinterpret_cast<const f32x4 *>(&bm.k_scale[g][T::row(at, g_lane)]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              y[4 * at + i] = g == 0 ? EIGHT ? __builtin_fmaf(scale[i], acc[0][4 * x + i], apart()) : scale[i] * acc[0][4 * x + i]
                                     : __builtin_fmaf(scale[i], acc[g][4 * x + i], y[4 * at + i]);
          }
        }
      }
    };
    auto raise_codes = [&](auto &...y) {
      raise([&](float alpha) {
#pragma unroll
        for (int g = 0; g < NG; ++g) acc_z[g] *= alpha;
        if (g_lane == 1 && !(EIGHT && col >= 8)) start[0] = start_slots(EIGHT ? -m : apart() - m, 0x00003F80u);
      }, y...);
    };
    // weights of a block's scores, and their sum
    auto weights = [&](const auto &bm, float (&y)[NY]) {
#pragma unroll
      for (int i = 0; i < NY; ++i) y[i] = exp2_bare(y[i]);
      float l2 = 0.0f;
#pragma unroll
      for (int x = 0; x < NA; ++x) {
        const f32x4 r = *reinterpret_cast<const f32x4 *>(&bm.v_rcp[T::row(x, g_lane)]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (x & 1) l2 = __builtin_fmaf(y[4 * x + i], r[i], l2);
          else l = __builtin_fmaf(y[4 * x + i], r[i], l);
        }
      }
      l += l2;
    };
    // values that stay in their words
    [[maybe_unused]] auto values = [&](const Words &v, const BlockMeta<NG> &bm, bool far, float (&y)[NY]) {
      u32x4 w[NG][NS];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int st = 0; st < NS; ++st) {
          const int lo = 4 * st, hi = 4 * st + NY / 2;
          if constexpr (NG == 2) {
            const f32x4 s0 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][T::row(lo / 4, g_lane)]), s1 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][T::row(hi / 4, g_lane)]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[g][st][i] = pack_f16x2(y[lo + i] * s0[i], y[hi + i] * s1[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[g][st][i] = pack_f16x2(y[lo + i], y[hi + i]);
          }
        }
      // ---- zero-points: sums with the rounded weights
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x == 0 || __builtin_expect(far, 0))
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int st = 0; st < NS; ++st) {
              const u32x4 z = *reinterpret_cast<const u32x4 *>(&bm.v_zero[x][g][8 * (2 * st + g_lane)]);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t wi = w[g][st][i], zi = z[i];  // (values of their own: a cast of a vector's element takes its first one)
                acc_z[g] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, wi), __builtin_bit_cast(f16x2, zi), acc_z[g], false);
              }
            }
      // ---- values: word nb / 2 of a chunk in half nb % 2, one channel block a word
      if constexpr (BITS == 4) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int wd = 0; wd < 4; ++wd) {
            const int g = NG == 2 ? wd >> 1 : 0, st = kWide ? x : 0, j = kWide ? wd : 2 * wd + x;
            const uint32_t lo = v.w[x][wd], hi = lo >> 8;
            o[j] = T::f16((u32x4){lo & 0x000F000Fu, lo & 0x00F000F0u, hi & 0x000F000Fu, hi & 0x00F000F0u}, w[g][st], o[j]);
          }
        return;
      }
      // ---- values: word (nb % 2, nb / 4) of a chunk, fields (nb / 2) % 2 a byte apart
#pragma unroll
      for (int wd = 0; wd < 4; ++wd) {
        const int g = NG == 2 ? (wd & 1) : 0, st = kWide ? wd >> 1 : 0;
        const int j = kWide ? 2 * (wd & 1) : 4 * (wd & 1) + (wd >> 1), j2 = kWide ? j + 1 : j + 2;
        const uint32_t x = v.w[0][wd], x8 = x >> 8;
        const u32x4 vx = {x & 0x00030003u, x & 0x000C000Cu, x & 0x00300030u, x & 0x00C000C0u};
        const u32x4 vy = {x8 & 0x00030003u, x8 & 0x000C000Cu, x8 & 0x00300030u, x8 & 0x00C000C0u};
        o[j] = T::f16(vx, w[g][st], o[j]);
        o[j2] = T::f16(vy, w[g][st], o[j2]);
      }
    };
    if constexpr (MANY) {
      // The wavefronts expand the next four blocks for all, two for each block: the first its meta words and a half of its values, the
      // second its keys and the other half.  What they need is asked for while the blocks before are worked on, and the pages'
      // numbers (lane l: of block from + l) a round earlier.
      const int mine = wave >> 1, part = wave & 1, h = g_lane;
      constexpr bool kGroupWeights = BITS == 4 && NG == 2;
      MetaWords<NG> words;
      u32x4 v_meta[2][NG];
      u32x4 k;  // (4 bits: of the first and the second chunk, two words of this wavefront's product)
      typename std::conditional<BITS == 2, u32x2, u32x4>::type v;
      int limit = 0;
      auto ask = [&](int from, int pages) {
        const Where at = find(min(from + mine, n_code - 1), __builtin_amdgcn_readlane(pages, mine));
        const uint32_t *meta = c.v_meta + (at.row + 4 * (2 * part + h)) * NG;  // of rows 4g + i and 16 + 4g + i, g = 2 part + h
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int y = 0; y < NG; ++y) v_meta[x][y] = *reinterpret_cast<const u32x4 *>(meta + 16 * NG * x + 4 * y);
        v = *reinterpret_cast<const decltype(v) *>(c.v_codes + at.row * (4 * BITS) + (16 * (2 * part + h) + n) * 4 + (BITS == 2 ? 2 : 256) * p);
        words = load_meta<NG>((part == 0 && lane < 32 ? c.k_meta : c.v_meta) + (at.row + (lane & 31)) * NG);
        if constexpr (BITS == 4) {
          const uint32_t *blk = c.k_codes + at.row * 16 + 256 * p + (16 * h + n) * 4 + 2 * part;
          const u32x2 x = *reinterpret_cast<const u32x2 *>(blk), y = *reinterpret_cast<const u32x2 *>(blk + 128);
          k = (u32x4){x[0], x[1], y[0], y[1]};
        } else if (part == 1) {
          k = load_codes(c.k_codes, at).w[0];
        }
        limit = at.limit;
      };
      auto expand = [&](int blk, CodeBlock<NG, BITS> &to, uint8_t &far_zero) {
        if constexpr (BITS == 4) {  // keys: a product's a wavefront
          // a nibble is a binary16 subnormal, code * 2^-24: as a 6-bit float of the scale 2^-21 it is code / 8, its bits as they were
          typedef __attribute__((ext_vector_type(16))) unsigned int u32x16;
          u32x16 x;
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = (k[i >> 2] >> (4 * (i & 3))) & 0x000F000Fu;
          const f16x32 codes32 = __builtin_bit_cast(f16x32, x);
          const u32x6 made = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_pk32_fp6_f16(codes32, 4.76837158203125e-07f));
          asm volatile("" ::"v"(codes32), "v"(made) : "memory");  // (as in make_digit)
          to.k[part][lane] = (u32x4){made[0], made[1], made[2], made[3]};
          to.k_more[part][lane] = (u32x2){made[4], made[5]};
        }
        if (part == 0) {
          const int r = lane & 31;  // lanes 0-31: keys, lanes 32-63: values
          const RowMeta<NG> row(words, blk * 32 + r < limit, lane >= 32);
          const float v_log = halves(NG == 2 ? power_log(row.top) + (kGroupWeights ? 1.0f : 0.0f) : log2_bare(row.top)).hi;
          if (lane < 32) {
            decode_key(row, v_log, to, r);
          } else {
            const float rcp = power_rcp(row.top) * (kGroupWeights ? 0.5f : 1.0f);
            to.v_rcp[r] = NG == 2 && row.part ? rcp : row.rcp;
            if constexpr (kGroupWeights)
#pragma unroll
              for (int g = 0; g < NG; ++g) to.v_share[g][r] = row.scale[g] * rcp;
          }
        } else {
          if constexpr (BITS == 2) {
            const u32x2 k0 = ex4(k[0]), k1 = ex4(k[1]), k2 = ex4(k[2]), k3 = ex4(k[3]);
            to.k[0][lane] = (u32x4){k0[0], k0[1], k2[0], k2[1]};
            to.k[1][lane] = (u32x4){k1[0], k1[1], k3[0], k3[1]};
          }
          int high[NG], any = 0;
#pragma unroll
          for (int g = 0; g < NG; ++g) any |= high[g] = zero_high(words.w[g]);
          const bool far = __ballot(any != 0) != 0ull;
          if (lane == 0) far_zero = far;
          if (__builtin_expect(far, 0)) {  // (two lanes a row)
            const int r = lane & 31;
            const RowMeta<NG> row(words, blk * 32 + r < limit, true);
            const int at = weight_place(r);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              const float z = -(float)high[g] * (NG == 2 && !kGroupWeights ? row.scale[g] * power_rcp(row.top) : 1.0f);
              const uint32_t a = float_to_half_bits_rne(z);
              to.v_far[0][g][at] = (uint16_t)a;
              if constexpr (NG == 2 && !kGroupWeights) to.v_far[1][g][at] = (uint16_t)float_to_half_bits_rne(z - half_bits_to_float(a));
            }
          }
        }
        // values: 1536 + code in place, less 1536 + the low part of the zero-point: exact (the rest of a far one is summed apart).  Two scales over the
        // larger one's power of two have their own bits in binary16, where they are above 2^-14.  Values of 2-bit codes are multiplied by them,
        // rounded once, 2^-11, and one set of weights serves both groups; 4-bit codes stay exact, and each group has weights of its own: error of the
        // output 2.9e-4 against 3.4e-4 of its norm, 4 x 2048 rows of 32 heads over 8192 cached ones 1.63 ms against 1.53.
        u32x4 less[NG];
        [[maybe_unused]] u32x4 share[NG];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          [[maybe_unused]] float sc[2][NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            uint32_t w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              w[x] = v_meta[x][NG == 2 ? i / 2 : 0][NG == 2 ? 2 * (i & 1) + g : i];
              sc[x][g] = half_bits_to_float(w[x] & 0x7FFFu);
            }
            less[g][i] = less_zero_low(w[0], w[1]);
          }
          if constexpr (NG == 2 && !kGroupWeights) {
            float inv[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) inv[x] = power_rcp(fmaxf(sc[x][0], sc[x][1]));
#pragma unroll
            for (int g = 0; g < 2; ++g) share[g][i] = pack_f16x2(sc[0][g] * inv[0], sc[1][g] * inv[1]);
          }
        }
        // rows that take no part may hold anything, and 0 * NaN is no 0
        u32x4 keep = {~0u, ~0u, ~0u, ~0u};
        const int row = blk * 32 + 4 * (2 * part + h);
        if (blk * 32 + 32 > limit)  // uniform
#pragma unroll
          for (int i = 0; i < 4; ++i) keep[i] = (row + i < limit ? 0xFFFFu : 0u) | (row + 16 + i < limit ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int wd = 0; wd < 2; ++wd)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int g = NG == 2 ? wd : 0;
            u32x4 o4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t word = BITS == 2 ? v[wd] >> (8 * x + 2 * i) : v[2 * wd + x] >> (4 * i), zi = less[g][i];
              const uint32_t code = (word & (BITS == 2 ? 0x00030003u : 0x000F000Fu)) | 0x66006600u;
              f16x2 val = __builtin_bit_cast(f16x2, code) + __builtin_bit_cast(f16x2, zi);
              if constexpr (NG == 2 && !kGroupWeights) {
                const uint32_t si = share[g][i];
                val *= __builtin_bit_cast(f16x2, si);
              }
              o4[i] = __builtin_bit_cast(uint32_t, val) & keep[i];
            }
            to.v[part][2 * wd + x][lane] = o4;
          }
      };
      auto block_scores = [&](const CodeBlock<NG, BITS> &bm, float (&y)[NY]) {
        scores(bm, y, [&](int pr, int) {
          if constexpr (BITS == 4) {
            const u32x4 a = bm.k[pr][lane];
            const u32x2 b = bm.k_more[pr][lane];
            return (u32x6){a[0], a[1], a[2], a[3], b[0], b[1]};
          } else {
            return bm.k[pr][lane];
          }
        });
      };
      auto block_values = [&](const CodeBlock<NG, BITS> &bm, bool far, float (&y)[NY]) {
        weights(bm, y);
        constexpr int NW = kGroupWeights ? NG : 1;
        u32x4 w[NW][NS];
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int g = 0; g < NW; ++g) {
            if constexpr (kGroupWeights) {
              const f32x4 s0 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][T::row(st, g_lane)]), s1 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][T::row(st + NA / 2, g_lane)]);
#pragma unroll
              for (int i = 0; i < 4; ++i) w[g][st][i] = scaled_f16x2(y[4 * st + i], y[4 * st + NY / 2 + i], s0[i], s1[i]);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) w[g][st][i] = pack_f16x2(y[4 * st + i], y[4 * st + NY / 2 + i]);
            }
#pragma unroll
            for (int j = g * NB / NW; j < (g + 1) * NB / NW; ++j) o[j] = T::f16(bm.v[st][j][lane], w[g][st], o[j]);
          }
        if (__builtin_expect(far, 0)) {  // rows far from zero: the same for all of a group's channels
#pragma unroll
          for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
              for (int x = 0; x < (kGroupWeights ? 1 : NG); ++x) {
                const u32x4 z = *reinterpret_cast<const u32x4 *>(&bm.v_far[x][g][8 * (2 * st + g_lane)]);
#pragma unroll
                for (int j = g * NB / NG; j < (g + 1) * NB / NG; ++j) o[j] = T::f16(z, w[kGroupWeights ? g : 0][st], o[j]);
              }
        }
      };
      auto ask_pages = [&](int from) { return table[page_of(min(from + lane, n_code - 1))]; };
      int of_blocks = ask_pages(first);
      ask(first, of_blocks);
      of_blocks = ask_pages(first + kStageBlocks);
      for (int from = first, turn = 0; from < code_end; from += kStageBlocks, turn ^= 1) {
        expand(min(from + mine, n_code - 1), sh.blocks[turn][mine], sh.far[turn][mine]);
        ask(from + kStageBlocks, of_blocks);
        of_blocks = ask_pages(from + 2 * kStageBlocks);
        lds_barrier();  // (the other set was last read in front of the barrier before)
        if (idle) continue;
        const int last = min(kStageBlocks, code_end - from);
        const uint32_t far = __builtin_amdgcn_readfirstlane(*reinterpret_cast<const uint32_t *>(&sh.far[turn][0]));  // (a byte a block)
        for (int x = 0; x < last; ++x) {
          const CodeBlock<NG, BITS> &bm = sh.blocks[turn][x];
          float y[NY];
          block_scores(bm, y);
          raise_codes(y);
          block_values(bm, ((far >> (8 * x)) & 1u) != 0u, y);
        }
      }
      lds_barrier();  // the stages of 16-bit rows lie where the blocks were
    } else {
      auto &bms = sh.own[wave].meta;
      auto codes_of = [&](int x) {
        return [&, x](int pr, int half) {
          if constexpr (BITS == 4 && kWide) {
            const u32x2 a = nibbles(few_k[x].w[0][2 * pr]), b = nibbles(few_k[x].w[0][2 * pr + 1]), c = nibbles(few_k[x].w[1][2 * pr]), d = nibbles(few_k[x].w[1][2 * pr + 1]);
            return (u32x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
          } else if constexpr (BITS == 4) {
            const u32x4 w = few_k[x].w[half];
            const u32x2 a = nibbles(w[0]), b = nibbles(w[1]), c = nibbles(w[2]), d = nibbles(w[3]);
            return (u32x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
          } else if constexpr (kWide) {
            const u32x2 lo = ex4(few_k[x].w[0][pr]), hi = ex4(few_k[x].w[0][2 + pr]);
            return (u32x4){lo[0], lo[1], hi[0], hi[1]};
          } else {  // a group's product takes zeros in the other's slots
            const u32x2 lo = ex4(few_k[x].w[0][2 * half]), hi = ex4(few_k[x].w[0][2 * half + 1]), none = {0u, 0u};
            const u32x2 a0 = NG == 2 && pr == 1 ? none : lo, a1 = NG == 2 && pr == 0 ? none : hi;
            return (u32x4){a0[0], a0[1], a1[0], a1[1]};
          }
        };
      };
      bool far = false;
      if (first < code_end) far = decode_pair<NG, BITS>(few_kw, few_vw, row_there(first, now), bms[0], lane);
      if (!EIGHT || first + 2 < code_end) ask_meta(next);
      wave_lds_sync();
      for (int blk = first, turn = 0; blk < code_end; blk += 2, turn ^= 1) {
        bool next_far = false;
        Pair after = next;
        // (up to eight rows: nothing is asked or waited for that is not used)
        const bool more = !EIGHT || blk + 2 < code_end;
        if (more) {
          next_far = decode_pair<NG, BITS>(few_kw, few_vw, row_there(blk + 2, next), bms[turn ^ 1], lane);
          after = locate(blk + 4);
          if (!EIGHT || blk + 4 < code_end) ask_meta(after);
        }
        // (EIGHT with two groups: one after the other, and codes asked for that may not be used, so that three workgroups run on a CU: one row over
        // 32768 rows of 128 units 108-112 us, both at once and two workgroups 117-120; a call of one pair of blocks each 10.5 against 10.4)
        const BlockMeta<NG> (&bm)[2] = bms[turn];
        if constexpr (kWide || (EIGHT && NG == 2)) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x == 1 && blk + 1 >= code_end) break;
            float y[NY];
            scores(bm[x], y, codes_of(x));
            few_k[x] = load_codes(c.k_codes, next.at[x]);
            raise_codes(y);
            weights(bm[x], y);
            values(few_v[kOneValue ? 0 : x], bm[x], far, y);
            if constexpr (kOneValue) few_v[0] = load_codes(c.v_codes, x == 0 ? now.at[1] : next.at[0]);
            else few_v[x] = load_codes(c.v_codes, next.at[x]);
          }
        } else {  // both at once: what one waits for the other covers
          float y0[NY], y1[NY];
          scores(bm[0], y0, codes_of(0));
          scores(bm[1], y1, codes_of(1));
          if (more)
#pragma unroll
            for (int x = 0; x < 2; ++x) few_k[x] = load_codes(c.k_codes, next.at[x]);
          raise_codes(y0, y1);
          weights(bm[0], y0);
          weights(bm[1], y1);
          values(few_v[0], bm[0], far, y0);
          values(few_v[1], bm[1], far, y1);
          if (more)
#pragma unroll
            for (int x = 0; x < 2; ++x) few_v[x] = load_codes(c.v_codes, next.at[x]);
        }
        if constexpr (kOneValue) now = next;
        next = after;
        far = next_far;
        wave_lds_sync();
      }
    }
    // codes were 2^-24 of themselves, zero-points 2^-6; a group's zero-points reach all of its channels
    if constexpr (!MANY) {
#pragma unroll
      for (int g = 0; g < NG; ++g) acc_z[g] = -64.0f * T::column_sum(acc_z[g]);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float z = acc_z[NG == 2 ? j / (NB / 2) : 0];
#pragma unroll
        for (int i = 0; i < (kWide ? 16 : 4); ++i) o[j][i] = __builtin_fmaf(o[j][i], 16777216.0f, z);
      }
    }
  }

  // Sixteen-bit keys and values of a workgroup of many rows go through LDS, a stage at a time: every thread brings two chunks of keys
  // and of values, asked for while the stage before is worked on.  from(key?, stage, row, chunk): where a chunk comes from;
  // at_v(row, chunk): where values go.
  [[maybe_unused]] auto staged = [&](int begin, int end, auto &&from, auto &&at_v, auto &&work) {  // stages [begin, end), uniform over the workgroup
    if constexpr (MANY) {
      if (begin >= end) return;
      u32x4 kx[2], vx[2];
      auto ask = [&](int stage) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int id = threadIdx.x + 512 * x, row = id >> 4, chunk = id & 15;
          kx[x] = *reinterpret_cast<const u32x4 *>(from(true, stage, row, chunk));
          vx[x] = *reinterpret_cast<const u32x4 *>(from(false, stage, row, chunk));
        }
      };
      ask(begin);
      for (int stage = begin; stage < end; ++stage) {
        const int buf = stage & 1;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int id = threadIdx.x + 512 * x, row = id >> 4, chunk = id & 15;
          *reinterpret_cast<u32x4 *>(&sh.k[buf][staged_at(row, chunk)]) = kx[x];
          *reinterpret_cast<u32x4 *>(&sh.v[buf][at_v(row, chunk)]) = vx[x];
        }
        if (stage + 1 < end) ask(stage + 1);
        lds_barrier();  // (the other buffer was last read in front of the barrier before)
        work(stage, buf);
      }
      lds_barrier();  // whoever comes next overwrites the stages
    }
  };
  // Scores of a block of 16-bit keys: key(half, k): the row operand of chunk k (W = 32: of all 32 rows, else of a half), q: column operands
  auto score16 = [&](float (&y)[NY], auto &&key, auto &&add) {
#pragma unroll
    for (int half = 0; half < (kWide ? 1 : 2); ++half) {
      Acc acc = T::zero();
#pragma unroll
      for (int k = 0; k < NC; ++k) acc = add(key(half, k), k, acc);
#pragma unroll
      for (int i = 0; i < (kWide ? 16 : 4); ++i) y[4 * half + i] = acc[i];
    }
  };
  auto row_of = [&](int i) { return T::row(i >> 2, g_lane) + (i & 3); };  // of y[i], in its block

  // ================= 16-bit rows of the cache =================
  if (wide_begin < wide_end) {
    const uint16_t *ks = c.k_sal + (size_t)unit * c.S_cap * kD, *vs = c.v_sal + (size_t)unit * c.S_cap * kD;
    auto key_at = [&](int blk, int half, int k) { return reinterpret_cast<const u32x4 *>(ks + (size_t)(blk * 32 + 16 * half + col) * kD + kD / NC * k + 8 * g_lane); };
    auto value_at = [&](int blk, int nb, int g) { return reinterpret_cast<const u32x4 *>(vs + (size_t)blk * 4096 + nb * 512 + 8 * (16 * g + n)); };
    {
      u32x4 raw[NC];
      float x[8 * NC];
      load_query(raw);
      rotated(raw, x);
      split_query(x);
    }
    // one block of 32 slots; value(nb, g): the 16 bytes of the tile for channels 16nb + n, rows 4g + i and 16 + 4g + i
    auto wide_block = [&](int blk, auto &&key, auto &&value) {
      float y[NY];
      score16(y, key, [&](u32x4 k, int at, Acc acc) { return T::bf16(k, q_hi[at], T::bf16(k, q_lo[at], acc)); });
#pragma unroll
      for (int i = 0; i < NY; ++i) y[i] = blk * 32 + row_of(i) < wide ? y[i] + (apart() - m) : kNoScore;
      weigh(y);
#pragma unroll
      for (int i = 0; i < NY; ++i) l += y[i];
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y0 = y[4 * st + i], y1 = y[4 * st + NY / 2 + i];
          hi[i] = pack_bf16x2(y0, y1);
          lo[i] = pack_bf16x2(y0 - __uint_as_float(hi[i] << 16), y1 - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
        const int g = 2 * st + g_lane;
        u32x4 keep = {~0u, ~0u, ~0u, ~0u};
        if (blk * 32 + 32 > wide)  // slots behind the last row may hold anything, and 0 * NaN is no 0
#pragma unroll
          for (int i = 0; i < 4; ++i)
            keep[i] = (blk * 32 + 4 * g + i < wide ? 0xFFFFu : 0u) | (blk * 32 + 16 + 4 * g + i < wide ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const u32x4 v = value(kWide ? 2 * j + p : j, g) & keep;
          o[j] = T::bf16(v, hi, T::bf16(v, lo, o[j]));
        }
      }
    };
    if constexpr (MANY) {
      staged(wide_begin / 2, (wide_end + 1) / 2,
             [&](bool key, int stage, int row, int chunk) { return (key ? ks : vs) + (size_t)stage * (kStage * kD) + row * kD + 8 * chunk; },
             [](int row, int chunk) { return row * kD + 8 * chunk; },  // (tiles: a wavefront reads 1 KB pieces as they lie)
             [&](int stage, int buf) {
               if (idle) return;
#pragma unroll
               for (int x = 0; x < 2; ++x)
                 if (2 * stage + x >= wide_begin && 2 * stage + x < wide_end)
                   wide_block(2 * stage + x,
                              [&](int half, int k) {
                                return *reinterpret_cast<const u32x4 *>(&sh.k[buf][staged_at(32 * x + 16 * half + col, 16 / NC * k + g_lane)]);
                              },
                              [&](int nb, int g) { return *reinterpret_cast<const u32x4 *>(&sh.v[buf][x * 4096 + nb * 512 + 8 * (16 * g + n)]); });
             });
    } else {
      for (int blk = wide_begin; blk < wide_end; ++blk)
        wide_block(blk, [&](int half, int k) { return *key_at(blk, half, k); }, [&](int nb, int g) { return *value_at(blk, nb, g); });
    }
  }
  // The cached rows' share is rotated back (H is its own inverse), and the chunk's rows join it.  Their weights are relative to the
  // sum so far: the reference of the code rows holds V scales as well.
  if (!kMergeFirst && !idle && (code_begin < code_end || wide_begin < wide_end)) {
    constexpr int NO = kWide ? 16 : 4;
    if (!a.out_rotated) {
      float x[NB * NO];
#pragma unroll
      for (int e = 0; e < NB * NO; ++e) x[e] = o[e / NO][e % NO];
      wht128_output<W>(x, lane);
#pragma unroll
      for (int e = 0; e < NB * NO; ++e) o[e / NO][e % NO] = x[e] * inv_sqrt128();
    }
    const float all = T::column_sum(l);
    if (all > 0.0f) {
      const float to = rintf(m + log2_bare(all)) - kRaiseTo, alpha = exp2_bare(m - to);
#pragma unroll
      for (int j = 0; j < NB; ++j) o[j] *= alpha;
      l *= alpha;
      m = to;
      limit = kRaiseAt;
    }
  }

  // (of a tile of 16) the sum of a row's two columns
  [[maybe_unused]] auto both = [&](float x) { return x + other_eight(x); };
  [[maybe_unused]] auto join_columns = [&](float &sum) {
    if (!twice) return;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = both(o[j][i]);
    sum = both(sum);
  };
  if constexpr (kMergeFirst) {
    float sum = T::column_sum(l);
    join_columns(sum);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      *reinterpret_cast<f32x4 *>(&sh.own[wk].o[col][T::channel(j, 0, g_lane)]) = (f32x4){o[j][0], o[j][1], o[j][2], o[j][3]};
      o[j] = T::zero();
    }
    if (g_lane == 0) {
      sh.m[wk][col] = limit < 0.0f ? kNoScore : m;
      sh.l[wk][col] = sum;
    }
    m = 0.0f;
    limit = 0.5f * kNoScore;
    l = 0.0f;
  }

  // ================= rows of the chunk =================
  if (self_begin < self_end) {
    const int low_token = row0 / R;                                        // of this wavefront's rows
    const int my_end = idle ? 0 : (min(row0 + W, rows) - 1) / R / 32 + 1;
    const uint16_t *ks = a.k + s.first * a.k_stride + head * kD, *vs = a.v + s.first * a.v_stride + head * kD;
    u32x4 raw[NC];
    load_query(raw);
    // one block of 32 rows; vt, vrow: where the block's values lie in LDS
    auto self_block = [&](int blk, auto &&key, const uint16_t *vt, int vrow) {
      float y[NY];
      score16(y, key, [&](u32x4 k, int at, Acc acc) { return T::f16(k, raw[at], acc); });
#pragma unroll
      for (int i = 0; i < NY; ++i) y[i] = __builtin_fmaf(y[i], sm2, apart() - m);
      if (blk * 32 + 31 > low_token) {  // uniform over the wavefront: some row may not look at all of the block
#pragma unroll
        for (int i = 0; i < NY; ++i)
          if (blk * 32 + row_of(i) > my_token) y[i] = kNoScore;
      }
      weigh(y);
      float l2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NY; i += 2) {
        l += y[i];
        l2 += y[i + 1];
      }
      l += l2;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const int lo = 4 * st, hi = 4 * st + NY / 2;  // rows 4g + i and 16 + 4g + i, here one after the other
        const u32x4 w = {pack_f16x2(y[lo], y[lo + 1]), pack_f16x2(y[lo + 2], y[lo + 3]), pack_f16x2(y[hi], y[hi + 1]), pack_f16x2(y[hi + 2], y[hi + 3])};
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          u32x4 v;
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // a transposing read: the lane gets its channel of rows 16 half + 4g .. + 3
            const int row = vrow + 16 * half + 4 * (2 * st + g_lane) + (n >> 2), nb = kWide ? 2 * j + p : j;
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(&vt[staged_at(row, 2 * nb + ((n & 3) >> 1)) + 4 * (n & 1)])));
            v[2 * half] = x[0];
            v[2 * half + 1] = x[1];
          }
          o[j] = T::f16(v, w, o[j]);
        }
      }
    };
    if constexpr (MANY) {
      staged(self_begin / 2, (self_end + 1) / 2,
             [&](bool key, int stage, int row, int chunk) {
               const int r = min(stage * kStage + row, s.rows - 1);
               return (key ? ks + r * a.k_stride : vs + r * a.v_stride) + 8 * chunk;
             },
             staged_at,
             [&](int stage, int buf) {
#pragma unroll
               for (int x = 0; x < 2; ++x) {
                 const int blk = 2 * stage + x;
                 if (blk >= self_begin && blk < min(self_end, my_end))
                   self_block(blk,
                              [&](int half, int k) {
                                return *reinterpret_cast<const u32x4 *>(&sh.k[buf][staged_at(32 * x + 16 * half + col, 16 / NC * k + g_lane)]);
                              },
                              sh.v[buf], 32 * x);
               }
             });
    } else {
      uint16_t *vt = sh.v[W == 16 ? 0 : wave];
      for (int blk = self_begin; blk < min(self_end, my_end); ++blk) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int row = 4 * x + (lane >> 4);
          *reinterpret_cast<u32x4 *>(&vt[staged_at(row, n)]) = *reinterpret_cast<const u32x4 *>(vs + min(blk * 32 + row, s.rows - 1) * a.v_stride + 8 * n);
        }
        wave_lds_sync();
        self_block(blk, [&](int half, int k) {
          return *reinterpret_cast<const u32x4 *>(ks + min(blk * 32 + 16 * half + col, s.rows - 1) * a.k_stride + kD / NC * k + 8 * g_lane);
        }, vt, 0);
        wave_lds_sync();
      }
    }
  }

  // ================= sums of the wavefronts, and out =================
  l = T::column_sum(l);
  if (limit < 0.0f) m = kNoScore;
  auto store = [&](int row, int ch, const f32x4 &x, float top, float sum) {  // four channels of a finished or partial row
    const int token = row / R, hq = head * R + row - token * R;
    const size_t at = (size_t)(s.first + token) * a.Hq + hq;
    if (a.n_split == 1) {
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      *reinterpret_cast<u32x2 *>(a.out + (s.first + token) * a.out_stride + hq * kD + ch) =
          (u32x2){pack_f16x2(x[0] * inv, x[1] * inv), pack_f16x2(x[2] * inv, x[3] * inv)};
      if (a.lse && ch == 0) a.lse[at] = sum > 0.0f ? (top + log2_bare(sum)) * kLn2 : -INFINITY;
    } else {
      float *to = a.partial + (at * a.n_split + split) * kPartialStride;
      *reinterpret_cast<f32x4 *>(to + 4 + ch) = x;
      if (ch == 0) { to[0] = top; to[1] = sum; }
    }
  };
  auto part_of = [&](int j, int x) { return (f32x4){o[j][4 * x], o[j][4 * x + 1], o[j][4 * x + 2], o[j][4 * x + 3]}; };
  if constexpr (MANY) {
    if (row0 + col < rows)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int x = 0; x < (kWide ? 4 : 1); ++x) store(row0 + col, T::channel(j, x, g_lane), part_of(j, x), m, l);
  } else if constexpr (kMergeFirst) {
    const bool with_self = group_begin <= self_at && run_start(split * WK + WK) > self_at;  // uniform: this workgroup has the chunk's block
    if (self_begin < self_end) {
      join_columns(l);
#pragma unroll
      for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4 *>(&sh.self[col][T::channel(j, 0, g_lane)]) = part_of(j, 0);
      if (g_lane == 0) { sh.m[WK][col] = m; sh.l[WK][col] = l; }
    }
    __syncthreads();
    // Sixteen lanes a row, eight channels each.  Lanes meet at distances of 1, 2, 7 and 15 (what the lane exchanges of a row reach), so
    // lane i takes chunk `place`, whose bits say how often each of them goes into i.
    const int r = threadIdx.x >> 4, i = threadIdx.x & 15;
    const int i1 = i ^ ((i & 8) ? 15 : 0), i2 = i1 ^ ((i1 & 4) ? 7 : 0), place = (i & 8) | (i1 & 4) | (i2 & 3), ch = 8 * place;
    float top = sh.m[0][r], sum = 0.0f, x[8];
    const float once = twice ? 1.0f / (1.0f + kApartFactor) : 1.0f;
#pragma unroll
    for (int w = 1; w < WK; ++w) top = fmaxf(top, sh.m[w][r]);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float f = exp2_bare(sh.m[w][r] - top) * once;
      sum += f * sh.l[w][r];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += f * sh.own[w].o[r][ch + e];
    }
    if (!a.out_rotated) {
      butterflies(x, 1);
      butterflies(x, 2);
      butterflies(x, 4);
      auto across = [&](auto exchange, int bit) {
        const float sign = (place & bit) ? -1.0f : 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int other = __builtin_amdgcn_update_dpp(0, __float_as_int(x[e]), decltype(exchange)::value, 0xF, 0xF, false);
          x[e] = __builtin_fmaf(sign, x[e], __int_as_float(other));
        }
      };
      across(Dpp<0xB1>(), 1);   // quad_perm [1,0,3,2]
      across(Dpp<0x4E>(), 2);   // quad_perm [2,3,0,1]
      across(Dpp<0x141>(), 4);  // row_half_mirror
      across(Dpp<0x140>(), 8);  // row_mirror
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= inv_sqrt128();
    }
    if (with_self) {
      const float self_m = sh.m[WK][r], all = fmaxf(top, self_m), f = exp2_bare(top - all), g = exp2_bare(self_m - all) * once;
      sum = f * sum + g * sh.l[WK][r];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = f * x[e] + g * sh.self[r][ch + e];
      top = all;
    }
    if (row0 + r < rows) {
      store(row0 + r, ch, (f32x4){x[0], x[1], x[2], x[3]}, top, sum);
      store(row0 + r, ch + 4, (f32x4){x[4], x[5], x[6], x[7]}, top, sum);
    }
  } else {
    __syncthreads();  // (the sums lie where other wavefronts may still read)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int x = 0; x < (kWide ? 4 : 1); ++x) *reinterpret_cast<f32x4 *>(&sh.o[wk][col][T::channel(j, x, g_lane)]) = part_of(j, x);
    if (g_lane == 0) { sh.m[wk][col] = m; sh.l[wk][col] = l; }
    __syncthreads();
    for (int at = threadIdx.x; at < W * 32; at += 64 * NW) {
      const int r = at >> 5, ch = 4 * (at & 31);
      if (row0 + r >= rows) break;
      float top = sh.m[0][r], sum = 0.0f;
#pragma unroll
      for (int x = 1; x < WK; ++x) top = fmaxf(top, sh.m[x][r]);
      f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < WK; ++x) {
        const float f = exp2_bare(sh.m[x][r] - top);
        sum += f * sh.l[x][r];
        all += f * *reinterpret_cast<const f32x4 *>(&sh.o[x][r][ch]);
      }
      store(row0 + r, ch, all, top, sum);
    }
  }
}

// Merges the splits of a row: one wavefront a row, four channels a lane, the halves of the lanes take every other split.  Sixteen splits are in
// flight at a time: one round trip to memory is all that most calls wait for.
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedAttentionArgs a) {
  const PagedArgs &c = a.c;
  const int lane = threadIdx.x & 63, half = lane >> 5, unit = blockIdx.y, b = unit / c.Hkv, head = unit % c.Hkv, R = a.Hq / c.Hkv;
  const int row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ChunkSpan s = chunk_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (row >= s.rows * R) return;
  const int token = row / R, hq = head * R + row - token * R, ch = 4 * (lane & 31);
  const size_t at = (size_t)(s.first + token) * a.Hq + hq;
  const float *p = a.partial + at * a.n_split * kPartialStride;
  float top = kNoScore, sum = 0.0f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int from = 0; from < a.n_split; from += 16) {
    float m[8], l[8];
    f32x4 part[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool there = from + 2 * i + half < a.n_split;
      const float *r = p + (there ? from + 2 * i + half : from) * kPartialStride;
      m[i] = there ? r[0] : kNoScore;
      l[i] = there ? r[1] : 0.0f;
      part[i] = *reinterpret_cast<const f32x4 *>(r + 4 + ch);
    }
    float all = top;
#pragma unroll
    for (int i = 0; i < 8; ++i) all = fmaxf(all, m[i]);
    all = halves_max(all);
    const float alpha = exp2_bare(top - all);
    top = all;
    sum *= alpha;
    x *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = from + 2 * i + half < a.n_split ? exp2_bare(m[i] - all) : 0.0f;
      sum = __builtin_fmaf(f, l[i], sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(f, part[i][e], x[e]);
    }
  }
  sum = halves_sum(sum);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = halves_sum(x[e]);
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  if (half == 0)
    *reinterpret_cast<u32x2 *>(a.out + (s.first + token) * a.out_stride + hq * kD + ch) = (u32x2){pack_f16x2(x[0] * inv, x[1] * inv), pack_f16x2(x[2] * inv, x[3] * inv)};
  if (a.lse && lane == 0) a.lse[at] = sum > 0.0f ? (top + log2_bare(sum)) * kLn2 : -INFINITY;
}

template <int G, int BITS>
void launch_variant(const PagedAttentionArgs &a, int rows, hipStream_t stream) {
  const int units = a.c.B * a.c.Hkv;
  auto grid = [&](int per) { return dim3(units, (rows + per - 1) / per, a.n_split); };
  constexpr int kFew = 64 * kFewWaves, kMany = 64 * kManyWaves;
  static_assert(kPagedManyRows == 32 * kManyWaves);
  const long per = paged_tile_rows(units, a.c.max_rows, a.Hq / a.c.Hkv, a.c.max_len, {BITS, G});
  if (BITS == 4 && per == 16 && rows <= 8) paged_attention_kernel<G, 16, false, BITS, BITS == 4><<<grid(16), kFew, 0, stream>>>(a);
  else if (per == 16) paged_attention_kernel<G, 16, false, BITS><<<grid(16), kFew, 0, stream>>>(a);
  else if (per == 32) paged_attention_kernel<G, 32, false, BITS><<<grid(32), kFew, 0, stream>>>(a);
  else paged_attention_kernel<G, 32, true, BITS><<<grid(kPagedManyRows), kMany, 0, stream>>>(a);
}

template <int BITS>
hipError_t launch_attention(const PagedAttentionArgs &a, int G, hipStream_t stream) {
  const int rows = a.c.max_rows * (a.Hq / a.c.Hkv);
  if (G == 128) launch_variant<128, BITS>(a, rows, stream);
  else launch_variant<64, BITS>(a, rows, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  paged_combine_kernel<<<dim3((rows + 3) / 4, a.c.B * a.c.Hkv), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace akvq
