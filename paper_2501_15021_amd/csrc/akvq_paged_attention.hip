// Attention of a chunk of new rows over the cache in pages and over the chunk itself.
//
//   out_i = softmax_j(sm_scale * s_ij) v_j,  j over the sequence's cached rows and the chunk's rows up to i;
//   cached: s_ij = (H q_i) . khat_j, khat = scale * (code - zero) or a 16-bit row, and H (sum_j p_ij vhat_j) is the cached rows' share;
//   new:    s_ij = q_i . k_j, with k and v as they arrive (binary16).
//
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, in 16 x 16 tiles: a query is a column, i.e. a lane (and the three
// lanes 16, 32, 48 further), so the softmax needs no exchange between lanes but for a raised reference, and the weights leave the
// score product in the very registers in which the value product takes them (rows 4q + i of the two 16-row halves of a block; the
// packed V words and the 16-bit V tiles pair the rows that way).  Nothing goes through LDS but the meta words (decoded once per
// wavefront, a row a lane) and the chunk's V rows (transposed by the reads).
//   K codes enter the scaled 16x16x128 product as 4-bit floats without decoding (three instructions per 16 codes), against the query as
// kDigits balanced base-32 digits that 6-bit floats hold exactly: 5 * kDigits bits of the query's largest channel, at the price of
// kDigits / 4 of a 16-bit product.  What else a score holds comes from one more product, that the codes' products are added onto: per row
// zero-point, 1 / scale and log2(V scale) / scale, per column the query's sum, the reference and 1, all in bfloat16 terms that
// together hold the 32-bit numbers.  One multiplication by the row's scale is left.
//   V codes are masked in place, which leaves binary16 subnormals code * 4^ii * 2^-24 (ii: the row's place in its word): one
// instruction per two codes.  The V scale and 4^-ii ride in the exponent of the weight, the denominator takes the weight back by
// 4^ii / scale, and zero-points are summed by one more product.  What is left to the vector units is the softmax, which bounds the
// long chunks together with the products; a few rows are bound by the cache's stream.
//   Weights are binary16 (half a step is 2^-12 of a weight), relative to a reference that keeps the largest between 2^7 and 2^15: a
// weight below 2^-21 of its row's largest loses bits, one below 2^-31 all of them.  Scores, references, sums and accumulators are 32-bit.
#include "akvq_device.h"
#include "akvq_kernels.h"

namespace akvq {
namespace {

constexpr int kDigits = 4;  // 3 or 4
constexpr int kFewWaves = 4;   // of a workgroup that has few rows: they share them and deal the keys among them
constexpr int kManyWaves = 8;  // of a workgroup that has many: each has its own, and all look at the same keys
constexpr float kNoScore = -1.0e30f;   // score of a row that takes no part, reference of a column without scores
constexpr float kRaiseAt = 15.0f;      // a score may exceed the reference by this (2^15 is the largest weight) ...
constexpr float kRaiseTo = 7.0f;       // ... and then gets a reference this far below it
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef const __attribute__((address_space(3))) s16x4 *lds_s16x4;

__device__ __forceinline__ float exp2_bare(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_bare(float x) { return __builtin_amdgcn_logf(x); }
// over the four lanes that share a column
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
  uint32_t r;
  asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
// rows: codes as 4-bit floats; columns: query digits as 6-bit floats, times 2^(byte DIGIT of scale - 127)
template <int DIGIT>
__device__ __forceinline__ f32x4 mfma_codes(u32x4 codes, u32x6 digits, uint32_t scale, f32x4 c) {
  constexpr int kE2M3 = 2, kE2M1 = 4;
  const i32x8 a = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
  const i32x8 b = {(int)digits[0], (int)digits[1], (int)digits[2], (int)digits[3], (int)digits[4], (int)digits[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kE2M1, kE2M3, 0, 127, DIGIT, (int)scale);
}
__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_b16(u32x4 a, u32x4 b, f32x4 c) {
  return mfma_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
}

// A query row over the four lanes of its column: lane (n, q) holds channels 32m + 8q + i as x[8m + i].  Un-normalised transform.
__device__ __forceinline__ void wht128_column(float (&x)[32], int q) {
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    if (s >= 8) continue;
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if ((e & s) == 0) {
        const float a = x[e], b = x[e + s];
        x[e] = a + b;
        x[e + s] = a - b;
      }
  }
#pragma unroll
  for (int s = 1; s < 4; s *= 2)
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const float p = __shfl_xor(x[e], 16 * s, kWave);
      x[e] = (q & s) ? p - x[e] : x[e] + p;
    }
#pragma unroll
  for (int s = 8; s < 32; s *= 2)
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if ((e & s) == 0) {
        const float a = x[e], b = x[e + s];
        x[e] = a + b;
        x[e + s] = a - b;
      }
}
// An output column: lane (n, q) holds channels 16nb + 4q + i as o[nb][i].
__device__ __forceinline__ void wht128_output(f32x4 (&o)[8], int q) {
#pragma unroll
  for (int nb = 0; nb < 8; ++nb) {
    const float a = o[nb][0] + o[nb][1], b = o[nb][0] - o[nb][1], c = o[nb][2] + o[nb][3], d = o[nb][2] - o[nb][3];
    o[nb] = (f32x4){a + c, b + d, a - c, b - d};
  }
#pragma unroll
  for (int s = 1; s < 4; s *= 2)
#pragma unroll
    for (int nb = 0; nb < 8; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __shfl_xor(o[nb][i], 16 * s, kWave);
        o[nb][i] = (q & s) ? p - o[nb][i] : o[nb][i] + p;
      }
#pragma unroll
  for (int s = 1; s < 8; s *= 2)
#pragma unroll
    for (int nb = 0; nb < 8; ++nb)
      if ((nb & s) == 0) {
        const f32x4 a = o[nb], b = o[nb + s];
        o[nb] = a + b;
        o[nb + s] = a - b;
      }
#pragma unroll
  for (int nb = 0; nb < 8; ++nb) o[nb] *= inv_sqrt128();
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

// What is decoded of a block's meta words, a row a lane, for all columns that look at the block.
template <int NG>
struct BlockMeta {
  // Row operands of the product that a score starts with, eight bfloat16 slots for each lane group q.  q = 0: -zero-point (low byte and
  // multiples of 256, three times each: times the three terms of the query's sum).  q = 1: terms of 1 / scale (times those of minus the reference).
  // q = 2: terms of log2(V scale) / scale - 2 ii / scale (times 1); a row that takes no part has kNoScore here, a scale of 1 and no other terms.
  __attribute__((aligned(16))) uint16_t start[32][4][8];
  __attribute__((aligned(16))) uint16_t start2[NG == 2 ? 32 : 1][8];  // q = 3, of the second group's product: its zero-point (the query's sum over it)
  __attribute__((aligned(16))) float k_scale[NG][32];
  __attribute__((aligned(16))) float v_rcp[32];                       // 4^ii / V scale, the larger one where there are two (no part: 0)
  __attribute__((aligned(16))) float v_share[NG == 2 ? 2 : 1][32];    // V scale / the larger one
  __attribute__((aligned(16))) uint16_t v_zero[2][NG][32];            // binary16, in the weights' order: zero-point * 4^(ii - 3), low part and multiples of 2048
  int far;                                                            // some zero-point has such multiples
};

template <int NG>
struct CodeBlock {
  u32x4 k, v;
  uint32_t meta[NG];  // lanes 0-31: K meta of row `lane`, lanes 32-63: V meta of row lane - 32
  int limit;          // rows from here on (of the sequence) take no part
};

__device__ __forceinline__ void lds_barrier() {  // leaves loads from memory in flight
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Rows of 16 chunks of 16 bytes in LDS: chunk c of row r lies at place c ^ 2 (r % 8), so that eight rows' chunks of the same number fall
// on all banks, read whole (a key operand) or as the two chunks of a transposing read.
__device__ __forceinline__ int staged_at(int row, int chunk) { return row * kD + ((chunk ^ (2 * (row & 7))) << 3); }
constexpr int kStage = 64;  // rows of 16-bit keys and values that a workgroup of many rows holds in LDS at a time (two such stages)

template <int G, int QT, bool MANY>
struct PagedShared;
template <int G, int QT>
struct PagedShared<G, QT, true> {
  BlockMeta<kD / G> meta[2][kManyWaves];  // of the blocks being worked on, and the next
  __attribute__((aligned(16))) uint16_t k[2][kStage * kD], v[2][kStage * kD];
  __attribute__((aligned(16))) uint16_t none[32];
};
template <int G, int QT>
struct PagedShared<G, QT, false> {
  BlockMeta<kD / G> meta[1][kFewWaves];
  __attribute__((aligned(16))) uint16_t v[kFewWaves][32 * kD];
  __attribute__((aligned(16))) float o[kFewWaves][16 * QT][kD + 4];
  float m[kFewWaves][16 * QT], l[kFewWaves][16 * QT];
  __attribute__((aligned(16))) uint16_t none[32];
};

template <int G, int QT, bool MANY>
__global__ __launch_bounds__(64 * (MANY ? kManyWaves : kFewWaves), 2) void paged_attention_kernel(PagedAttentionArgs a) {
  constexpr int NG = kD / G, NW = MANY ? kManyWaves : kFewWaves, WR = MANY ? NW : 1, WK = NW / WR, kRows = 16 * QT;
  __shared__ PagedShared<G, QT, MANY> sh;
  const PagedArgs &c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int wk = MANY ? 0 : wave, wr = MANY ? wave : 0;
  const int unit = blockIdx.y, b = unit / c.Hkv, head = unit % c.Hkv, R = a.Hq / c.Hkv, split = blockIdx.z;
  const ChunkSpan s = chunk_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  const int rows = s.rows * R;                                  // of this unit: token by token, the heads of the group
  const int wg_row = blockIdx.x * (WR * kRows);                 // first row of the workgroup
  if (wg_row >= rows) return;                                   // whole workgroup
  const int row0 = wg_row + wr * kRows;                         // first row of the wavefront
  const bool idle = row0 >= rows;                               // (of a workgroup whose wavefronts have rows of their own)
  const float sm2 = a.sm_scale * kLog2e;

  // ---- the keys of this workgroup: blocks of 32 code rows, of 32 overlay slots, of 32 chunk rows, dealt to the splits as one list
  const int32_t *sidx = c.sal_idx + (size_t)unit * c.S_cap;
  int wide = min(max(c.sal_cnt[unit], 0), c.S_cap);             // overlay slots of cached rows (the list may be final for new rows, too)
  {
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
  const int last_row = min(wg_row + WR * kRows, rows) - 1;
  const int n_code = (s.len + 31) >> 5, n_wide = (wide + 31) >> 5, n_self = last_row / R / 32 + 1;
  int u0, u1;
  decode_split_range(n_code + n_wide + n_self, a.n_split, split, u0, u1);

  f32x4 o[QT][8];
  // per column: the reference that weights are relative to, from which excess over it it is raised (before the first score: any), and
  // this lane's share of the sum
  float m[QT], limit[QT], l[QT];
  const uint16_t *q_at[QT];  // of this lane's column
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) o[t][nb] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m[t] = 0.0f;
    limit[t] = 0.5f * kNoScore;
    l[t] = 0.0f;
    const int row = min(row0 + 16 * t + n, rows - 1), token = row / R;
    q_at[t] = a.q + (s.first + token) * a.q_stride + (head * R + row - token * R) * kD + 8 * q;
  }
  // the query as it arrives: lane (n, q) holds channels 32m + 8q .. + 7 of its column's row (read again by each kind of keys: kept, it
  // would take 32 registers all along)
  auto load_query = [&](int t, u32x4 (&raw)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[k] = *reinterpret_cast<const u32x4 *>(q_at[t] + 32 * k);
  };
  // the rotated query, times sm_scale * log2(e): products with it are base-2 logits
  auto rotated = [&](int t, float (&x)[32]) {
    u32x4 raw[4];
    load_query(t, raw);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        x[8 * k + 2 * w] = half_bits_to_float(raw[k][w] & 0xFFFFu);
        x[8 * k + 2 * w + 1] = half_bits_to_float(raw[k][w] >> 16);
      }
    float f = sm2;
    if (!a.q_rotated) {
      wht128_column(x, q);
      f *= inv_sqrt128();
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] *= f;
  };
  // Weights of the tiles' scores relative to the reference (rows 4q + i of the two halves of a block; no part: far below).  The
  // reference is raised, and what was summed against it rescaled (`more`: the rest of it), only when a score exceeds it by kRaiseAt.
  auto weigh = [&](float (&y)[QT][2][4], auto &&more) {
    float top[QT];
    bool raise = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      top[t] = y[t][0][0];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], y[t][h][i]);
      raise = raise || top[t] > limit[t];
    }
    if (__builtin_expect(__ballot(raise) != 0ull, 0)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float all = column_max(top[t]);
        float by = 0.0f;
        if (all > limit[t]) {  // the four lanes of a column agree
          const float to = rintf(m[t] + all) - kRaiseTo;
          by = to - m[t];
          const float alpha = limit[t] < 0.0f ? 0.0f : exp2_bare(-by);  // (there was nothing before the first score)
#pragma unroll
          for (int nb = 0; nb < 8; ++nb) o[t][nb] *= alpha;
          l[t] *= alpha;
          m[t] = to;
          limit[t] = kRaiseAt;
          more(t, alpha);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][h][i] -= by;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][h][i] = exp2_bare(y[t][h][i]);
  };

  // ================= code rows =================
  const int code_end = min(u1, n_code);
  if (MANY ? u0 < code_end : u0 + wk < code_end) {
    u32x6 digits[QT][kDigits];
    uint32_t unit_exp[QT];
    u32x4 start[QT];  // column operands of the first product: terms of the query's sums, of minus the reference, ones
    auto start_slots = [&](float v) {
      const Terms x = split_terms(v);
      return (u32x4){upper_halves(x.a, x.b), upper_halves(x.c, x.a), upper_halves(x.b, q == 1 ? x.a : x.c), 0u};
    };
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float x[32], mx = 0.0f;
      rotated(t, x);
#pragma unroll
      for (int e = 0; e < 32; ++e) mx = fmaxf(mx, fabsf(x[e]));
      mx = column_max(mx);
      // integers of up to 5 kDigits - 1 bits and a sign in units of a power of two U, |x| < 2^(5 kDigits - 1) U
      const uint32_t e_biased = min(max(__float_as_uint(mx) >> 23, 20u), 250u);  // mx < 2^(e_biased - 126)
      const float unit_inv = __uint_as_float((252u + 5u * kDigits - e_biased) << 23), u = 1.0f / unit_inv;
      float sum[2] = {0.0f, 0.0f};
      constexpr int kLower = kDigits == 4 ? 16 * (1 + 32 + 1024) : 16 * (1 + 32);  // lower digits offset to 0 .. 31
      int v[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float nf = rintf(x[e] * unit_inv);
        sum[e >> 4] += nf * u;
        v[e] = (int)nf + kLower;
      }
#pragma unroll
      for (int d = 0; d < kDigits; ++d) {
        f32x16 dig[2];  // even and odd slots, as the packing conversion takes them
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          // slot of a lane: what ExpandF4 makes of the code words, word slot / 16, field 2 (slot % 8) + (slot / 8) % 2
          const int i = e & 7, slot = 8 * (i & 1) + 4 * ((e >> 3) & 1) + (i >> 1) + 16 * (e >> 4);
          dig[slot & 1][slot >> 1] = 0.125f * (float)(d == kDigits - 1 ? v[e] >> (5 * d) : ((v[e] >> (5 * d)) & 31) - 16);
        }
        digits[t][d] = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(dig[0], dig[1], 1.0f));
        asm volatile("" ::: "memory");  // one digit after the other: all of them at once take 128 registers
      }
      float qs = 0.0f;
      if constexpr (NG == 2) {
        const float s0 = column_sum(sum[0]), s1 = column_sum(sum[1]);
        qs = q == 0 ? s0 : q == 3 ? s1 : 0.0f;
      } else {
        const float s0 = column_sum(sum[0] + sum[1]);
        qs = q == 0 ? s0 : 0.0f;
      }
      start[t] = start_slots(qs);
      if (q == 2) start[t] = (u32x4){0x3F803F80u, 0x00003F80u, 0u, 0u};
      unit_exp[t] = (e_biased + 6u - 5u * kDigits) * 0x01010101u + 0x0F0A0500u;  // a byte a digit: each 32 times the one below
    }
    // sums of weight * zero-point: one row of products serves all channels of a group, so rows 0-7 sum the first group's and rows 8-15
    // the second's (lanes q = 0, 1 and 2, 3 of the result)
    f32x4 acc_z[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) acc_z[t] = (f32x4){0.f, 0.f, 0.f, 0.f};

    if (lane < 16) reinterpret_cast<uint32_t *>(sh.none)[lane] = 0u;  // (by every wavefront for itself)
    const ExpandF4 ex4;
    // page numbers by scalar loads (the constant address space), whose wait stands in front of the first use: a vector load of them would
    // be waited for where it is issued, and every other load with it
    const auto *table = reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(
        reinterpret_cast<uintptr_t>(c.table + (size_t)b * c.max_pages));
    auto page_of = [&](int blk) { return table[min(blk * 32, s.len - 1) >> c.page_shift]; };
    struct Where { size_t row; int limit; };  // first row of a block in the pools; rows from `limit` on (of the sequence) take no part
    auto find = [&](int blk, int page) {
      const bool there = page >= 0 && page < c.n_pages;
      return Where{(((size_t)(there ? page : 0) * c.Hkv + head) << c.page_shift) + ((blk * 32) & ((1 << c.page_shift) - 1)), there ? s.len : 0};
    };
    auto load_meta = [&](const Where &at, CodeBlock<NG> &t) {
      const uint32_t *meta = (lane < 32 ? c.k_meta : c.v_meta) + (at.row + (lane & 31)) * NG;
      if constexpr (NG == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(meta);
        t.meta[0] = w[0]; t.meta[1] = w[1];
      } else {
        t.meta[0] = *meta;
      }
      t.limit = at.limit;
    };
    auto load_keys = [&](const Where &at, CodeBlock<NG> &t) { t.k = *reinterpret_cast<const u32x4 *>(c.k_codes + at.row * 8 + 4 * lane); };
    auto load_values = [&](const Where &at, CodeBlock<NG> &t) { t.v = *reinterpret_cast<const u32x4 *>(c.v_codes + at.row * 8 + 4 * lane); };
    // A block's meta words, a row a lane: lanes 0-31 what concerns keys, lanes 32-63 values.
    auto decode = [&](const CodeBlock<NG> &cur, int blk, BlockMeta<NG> &bm) {
      const int r = lane & 31, ii = r & 3;
      const bool part = blk * 32 + r < cur.limit && (cur.meta[0] & 0x8000u) == 0u;
      float scale[NG], zero[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        scale[g] = part ? half_bits_to_float(cur.meta[g] & 0x7FFFu) : 1.0f;
        zero[g] = part ? (float)((int)cur.meta[g] >> 16) : 0.0f;
      }
      const float top = NG == 2 && lane >= 32 ? fmaxf(scale[0], scale[NG - 1]) : scale[0], rcp = part ? __builtin_amdgcn_rcpf(top) : 0.0f;
      const float v_log = __shfl_xor(log2_bare(top), 32, kWave) - 2.0f * (float)ii;  // (keys' lanes: of their row's values)
      bool far = false;  // a zero-point that 11 bits do not hold
      if (lane < 32) {
        const Terms inv = split_terms(rcp), log = split_terms(part ? v_log * rcp : kNoScore);
        const float zh = rintf(zero[0] * (1.0f / 256.0f)) * -256.0f, zl = -zero[0] - zh;
        u32x4 *to = reinterpret_cast<u32x4 *>(&bm.start[r][0][0]);
        to[0] = (u32x4){upper_halves(zl, zl), upper_halves(zl, zh), upper_halves(zh, zh), 0u};
        to[1] = (u32x4){upper_halves(inv.a, inv.a), upper_halves(inv.a, inv.b), upper_halves(inv.b, inv.c), 0u};
        to[2] = (u32x4){upper_halves(log.a, log.b), upper_halves(log.c, 0.0f), 0u, 0u};
        to[3] = (u32x4){0u, 0u, 0u, 0u};
        if constexpr (NG == 2) {
          const float yh = rintf(zero[1] * (1.0f / 256.0f)) * -256.0f, yl = -zero[1] - yh;
          *reinterpret_cast<u32x4 *>(&bm.start2[r][0]) = (u32x4){upper_halves(yl, yl), upper_halves(yl, yh), upper_halves(yh, yh), 0u};
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) bm.k_scale[g][r] = part || g == 0 ? scale[g] : 0.0f;
      } else {
        const int at = 2 * (4 * ((r & 15) >> 2) + ii) + (r >> 4);  // the weights' order: pairs (r, r + 16)
        const float four = (float)(1 << (2 * ii));
        bm.v_rcp[r] = rcp * four;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if constexpr (NG == 2) bm.v_share[g][r] = scale[g] * rcp;
          const float hi = rintf(zero[g] * (1.0f / 2048.0f)) * 2048.0f, f = four * (1.0f / 64.0f);
          bm.v_zero[0][g][at] = (uint16_t)float_to_half_bits_rne((zero[g] - hi) * f);
          bm.v_zero[1][g][at] = (uint16_t)float_to_half_bits_rne(hi * f);
          far = far || hi != 0.0f;
        }
      }
      bm.far = __ballot(far) != 0ull;
    };
    // one block; done_keys, done_values: called when that part of `cur` has been taken
    auto process = [&](CodeBlock<NG> &cur, const BlockMeta<NG> &bm, auto &&done_keys, auto &&done_values) {
      // ---- scores and weights
      const int far = bm.far;
      float y[QT][2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2 lo = ex4(cur.k[2 * h]), hi = ex4(cur.k[2 * h + 1]);
        u32x4 codes[NG], first[NG];
        f32x4 k_scale[NG];
        first[0] = *reinterpret_cast<const u32x4 *>(&bm.start[16 * h + n][q][0]);
        if constexpr (NG == 2) {  // a group's product takes zeros in the other group's slots
          codes[0] = (u32x4){lo[0], lo[1], 0u, 0u};
          codes[1] = (u32x4){0u, 0u, hi[0], hi[1]};
          first[1] = *reinterpret_cast<const u32x4 *>(q == 3 ? &bm.start2[16 * h + n][0] : &sh.none[0]);
        } else {
          codes[0] = (u32x4){lo[0], lo[1], hi[0], hi[1]};
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) k_scale[g] = *reinterpret_cast<const f32x4 *>(&bm.k_scale[g][16 * h + 4 * q]);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          f32x4 acc[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            acc[g] = mfma_b16(first[g], start[t], (f32x4){0.f, 0.f, 0.f, 0.f});
            acc[g] = mfma_codes<0>(codes[g], digits[t][0], unit_exp[t], acc[g]);
            acc[g] = mfma_codes<1>(codes[g], digits[t][1], unit_exp[t], acc[g]);
            acc[g] = mfma_codes<2>(codes[g], digits[t][2], unit_exp[t], acc[g]);
            if constexpr (kDigits == 4) acc[g] = mfma_codes<kDigits - 1>(codes[g], digits[t][kDigits - 1], unit_exp[t], acc[g]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[t][h][i] = k_scale[0][i] * acc[0][i];
            if constexpr (NG == 2) y[t][h][i] = __builtin_fmaf(k_scale[1][i], acc[1][i], y[t][h][i]);
          }
        }
      }
      done_keys();
      u32x4 w[QT][NG];
      const f32x4 r0 = *reinterpret_cast<const f32x4 *>(&bm.v_rcp[4 * q]), r1 = *reinterpret_cast<const f32x4 *>(&bm.v_rcp[16 + 4 * q]);
      weigh(y, [&](int t, float alpha) {
        acc_z[t] *= alpha;
        if (q == 1) start[t] = start_slots(-m[t]);
      });
#pragma unroll
      for (int t = 0; t < QT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) l[t] = __builtin_fmaf(y[t][0][i], r0[i], __builtin_fmaf(y[t][1][i], r1[i], l[t]));
        if constexpr (NG == 2) {
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const f32x4 s0 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][4 * q]), s1 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][16 + 4 * q]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[t][g][i] = pack_f16x2(y[t][0][i] * s0[i], y[t][1][i] * s1[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[t][0][i] = pack_f16x2(y[t][0][i], y[t][1][i]);
        }
      }
      // ---- values
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x == 0 || __builtin_expect(__builtin_amdgcn_readfirstlane(far) != 0, 0))
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const u32x4 z = *reinterpret_cast<const u32x4 *>(NG == 1 || n / 8 == g ? &bm.v_zero[x][g][8 * q] : &sh.none[0]);
#pragma unroll
            for (int t = 0; t < QT; ++t) acc_z[t] = mfma_f16(z, w[t][g], acc_z[t]);
          }
#pragma unroll
      for (int wd = 0; wd < 4; ++wd) {
        const int g = NG == 2 ? (wd & 1) : 0, nb = 4 * (wd & 1) + (wd >> 1);
        const uint32_t x = cur.v[wd], y8 = x >> 8;
        const u32x4 vx = {x & 0x00030003u, x & 0x000C000Cu, x & 0x00300030u, x & 0x00C000C0u};
        const u32x4 vy = {y8 & 0x00030003u, y8 & 0x000C000Cu, y8 & 0x00300030u, y8 & 0x00C000C0u};
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          o[t][nb] = mfma_f16(vx, w[t][g], o[t][nb]);
          o[t][nb + 2] = mfma_f16(vy, w[t][g], o[t][nb + 2]);
        }
      }
      done_values();
    };
    // The next block is requested while one is worked on, and its page's number one block earlier.
    const int first = u0 + wk;
    if constexpr (MANY) {
      // Every wavefront decodes one block of the next eight for all; codes go into their registers again as soon as they are free (another
      // set would be ten registers too many).
      CodeBlock<NG> buf, words;
      auto ask_words = [&](int from) {
        const int blk = min(from + wave, n_code - 1);
        load_meta(find(blk, page_of(blk)), words);
      };
      ask_words(first);
      Where at = find(first, page_of(first));
      load_keys(at, buf);
      load_values(at, buf);
      int page = page_of(min(first + 1, n_code - 1));
      for (int from = first, turn = 0; from < code_end; from += kManyWaves, turn ^= 1) {
        decode(words, min(from + wave, n_code - 1), sh.meta[turn][wave]);
        if (from + kManyWaves < code_end) ask_words(from + kManyWaves);
        lds_barrier();  // (the other set was last read in front of the barrier before)
        if (idle) continue;
        for (int blk = from; blk < min(from + kManyWaves, code_end); ++blk) {
          at = find(min(blk + 1, n_code - 1), page);
          page = page_of(min(blk + 2, n_code - 1));
          process(buf, sh.meta[turn][blk - from], [&] { load_keys(at, buf); }, [&] { load_values(at, buf); });
        }
      }
    } else {
      // bound by the stream: another set of registers, asked for as a whole
      CodeBlock<NG> buf[2];
      BlockMeta<NG> &bm = sh.meta[0][wave];
      Where at = find(first, page_of(first));
      int page = page_of(min(first + WK, n_code - 1));
      load_meta(at, buf[0]);
      load_keys(at, buf[0]);
      load_values(at, buf[0]);
      for (int blk = first; blk < code_end; blk += 2 * WK) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int now = blk + x * WK;
          if (now >= code_end) break;
          at = find(min(now + WK, n_code - 1), page);
          page = page_of(min(now + 2 * WK, n_code - 1));
          load_meta(at, buf[1 - x]);
          load_keys(at, buf[1 - x]);
          load_values(at, buf[1 - x]);
          wave_lds_sync();  // the block before is done with its words
          decode(buf[x], now, bm);
          wave_lds_sync();
          process(buf[x], bm, [] {}, [] {});
        }
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float mine = -64.0f * acc_z[t][0], other = NG == 2 ? __shfl_xor(mine, 32, kWave) : mine;
      const float z[2] = {q < 2 ? mine : other, q < 2 ? other : mine};
#pragma unroll
      for (int nb = 0; nb < 8; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][nb][i] = __builtin_fmaf(o[t][nb][i], 16777216.0f, z[NG == 2 ? nb / 4 : 0]);
    }
  }

  // Sixteen-bit keys and values of a workgroup of many rows go through LDS, a stage at a time: every thread brings two chunks of keys
  // and of values, asked for while the stage before is worked on.  `from(key?, row, chunk)`: where a chunk comes from.
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

  // ================= 16-bit rows of the cache =================
  const int wide_begin = max(u0 - n_code, 0), wide_end = min(u1 - n_code, n_wide);
  if (wide_begin < wide_end) {
    u32x4 q_hi[QT][4], q_lo[QT][4];  // two bfloat16 terms: 16 bits of the query
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float x[32];
      rotated(t, x);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = x[8 * k + 2 * i], x1 = x[8 * k + 2 * i + 1];
          const uint32_t hi = pack_bf16x2(x0, x1);
          q_hi[t][k][i] = hi;
          q_lo[t][k][i] = pack_bf16x2(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xFFFF0000u));
        }
    }
    const uint16_t *ks = c.k_sal + (size_t)unit * c.S_cap * kD, *vs = c.v_sal + (size_t)unit * c.S_cap * kD;
    // one block of 32 slots; key(h, ch), value(nb): operands
    auto wide_block = [&](int blk, auto &&key, auto &&value) {
      u32x4 hi[QT], lo[QT];
      float y[QT][2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 acc[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          const u32x4 k = key(h, ch);
#pragma unroll
          for (int t = 0; t < QT; ++t) acc[t] = mfma_b16(k, q_hi[t][ch], mfma_b16(k, q_lo[t][ch], acc[t]));
        }
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][h][i] = blk * 32 + 16 * h + 4 * q + i < wide ? acc[t][i] - m[t] : kNoScore;
      }
      weigh(y, [](int, float) {});
#pragma unroll
      for (int t = 0; t < QT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          l[t] += y[t][0][i] + y[t][1][i];
          hi[t][i] = pack_bf16x2(y[t][0][i], y[t][1][i]);
          lo[t][i] = pack_bf16x2(y[t][0][i] - __uint_as_float(hi[t][i] << 16), y[t][1][i] - __uint_as_float(hi[t][i] & 0xFFFF0000u));
        }
      }
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        u32x4 v = value(nb);
        if (blk * 32 + 32 > wide)  // slots behind the last row may hold anything, and 0 * NaN is no 0
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] &= (blk * 32 + 4 * q + i < wide ? 0xFFFFu : 0u) | (blk * 32 + 16 + 4 * q + i < wide ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int t = 0; t < QT; ++t) o[t][nb] = mfma_b16(v, hi[t], mfma_b16(v, lo[t], o[t][nb]));
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
                              [&](int h, int ch) { return *reinterpret_cast<const u32x4 *>(&sh.k[buf][staged_at(32 * x + 16 * h + n, 4 * ch + q)]); },
                              [&](int nb) { return *reinterpret_cast<const u32x4 *>(&sh.v[buf][x * 4096 + nb * 512 + 8 * lane]); });
             });
    } else {
      for (int blk = wide_begin + wk; blk < wide_end; blk += WK)
        wide_block(blk, [&](int h, int ch) { return *reinterpret_cast<const u32x4 *>(ks + (size_t)(blk * 32 + 16 * h + n) * kD + 32 * ch + 8 * q); },
                   [&](int nb) { return *reinterpret_cast<const u32x4 *>(vs + (size_t)blk * 4096 + nb * 512 + 8 * lane); });
    }
  }
  // The cached rows' share is rotated back (H is its own inverse), and the chunk's rows join it.  Their weights are relative to the
  // sum so far: the reference of the code rows holds V scales as well.
  if (!idle && u0 + wk < n_code + n_wide) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (!a.out_rotated) wht128_output(o[t], q);
      const float all = column_sum(l[t]);
      if (all > 0.0f) {
        const float to = rintf(m[t] + log2_bare(all)) - kRaiseTo, alpha = exp2_bare(m[t] - to);
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) o[t][nb] *= alpha;
        l[t] *= alpha;
        m[t] = to;
        limit[t] = kRaiseAt;
      }
    }
  }

  // ================= rows of the chunk =================
  const int self_begin = max(u0 - n_code - n_wide, 0), self_end = min(u1 - n_code - n_wide, n_self);
  if (self_begin < self_end) {
    const int low_token = row0 / R;                                        // of this wavefront's rows
    const int my_end = idle ? 0 : (min(row0 + kRows, rows) - 1) / R / 32 + 1;
    const uint16_t *ks = a.k + s.first * a.k_stride + head * kD, *vs = a.v + s.first * a.v_stride + head * kD;
    int token[QT];
    u32x4 raw[QT][4];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      token[t] = min(row0 + 16 * t + n, rows - 1) / R;
      load_query(t, raw[t]);
    }
    // one block of 32 rows; key(h, ch): operand; vt, vrow: where the block's values lie in LDS
    auto self_block = [&](int blk, auto &&key, const uint16_t *vt, int vrow) {
      u32x4 w[QT];
      float y[QT][2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 acc[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          const u32x4 k = key(h, ch);
#pragma unroll
          for (int t = 0; t < QT; ++t) acc[t] = mfma_f16(k, raw[t][ch], acc[t]);
        }
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][h][i] = __builtin_fmaf(acc[t][i], sm2, -m[t]);
      }
      if (blk * 32 + 31 > low_token) {  // uniform over the wavefront: some row may not look at all of the block
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (blk * 32 + 16 * h + 4 * q + i > token[t]) y[t][h][i] = kNoScore;
      }
      weigh(y, [](int, float) {});
#pragma unroll
      for (int t = 0; t < QT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          l[t] += (y[t][h][0] + y[t][h][1]) + (y[t][h][2] + y[t][h][3]);
          w[t][2 * h] = pack_f16x2(y[t][h][0], y[t][h][1]);
          w[t][2 * h + 1] = pack_f16x2(y[t][h][2], y[t][h][3]);
        }
      }
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        u32x4 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // a transposing read: the lane gets its channel of rows 16h + 4q .. + 3
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4 *)(&vt[staged_at(vrow + 16 * h + 4 * q + (n >> 2), 2 * nb + ((n & 3) >> 1)) + 4 * (n & 1)])));
          v[2 * h] = x[0];
          v[2 * h + 1] = x[1];
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) o[t][nb] = mfma_f16(v, w[t], o[t][nb]);
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
                   self_block(blk, [&](int h, int ch) { return *reinterpret_cast<const u32x4 *>(&sh.k[buf][staged_at(32 * x + 16 * h + n, 4 * ch + q)]); },
                              sh.v[buf], 32 * x);
               }
             });
    } else {
      uint16_t *vt = sh.v[wave];
      for (int blk = self_begin + wk; blk < min(self_end, my_end); blk += WK) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
          *reinterpret_cast<u32x4 *>(&vt[staged_at(4 * x + q, n)]) =
              *reinterpret_cast<const u32x4 *>(vs + min(blk * 32 + 4 * x + q, s.rows - 1) * a.v_stride + 8 * n);
        wave_lds_sync();
        self_block(blk, [&](int h, int ch) {
          return *reinterpret_cast<const u32x4 *>(ks + min(blk * 32 + 16 * h + n, s.rows - 1) * a.k_stride + 32 * ch + 8 * q);
        }, vt, 0);
        wave_lds_sync();
      }
    }
  }

  // ================= sums of the wavefronts, and out =================
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] = column_sum(l[t]);
    if (limit[t] < 0.0f) m[t] = kNoScore;
  }
  auto store = [&](int row, int ch, const f32x4 &x, float top, float sum) {  // four channels of a finished or partial row
    const int token = row / R, hq = head * R + row - token * R;
    const size_t at = (size_t)(s.first + token) * a.Hq + hq;
    if (a.n_split == 1) {
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      *reinterpret_cast<u32x2 *>(a.out + (s.first + token) * a.out_stride + hq * kD + ch) =
          (u32x2){pack_f16x2(x[0] * inv, x[1] * inv), pack_f16x2(x[2] * inv, x[3] * inv)};
      if (a.lse && ch == 0) a.lse[at] = sum > 0.0f ? (top + log2_bare(sum)) * kLn2 : -INFINITY;
    } else {
      float *p = a.partial + (at * a.n_split + split) * kPartialStride;
      *reinterpret_cast<f32x4 *>(p + 4 + ch) = x;
      if (ch == 0) { p[0] = top; p[1] = sum; }
    }
  };
  if constexpr (MANY) {
    if (idle) return;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int row = row0 + 16 * t + n;
      if (row < rows)
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) store(row, 16 * nb + 4 * q, o[t][nb], m[t], l[t]);
    }
  } else {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) *reinterpret_cast<f32x4 *>(&sh.o[wk][16 * t + n][16 * nb + 4 * q]) = o[t][nb];
      if (q == 0) { sh.m[wk][16 * t + n] = m[t]; sh.l[wk][16 * t + n] = l[t]; }
    }
    __syncthreads();
    for (int at = threadIdx.x; at < kRows * 32; at += 64 * NW) {
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

// Merges the splits of a row: one wavefront a row, two channels a lane.
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedAttentionArgs a) {
  const PagedArgs &c = a.c;
  const int lane = threadIdx.x & 63, unit = blockIdx.y, b = unit / c.Hkv, head = unit % c.Hkv, R = a.Hq / c.Hkv;
  const int row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ChunkSpan s = chunk_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (row >= s.rows * R) return;
  const int token = row / R, hq = head * R + row - token * R;
  const size_t at = (size_t)(s.first + token) * a.Hq + hq;
  const float *p = a.partial + at * a.n_split * kPartialStride;
  float top = kNoScore, sum = 0.0f, x0 = 0.0f, x1 = 0.0f;
  for (int i = 0; i < a.n_split; ++i) top = fmaxf(top, p[i * kPartialStride]);
  for (int i = 0; i < a.n_split; ++i) {
    const float *r = p + i * kPartialStride, f = exp2_bare(r[0] - top);
    sum += f * r[1];
    x0 += f * r[4 + 2 * lane];
    x1 += f * r[5 + 2 * lane];
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  *reinterpret_cast<uint32_t *>(a.out + (s.first + token) * a.out_stride + hq * kD + 2 * lane) = pack_f16x2(x0 * inv, x1 * inv);
  if (a.lse && lane == 0) a.lse[at] = sum > 0.0f ? (top + log2_bare(sum)) * kLn2 : -INFINITY;
}

template <int G>
void launch_variant(const PagedAttentionArgs &a, int rows, hipStream_t stream) {
  const int units = a.c.B * a.c.Hkv;
  auto grid = [&](int per) { return dim3((rows + per - 1) / per, units, a.n_split); };
  constexpr int kFew = 64 * kFewWaves, kMany = 64 * kManyWaves;
  if (rows <= 16) paged_attention_kernel<G, 1, false><<<grid(16), kFew, 0, stream>>>(a);
  else if (rows <= 64) paged_attention_kernel<G, 2, false><<<grid(32), kFew, 0, stream>>>(a);
  else paged_attention_kernel<G, 2, true><<<grid(32 * kManyWaves), kMany, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttentionArgs &a, int G, hipStream_t stream) {
  const int rows = a.c.max_rows * (a.Hq / a.c.Hkv);
  if (G == 128) launch_variant<128>(a, rows, stream);
  else launch_variant<64>(a, rows, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  paged_combine_kernel<<<dim3((rows + 3) / 4, a.c.B * a.c.Hkv), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace akvq
