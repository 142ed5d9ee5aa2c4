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
// kDigits / 4 of a 16-bit product.  Scale and zero-point of a row are applied to its score.
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

constexpr int kDigits = 4;
constexpr int kPagedWaves = 4;
constexpr float kNoScore = -1.0e30f;   // reference before the first score
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
// rows: codes as 4-bit floats; columns: query digits as 6-bit floats, times 2^(scale - 127)
__device__ __forceinline__ f32x4 mfma_codes(u32x4 codes, u32x6 digits, uint32_t scale, f32x4 c) {
  constexpr int kE2M3 = 2, kE2M1 = 4;
  const i32x8 a = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
  const i32x8 b = {(int)digits[0], (int)digits[1], (int)digits[2], (int)digits[3], (int)digits[4], (int)digits[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kE2M1, kE2M3, 0, 127, 0, (int)scale);
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

// What a wavefront decodes of a block's meta words, a row a lane, for all its columns.
template <int NG>
struct BlockMeta {
  float k_scale[NG][32], k_zero[NG][32];  // a row that takes no part: 0
  float v_log[32];                        // log2(scale) - 2 ii, of the larger scale where there are two (no part: -inf)
  float v_rcp[32];                        // 4^ii / that scale (no part: 0)
  float v_share[NG][32];                  // scale / that scale (two groups only)
  uint16_t v_zero[2][NG][32];             // binary16, in the weights' order: zero-point * 4^(ii - 3), low part and multiples of 2048
};

template <int NG>
struct CodeBlock {
  u32x4 k, v;
  uint32_t meta[NG];  // lanes 0-31: K meta of row `lane`, lanes 32-63: V meta of row lane - 32
  int limit;          // rows from here on (of the sequence) take no part
};

// WK of the four wavefronts of a workgroup share its rows and deal the keys among them; the others have rows of their own.
template <int G, int QT, int WK>
struct PagedShared {
  static constexpr int NG = kD / G;
  static constexpr int kRows = 16 * QT;      // of a wavefront
  static constexpr int kVStride = kD + 16;   // binary16 values: the rows of a transposing read fall on different banks
  BlockMeta<NG> meta[kPagedWaves];
  __attribute__((aligned(16))) uint16_t v[kPagedWaves][32][kVStride];
  float o[WK > 1 ? WK : 1][WK > 1 ? kRows : 1][WK > 1 ? kD + 4 : 1];
  float m[WK][kRows], l[WK][kRows];
};

template <int G, int QT, int WK>
__global__ __launch_bounds__(64 * kPagedWaves) void paged_attention_kernel(PagedAttentionArgs a) {
  constexpr int NG = kD / G, WR = kPagedWaves / WK, kRows = 16 * QT;
  using Shared = PagedShared<G, QT, WK>;
  __shared__ Shared sh;
  const PagedArgs &c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int wk = WK > 1 ? wave : 0, wr = WK > 1 ? 0 : wave;
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
  float m[QT], l[QT];
  u32x4 raw[QT][4];  // the queries as they arrive: lane (n, q) holds channels 32m + 8q .. + 7 of its column's row
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) o[t][nb] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m[t] = kNoScore;
    l[t] = 0.0f;
    const int row = min(row0 + 16 * t + n, rows - 1), token = row / R;
    const uint16_t *p = a.q + (s.first + token) * a.q_stride + (head * R + row - token * R) * kD + 8 * q;
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[t][k] = *reinterpret_cast<const u32x4 *>(p + 32 * k);
  }
  // the rotated query, times sm_scale * log2(e): products with it are base-2 logits
  auto rotated = [&](int t, float (&x)[32]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        x[8 * k + 2 * w] = half_bits_to_float(raw[t][k][w] & 0xFFFFu);
        x[8 * k + 2 * w + 1] = half_bits_to_float(raw[t][k][w] >> 16);
      }
    float f = sm2;
    if (!a.q_rotated) {
      wht128_column(x, q);
      f *= inv_sqrt128();
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] *= f;
  };
  // Weights of a tile's eight scores (rows 4q + i of the two halves of a block; -inf: no part).  The reference of a column is raised, and what
  // was summed against it rescaled by `more`, only when a score exceeds it by kRaiseAt.
  auto weigh = [&](int t, float (&y)[2][4], auto &&more) {
    float top = y[0][0];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, y[h][i]);
    if (__ballot(top > m[t] + kRaiseAt) != 0ull) {
      const float all = column_max(top);
      if (all > m[t] + kRaiseAt) {
        const float alpha = exp2_bare(m[t] - (all - kRaiseTo));  // 0 while there was no score
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) o[t][nb] *= alpha;
        l[t] *= alpha;
        more(alpha);
        m[t] = all - kRaiseTo;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[h][i] = exp2_bare(y[h][i] - m[t]);
  };

  // ================= code rows =================
  const int code_end = min(u1, n_code);
  if (!idle && u0 + wk < code_end) {
    u32x6 digits[QT][kDigits];
    uint32_t unit_exp[QT];
    float qsum[QT][NG];
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
      f32x16 dig[kDigits][2];  // even and odd slots, as the packing conversion takes them
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int f8 = 0; f8 < 2; ++f8)
#pragma unroll
          for (int i = 0; i < 8; ++i) {  // slot v of a lane is what ExpandF4 makes of the code words: word v / 16, field 2 (v % 8) + (v / 8) % 2
            const float nf = rintf(x[8 * (2 * w + f8) + i] * unit_inv);
            sum[w] += nf * u;
            constexpr int kLower = kDigits == 4 ? 16 * (1 + 32 + 1024) : 16 * (1 + 32);
            const int v = (int)nf + kLower, slot = 8 * (i & 1) + 4 * f8 + (i >> 1) + 16 * w;
#pragma unroll
            for (int d = 0; d < kDigits; ++d)
              dig[d][slot & 1][slot >> 1] = 0.125f * (float)(d == kDigits - 1 ? v >> (5 * d) : ((v >> (5 * d)) & 31) - 16);
          }
#pragma unroll
      for (int d = 0; d < kDigits; ++d)
        digits[t][d] = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(dig[d][0], dig[d][1], 1.0f));
      if constexpr (NG == 2) {
        qsum[t][0] = column_sum(sum[0]);
        qsum[t][1] = column_sum(sum[1]);
      } else {
        qsum[t][0] = column_sum(sum[0] + sum[1]);
      }
      unit_exp[t] = e_biased + 6u - 5u * kDigits;
    }
    f32x4 acc_z[QT][NG];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int g = 0; g < NG; ++g) acc_z[t][g] = (f32x4){0.f, 0.f, 0.f, 0.f};

    BlockMeta<NG> &bm = sh.meta[wave];
    const ExpandF4 ex4;
    const int32_t *table = c.table + (size_t)b * c.max_pages;
    auto page_of = [&](int blk) { return table[min(blk * 32, s.len - 1) >> c.page_shift]; };
    auto load_block = [&](int blk, int page, CodeBlock<NG> &t) {
      const bool there = page >= 0 && page < c.n_pages;
      const int in_page = (blk * 32) & ((1 << c.page_shift) - 1);
      const size_t row = (((size_t)(there ? page : 0) * c.Hkv + head) << c.page_shift) + in_page;
      t.limit = there ? s.len : 0;
      t.k = *reinterpret_cast<const u32x4 *>(c.k_codes + row / 32 * kBlockWords + 4 * lane);
      t.v = *reinterpret_cast<const u32x4 *>(c.v_codes + row / 32 * kBlockWords + 4 * lane);
      const uint32_t *meta = (lane < 32 ? c.k_meta : c.v_meta) + (row + (lane & 31)) * NG;
      if constexpr (NG == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(meta);
        t.meta[0] = w[0]; t.meta[1] = w[1];
      } else {
        t.meta[0] = *meta;
      }
    };
    auto process = [&](const CodeBlock<NG> &cur, int blk) {
      // ---- meta words: a row a lane
      bool far = false;  // a zero-point that 11 bits do not hold
      {
        const int r = lane & 31, ii = r & 3, at = 2 * (4 * ((r & 15) >> 2) + ii) + (r >> 4);  // the weights' order: pairs (r, r + 16)
        const bool part = blk * 32 + r < cur.limit && (cur.meta[0] & 0x8000u) == 0u;
        float scale[NG], zero[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          scale[g] = part ? half_bits_to_float(cur.meta[g] & 0x7FFFu) : 0.0f;
          zero[g] = part ? (float)((int)cur.meta[g] >> 16) : 0.0f;
        }
        if (lane < 32) {
#pragma unroll
          for (int g = 0; g < NG; ++g) { bm.k_scale[g][r] = scale[g]; bm.k_zero[g][r] = zero[g]; }
        } else {
          const float top = NG == 2 ? fmaxf(scale[0], scale[NG - 1]) : scale[0];
          const bool any = top > 0.0f;
          const float inv = any ? 1.0f / top : 0.0f;
          bm.v_log[r] = any ? log2_bare(top) - 2.0f * (float)ii : -INFINITY;
          bm.v_rcp[r] = inv * (float)(1 << (2 * ii));
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            if constexpr (NG == 2) bm.v_share[g][r] = scale[g] * inv;
            const float hi = rintf(zero[g] * (1.0f / 2048.0f)) * 2048.0f, f = (float)(1 << (2 * ii)) * (1.0f / 64.0f);
            bm.v_zero[0][g][at] = (uint16_t)float_to_half_bits_rne((zero[g] - hi) * f);
            bm.v_zero[1][g][at] = (uint16_t)float_to_half_bits_rne(hi * f);
            far = far || hi != 0.0f;
          }
        }
      }
      const bool any_far = __ballot(far) != 0ull;
      wave_lds_sync();
      f32x4 k_scale[NG][2], k_zero[NG][2], v_log[2], v_rcp[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          k_scale[g][h] = *reinterpret_cast<const f32x4 *>(&bm.k_scale[g][16 * h + 4 * q]);
          k_zero[g][h] = *reinterpret_cast<const f32x4 *>(&bm.k_zero[g][16 * h + 4 * q]);
        }
        v_log[h] = *reinterpret_cast<const f32x4 *>(&bm.v_log[16 * h + 4 * q]);
        v_rcp[h] = *reinterpret_cast<const f32x4 *>(&bm.v_rcp[16 * h + 4 * q]);
      }
      // ---- scores and weights
      u32x4 codes[2][NG];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2 lo = ex4(cur.k[2 * h]), hi = ex4(cur.k[2 * h + 1]);
        if constexpr (NG == 2) {
          codes[h][0] = (u32x4){lo[0], lo[1], 0u, 0u};
          codes[h][1] = (u32x4){0u, 0u, hi[0], hi[1]};
        } else {
          codes[h][0] = (u32x4){lo[0], lo[1], hi[0], hi[1]};
        }
      }
      u32x4 w[QT][NG];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float y[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 acc[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            acc[g] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < kDigits; ++d) acc[g] = mfma_codes(codes[h][g], digits[t][d], unit_exp[t] + 5u * d, acc[g]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = v_log[h][i];
#pragma unroll
            for (int g = 0; g < NG; ++g)
              v = __builtin_fmaf(k_scale[g][h][i], __builtin_fmaf(-k_zero[g][h][i], qsum[t][g], acc[g][i]), v);
            y[h][i] = v;
          }
        }
        weigh(t, y, [&](float alpha) {
#pragma unroll
          for (int g = 0; g < NG; ++g) acc_z[t][g] *= alpha;
        });
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) l[t] = __builtin_fmaf(y[h][i], v_rcp[h][i], l[t]);
        if constexpr (NG == 2) {
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const f32x4 s0 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][4 * q]), s1 = *reinterpret_cast<const f32x4 *>(&bm.v_share[g][16 + 4 * q]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[t][g][i] = pack_f16x2(y[0][i] * s0[i], y[1][i] * s1[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[t][0][i] = pack_f16x2(y[0][i], y[1][i]);
        }
      }
      // ---- values
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const u32x4 z = *reinterpret_cast<const u32x4 *>(&bm.v_zero[0][g][8 * q]);
#pragma unroll
        for (int t = 0; t < QT; ++t) acc_z[t][g] = mfma_f16(z, w[t][g], acc_z[t][g]);
        if (any_far) {
          const u32x4 z2 = *reinterpret_cast<const u32x4 *>(&bm.v_zero[1][g][8 * q]);
#pragma unroll
          for (int t = 0; t < QT; ++t) acc_z[t][g] = mfma_f16(z2, w[t][g], acc_z[t][g]);
        }
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
      wave_lds_sync();  // the next block's meta words overwrite this one's
    };
    // a block is requested while the one before it is worked on, its page's number one block earlier
    CodeBlock<NG> buf[2];
    const int first = u0 + wk;
    load_block(first, page_of(first), buf[0]);
    int next_page = page_of(min(first + WK, n_code - 1));
    for (int blk = first; blk < code_end; blk += 2 * WK) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int now = blk + x * WK;
        if (now >= code_end) break;
        load_block(min(now + WK, n_code - 1), next_page, buf[1 - x]);
        next_page = page_of(min(now + 2 * WK, n_code - 1));
        process(buf[x], now);
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int nb = 0; nb < 8; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][nb][i] = __builtin_fmaf(o[t][nb][i], 16777216.0f, -64.0f * acc_z[t][NG == 2 ? nb / 4 : 0][i]);
  }

  // ================= 16-bit rows of the cache =================
  const int wide_begin = max(u0 - n_code, 0), wide_end = min(u1 - n_code, n_wide);
  if (!idle && wide_begin + wk < wide_end) {
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
    for (int blk = wide_begin + wk; blk < wide_end; blk += WK) {
      u32x4 k[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
          k[h][ch] = *reinterpret_cast<const u32x4 *>(ks + (size_t)(blk * 32 + 16 * h + n) * kD + 32 * ch + 8 * q);
      u32x4 v[8];
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        v[nb] = *reinterpret_cast<const u32x4 *>(vs + (size_t)blk * 4096 + nb * 512 + 8 * lane);
        if (blk * 32 + 32 > wide)  // slots behind the last row may hold anything, and 0 * NaN is no 0
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[nb][i] &= (blk * 32 + 4 * q + i < wide ? 0xFFFFu : 0u) | (blk * 32 + 16 + 4 * q + i < wide ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float y[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) acc = mfma_b16(k[h][ch], q_hi[t][ch], mfma_b16(k[h][ch], q_lo[t][ch], acc));
#pragma unroll
          for (int i = 0; i < 4; ++i) y[h][i] = blk * 32 + 16 * h + 4 * q + i < wide ? acc[i] : -INFINITY;
        }
        weigh(t, y, [](float) {});
        u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          l[t] += y[0][i] + y[1][i];
          hi[i] = pack_bf16x2(y[0][i], y[1][i]);
          lo[i] = pack_bf16x2(y[0][i] - __uint_as_float(hi[i] << 16), y[1][i] - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) o[t][nb] = mfma_b16(v[nb], hi, mfma_b16(v[nb], lo, o[t][nb]));
      }
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
        const float to = m[t] + log2_bare(all) - kRaiseTo, alpha = exp2_bare(m[t] - to);
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) o[t][nb] *= alpha;
        l[t] *= alpha;
        m[t] = to;
      }
    }
  }

  // ================= rows of the chunk =================
  const int self_begin = max(u0 - n_code - n_wide, 0);
  int self_end = min(u1 - n_code - n_wide, n_self);
  const int low_token = row0 / R;                                             // of this wavefront's rows
  self_end = min(self_end, (min(row0 + kRows, rows) - 1) / R / 32 + 1);       // (before an idle wavefront's first row: nothing to do)
  if (!idle) {
    auto &vt = sh.v[wave];
    const uint16_t *ks = a.k + s.first * a.k_stride + head * kD, *vs = a.v + s.first * a.v_stride + head * kD;
    int token[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) token[t] = min(row0 + 16 * t + n, rows - 1) / R;
    for (int blk = self_begin + wk; blk < self_end; blk += WK) {
      u32x4 k[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
          k[h][ch] = *reinterpret_cast<const u32x4 *>(ks + min(blk * 32 + 16 * h + n, s.rows - 1) * a.k_stride + 32 * ch + 8 * q);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        *reinterpret_cast<u32x4 *>(&vt[4 * x + q][8 * n]) =
            *reinterpret_cast<const u32x4 *>(vs + min(blk * 32 + 4 * x + q, s.rows - 1) * a.v_stride + 8 * n);
      wave_lds_sync();
      u32x4 w[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float y[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) acc = mfma_f16(k[h][ch], raw[t][ch], acc);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[h][i] = acc[i] * sm2;
        }
        if (blk * 32 + 31 > low_token) {  // uniform over the wavefront: some row may not look at all of the block
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (blk * 32 + 16 * h + 4 * q + i > token[t]) y[h][i] = -INFINITY;
        }
        weigh(t, y, [](float) {});
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          l[t] += (y[h][0] + y[h][1]) + (y[h][2] + y[h][3]);
          w[t][2 * h] = pack_f16x2(y[h][0], y[h][1]);
          w[t][2 * h + 1] = pack_f16x2(y[h][2], y[h][3]);
        }
      }
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        u32x4 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // a transposing read: the lane gets its channel of rows 16h + 4q .. + 3
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4 *)(&vt[16 * h + 4 * q + (n >> 2)][16 * nb + 4 * (n & 3)])));
          v[2 * h] = x[0];
          v[2 * h + 1] = x[1];
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) o[t][nb] = mfma_f16(v, w[t], o[t][nb]);
      }
      wave_lds_sync();
    }
  }

  // ================= sums of the wavefronts, and out =================
#pragma unroll
  for (int t = 0; t < QT; ++t) l[t] = column_sum(l[t]);
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
  if constexpr (WK == 1) {
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
    for (int at = threadIdx.x; at < kRows * 32; at += 64 * kPagedWaves) {
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
  const dim3 block(64 * kPagedWaves);
  if (rows <= 16) paged_attention_kernel<G, 1, 4><<<grid(16), block, 0, stream>>>(a);
  else if (rows <= 64) paged_attention_kernel<G, 2, 4><<<grid(32), block, 0, stream>>>(a);
  else paged_attention_kernel<G, 2, 1><<<grid(128), block, 0, stream>>>(a);
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
