// One 32-row block of the cache in pages, and one row of it, as the calls that write chunks into pages share them: rows are rotated, quantized and
// packed as in akvq_quantize.hip (the same arithmetic, akvq_blockquant.h), to 2 or 4 bits a code.
#pragma once
#include "akvq_blockquant.h"
#include "akvq_device.h"
#include "akvq_kernels.h"
#include "akvq_rowquant.h"

#include <type_traits>

namespace akvq {
namespace {

template <int BITS>
__device__ __forceinline__ TierQ tier_of() {  // levels, and the largest scale that binary16 holds
  return {__uint_as_float(BITS == 2 ? 0x3EAAAAABu : 0x3D888889u), 0x7BFFu};
}
// Eq. 3 for one value: the bits of 1.5 * 2^23 + code
template <int BITS>
__device__ __forceinline__ uint32_t code_bits_of(float u, const GroupQ &g) {
  float t = __fmaf_rn(u, g.rcpu, g.magic_zero);
  t = fminf(fmaxf(t, kMagic), kMagic + (float)((1 << BITS) - 1));
  return __float_as_uint(t);
}
constexpr uint32_t kPack8Bias = (uint32_t)(0x4B400000ull * 0x11111111ull);  // sum over s < 8 of kMagicBits << 4s

// Eight words, each or-ed over the four lanes that lie 4 apart in a row of 16.  Assembly, because the compiler spends a move on every other one of these.
// (The leading s_nop covers the wait states of a DPP read after a VALU write of its source and after an EXEC write; inside, seven
// instructions lie between a write and its read.)
__device__ __forceinline__ void or_over_rows(uint32_t (&x)[8]) {
#define AKVQ_OR8(CTRL)                                                                                                     \
  "v_or_b32_dpp %0, %0, %0 " CTRL "\n\tv_or_b32_dpp %1, %1, %1 " CTRL "\n\tv_or_b32_dpp %2, %2, %2 " CTRL                 \
  "\n\tv_or_b32_dpp %3, %3, %3 " CTRL "\n\tv_or_b32_dpp %4, %4, %4 " CTRL "\n\tv_or_b32_dpp %5, %5, %5 " CTRL             \
  "\n\tv_or_b32_dpp %6, %6, %6 " CTRL "\n\tv_or_b32_dpp %7, %7, %7 " CTRL "\n\t"
  asm volatile("s_nop 4\n\t" AKVQ_OR8("row_ror:4 row_mask:0xf bank_mask:0xf") AKVQ_OR8("row_ror:8 row_mask:0xf bank_mask:0xf")
               : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
#undef AKVQ_OR8
}

// slot_of[r] = rank in the ascending list of the block's row t0 + r, or -1.  The block's entries are one run of at most 32: the list is
// sampled until the run starts within 64 entries of a sample, and two loads cover it.
__device__ __forceinline__ void block_slots(const int32_t *sidx, int cnt, int t0, int lane, int *slot_of) {
  if (lane < kTokBlock) slot_of[lane] = -1;
  int base = 0, span = cnt;
  while (span > 64) {
    const int step = (span + 63) >> 6, at = base + lane * step;
    const int e = lane * step < span && at < cnt ? sidx[at] : 0x7FFFFFFF;
    const int below = __popcll(__ballot(e < t0));
    base += max(below - 1, 0) * step;
    span = step;
  }
  int e[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) e[x] = base + 64 * x + lane < cnt ? sidx[base + 64 * x + lane] : 0x7FFFFFFF;
  wave_lds_sync();
#pragma unroll
  for (int x = 0; x < 2; ++x)
    if (e[x] >= t0 && e[x] < t0 + kTokBlock) slot_of[e[x] - t0] = base + 64 * x + lane;
  wave_lds_sync();
}

// One wavefront writes the new rows of a block of one (sequence, KV head) and tensor: rows t0 .. t0 + 31 of the sequence, whose first one is row
// row0 of the pools.  raw[h]: row 16h + r as it arrives, lane (r, j): channels 32m + 8j .. + 7; valid[h]: whether it is new; partial_blk: some
// row is not (uniform over the wavefront).
template <int G, int BITS, int TENSOR>
__device__ __forceinline__ void append_block(const PagedArgs &c, size_t unit, int t0, size_t row0, const u32x4 (&raw)[2][4], const bool (&valid)[2],
                                             bool partial_blk, bool rotate, float clip, int *slot_of, int lane) {
  constexpr int NG = kD / G;
  const int r = lane >> 2, j = lane & 3, ii = r & 3, q = r >> 2;
  const size_t blk_word = row0 / kTokBlock * (BITS * kBlockWords / 2);
  const float kappa = rotate ? inv_sqrt128() : 1.0f;
  const float lane_sign = rotate ? quad_sign(j) : 1.0f;  // this lane holds lane_sign * (transformed values)
  const float kappa_s = lane_sign * kappa;
  // a block that is only partly new keeps the other rows' bits of its V words, read before they are needed
  typedef typename std::conditional<BITS == 2, u32x2, u32x4>::type VWords;  // of one chunk and channel block half
  auto v_at = [&](int x) {  // eight chunks of four rows: two a row
    const int chunk = 16 * q + 8 * (j & 1) + 2 * ii + x;
    return reinterpret_cast<VWords *>(c.v_codes + blk_word + (BITS == 2 ? chunk * 4 + 2 * (j >> 1) : (j >> 1) * 256 + chunk * 4));
  };
  VWords v_old[2] = {};
  if (TENSOR == 1 && partial_blk) {
#pragma unroll
    for (int x = 0; x < 2; ++x) v_old[x] = *v_at(x);
  }
  block_slots(c.sal_idx + unit * c.S_cap, min(max(c.sal_cnt[unit], 0), c.S_cap), t0, lane, slot_of);

  uint32_t kw[2][BITS], vcode[BITS][8], vmask_part = 0, meta_out[2][NG];  // (words of a row; of the block's values, before they are joined)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int slot = slot_of[16 * h + r];
    float u[4][8];
    if (rotate) {
      wht128_quad(raw[h], u, j);
    } else {
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          u[m][2 * w] = half_bits_to_float(raw[h][m][w] & 0xFFFFu);
          u[m][2 * w + 1] = half_bits_to_float(raw[h][m][w] >> 16);
        }
    }
    if (valid[h] && slot >= 0)
      store_bf16_row<TENSOR>(u, kappa_s, j, c.k_sal + unit * c.S_cap * kD, c.v_sal + unit * c.S_cap * kD, slot, true);
    GroupQ gq[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      constexpr int MPG = 4 / NG;  // m-slices per group
      float mn = u[g * MPG][0], mx = u[g * MPG][0];
#pragma unroll
      for (int m = g * MPG; m < (g + 1) * MPG; ++m)
#pragma unroll
        for (int i = 0; i < 8; i += 2) minmax3(mn, mx, u[m][i], u[m][i + 1]);
      if (lane_sign < 0.0f) {  // extrema of the true values
        const float t = mn;
        mn = -mx;
        mx = -t;
      }
      quad_minmax(mn, mx);
      gq[g] = group_params(mn, mx, kappa, clip, tier_of<BITS>());
      meta_out[h][g] = gq[g].meta | (slot >= 0 ? 0x8000u : 0u);
      gq[g].rcpu *= lane_sign;  // codes are taken from the signed values this lane holds
    }
    if (TENSOR == 0) {
      // K word m/2: slot 8*(m%2)+i at bits 2*slot, or word m: i at bits 4*i; built from the top slot down by shift-adds
      constexpr int kSlots = 32 / BITS;
#pragma unroll
      for (int wq = 0; wq < BITS; ++wq) {
        uint32_t word = 0;
#pragma unroll
        for (int at = kSlots - 1; at >= 0; --at) {
          const int m = BITS == 2 ? 2 * wq + (at >> 3) : wq, i = at & 7;
          word = (word << BITS) + code_bits_of<BITS>(u[m][i], gq[m / (4 / NG)]);
          asm("" : "+v"(word));  // keep the chain one shift-add per code
        }
        kw[h][wq] = word - (BITS == 2 ? kPack16Bias : kPack8Bias);
      }
    } else if constexpr (BITS == 2) {
      // V: byte lanes of a partial word: row half h, channel blocks X (m even) / Y (m odd); biases removed after both halves
#pragma unroll
      for (int mp = 0; mp < 2; ++mp)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t part = (code_bits_of<2>(u[2 * mp + 1][i], gq[(2 * mp + 1) / (4 / NG)]) << 8) + code_bits_of<2>(u[2 * mp][i], gq[(2 * mp) / (4 / NG)]);
          vcode[mp][i] = h == 0 ? part : (part << 16) + vcode[mp][i];
        }
      if (valid[h]) vmask_part |= 0x0303u << (16 * h);
    } else {
      // V: one channel a word, row half h (the upper half's bias leaves the word)
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t part = code_bits_of<4>(u[m][i], gq[m / (4 / NG)]);
          vcode[m][i] = h == 0 ? part : (part << 16) + vcode[m][i];
        }
      if (valid[h]) vmask_part |= 0xFu << (16 * h);
    }
  }

  if (j == 0) {
    uint32_t *meta = TENSOR == 0 ? c.k_meta : c.v_meta;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (valid[h]) {
#pragma unroll
        for (int g = 0; g < NG; ++g) meta[(row0 + 16 * h + r) * NG + g] = meta_out[h][g];
      }
  }
  if (TENSOR == 0) {
    if constexpr (BITS == 2) {
      // chunk 16*j + r: words {2h, 2h+1} belong to row half h
      uint32_t *chunk = c.k_codes + blk_word + (size_t)(16 * j + r) * 4;
      if (valid[0] && valid[1]) *reinterpret_cast<u32x4 *>(chunk) = (u32x4){kw[0][0], kw[0][1], kw[1][0], kw[1][1]};
      else if (valid[0]) *reinterpret_cast<u32x2 *>(chunk) = (u32x2){kw[0][0], kw[0][1]};
      else if (valid[1]) *reinterpret_cast<u32x2 *>(chunk + 2) = (u32x2){kw[1][0], kw[1][1]};
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)  // a row's words are its own
        if (valid[h]) *reinterpret_cast<u32x4 *>(c.k_codes + blk_word + 256 * h + (size_t)(16 * j + r) * 4) = (u32x4){kw[h][0], kw[h][1], kw[h][2], kw[h][3]};
    }
  } else {
    // shift the codes to this row's place (ii), then OR over the four rows that share a chunk (all lanes take part)
    uint32_t mask = vmask_part << (BITS * ii);
    mask |= dpp_move_u<kRowRor4>(mask);
    mask |= dpp_move_u<kRowRor8>(mask);
    const uint32_t shifted_bias = 0u - ((BITS == 2 ? kPack4Bias : kMagicBits) << (BITS * ii));
    uint32_t w[BITS][8];
#pragma unroll
    for (int mp = 0; mp < BITS; ++mp) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[mp][i] = (vcode[mp][i] << (BITS * ii)) + shifted_bias;
      or_over_rows(w[mp]);
    }
    if (mask == 0u) return;  // no new row in this lane's chunk
    // each of the four rows stores two of the eight chunks: i = 2*ii and 2*ii + 1 (pinned to registers: an indexed array would be
    // moved to LDS)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      VWords o;
#pragma unroll
      for (int mp = 0; mp < BITS; ++mp) {
        uint32_t y[4] = {w[mp][x], w[mp][2 + x], w[mp][4 + x], w[mp][6 + x]};
#pragma unroll
        for (int p = 0; p < 4; ++p) asm("" : "+v"(y[p]));
        const uint32_t lo = (ii & 1) ? y[1] : y[0], hi = (ii & 1) ? y[3] : y[2], v = (ii & 2) ? hi : lo;
        o[mp] = (v_old[x][mp] & ~mask) | (v & mask);
      }
      *v_at(x) = o;
    }
  }
}

// A row's place in its list of salient rows as RowSlot, but sampled: lists of pages are as long as the prompts' text.
struct SampledSlot : RowSlot {
  using RowSlot::RowSlot;
  __device__ __forceinline__ int find(int t) const {
    const int n = min(max(cnt, 0), cap);
    int base = 0, e = first_entry;
    if (n > kWave) {
      for (int span = n; span > 1;) {  // the row's entry, if there is one, is in [base, base + span)
        const int step = (span + 63) >> 6, at = base + lane * step;
        e = lane * step < span && at < n ? sidx[at] : 0x7FFFFFFF;
        base += max(__popcll(__ballot(e <= t)) - 1, 0) * step;
        span = step;
      }
      return __ballot(e == t) != 0ull ? base : -1;
    }
    const unsigned long long hit = __ballot(lane < n && e == t);
    return hit != 0ull ? __builtin_ctzll(hit) : -1;
  }
};
// what RowSlot reads of its arguments
__device__ __forceinline__ QuantArgs list_of(const PagedArgs &c) {
  QuantArgs q = {};
  q.sal_idx = c.sal_idx;
  q.sal_cnt = c.sal_cnt;
  q.S_cap = c.S_cap;
  return q;
}

// One row of a block, by one wavefront: lane l holds channels l (x0) and l + 64 (x1) as numbers, not yet rotated.  row0: the pools' row of the
// block's first one; code_lds, row_lds: this wavefront's alone.  As append_row_wave (akvq_rowquant.h), to 2 or 4 bits a code.
template <int G, int BITS, int TENSOR>
__device__ __forceinline__ void append_row(const PagedArgs &c, size_t unit, int t, size_t row0, float x0, float x1, int slot, uint32_t (&old)[2],
                                           bool rotate, float clip, int lane, uint8_t *code_lds, uint16_t *row_lds) {
  constexpr int NG = kD / G;
  const int half = (t % kTokBlock) >> 4, n16 = t & 15, q = n16 >> 2, ii = n16 & 3;
  const float kappa = rotate ? inv_sqrt128() : 1.0f;
  if (rotate) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      x0 = xor_butterfly(x0, s, lane);
      x1 = xor_butterfly(x1, s, lane);
    }
    const float lo = x0 + x1, hi = x0 - x1;
    x0 = lo;
    x1 = hi;
  }
  GroupQ gq[2];
  if constexpr (NG == 1) {
    gq[0] = gq[1] = group_params(wave_min_all(fminf(x0, x1)), wave_max_all(fmaxf(x0, x1)), kappa, clip, tier_of<BITS>());
  } else {
    gq[0] = group_params(wave_min_all(x0), wave_max_all(x0), kappa, clip, tier_of<BITS>());
    gq[1] = group_params(wave_min_all(x1), wave_max_all(x1), kappa, clip, tier_of<BITS>());
  }
  constexpr uint32_t kMask = (1u << BITS) - 1u;
  code_lds[lane] = (uint8_t)(code_bits_of<BITS>(x0, gq[0]) & kMask);
  code_lds[lane + 64] = (uint8_t)(code_bits_of<BITS>(x1, gq[1]) & kMask);
  const uint32_t y0 = pack_bf16x2(scaled_row_value(x0, kappa), 0.0f) & 0xFFFFu, y1 = pack_bf16x2(scaled_row_value(x1, kappa), 0.0f) & 0xFFFFu;
  if (TENSOR == 0) {
    row_lds[lane] = (uint16_t)y0;
    row_lds[lane + 64] = (uint16_t)y1;
  }
  wave_lds_sync();
  if (lane == 0) {
    uint32_t *meta = (TENSOR == 0 ? c.k_meta : c.v_meta) + (row0 + t % kTokBlock) * NG;
#pragma unroll
    for (int g = 0; g < NG; ++g) meta[g] = gq[g].meta | (slot >= 0 ? 0x8000u : 0u);
  }
  const size_t blk_word = row0 / kTokBlock * (BITS * kBlockWords / 2);
  if (TENSOR == 0) {
    if (lane < 4 * BITS) {  // the words hold this row's codes only
      const int j = lane / BITS, w = lane % BITS;
      uint32_t word = 0u;
#pragma unroll
      for (int x = 0; x < 4 / BITS; ++x) {  // slices of eight channels
        const u32x2 eight = *reinterpret_cast<const u32x2 *>(&code_lds[32 * (BITS == 2 ? 2 * w + x : w) + 8 * j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) word |= ((eight[i >> 2] >> (8 * (i & 3))) & kMask) << (BITS * (8 * x + i));
      }
      c.k_codes[blk_word + (BITS == 2 ? (16 * j + n16) * 4 + 2 * half + w : 256 * half + (16 * j + n16) * 4 + w)] = word;
    }
  } else {
    uint32_t *at = c.v_codes + blk_word + 64 * q + lane;  // word w = lane % 4 of chunk 16q + lane / 4
    const int n = lane >> 2, w = lane & 3;
    if constexpr (BITS == 2) {  // channel blocks nb = w / 2 + 4 (w % 2) and nb + 2, 8 bits apart
      const int nb = (w >> 1) + 4 * (w & 1), bit = 16 * half + 2 * ii;
      const uint32_t mask = (3u << bit) | (3u << (bit + 8));
      *at = (old[0] & ~mask) | ((uint32_t)code_lds[16 * nb + n] << bit) | ((uint32_t)code_lds[16 * (nb + 2) + n] << (bit + 8));
    } else {  // channel blocks 2w and 2w + 1, 256 words apart
      const int bit = 16 * half + 4 * ii;
#pragma unroll
      for (int x = 0; x < 2; ++x) at[256 * x] = (old[x] & ~(15u << bit)) | ((uint32_t)code_lds[16 * (2 * w + x) + n] << bit);
    }
  }
  if (slot < 0) return;
  if (TENSOR == 0) {
    reinterpret_cast<uint32_t *>(c.k_sal + (unit * c.S_cap + slot) * kD)[lane] = reinterpret_cast<const uint32_t *>(row_lds)[lane];
  } else {
    const int sb = slot >> 5, sh = (slot & 31) >> 4, sr = slot & 15, sq = sr >> 2, sii = sr & 3;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = lane + 64 * k, nb = e >> 4, n = e & 15;
      c.v_sal[unit * c.S_cap * kD + (size_t)sb * 4096 + nb * 512 + (16 * sq + n) * 8 + 2 * sii + sh] = (uint16_t)(k == 0 ? y0 : y1);
    }
  }
}
// The V words that a row's codes go into, as they are (asked for early)
template <int BITS>
__device__ __forceinline__ void old_v_words(const PagedArgs &c, int t, size_t row0, int lane, uint32_t (&old)[2]) {
  const uint32_t *at = c.v_codes + row0 / kTokBlock * (BITS * kBlockWords / 2) + 64 * ((t & 15) >> 2) + lane;
  old[0] = at[0];
  old[1] = BITS == 4 ? at[256] : 0u;
}

}  // namespace
}  // namespace akvq
