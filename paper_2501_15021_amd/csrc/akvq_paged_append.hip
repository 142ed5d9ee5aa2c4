// The write path into pages: rows of a packed chunk are rotated, quantized and packed as in akvq_quantize.hip (the same arithmetic,
// akvq_blockquant.h), each into the page its sequence's table names.
//
// One wavefront owns one 32-row block of one (sequence, kv-head, tensor), as there: pages hold whole blocks, so a block has one page,
// and a block that is only partly new has one writer.  Memory and instruction issue bound it alike (512 bytes in, 72 or 80 out and 11
// operations an element): sixteen prompts of 4096 rows, 32 heads, 251 us, 4.9 TB/s (a large copy: 5.47).  Chunks of 500 to 1000 rows, 13
// sequences of 4 heads, a seventh of the rows 16-bit, 13 us: a round of wavefronts, latency (the list's samples 2 us of it, the overlay 1).
#include "../../include/akvq.h"
#include "akvq_device.h"
#include "akvq_kernels.h"
#include "akvq_rowquant.h"
#include "akvq_blockquant.h"

namespace akvq {

namespace {

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

template <int G, int TENSOR>
__device__ __forceinline__ void paged_append_body(const PagedAppendArgs &a, int *slot_of) {
  constexpr int NG = kD / G;
  const PagedArgs &c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.y / c.Hkv, head = blockIdx.y % c.Hkv, r = lane >> 2, j = lane & 3;
  const ChunkSpan s = append_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (s.rows == 0) return;  // whole wavefront leaves (here and below); no workgroup barrier below
  const int t_end = min(s.len + s.rows, c.row_cap);
  const int blk = s.len / kTokBlock + blockIdx.x * 4 + wave, t0 = blk * kTokBlock;
  if (t0 >= t_end) return;
  const int page = c.table[(size_t)b * c.max_pages + (t0 >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return;
  const int t_page = t0 & ((1 << c.page_shift) - 1);  // the block's first row in its page
  const size_t row0 = (((size_t)page * c.Hkv + head) << c.page_shift) + t_page, blk_word = row0 / kTokBlock * kBlockWords;

  const bool rotate = (TENSOR == 0 ? a.rotate_k : a.rotate_v) != 0;
  const float kappa = rotate ? inv_sqrt128() : 1.0f;
  const float lane_sign = rotate ? quad_sign(j) : 1.0f;  // this lane holds lane_sign * (transformed values)
  const float kappa_s = lane_sign * kappa;
  const uint16_t *src = (TENSOR == 0 ? a.k : a.v) + head * kD;
  const long long stride = TENSOR == 0 ? a.k_stride : a.v_stride;

  bool valid[2];
  u32x4 raw[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int t = t0 + 16 * h + r;
    valid[h] = t >= s.len && t < t_end;
    // rows outside the chunk read a clamped (valid) address; nothing derived from them is stored
    const uint16_t *row = src + (s.first + min(max(t - s.len, 0), s.rows - 1)) * stride;
#pragma unroll
    for (int m = 0; m < 4; ++m) raw[h][m] = *reinterpret_cast<const u32x4 *>(row + 32 * m + 8 * j);
  }
  // a block that is only partly new keeps the other rows' bits of its V words, read before they are needed
  const int ii = r & 3, q = r >> 2;
  const bool partial_blk = t0 < s.len || t0 + kTokBlock > t_end;  // uniform over the wavefront
  u32x2 v_old[2] = {{0u, 0u}, {0u, 0u}};
  if (TENSOR == 1 && partial_blk) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
      v_old[x] = *reinterpret_cast<const u32x2 *>(c.v_codes + blk_word + (size_t)(16 * q + 8 * (j & 1) + 2 * ii + x) * 4 + 2 * (j >> 1));
  }
  const size_t unit = blockIdx.y;
  block_slots(c.sal_idx + unit * c.S_cap, min(max(c.sal_cnt[unit], 0), c.S_cap), t0, lane, slot_of);

  uint32_t kw[2][2], vcode[2][8], vmask_part = 0, meta_out[2][NG];
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
      gq[g] = group_params(mn, mx, kappa, a.clip, tier_two_bit());
      meta_out[h][g] = gq[g].meta | (slot >= 0 ? 0x8000u : 0u);
      gq[g].rcpu *= lane_sign;  // codes are taken from the signed values this lane holds
    }
    if (TENSOR == 0) {
      // K word m/2: slot 8*(m%2)+i at bits 2*slot; built from the top slot down by shift-adds
#pragma unroll
      for (int wq = 0; wq < 2; ++wq) {
        uint32_t word = 0;
#pragma unroll
        for (int at = 15; at >= 0; --at) {
          const int m = 2 * wq + (at >> 3), i = at & 7;
          word = (word << 2) + code_bits(u[m][i], gq[m / (4 / NG)]);
          asm("" : "+v"(word));  // keep the chain one shift-add per code
        }
        kw[h][wq] = word - kPack16Bias;
      }
    } else {
      // V: byte lanes of a partial word: row half h, channel blocks X (m even) / Y (m odd); biases removed after both halves
#pragma unroll
      for (int mp = 0; mp < 2; ++mp)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t part = (code_bits(u[2 * mp + 1][i], gq[(2 * mp + 1) / (4 / NG)]) << 8) + code_bits(u[2 * mp][i], gq[(2 * mp) / (4 / NG)]);
          vcode[mp][i] = h == 0 ? part : (part << 16) + vcode[mp][i];
        }
      if (valid[h]) vmask_part |= 0x0303u << (16 * h);
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
    // chunk 16*j + r: words {2h, 2h+1} belong to row half h
    uint32_t *chunk = c.k_codes + blk_word + (size_t)(16 * j + r) * 4;
    if (valid[0] && valid[1]) *reinterpret_cast<u32x4 *>(chunk) = (u32x4){kw[0][0], kw[0][1], kw[1][0], kw[1][1]};
    else if (valid[0]) *reinterpret_cast<u32x2 *>(chunk) = (u32x2){kw[0][0], kw[0][1]};
    else if (valid[1]) *reinterpret_cast<u32x2 *>(chunk + 2) = (u32x2){kw[1][0], kw[1][1]};
  } else {
    // shift the byte lanes to this row's pair position (ii), then OR over the four rows that share a chunk (all lanes take part)
    uint32_t mask = vmask_part << (2 * ii);
    mask |= dpp_move_u<kRowRor4>(mask);
    mask |= dpp_move_u<kRowRor8>(mask);
    const uint32_t shifted_bias = 0u - (kPack4Bias << (2 * ii));
    uint32_t w[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int mp = 0; mp < 2; ++mp) {
        uint32_t x = (vcode[mp][i] << (2 * ii)) + shifted_bias;
        x |= dpp_move_u<kRowRor4>(x);
        x |= dpp_move_u<kRowRor8>(x);
        w[mp][i] = x;
      }
    if (mask == 0u) return;  // no new row in this lane's chunk
    // each of the four rows stores two of the eight chunks: i = 2*ii and 2*ii + 1 (pinned to registers: an indexed array would be
    // moved to LDS)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      u32x2 o;
#pragma unroll
      for (int mp = 0; mp < 2; ++mp) {
        uint32_t y[4] = {w[mp][x], w[mp][2 + x], w[mp][4 + x], w[mp][6 + x]};
#pragma unroll
        for (int p = 0; p < 4; ++p) asm("" : "+v"(y[p]));
        const uint32_t lo = (ii & 1) ? y[1] : y[0], hi = (ii & 1) ? y[3] : y[2], v = (ii & 2) ? hi : lo;
        o[mp] = (v_old[x][mp] & ~mask) | (v & mask);
      }
      *reinterpret_cast<u32x2 *>(c.v_codes + blk_word + (size_t)(16 * q + 8 * (j & 1) + 2 * ii + x) * 4 + 2 * (j >> 1)) = o;
    }
  }
}

template <int G>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  __shared__ int slot_of_lds[4][kTokBlock];
  int *slot_of = slot_of_lds[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
  if (blockIdx.z == 0) paged_append_body<G, 0>(a, slot_of);
  else paged_append_body<G, 1>(a, slot_of);
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

// One generated token of every sequence: a wavefront a row and tensor (append_row_wave), the block's place in its page put under the place
// that the row would have in a plane of its own.  Latency bound: sixteen sequences, 32 heads, 3.2 us (the block kernel 4.9).
template <int G>
__global__ __launch_bounds__(64) void paged_append_row_kernel(PagedAppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t code_lds[kD];
  __shared__ __attribute__((aligned(16))) uint16_t row_lds[kD];
  const PagedArgs &c = a.c;
  const int unit = blockIdx.x, b = unit / c.Hkv, head = unit % c.Hkv;
  const ChunkSpan s = append_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (s.rows == 0) return;
  const int page = c.table[(size_t)b * c.max_pages + (s.len >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return;
  const int t0 = s.len & ~(kTokBlock - 1);
  const long long row0 = ((((long long)page * c.Hkv + head) << c.page_shift) + (t0 & ((1 << c.page_shift) - 1))) - t0;
  QuantArgs q = {};
  q.k_new = a.k + s.first * a.k_stride + (head - unit) * kD;  // (append_row_wave adds what the unit's row and planes lie behind)
  q.v_new = a.v + s.first * a.v_stride + (head - unit) * kD;
  q.k_codes = c.k_codes + row0 * (kBlockWords / kTokBlock);
  q.v_codes = c.v_codes + row0 * (kBlockWords / kTokBlock);
  q.k_meta = c.k_meta + row0 * (kD / G);
  q.v_meta = c.v_meta + row0 * (kD / G);
  q.k_sal = c.k_sal;
  q.v_sal = c.v_sal;
  q.sal_idx = c.sal_idx;
  q.sal_cnt = c.sal_cnt;
  q.Hkv = c.Hkv;
  q.S_cap = c.S_cap;
  q.T_len = s.len;
  q.clip = a.clip;
  q.rotate_k = a.rotate_k;
  q.rotate_v = a.rotate_v;
  append_row_wave<G, SampledSlot>(q, unit, blockIdx.y, threadIdx.x, code_lds, row_lds);
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs &a, int G, hipStream_t stream) {
  if (a.c.max_rows == 1) {
    const dim3 grid(a.c.B * a.c.Hkv, 2);
    if (G == 128) paged_append_row_kernel<128><<<grid, dim3(64), 0, stream>>>(a);
    else paged_append_row_kernel<64><<<grid, dim3(64), 0, stream>>>(a);
    return hipGetLastError();
  }
  const int blocks = (a.c.max_rows + 30) / kTokBlock + 1;  // that max_rows rows can touch, wherever they start
  const dim3 grid((blocks + 3) / 4, a.c.B * a.c.Hkv, 2), block(256);
  if (G == 128) paged_append_kernel<128><<<grid, block, 0, stream>>>(a);
  else paged_append_kernel<64><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace akvq
