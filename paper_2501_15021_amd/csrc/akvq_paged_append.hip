// The write path into pages: rows of a packed chunk are rotated, quantized and packed as in akvq_quantize.hip (the same arithmetic,
// akvq_pageblock.h), each into the page its sequence's table names.
//
// One wavefront owns one 32-row block of one (sequence, kv-head, tensor), as there: pages hold whole blocks, so a block has one page,
// and a block that is only partly new has one writer.  Memory and instruction issue bound it alike (512 bytes in, 72 or 80 out and 11
// operations an element): sixteen prompts of 4096 rows, 32 heads, 251 us, 4.9 TB/s (a large copy: 5.47).  Chunks of 540 to 1024 rows of
// 12 sequences, 4 heads, a seventh of the rows 16-bit, 14.7 us from memory and 11.4 where the last cache has the rows, without 16-bit ones 11.2 and
// 9.3: a round of wavefronts, latency.
//   4 bits a code (twice the words, the same loads and rotation; 13 operations an element): 12 prompts of up to 4095 rows, 32 heads, 149 us,
// 4.7 TB/s, the vector unit 77 % busy; one row of each of 16 sequences as with 2 bits.
#include "../../include/akvq.h"
#include "akvq_device.h"
#include "akvq_kernels.h"
#include "akvq_pageblock.h"

namespace akvq {

namespace {

template <int G, int BITS, int TENSOR>
__device__ __forceinline__ void paged_append_body(const PagedAppendArgs &a, int *slot_of) {
  const PagedArgs &c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int at = a.heads_first ? blockIdx.x : blockIdx.y, over = at / c.Hkv, head = at % c.Hkv;
  const int b = a.heads_first ? blockIdx.y : over, group = a.heads_first ? over : blockIdx.x, r = lane >> 2, j = lane & 3;
  const ChunkSpan s = append_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (s.rows == 0) return;  // whole wavefront leaves (here and below); no workgroup barrier below
  const int t_end = min(s.len + s.rows, c.row_cap);
  const int blk = s.len / kTokBlock + group * 4 + wave, t0 = blk * kTokBlock;
  if (t0 >= t_end) return;
  const int page = c.table[(size_t)b * c.max_pages + (t0 >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return;
  const int t_page = t0 & ((1 << c.page_shift) - 1);  // the block's first row in its page
  const size_t row0 = (((size_t)page * c.Hkv + head) << c.page_shift) + t_page;

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
  append_block<G, BITS, TENSOR>(c, b * c.Hkv + head, t0, row0, raw, valid, t0 < s.len || t0 + kTokBlock > t_end,
                                (TENSOR == 0 ? a.rotate_k : a.rotate_v) != 0, a.clip, slot_of, lane);
}

template <int G, int BITS>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  __shared__ int slot_of_lds[4][kTokBlock];
  int *slot_of = slot_of_lds[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
  if (blockIdx.z == 0) paged_append_body<G, BITS, 0>(a, slot_of);
  else paged_append_body<G, BITS, 1>(a, slot_of);
}

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

// The same into pages of 4-bit codes: the row's words are joined with their neighbours' nibbles, which for values lie in words of four rows.
template <int G>
__global__ __launch_bounds__(64) void paged4_append_row_kernel(PagedAppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t code_lds[kD];
  __shared__ __attribute__((aligned(16))) uint16_t row_lds[kD];
  const PagedArgs &c = a.c;
  const int unit = blockIdx.x, b = unit / c.Hkv, head = unit % c.Hkv, lane = threadIdx.x;
  const ChunkSpan s = append_span(c.seq_len[b], c.row_start[b], c.row_start[b + 1], c);
  if (s.rows == 0) return;
  const int page = c.table[(size_t)b * c.max_pages + (s.len >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return;
  const size_t row0 = (((size_t)page * c.Hkv + head) << c.page_shift) + (s.len & ((1 << c.page_shift) - 1) & ~(kTokBlock - 1));
  const uint16_t *row = blockIdx.y == 0 ? a.k + s.first * a.k_stride + head * kD : a.v + s.first * a.v_stride + head * kD;
  const SampledSlot list(list_of(c), unit, lane);
  const float x0 = half_bits_to_float(row[lane]), x1 = half_bits_to_float(row[lane + 64]);
  uint32_t old[2] = {0u, 0u};
  if (blockIdx.y == 1) old_v_words<4>(c, s.len, row0, lane, old);
  const int slot = list.find(s.len);
  if (blockIdx.y == 0) append_row<G, 4, 0>(c, unit, s.len, row0, x0, x1, slot, old, a.rotate_k != 0, a.clip, lane, code_lds, row_lds);
  else append_row<G, 4, 1>(c, unit, s.len, row0, x0, x1, slot, old, a.rotate_v != 0, a.clip, lane, code_lds, row_lds);
}

template <int G, int BITS>
hipError_t launch_blocks(PagedAppendArgs a, hipStream_t stream) {
  const int blocks = (a.c.max_rows + 30) / kTokBlock + 1, groups = (blocks + 3) / 4;  // blocks that max_rows rows can touch, wherever they start
  // Few workgroups: those of the same rows, whose heads lie next to each other in the chunk, run together.  Measured, us, that way and a head's together:
  // 12 chunks of 540 to 1024 rows, 4 of 36 heads (936 workgroups in the grid, rows from memory) 11.1 and 11.4, with a seventh of them 16-bit 14.5 and 14.6, 40 of 700 (1920) 15.7 and 16.3, 1 of 300, 32 heads (192) 4.5 and 4.8;
  // 6 of 4000, 8 heads (3072) 25.6 and 25.2, 12 of up to 4095, 32 heads (25344) 140 and 137; 4 bits alike.
  a.heads_first = 2ll * groups * a.c.B * a.c.Hkv <= 2048 ? 1 : 0;
  const dim3 grid = a.heads_first ? dim3(groups * a.c.Hkv, a.c.B, 2) : dim3(groups, a.c.B * a.c.Hkv, 2);
  paged_append_kernel<G, BITS><<<grid, dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs &a, int G, hipStream_t stream) {
  if (a.c.max_rows > 1) return G == 128 ? launch_blocks<128, 2>(a, stream) : launch_blocks<64, 2>(a, stream);
  const dim3 grid(a.c.B * a.c.Hkv, 2);
  if (G == 128) paged_append_row_kernel<128><<<grid, dim3(64), 0, stream>>>(a);
  else paged_append_row_kernel<64><<<grid, dim3(64), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged4_append(const PagedAppendArgs &a, int G, hipStream_t stream) {
  if (a.c.max_rows > 1) return G == 128 ? launch_blocks<128, 4>(a, stream) : launch_blocks<64, 4>(a, stream);
  const dim3 grid(a.c.B * a.c.Hkv, 2);
  if (G == 128) paged4_append_row_kernel<128><<<grid, dim3(64), 0, stream>>>(a);
  else paged4_append_row_kernel<64><<<grid, dim3(64), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace akvq
