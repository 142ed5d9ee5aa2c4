// A chunk on its way into the cache in pages, in one launch: queries and keys are turned by their positions (akvq_turn.h), turned keys and
// values are rotated, quantized and packed (akvq_pageblock.h), to 2 or 4 bits a code.
//
// A workgroup takes 32 rows of a sequence that share a block of the cache, and some of their heads.  The angles of these rows, 64 bits each, are
// formed once for all heads and lie in LDS; then its eight wavefronts take a head each: of the queries (turned: 16 bytes a lane, both sides of eight
// pairs), of the keys (turned in the layout of the transform, written out and quantized) or of the values (quantized).
//   Queries and keys out are written with the non-temporal hint: 8 x 4096 rows of 32 heads 302 us, 4.9 TB/s (a large copy: 5.47; plain stores 313,
// with four wavefronts a workgroup 324), and attention after it takes as long.  Chunks of 540 to 1024 rows of 12 sequences, 28 / 4 heads, a seventh of
// the rows 16-bit, 2 bits: 46 us from memory, 36 where the last cache has the rows (without 16-bit rows 43 from memory).  888 workgroups with rows, of
// which 512 run at a time, and every third has four heads for its eight wavefronts; each is a chain of lengths, positions, angles and two heads a
// wavefront.  The next head asked for ahead (151 registers in place of 120) takes as long.
#include "akvq_device.h"
#include "akvq_kernels.h"
#include "akvq_pageblock.h"
#include "akvq_turn.h"

namespace akvq {
namespace {

constexpr int kTurnWaves = 8;
constexpr int kTurnStride = 68;  // of a row's cosines in LDS: sixteen rows' 16-byte pieces fall on all banks

// The rows that a call turns, and where they go: rows first .. first + rows - 1 of the chunk are rows base, base + 1, ... of the sequence; those
// in front of `end` have a place in the cache.  A length that names no row of the table leaves none, and the rows are turned all the same.
struct TurnSpan { int base, first, rows, end; };
__device__ __forceinline__ TurnSpan turn_span(const PagedArgs &c, int b) {
  const int len = c.seq_len[b];
  const ChunkSpan s = chunk_span(0, c.row_start[b], c.row_start[b + 1], c);
  const bool place = len >= 0 && len < c.row_cap;
  const int base = place ? len : 0;
  return {base, s.first, s.rows, place ? min(base + s.rows, c.row_cap) : 0};
}

template <int G, int BITS, bool INTERLEAVED>
__global__ __launch_bounds__(64 * kTurnWaves, 4) void paged_turn_kernel(PagedTurnArgs a, int heads_per_group) {
  __shared__ __attribute__((aligned(16))) float cos_lds[kTokBlock][kTurnStride], sin_lds[kTokBlock][kTurnStride];
  __shared__ int slot_of_lds[kTurnWaves][kTokBlock];
  const PagedArgs &c = a.append.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.y, Hkv = c.Hkv, turned_heads = Hkv + a.Hq, heads = turned_heads + Hkv;  // keys, queries, values
  const int first_head = blockIdx.z * heads_per_group, end_head = min(first_head + heads_per_group, heads);
  const TurnSpan s = turn_span(c, b);
  const int t0 = (s.base / kTokBlock + blockIdx.x) * kTokBlock, t_turned = s.base + s.rows;
  if (s.rows == 0 || t0 >= t_turned) return;  // whole workgroup
  int page = -1;
  if (t0 < s.end) page = c.table[(size_t)b * c.max_pages + (t0 >> c.page_shift)];
  const bool stored = page >= 0 && page < c.n_pages;
  const int dim = a.plan.dim;
  if (first_head < turned_heads) {  // uniform
    for (int r = wave; r < kTokBlock; r += kTurnWaves)
      if (t0 + r >= s.base && t0 + r < t_turned && lane < dim / 2) {
        const Turn t = pair_turn(a.plan, lane, s.first + (t0 + r - s.base));
        cos_lds[r][lane] = t.c;
        sin_lds[r][lane] = t.s;
      }
    __syncthreads();
  }
  // the chunk's row that is row t of the sequence; rows outside of the chunk read a clamped (valid) one, and nothing derived from it is stored
  auto chunk_row = [&](int t) { return (long long)s.first + min(max(t - s.base, 0), s.rows - 1); };
  auto turns_row = [&](int t) { return t >= s.base && t < t_turned; };
  const bool partial = t0 < s.base || t0 + kTokBlock > s.end;
  auto pool_row = [&](int head) { return (((size_t)max(page, 0) * Hkv + head) << c.page_shift) + (t0 & ((1 << c.page_shift) - 1)); };
  // Sines, cosines and addresses are made again for every head: kept for all of them they take 100 registers, and two wavefronts a SIMD are left.
  auto again = [&] {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  auto load_rows = [&](const uint16_t *from, long long stride, int l, u32x4 (&raw)[2][4], bool (&valid)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = t0 + 16 * h + (l >> 2);
      valid[h] = t >= s.base && t < s.end;
      const uint16_t *row = from + chunk_row(t) * stride + 8 * (l & 3);
#pragma unroll
      for (int m = 0; m < 4; ++m) raw[h][m] = *reinterpret_cast<const u32x4 *>(row + 32 * m);
    }
  };

  auto write = [&](u32x4 *to, const u32x4 &x) {
    __builtin_nontemporal_store(x, to);
  };

  int job = first_head + wave;
  for (; job < min(end_head, Hkv); job += kTurnWaves) {  // a key head
    const int l = again(), r = l >> 2, j = l & 3;
    const uint16_t *from = a.append.k + job * kD;
    bool valid[2];
    u32x4 raw[2][4];
    load_rows(from, a.append.k_stride, l, raw, valid);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = 16 * h + r;
      if (!INTERLEAVED && dim < kD) {  // the other side of a chunk's pairs may be another lane's: read again
        const int half = dim / 16;  // in chunks
        const uint16_t *at = from + chunk_row(t0 + row) * a.append.k_stride;
        u32x4 other[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int chunk = 4 * m + j;
          other[m] = *reinterpret_cast<const u32x4 *>(at + 8 * (chunk < half ? chunk + half : chunk < 2 * half ? chunk - half : chunk));
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int chunk = 4 * m + j, pair = 8 * (chunk < half ? chunk : chunk - half);
          if (chunk < 2 * half) {
            const uint32_t flip = chunk < half ? 0x80000000u : 0u;  // (x, y) -> x c - y s; y c + x s
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              float v[2];
              const uint32_t ow = raw[h][m][w], pw = other[m][w];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float cs = cos_lds[row][pair + 2 * w + e], sn = __uint_as_float(__float_as_uint(sin_lds[row][pair + 2 * w + e]) ^ flip);
                const float own = half_bits_to_float(e ? ow >> 16 : ow & 0xFFFFu), oth = half_bits_to_float(e ? pw >> 16 : pw & 0xFFFFu);
                v[e] = __fmaf_rn(own, cs, __fmul_rn(oth, sn));
              }
              raw[h][m][w] = turned_pair(v[0], v[1]);
            }
          }
        }
      } else if (INTERLEAVED) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int pair = 4 * (4 * m + j);
          if (2 * pair < dim) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              float v0, v1;
              const uint32_t x = raw[h][m][w];
              turn_word(x, cos_lds[row][pair + w], sin_lds[row][pair + w], v0, v1);
              raw[h][m][w] = turned_pair(v0, v1);
            }
          }
        }
      } else {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float cs[8], sn[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) { cs[e] = cos_lds[row][32 * m + 8 * j + e]; sn[e] = sin_lds[row][32 * m + 8 * j + e]; }
          turn_chunks<false>(raw[h][m], raw[h][m + 2], cs, sn);
        }
      }
      if (turns_row(t0 + row)) {
        uint16_t *dst = a.k_out + chunk_row(t0 + row) * a.k_out_stride + job * kD + 8 * j;
#pragma unroll
        for (int m = 0; m < 4; ++m) write(reinterpret_cast<u32x4 *>(dst + 32 * m), raw[h][m]);
      }
    }
    if (stored) append_block<G, BITS, 0>(c, (size_t)b * Hkv + job, t0, pool_row(job), raw, valid, partial, true, a.append.clip, slot_of_lds[wave], l);
  }
  for (; job < min(end_head, turned_heads); job += kTurnWaves) {  // a query head: eight rows at a time
    const int l = again(), head = job - Hkv, o = l & 7, turning = dim / 16;
    const bool turns = o < turning;
    const int at0 = INTERLEAVED ? 16 * o : turns ? 8 * o : dim + 16 * (o - turning), at1 = at0 + (!INTERLEAVED && turns ? dim / 2 : 8);
    u32x4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t *src = a.q + chunk_row(t0 + 8 * i + (l >> 3)) * a.q_stride + head * kD;
      x[i] = *reinterpret_cast<const u32x4 *>(src + at0);
      y[i] = *reinterpret_cast<const u32x4 *>(src + at1);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + (l >> 3);
      if (turns) {
        float cs[8], sn[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = cos_lds[row][8 * o + e]; sn[e] = sin_lds[row][8 * o + e]; }
        turn_chunks<INTERLEAVED>(x[i], y[i], cs, sn);
      }
      if (turns_row(t0 + row)) {
        uint16_t *dst = a.q_out + chunk_row(t0 + row) * a.q_out_stride + head * kD;
        write(reinterpret_cast<u32x4 *>(dst + at0), x[i]);
        write(reinterpret_cast<u32x4 *>(dst + at1), y[i]);
      }
    }
  }
  if (!stored) return;
  for (; job < end_head; job += kTurnWaves) {  // a value head
    const int l = again(), head = job - turned_heads;
    bool valid[2];
    u32x4 raw[2][4];
    load_rows(a.append.v + head * kD, a.append.v_stride, l, raw, valid);
    append_block<G, BITS, 1>(c, (size_t)b * Hkv + head, t0, pool_row(head), raw, valid, partial, a.append.rotate_v != 0, a.append.clip, slot_of_lds[wave], l);
  }
}

// One generated token of every sequence: a wavefront a head.  Latency bound.
template <int G, int BITS>
__global__ __launch_bounds__(64) void paged_turn_row_kernel(PagedTurnArgs a) {
  __shared__ float cos_lds[64], sin_lds[64];
  __shared__ __attribute__((aligned(16))) uint8_t code_lds[kD];
  __shared__ __attribute__((aligned(16))) uint16_t row_lds[kD];
  const PagedArgs &c = a.append.c;
  const int heads = a.Hq + 2 * c.Hkv, b = blockIdx.x / heads, job = blockIdx.x % heads, lane = threadIdx.x;
  const bool value = job >= a.Hq + c.Hkv, query = job >= c.Hkv && !value;
  const int head = value ? job - a.Hq - c.Hkv : query ? job - c.Hkv : job;
  const TurnSpan s = turn_span(c, b);
  if (s.rows == 0) return;
  const bool place = s.base < s.end && !query;
  int page = -1;
  if (place) page = c.table[(size_t)b * c.max_pages + (s.base >> c.page_shift)];
  const bool stored = page >= 0 && page < c.n_pages;
  const size_t row0 = (((size_t)max(page, 0) * c.Hkv + head) << c.page_shift) + (s.base & ((1 << c.page_shift) - 1) & ~(kTokBlock - 1));
  const uint16_t *row = (value ? a.append.v + s.first * a.append.v_stride : query ? a.q + s.first * a.q_stride : a.append.k + s.first * a.append.k_stride) + head * kD;
  uint32_t own[2] = {row[lane], row[lane + 64]};
  float x[2];
  if (!value) {
    const int dim = a.plan.dim, half = dim / 2;
    int pair[2];
    uint32_t other[2];
    bool first[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = lane + 64 * k;
      first[k] = a.plan.interleaved ? (e & 1) == 0 : e < half;
      pair[k] = a.plan.interleaved ? e >> 1 : e < half ? e : e - half;
      other[k] = row[e >= dim ? e : a.plan.interleaved ? e ^ 1 : first[k] ? e + half : e - half];
    }
    if (lane < half) {
      const Turn t = pair_turn(a.plan, lane, s.first);
      cos_lds[lane] = t.c;
      sin_lds[lane] = t.s;
    }
    wave_lds_sync();
    uint16_t *dst = (query ? a.q_out + s.first * a.q_out_stride : a.k_out + s.first * a.k_out_stride) + head * kD;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = lane + 64 * k;
      if (e < dim) {
        const float sn = first[k] ? -sin_lds[pair[k]] : sin_lds[pair[k]];
        float y = __fmaf_rn(half_bits_to_float(own[k]), cos_lds[pair[k]], __fmul_rn(half_bits_to_float(other[k]), sn));
        asm("" : "+v"(y));  // keeps the rounding to 32 bits and the one to binary16 apart
        own[k] = float_to_half_bits_rne(y);
      }
      dst[e] = (uint16_t)own[k];
    }
  }
  if (!stored) return;
  const size_t unit = (size_t)b * c.Hkv + head;
  const SampledSlot list(list_of(c), (int)unit, lane);
  x[0] = half_bits_to_float(own[0]);
  x[1] = half_bits_to_float(own[1]);
  uint32_t old[2] = {0u, 0u};
  if (value) old_v_words<BITS>(c, s.base, row0, lane, old);
  const int slot = list.find(s.base);
  if (value) append_row<G, BITS, 1>(c, unit, s.base, row0, x[0], x[1], slot, old, a.append.rotate_v != 0, a.append.clip, lane, code_lds, row_lds);
  else append_row<G, BITS, 0>(c, unit, s.base, row0, x[0], x[1], slot, old, true, a.append.clip, lane, code_lds, row_lds);
}

template <int G, int BITS>
void launch_variant(const PagedTurnArgs &a, hipStream_t stream) {
  const PagedArgs &c = a.append.c;
  const long long heads = a.Hq + 2ll * c.Hkv;
  if (c.max_rows == 1 && heads * c.B < 1ll << 25) {
    paged_turn_row_kernel<G, BITS><<<dim3((unsigned)(heads * c.B)), dim3(64), 0, stream>>>(a);
    return;
  }
  const int blocks = (c.max_rows + 30) / kTokBlock + 1;  // that max_rows rows can touch, wherever they start
  // Heads of a workgroup, whose angles serve them all: two a wavefront, or one where that leaves the chip room.  Measured, us, 8 and 16 heads: 16 x 16
  // rows of 96 heads in all (192 workgroups of 16 heads, in the grid) 12.6 and 13.6, 4 x 1024 (792) 42.7 and 47.3, 8 x 4096 (6192) 356 and 302; 2 x 1024 of 48
  // (198) 13.2 and 13.9; of 36 heads 512 (51) 9.0 and 10.1, 32 x 8 (192) 9.2 and 8.5, 8 x 700 (552) 22.5 and 21.6, 13 of up to 1024 45.7 and 45.4.
  const long long groups = (long long)blocks * c.B * ((heads + 15) / 16);
  const int per = groups < (heads >= 48 ? 1024 : 64) ? 8 : 16;
  const dim3 grid(blocks, c.B, (unsigned)((heads + per - 1) / per)), block(64 * kTurnWaves);
  if (a.plan.interleaved) paged_turn_kernel<G, BITS, true><<<grid, block, 0, stream>>>(a, per);
  else paged_turn_kernel<G, BITS, false><<<grid, block, 0, stream>>>(a, per);
}

}  // namespace

hipError_t launch_paged_turn(const PagedTurnArgs &a, int G, int bits, hipStream_t stream) {
  if (G == 128) {
    if (bits == 2) launch_variant<128, 2>(a, stream);
    else launch_variant<128, 4>(a, stream);
  } else {
    if (bits == 2) launch_variant<64, 2>(a, stream);
    else launch_variant<64, 4>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace akvq
