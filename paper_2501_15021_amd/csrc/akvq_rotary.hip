// Rotary positions in either layout, of the whole head or its first channels: pair i of a row turns by pos[axis(i)][row] * inv_freq(i).
//
//   (x, y) -> (x c - y s, y c + x s), c and s the cosine and sine times the magnitude.
//
// Memory bound: every element is read and written once for three operations.  One wavefront takes a row: lane i forms the angle of pair i once
// for all heads (64 bits, 50 instructions) and leaves its sine and cosine in LDS, from where lane (h, o) takes those of pairs 8o .. 8o + 7 for
// every eighth head.  A lane owns two chunks of eight channels, which hold both sides of its eight pairs in either layout (half: chunks that
// lie dim / 2 apart; interleaved: neighbours), or two chunks that do not turn: so a row may be turned in place.
//   8 x 8191 rows of 28 / 4 heads, 64 of 128 channels turning: 137 us, 5.2 TB/s (a large copy: 5.47; written with the non-temporal hint 161).
// 16 rows of 64 heads: 2.65 us, a chain of one load, the angle and one store.
#include "akvq_device.h"
#include "akvq_kernels.h"
#include "akvq_turn.h"

namespace akvq {
namespace {

constexpr int kRotaryWaves = 4;

template <bool INTERLEAVED>
__global__ __launch_bounds__(64 * kRotaryWaves) void rotary_rows_kernel(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) float cos_lds[kRotaryWaves][64], sin_lds[kRotaryWaves][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRotaryWaves + wave;
  if (row >= a.n_rows) return;  // whole wavefront; no workgroup barrier below
  const int o = lane & 7, first = blockIdx.y * a.heads_per_wave, end = min(first + a.heads_per_wave, a.Hq + a.Hkv);
  const int dim = a.plan.dim, turning = dim / 16;
  const bool turns = o < turning;
  const int at0 = INTERLEAVED ? 16 * o : turns ? 8 * o : dim + 16 * (o - turning), at1 = at0 + (!INTERLEAVED && turns ? dim / 2 : 8);
  // a head's row, or the last one's: asked for a head ahead, the first in front of the angle
  auto source = [&](int h) {
    h = min(h, a.Hq + a.Hkv - 1);
    return h >= a.Hq ? a.k + row * a.k_stride + (h - a.Hq) * kD : a.q + row * a.q_stride + h * kD;
  };
  const uint16_t *src = source(first + (lane >> 3));
  u32x4 next0 = *reinterpret_cast<const u32x4 *>(src + at0), next1 = *reinterpret_cast<const u32x4 *>(src + at1);
  if (lane < dim / 2) {
    const Turn t = pair_turn(a.plan, lane, row);
    cos_lds[wave][lane] = t.c;
    sin_lds[wave][lane] = t.s;
  }
  wave_lds_sync();
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = cos_lds[wave][8 * o + i]; s[i] = sin_lds[wave][8 * o + i]; }  // (of chunks that do not turn: anything)
  for (int h = first + (lane >> 3); h < end; h += 8) {
    uint16_t *dst = h >= a.Hq ? a.k_out + row * a.k_out_stride + (h - a.Hq) * kD : a.q_out + row * a.q_out_stride + h * kD;
    u32x4 x = next0, y = next1;
    if (h + 8 < end) {
      src = source(h + 8);
      next0 = *reinterpret_cast<const u32x4 *>(src + at0);
      next1 = *reinterpret_cast<const u32x4 *>(src + at1);
    }
    if (turns) turn_chunks<INTERLEAVED>(x, y, c, s);
    *reinterpret_cast<u32x4 *>(dst + at0) = x;
    *reinterpret_cast<u32x4 *>(dst + at1) = y;
  }
}

}  // namespace

hipError_t launch_rotary_rows(RotaryArgs a, hipStream_t stream) {
  const unsigned blocks = ((unsigned)a.n_rows + kRotaryWaves - 1) / kRotaryWaves;
  const int heads = a.Hq + a.Hkv;
  // few rows: their heads are dealt to as many wavefronts as fill the chip twice, eight heads (one round) each or more
  const long long per = ((long long)a.n_rows * heads + 2047) / 2048;
  a.heads_per_wave = per >= heads ? heads : (int)((per + 7) / 8 * 8);
  const unsigned parts = (heads + a.heads_per_wave - 1) / a.heads_per_wave;
  const dim3 grid(blocks, parts), block(64 * kRotaryWaves);
  if (a.plan.interleaved) rotary_rows_kernel<true><<<grid, block, 0, stream>>>(a);
  else rotary_rows_kernel<false><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace akvq
