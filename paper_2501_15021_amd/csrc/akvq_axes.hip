// Rotary positions with several axes: pair i of a row (channels i, i + 64) is turned by pos[axis(i)][row] * inv_freq(i).
//
// Memory bound: every element is read and written once for three operations.  One wavefront takes a row: lane i forms the angle of
// pair i once for all heads (a 64-bit product and its rest, whose whole turns are dropped before 32 bits hold it: a 32-bit angle would be off by
// 2^-24 of itself, 6e-3 at position 100000) and leaves its sine and cosine in LDS, from where lane (h, o) takes those of pairs
// 8o .. 8o + 7 for every eighth head: two 128-bit loads and stores a head, 128 contiguous bytes for eight lanes.
//   Measured: 8 x 8191 rows of 32 heads 131 us, 5.4 TB/s (a large copy: 5.47); sixteen rows of 64 heads 2.3 us, a launch and one round
// trip to memory (4.4 with a wavefront a row, and the first head behind the angle).
#include "akvq_device.h"
#include "akvq_kernels.h"

namespace akvq {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
constexpr int kAxesWaves = 4;

// cosine and sine of a row's pair
__device__ __forceinline__ void pair_turn(const AxesArgs &a, int pair, int row, float &c, float &s) {
  const double p = a.pos[a.axis[pair] * a.pos_stride + row], f = a.turns[pair], t = p * f;
  // what the rounded product and frequency leave: up to 5e-7 of an angle of 2^31, in place of 1e-7 for all
  const double rest = __builtin_fma(p, f, -t) + p * (double)a.turns_rest[pair];
  sincospif(2.0f * (float)((t - rint(t)) + rest), &s, &c);
}

__global__ __launch_bounds__(64 * kAxesWaves) void rope_axes_kernel(AxesArgs a) {
  __shared__ __attribute__((aligned(16))) float cos_lds[kAxesWaves][64], sin_lds[kAxesWaves][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = blockIdx.x * kAxesWaves + wave;
  if (row >= a.n_rows) return;  // whole wavefront; no workgroup barrier below
  const int o = lane & 7, first = blockIdx.y * a.heads_per_wave, end = min(first + a.heads_per_wave, a.Hq + a.Hkv);
  // a head's row, or the last one's: asked for a head ahead, the first in front of the angle
  auto source = [&](int h) {
    h = min(h, a.Hq + a.Hkv - 1);
    return (h >= a.Hq ? a.k + row * a.k_stride + (h - a.Hq) * kD : a.q + row * a.q_stride + h * kD) + 8 * o;
  };
  const uint16_t *src = source(first + (lane >> 3));
  f16x8 next_lo = *reinterpret_cast<const f16x8 *>(src), next_hi = *reinterpret_cast<const f16x8 *>(src + 64);
  float c1, s1;
  pair_turn(a, lane, row, c1, s1);
  cos_lds[wave][lane] = c1;
  sin_lds[wave][lane] = a.inverse ? -s1 : s1;
  wave_lds_sync();
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = cos_lds[wave][8 * o + i]; s[i] = sin_lds[wave][8 * o + i]; }
  for (int h = first + (lane >> 3); h < end; h += 8) {
    uint16_t *dst = h >= a.Hq ? a.k_out + row * a.k_out_stride + (h - a.Hq) * kD : a.q_out + row * a.q_out_stride + h * kD;
    const f16x8 lo = next_lo, hi = next_hi;
    if (h + 8 < end) {
      src = source(h + 8);
      next_lo = *reinterpret_cast<const f16x8 *>(src);
      next_hi = *reinterpret_cast<const f16x8 *>(src + 64);
    }
    f16x8 lo2, hi2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = (float)lo[i], y = (float)hi[i];
      lo2[i] = (_Float16)__fmaf_rn(x, c[i], -__fmul_rn(y, s[i]));
      hi2[i] = (_Float16)__fmaf_rn(y, c[i], __fmul_rn(x, s[i]));
    }
    *reinterpret_cast<f16x8 *>(dst + 8 * o) = lo2;
    *reinterpret_cast<f16x8 *>(dst + 64 + 8 * o) = hi2;
  }
}

__global__ __launch_bounds__(256) void rope_axes_table_kernel(AxesArgs a) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.n_rows) return;
  float c, s;
  pair_turn(a, lane, row, c, s);
  a.q_out[(size_t)row * 64 + lane] = (uint16_t)float_to_half_bits_rne(c);
  a.k_out[(size_t)row * 64 + lane] = (uint16_t)float_to_half_bits_rne(s);
}

}  // namespace

hipError_t launch_rope_axes(AxesArgs a, hipStream_t stream) {
  const unsigned blocks = ((unsigned)a.n_rows + kAxesWaves - 1) / kAxesWaves;
  const int heads = a.Hq + a.Hkv;
  // few rows: their heads are dealt to as many wavefronts as fill the chip twice, eight heads (one round) each or more
  const long long per = ((long long)a.n_rows * heads + 2047) / 2048;
  a.heads_per_wave = per >= heads ? heads : (int)((per + 7) / 8 * 8);
  const unsigned parts = (heads + a.heads_per_wave - 1) / a.heads_per_wave;
  rope_axes_kernel<<<dim3(blocks, parts), dim3(64 * kAxesWaves), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rope_axes_table(const AxesArgs &a, hipStream_t stream) {
  rope_axes_table_kernel<<<dim3(((unsigned)a.n_rows + 3) / 4), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace akvq
