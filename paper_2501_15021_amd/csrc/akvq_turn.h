// Sine and cosine of rotary angles, and the turn of a pair, as the calls that turn rows share them.
//
// The angle pos * f is formed in turns, in 64 bits: 1 / 2 pi is taken as its first 29 bits, whose product with a 32-bit number is exact,
// and the rest, so frequency and product are sums of two numbers whose whole turns are dropped exactly.  What is left, at most an eighth of a turn
// from a quarter's multiple, goes into the series of sine and cosine up to z^17 and z^16 (below 2^-54 there).  So what is rounded to 32 bits is right
// to 1e-15, and the rounded numbers are those of any other 64-bit computation but for one in 10^7.
#pragma once
#include "akvq_device.h"
#include "akvq_kernels.h"

namespace akvq {
namespace {

struct Turn { float c, s; };

__device__ __forceinline__ Turn pair_turn(const RotaryPlan &plan, int pair, long long row) {
  constexpr double kTurns = 0x1.45f306dp-3, kTurnsRest = 0x1.9391054a7f09dp-32;  // 1 / 2 pi
  const double p = plan.pos[plan.axis[pair] * plan.pos_stride + row], f = plan.inv_freq[pair];
  const double whole = f * kTurns, rest = f * kTurnsRest, turns = whole + rest, turns_rest = rest - (turns - whole);
  const double t = p * turns;
  const double x = (t - rint(t)) + (__builtin_fma(p, turns, -t) + p * turns_rest);
  const double n = rint(4.0 * x);
  const double z = (x - 0.25 * n) * 6.283185307179586, zz = z * z;
  // 1 / k!
  double s = __builtin_fma(zz, 2.8114572543455206e-15, -7.647163731819816e-13);
  s = __builtin_fma(zz, s, 1.6059043836821613e-10);
  s = __builtin_fma(zz, s, -2.505210838544172e-08);
  s = __builtin_fma(zz, s, 2.7557319223985893e-06);
  s = __builtin_fma(zz, s, -1.984126984126984e-04);
  s = __builtin_fma(zz, s, 8.333333333333333e-03);
  s = __builtin_fma(zz, s, -1.6666666666666666e-01);
  s = __builtin_fma(z * zz, s, z);
  double c = __builtin_fma(zz, 4.779477332387385e-14, -1.1470745597729725e-11);
  c = __builtin_fma(zz, c, 2.08767569878681e-09);
  c = __builtin_fma(zz, c, -2.755731922398589e-07);
  c = __builtin_fma(zz, c, 2.48015873015873e-05);
  c = __builtin_fma(zz, c, -1.388888888888889e-03);
  c = __builtin_fma(zz, c, 4.1666666666666664e-02);
  c = __builtin_fma(zz, c, -0.5);
  c = __builtin_fma(zz, c, 1.0);
  const int q = (int)n & 3;  // quarter turns: (c, s) -> (-s, c)
  const double c1 = (q & 1) ? s : c, s1 = (q & 1) ? c : s;
  const double m = plan.magnitude, cm = ((q + 1) & 2) ? -m : m, sm = ((q & 2) != 0) != (plan.inverse != 0) ? -m : m;
  return {(float)(c1 * cm), (float)(s1 * sm)};
}

// One pair of binary16 numbers in one half of their words, turned: the product with the sine is rounded to 32 bits, its sum with the other once.
// (As __fmul_rn and __fmaf_rn would, with the binary16 numbers read in place: 0 where it is the words' lower half.)
template <int HI>
__device__ __forceinline__ void turn_halves(uint32_t x, uint32_t y, float c, float s, float &x2, float &y2) {
  const float neg_zero = -0.0f;  // product + (-0) is the product itself, signed zeros included
  float ys, xs;
  if (HI) {
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(ys) : "v"(y), "v"(s), "v"(neg_zero));
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(xs) : "v"(x), "v"(s), "v"(neg_zero));
    asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(x2) : "v"(x), "v"(c), "v"(ys));
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y2) : "v"(y), "v"(c), "v"(xs));
  } else {
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(ys) : "v"(y), "v"(s), "v"(neg_zero));
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(xs) : "v"(x), "v"(s), "v"(neg_zero));
    asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(x2) : "v"(x), "v"(c), "v"(ys));
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(y2) : "v"(y), "v"(c), "v"(xs));
  }
}
// ... x in the lower half, y in the upper half of one word
__device__ __forceinline__ void turn_word(uint32_t w, float c, float s, float &x2, float &y2) {
  const float neg_zero = -0.0f;
  float ys, xs;
  asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(ys) : "v"(w), "v"(s), "v"(neg_zero));
  asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(xs) : "v"(w), "v"(s), "v"(neg_zero));
  asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(x2) : "v"(w), "v"(c), "v"(ys));
  asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y2) : "v"(w), "v"(c), "v"(xs));
}
// two floats -> packed binary16 pair, each rounded to nearest even
__device__ __forceinline__ uint32_t turned_pair(float a, float b) {
  uint32_t r;
  asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// Eight pairs, whose turns are t[0 .. 7]: of chunk x with chunk y (half layout), or neighbours in x and then in y (interleaved).
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_chunks(u32x4 &x, u32x4 &y, const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float a0, a1, b0, b1;
    const uint32_t xw = x[w], yw = y[w];
    if (INTERLEAVED) {
      turn_word(xw, c[w], s[w], a0, a1);
      turn_word(yw, c[4 + w], s[4 + w], b0, b1);
    } else {
      turn_halves<0>(xw, yw, c[2 * w], s[2 * w], a0, b0);
      turn_halves<1>(xw, yw, c[2 * w + 1], s[2 * w + 1], a1, b1);
    }
    x[w] = turned_pair(a0, a1);
    y[w] = turned_pair(b0, b1);
  }
}

}  // namespace
}  // namespace akvq
