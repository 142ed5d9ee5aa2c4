// Arithmetic of one 32-row block in the write path, shared by the kernels that write contiguous planes and the one that writes
// pages: the transform over the four lanes that own a token pair, extrema, packing constants, 16-bit rows.
//
// Four neighbouring lanes own a token pair (t, t+16) of the block: lane (r, j) holds channels e = 32*m + 8*j + i (m<4, i<8), so
// every load of rows is a 128-bit load and a quad covers 64 contiguous bytes.  Butterfly strides 1,2,4 and 32,64 stay in
// registers; strides 8,16 cross the quad with DPP quad_perm.
#pragma once
#include "akvq_rowquant.h"

namespace akvq {
namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
// Running extrema, three operands at a time, and their reduction over the four lanes of a quad with the partner's
// value read through DPP by the min / max itself.  Assembly, because the compiler's fminf / fmaxf first canonicalise
// operands it cannot prove quiet (one more instruction each) and reach a partner lane through a separate move.
__device__ __forceinline__ void minmax3(float &mn, float &mx, float a, float b) {
  asm("v_min3_f32 %0, %0, %1, %2" : "+v"(mn) : "v"(a), "v"(b));
  asm("v_max3_f32 %0, %0, %1, %2" : "+v"(mx) : "v"(a), "v"(b));
}
// (the leading s_nop covers the wait states of a DPP read after a VALU write of its source and after an EXEC write)
__device__ __forceinline__ void quad_minmax(float &mn, float &mx) {
  asm volatile("s_nop 4\n\t"
               "v_min_f32_dpp %0, %0, %0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
               "v_max_f32_dpp %1, %1, %1 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
               "s_nop 1\n\t"
               "v_min_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
               "v_max_f32_dpp %1, %1, %1 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf"
               : "+v"(mn), "+v"(mx));
}
constexpr int kRowRor4 = 0x124;  // rotate right by 4 inside a row of 16 lanes
constexpr int kRowRor8 = 0x128;

// A cross-lane butterfly level: the lane whose index bit is clear keeps a+b, its partner should keep a-b (a = the
// lower lane's value).  One DPP multiply-add per element does it: own += c * partner with c = +1 in the lower lane and
// -1 in the upper one.  The product is exact and the sum is rounded once, exactly like the add of the specification;
// the upper lane ends up with b-a, i.e. the negated result, and since every later level is linear that lane simply
// carries all its values negated from then on (rounding to nearest is symmetric in sign).  After both cross-lane
// levels lanes j = 1, 2 hold negated values; quad_sign(j) is folded into the per-lane constants that consume them.
__device__ __forceinline__ float quad_sign(int j) { return (j == 1 || j == 2) ? -1.0f : 1.0f; }

// Eight elements of one level.  The leading s_nop covers the wait states a DPP read needs after the VALU write of
// its source register (and after an EXEC write): the compiler does not track hazards of inline assembly.
#define AKVQ_DPP_FMAC8(CTRL, NOP)                                                                              \
  asm volatile("s_nop " NOP "\n\t"                                                                            \
               "v_fmac_f32_dpp %0, %0, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %1, %1, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %2, %2, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %3, %3, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %4, %4, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %5, %5, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %6, %6, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"                            \
               "v_fmac_f32_dpp %7, %7, %8 " CTRL " row_mask:0xf bank_mask:0xf"                                \
               : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]) \
               : "v"(c))
__device__ __forceinline__ void quad_level_xor1(float (&x)[8], float c, bool first) {
  if (first) AKVQ_DPP_FMAC8("quad_perm:[1,0,3,2]", "4"); else AKVQ_DPP_FMAC8("quad_perm:[1,0,3,2]", "1");
}
__device__ __forceinline__ void quad_level_xor2(float (&x)[8], float c, bool first) {
  if (first) AKVQ_DPP_FMAC8("quad_perm:[2,3,0,1]", "4"); else AKVQ_DPP_FMAC8("quad_perm:[2,3,0,1]", "1");
}
#undef AKVQ_DPP_FMAC8

// First level (stride 1) straight from the packed binary16 pair: lo + hi and lo - hi, each one mixed-precision
// multiply-add (the widening is exact, the sum is rounded once, as widening followed by an fp32 add would be).
__device__ __forceinline__ void level1_from_half2(uint32_t w, float &sum, float &diff) {
  asm("v_fma_mix_f32 %0, %1, 1.0, %1 op_sel:[0,0,1] op_sel_hi:[1,0,1]" : "=v"(sum) : "v"(w));
  asm("v_fma_mix_f32 %0, %1, 1.0, -%1 op_sel:[0,0,1] op_sel_hi:[1,0,1]" : "=v"(diff) : "v"(w));
}

// un-normalised 128-point butterfly of one row held as raw[m] (eight binary16 channels 32m+8j..+7 per m) with the j
// index spread over the quad; the result in lane j is quad_sign(j) times the transform
__device__ __forceinline__ void wht128_quad(const u32x4 (&raw)[4], float (&u)[4][8], int j) {
  // stride 1
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int w = 0; w < 4; ++w) level1_from_half2(raw[m][w], u[m][2 * w], u[m][2 * w + 1]);
  // strides 2, 4: inside i
#pragma unroll
  for (int h = 2; h < 8; h *= 2)
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((i & h) == 0) {
          float a = u[m][i], b = u[m][i + h];
          u[m][i] = a + b;
          u[m][i + h] = a - b;
        }
  // strides 8, 16: across the quad (j bit 0, j bit 1)
  const float c1 = (j & 1) ? -1.0f : 1.0f, c2 = (j & 2) ? -1.0f : 1.0f;
#pragma unroll
  for (int m = 0; m < 4; ++m) quad_level_xor1(u[m], c1, m == 0);
#pragma unroll
  for (int m = 0; m < 4; ++m) quad_level_xor2(u[m], c2, m == 0);
  // strides 32, 64: inside m
#pragma unroll
  for (int h = 1; h < 4; h *= 2)
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if ((m & h) == 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float a = u[m][i], b = u[m + h][i];
          u[m][i] = a + b;
          u[m + h][i] = a - b;
        }
}

// Rotary position embedding of one row held as raw[m] (see wht128_quad): channel e pairs with e + 64, i.e. raw[mm] with
// raw[mm + 2] word by word, both in this lane; cw / sw hold the binary16 cos / sin of channels 32*mm + 8*j .. + 7.
// Both products are exact in fp32 and the multiply-add rounds their sum once; the result is then rounded to binary16.
// The mixed-precision instructions read the binary16 halves in place (HI selects the upper half of every word); being
// assembly, they also keep the compiler from merging the two roundings into one.
template <int HI>
__device__ __forceinline__ float rope_mix(uint32_t x, uint32_t c, uint32_t xp, uint32_t sn, bool subtract) {
  float t, r;
  const float neg_zero = -0.0f;  // product + (-0) is the product itself, signed zeros included
  if (HI) asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,1,0] op_sel_hi:[1,1,0]" : "=v"(t) : "v"(xp), "v"(sn), "v"(neg_zero));
  else asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,1,0]" : "=v"(t) : "v"(xp), "v"(sn), "v"(neg_zero));
  if (subtract) {
    if (HI) asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[1,1,0] op_sel_hi:[1,1,0]" : "=v"(r) : "v"(x), "v"(c), "v"(t));
    else asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,0] op_sel_hi:[1,1,0]" : "=v"(r) : "v"(x), "v"(c), "v"(t));
  } else {
    if (HI) asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[1,1,0] op_sel_hi:[1,1,0]" : "=v"(r) : "v"(x), "v"(c), "v"(t));
    else asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,0,0] op_sel_hi:[1,1,0]" : "=v"(r) : "v"(x), "v"(c), "v"(t));
  }
  return r;
}
// two floats -> packed binary16 pair (lo = a, hi = b), round to nearest even, one conversion instruction
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  uint32_t r;
  asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ void rope_row_quad(u32x4 (&raw)[4], const u32x4 (&cw)[2], const u32x4 (&sw)[2]) {
#pragma unroll
  for (int mm = 0; mm < 2; ++mm)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t lo = raw[mm][w], hi = raw[mm + 2][w], c = cw[mm][w], sn = sw[mm][w];
      raw[mm][w] = pack_half2(rope_mix<0>(lo, c, hi, sn, true), rope_mix<1>(lo, c, hi, sn, true));
      raw[mm + 2][w] = pack_half2(rope_mix<0>(hi, c, lo, sn, false), rope_mix<1>(hi, c, lo, sn, false));
    }
}

// Packing adds the raw patterns with shifts (one shift-add per code); what the constant part of every pattern
// contributes is a compile-time constant (mod 2^32) that is subtracted once per word.
constexpr uint32_t kPack16Bias = (uint32_t)(0x4B400000ull * 0x55555555ull);   // sum over s<16 of kMagicBits << 2s
constexpr uint32_t kPack4Bias = (uint32_t)(0x4B400000ull * 0x01010101ull);    // sum over b<4 of kMagicBits << 8b

// One row as bfloat16 (u holds its sign-carrying transform, scale undoes that) into slot `slot` of row-major K rows or of
// 32-slot V tiles; zeros for a row that carries no token.
template <int TENSOR>
__device__ __forceinline__ void store_bf16_row(const float (&u)[4][8], float scale, int j, uint16_t *k_rows, uint16_t *v_plane,
                                               int slot, bool token) {
  if (TENSOR == 0) {
    uint16_t *dst = k_rows + (size_t)slot * kD;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      u32x4 o;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        o[w] = token ? pack_bf16x2(scaled_row_value(u[m][2 * w], scale), scaled_row_value(u[m][2 * w + 1], scale)) : 0u;
      *reinterpret_cast<u32x4 *>(dst + 32 * m + 8 * j) = o;
    }
  } else {
    const int sb = slot >> 5, sh = (slot & 31) >> 4, sr = slot & 15, sq = sr >> 2, sii = sr & 3;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = 32 * m + 8 * j + i, nb = e >> 4, n = e & 15;
        v_plane[(size_t)sb * 4096 + nb * 512 + (16 * sq + n) * 8 + 2 * sii + sh] =
            token ? (uint16_t)pack_bf16x2(scaled_row_value(u[m][i], scale), 0.0f) : (uint16_t)0;
      }
  }
}

}  // namespace
}  // namespace akvq
