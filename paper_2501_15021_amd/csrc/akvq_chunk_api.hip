// C ABI of the chunk entry points (declared in include/akvq.h): argument validation and dispatch.  As in akvq_api.hip nothing is
// allocated, freed or synchronised; every call enqueues on the caller's stream and returns.
#include "../../include/akvq.h"

#include <hip/hip_runtime.h>

#include "akvq_chunk_checks.h"
#include "akvq_kernels.h"

namespace {

// 1 / 2 pi as its first 29 bits, whose product with a 32-bit float is exact, and the rest
constexpr double kTurns = 0x1.45f306dp-3, kTurnsRest = 0x1.9391054a7f09dp-32;

int axes_args(const akvq_axes *axes, const int32_t *pos, int64_t pos_stride, int n_rows, akvq::AxesArgs &a) {
  if (!axes || n_rows < 0) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes < 1) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes > 4 || n_rows > kMaxChunkRows) return AKVQ_ERR_UNSUPPORTED;
  for (int i = 0; i < 64; ++i) {
    if (axes->axis[i] >= axes->n_axes) return AKVQ_ERR_INVALID_ARG;
    if (!__builtin_isfinite(axes->inv_freq[i])) return AKVQ_ERR_INVALID_ARG;
    const double whole = axes->inv_freq[i] * kTurns, rest = axes->inv_freq[i] * kTurnsRest;
    a.turns[i] = whole + rest;
    a.turns_rest[i] = (float)(rest - (a.turns[i] - whole));
    a.axis[i] = axes->axis[i];
  }
  if (n_rows > 0 && (!pos || !aligned(pos, 4))) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes > 1 && pos_stride < n_rows) return AKVQ_ERR_INVALID_ARG;
  a.pos = pos; a.pos_stride = pos_stride; a.n_rows = n_rows;
  return AKVQ_OK;
}

}  // namespace

extern "C" {

int akvq_paged_bytes(const akvq_paged *shape, size_t out_bytes[8]) { return paged_bytes(shape, 2, out_bytes); }

int akvq_paged_append(const akvq_paged *c, const akvq_chunk *rows, const void *k, int64_t k_stride, const void *v,
                      int64_t v_stride, float clip, uint32_t flags, void *stream) {
  akvq::PagedAppendArgs a{};
  const int st = append_args(c, rows, k, k_stride, v, v_stride, clip, flags, AKVQ_K_PREROTATED | AKVQ_V_PREROTATED, a);
  if (st != AKVQ_OK || a.c.max_rows == 0) return st;
  return akvq::launch_status(akvq::launch_paged_append(a, c->G, static_cast<hipStream_t>(stream)));
}

int akvq_rope_axes(const akvq_axes *axes, const int32_t *pos, int64_t pos_stride, int n_rows, const void *q, int64_t q_stride,
                   int Hq, const void *k, int64_t k_stride, int Hkv, void *q_out, int64_t q_out_stride, void *k_out,
                   int64_t k_out_stride, uint32_t flags, void *stream) {
  akvq::AxesArgs a{};
  int st = axes_args(axes, pos, pos_stride, n_rows, a);
  if (st != AKVQ_OK) return st;
  if (Hq < 0 || Hkv < 0 || (Hq == 0 && Hkv == 0)) return AKVQ_ERR_INVALID_ARG;
  if (Hq > 65535 || Hkv > 65535) return AKVQ_ERR_UNSUPPORTED;
  if (flags & ~(uint32_t)AKVQ_ROPE_INVERSE) return AKVQ_ERR_INVALID_ARG;
  if (n_rows == 0) return AKVQ_OK;
  if (Hq > 0) {
    if (check_rows(q, q_stride, Hq) != AKVQ_OK || check_rows(q_out, q_out_stride, Hq) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
    if (q == q_out && q_stride != q_out_stride) return AKVQ_ERR_INVALID_ARG;
  }
  if (Hkv > 0) {
    if (check_rows(k, k_stride, Hkv) != AKVQ_OK || check_rows(k_out, k_out_stride, Hkv) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
    if (k == k_out && k_stride != k_out_stride) return AKVQ_ERR_INVALID_ARG;
  }
  a.q = static_cast<const uint16_t *>(q); a.k = static_cast<const uint16_t *>(k);
  a.q_out = static_cast<uint16_t *>(q_out); a.k_out = static_cast<uint16_t *>(k_out);
  a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  a.Hq = Hq; a.Hkv = Hkv; a.inverse = (flags & AKVQ_ROPE_INVERSE) ? 1 : 0;
  return akvq::launch_status(akvq::launch_rope_axes(a, static_cast<hipStream_t>(stream)));
}

int akvq_rope_axes_table(const akvq_axes *axes, const int32_t *pos, int64_t pos_stride, int n_rows, void *cos, void *sin,
                         void *stream) {
  akvq::AxesArgs a{};
  const int st = axes_args(axes, pos, pos_stride, n_rows, a);
  if (st != AKVQ_OK) return st;
  if (n_rows == 0) return AKVQ_OK;
  if (!cos || !sin || !aligned(cos, 16) || !aligned(sin, 16)) return AKVQ_ERR_INVALID_ARG;
  a.q_out = static_cast<uint16_t *>(cos); a.k_out = static_cast<uint16_t *>(sin);
  return akvq::launch_status(akvq::launch_rope_axes_table(a, static_cast<hipStream_t>(stream)));
}

size_t akvq_paged_workspace_bytes(int n_rows, int Hq, int n_split) {
  if (n_rows <= 0 || Hq <= 0 || n_split <= 1) return 0;
  return (size_t)n_rows * Hq * n_split * akvq::kPartialStride * sizeof(float);
}

int akvq_paged_default_splits(const akvq_paged *c, int Hq, int max_rows) { return default_splits(c, Hq, max_rows, 2); }

int akvq_paged_attention(const akvq_paged *c, const akvq_chunk *rows, const void *q, int64_t q_stride, int Hq, const void *k,
                         int64_t k_stride, const void *v, int64_t v_stride, float sm_scale, void *out, int64_t out_stride,
                         float *lse_out, int n_split, void *workspace, size_t workspace_bytes, uint32_t flags, void *stream) {
  akvq::PagedAttentionArgs a{};
  const int st = attention_args(c, rows, q, q_stride, Hq, k, k_stride, v, v_stride, sm_scale, out, out_stride, lse_out, n_split, workspace,
                                workspace_bytes, flags, [&] { return akvq_paged_default_splits(c, Hq, rows->max_rows); }, a);
  if (st != AKVQ_OK || a.c.max_rows == 0) return st;
  return akvq::launch_status(akvq::launch_paged_attention(a, c->G, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
