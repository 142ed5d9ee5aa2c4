// C ABI of rotary positions in either layout, of pages of 4-bit codes and of the call that turns a chunk on its way into the pages (declared in
// include/akvq.h): argument validation and dispatch.  As in akvq_api.hip nothing is allocated, freed or synchronised; every call
// enqueues on the caller's stream and returns.
#include "../../include/akvq.h"

#include <hip/hip_runtime.h>

#include "akvq_chunk_checks.h"
#include "akvq_kernels.h"

namespace {

int rotary_plan(const akvq_rotary *r, const int32_t *pos, int64_t pos_stride, int n_rows, akvq::RotaryPlan &plan) {
  if (!r || n_rows < 0 || r->n_axes < 1) return AKVQ_ERR_INVALID_ARG;
  if (r->n_axes > 4 || n_rows > kMaxChunkRows) return AKVQ_ERR_UNSUPPORTED;
  if (r->layout != AKVQ_ROTARY_HALF && r->layout != AKVQ_ROTARY_INTERLEAVED) return AKVQ_ERR_INVALID_ARG;
  if (r->dim < 16 || r->dim > 128 || r->dim % 16 != 0) return AKVQ_ERR_UNSUPPORTED;
  if (!__builtin_isfinite(r->magnitude)) return AKVQ_ERR_INVALID_ARG;
  for (int i = 0; i < 64; ++i) {
    const bool turns = i < r->dim / 2;
    if (turns && (r->axis[i] >= r->n_axes || !__builtin_isfinite(r->inv_freq[i]))) return AKVQ_ERR_INVALID_ARG;
    plan.inv_freq[i] = turns ? r->inv_freq[i] : 0.0f;
    plan.axis[i] = turns ? r->axis[i] : (uint8_t)0;
  }
  if (n_rows > 0 && (!pos || !aligned(pos, 4))) return AKVQ_ERR_INVALID_ARG;
  if (r->n_axes > 1 && pos_stride < n_rows) return AKVQ_ERR_INVALID_ARG;
  plan.pos = pos; plan.pos_stride = pos_stride;
  plan.magnitude = r->magnitude; plan.dim = r->dim;
  plan.interleaved = r->layout == AKVQ_ROTARY_INTERLEAVED ? 1 : 0;
  return AKVQ_OK;
}

// rows that are read and rows that are written, which may be the same
int check_turned(const void *in, int64_t stride, const void *out, int64_t out_stride, int heads) {
  if (check_rows(in, stride, heads) != AKVQ_OK || check_rows(out, out_stride, heads) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  return in == out && stride != out_stride ? AKVQ_ERR_INVALID_ARG : AKVQ_OK;
}

}  // namespace

extern "C" {

int akvq_paged_nibble_bytes(const akvq_paged *shape, size_t out_bytes[8]) { return paged_bytes(shape, 4, out_bytes); }

int akvq_paged_nibble_append(const akvq_paged *c, const akvq_chunk *rows, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, float clip, uint32_t flags, void *stream) {
  akvq::PagedAppendArgs a{};
  const int st = append_args(c, rows, k, k_stride, v, v_stride, clip, flags, AKVQ_K_PREROTATED | AKVQ_V_PREROTATED, a);
  if (st != AKVQ_OK || a.c.max_rows == 0) return st;
  return akvq::launch_status(akvq::launch_paged4_append(a, c->G, static_cast<hipStream_t>(stream)));
}

int akvq_paged_nibble_default_splits(const akvq_paged *c, int Hq, int max_rows) { return default_splits(c, Hq, max_rows, 4); }

int akvq_paged_nibble_attention(const akvq_paged *c, const akvq_chunk *rows, const void *q, int64_t q_stride, int Hq, const void *k,
                          int64_t k_stride, const void *v, int64_t v_stride, float sm_scale, void *out, int64_t out_stride,
                          float *lse_out, int n_split, void *workspace, size_t workspace_bytes, uint32_t flags, void *stream) {
  akvq::PagedAttentionArgs a{};
  const int st = attention_args(c, rows, q, q_stride, Hq, k, k_stride, v, v_stride, sm_scale, out, out_stride, lse_out, n_split, workspace,
                                workspace_bytes, flags, [&] { return akvq_paged_nibble_default_splits(c, Hq, rows->max_rows); }, a);
  if (st != AKVQ_OK || a.c.max_rows == 0) return st;
  return akvq::launch_status(akvq::launch_paged4_attention(a, c->G, static_cast<hipStream_t>(stream)));
}

int akvq_rotary_rows(const akvq_rotary *rotary, const int32_t *pos, int64_t pos_stride, int n_rows, const void *q, int64_t q_stride,
                     int Hq, const void *k, int64_t k_stride, int Hkv, void *q_out, int64_t q_out_stride, void *k_out,
                     int64_t k_out_stride, uint32_t flags, void *stream) {
  akvq::RotaryArgs a{};
  const int st = rotary_plan(rotary, pos, pos_stride, n_rows, a.plan);
  if (st != AKVQ_OK) return st;
  if (Hq < 0 || Hkv < 0 || (Hq == 0 && Hkv == 0)) return AKVQ_ERR_INVALID_ARG;
  if (Hq > 65535 || Hkv > 65535) return AKVQ_ERR_UNSUPPORTED;
  if (flags & ~(uint32_t)AKVQ_ROPE_INVERSE) return AKVQ_ERR_INVALID_ARG;
  if (n_rows == 0) return AKVQ_OK;
  if (Hq > 0 && check_turned(q, q_stride, q_out, q_out_stride, Hq) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  if (Hkv > 0 && check_turned(k, k_stride, k_out, k_out_stride, Hkv) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  a.plan.inverse = (flags & AKVQ_ROPE_INVERSE) ? 1 : 0;
  a.n_rows = n_rows; a.Hq = Hq; a.Hkv = Hkv;
  a.q = static_cast<const uint16_t *>(q); a.k = static_cast<const uint16_t *>(k);
  a.q_out = static_cast<uint16_t *>(q_out); a.k_out = static_cast<uint16_t *>(k_out);
  a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  return akvq::launch_status(akvq::launch_rotary_rows(a, static_cast<hipStream_t>(stream)));
}

int akvq_paged_append_rotary(const akvq_paged *c, int bits, const akvq_chunk *rows, const akvq_rotary *rotary, const int32_t *pos,
                             int64_t pos_stride, const void *q, int64_t q_stride, int Hq, const void *k, int64_t k_stride,
                             const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride,
                             float clip, uint32_t flags, void *stream) {
  akvq::PagedTurnArgs a{};
  int st = append_args(c, rows, k, k_stride, v, v_stride, clip, flags, AKVQ_V_PREROTATED, a.append);
  if (st != AKVQ_OK) return st;
  if (bits != 2 && bits != 4) return AKVQ_ERR_UNSUPPORTED;
  st = rotary_plan(rotary, pos, pos_stride, rows->n_rows, a.plan);
  if (st != AKVQ_OK) return st;
  if (Hq < 0) return AKVQ_ERR_INVALID_ARG;
  if (Hq > 65535) return AKVQ_ERR_UNSUPPORTED;
  if (a.append.c.max_rows == 0) return AKVQ_OK;
  if (check_turned(k, k_stride, k_out, k_out_stride, c->Hkv) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  if (Hq > 0 && check_turned(q, q_stride, q_out, q_out_stride, Hq) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  a.Hq = Hq;
  a.q = static_cast<const uint16_t *>(q);
  a.q_out = static_cast<uint16_t *>(q_out); a.k_out = static_cast<uint16_t *>(k_out);
  a.q_stride = q_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  return akvq::launch_status(akvq::launch_paged_turn(a, c->G, bits, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
