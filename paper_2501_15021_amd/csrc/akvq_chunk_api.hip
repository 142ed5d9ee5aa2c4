// C ABI of the chunk entry points (declared in include/akvq.h): argument validation and dispatch.  As in akvq_api.hip nothing is
// allocated, freed or synchronised; every call enqueues on the caller's stream and returns.
#include "../../include/akvq.h"

#include <hip/hip_runtime.h>

#include "akvq_kernels.h"

namespace {

// one wavefront a row and 64 lanes a wavefront: a grid holds fewer than 2^32 of them
constexpr int kMaxChunkRows = 1 << 25;

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// packed rows of `heads` heads, `stride` elements apart
int check_rows(const void *rows, int64_t stride, int heads) {
  if (!rows || !aligned(rows, 16)) return AKVQ_ERR_INVALID_ARG;
  if (stride % 8 != 0 || stride < (int64_t)heads * 128) return AKVQ_ERR_INVALID_ARG;
  return AKVQ_OK;
}

int axes_args(const akvq_axes *axes, const int32_t *pos, int64_t pos_stride, int n_rows, akvq::AxesArgs &a) {
  if (!axes || n_rows < 0) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes < 1) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes > 4 || n_rows > kMaxChunkRows) return AKVQ_ERR_UNSUPPORTED;
  for (int i = 0; i < 64; ++i) {
    if (axes->axis[i] >= axes->n_axes) return AKVQ_ERR_INVALID_ARG;
    if (!__builtin_isfinite(axes->inv_freq[i])) return AKVQ_ERR_INVALID_ARG;
    a.turns[i] = (double)axes->inv_freq[i] / 6.283185307179586476925;
    a.axis[i] = axes->axis[i];
  }
  if (n_rows > 0 && (!pos || !aligned(pos, 4))) return AKVQ_ERR_INVALID_ARG;
  if (axes->n_axes > 1 && pos_stride < n_rows) return AKVQ_ERR_INVALID_ARG;
  a.pos = pos; a.pos_stride = pos_stride; a.n_rows = n_rows;
  return AKVQ_OK;
}

}  // namespace

extern "C" {

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

}  // extern "C"
