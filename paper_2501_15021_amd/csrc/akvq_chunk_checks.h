// Host checks that the calls for chunks share: packed rows, the cache in pages, a chunk's rows.
#pragma once
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

int check_paged_shape(const akvq_paged *c) {
  if (!c || c->B <= 0 || c->Hkv <= 0 || c->page_rows <= 0 || c->n_pages <= 0 || c->max_pages <= 0 || c->S_cap <= 0 || c->max_len < 0)
    return AKVQ_ERR_INVALID_ARG;
  if (c->G != 64 && c->G != 128) return AKVQ_ERR_UNSUPPORTED;
  if (c->S_cap % 64 != 0) return AKVQ_ERR_INVALID_ARG;
  if (c->page_rows < 32 || c->page_rows > 65536 || (c->page_rows & (c->page_rows - 1)) != 0) return AKVQ_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_rows >= (1 << 30)) return AKVQ_ERR_UNSUPPORTED;
  if ((int64_t)c->B * c->Hkv > 65535) return AKVQ_ERR_UNSUPPORTED;  // units index a grid dimension
  return AKVQ_OK;
}

int paged_args(const akvq_paged *c, const akvq_chunk *rows, akvq::PagedArgs &a) {
  const int st = check_paged_shape(c);
  if (st != AKVQ_OK) return st;
  const void *p[8] = {c->k_codes, c->v_codes, c->k_meta, c->v_meta, c->k_sal, c->v_sal, c->sal_idx, c->sal_cnt};
  for (const void *x : p)
    if (!x || !aligned(x, 16)) return AKVQ_ERR_INVALID_ARG;
  if (!c->table || !c->seq_len || !aligned(c->table, 4) || !aligned(c->seq_len, 4)) return AKVQ_ERR_INVALID_ARG;
  if (!rows || !rows->row_start || !aligned(rows->row_start, 4) || rows->n_rows < 0 || rows->max_rows < 0) return AKVQ_ERR_INVALID_ARG;
  if (rows->n_rows > kMaxChunkRows) return AKVQ_ERR_UNSUPPORTED;
  a = akvq::PagedArgs{};
  a.k_codes = c->k_codes; a.v_codes = c->v_codes; a.k_meta = c->k_meta; a.v_meta = c->v_meta;
  a.k_sal = c->k_sal; a.v_sal = c->v_sal; a.sal_idx = c->sal_idx; a.sal_cnt = c->sal_cnt;
  a.table = c->table; a.seq_len = c->seq_len;
  a.B = c->B; a.Hkv = c->Hkv; a.n_pages = c->n_pages; a.max_pages = c->max_pages; a.S_cap = c->S_cap;
  a.page_shift = __builtin_ctz((unsigned)c->page_rows);
  a.row_cap = c->max_pages * c->page_rows;
  a.max_len = c->max_len < a.row_cap ? c->max_len : a.row_cap;
  a.row_start = rows->row_start; a.n_rows = rows->n_rows;
  a.max_rows = rows->max_rows < rows->n_rows ? rows->max_rows : rows->n_rows;
  return AKVQ_OK;
}

int paged_bytes(const akvq_paged *shape, int bits, size_t out_bytes[8]) {
  const int st = check_paged_shape(shape);
  if (st != AKVQ_OK) return st;
  if (!out_bytes) return AKVQ_ERR_INVALID_ARG;
  const size_t rows = (size_t)shape->n_pages * shape->Hkv * shape->page_rows, units = (size_t)shape->B * shape->Hkv;
  out_bytes[0] = out_bytes[1] = rows * 16 * bits;
  out_bytes[2] = out_bytes[3] = rows * (128 / shape->G) * 4;
  out_bytes[4] = out_bytes[5] = units * shape->S_cap * 256;
  out_bytes[6] = units * shape->S_cap * 4;
  out_bytes[7] = (units * 4 + 15) / 16 * 16;
  return AKVQ_OK;
}

// Arguments of a call that writes rows into pages; allowed: its flags.  a.c.max_rows is 0 where there is nothing to do.
int append_args(const akvq_paged *c, const akvq_chunk *rows, const void *k, int64_t k_stride, const void *v, int64_t v_stride, float clip,
                uint32_t flags, uint32_t allowed, akvq::PagedAppendArgs &a) {
  const int st = paged_args(c, rows, a.c);
  if (st != AKVQ_OK) return st;
  if (!(clip > 0.0f) || clip > 1.0f) return AKVQ_ERR_INVALID_ARG;
  if (flags & ~allowed) return AKVQ_ERR_INVALID_ARG;
  if (a.c.max_rows == 0) return AKVQ_OK;
  if (check_rows(k, k_stride, c->Hkv) != AKVQ_OK || check_rows(v, v_stride, c->Hkv) != AKVQ_OK) return AKVQ_ERR_INVALID_ARG;
  a.k = static_cast<const uint16_t *>(k); a.v = static_cast<const uint16_t *>(v);
  a.k_stride = k_stride; a.v_stride = v_stride;
  a.clip = clip;
  a.rotate_k = (flags & AKVQ_K_PREROTATED) ? 0 : 1;
  a.rotate_v = (flags & AKVQ_V_PREROTATED) ? 0 : 1;
  return AKVQ_OK;
}

int default_splits(const akvq_paged *c, int Hq, int max_rows, int bits) {
  if (check_paged_shape(c) != AKVQ_OK || Hq <= 0 || Hq % c->Hkv != 0 || max_rows <= 0) return 1;
  const int64_t cap = (int64_t)c->max_pages * c->page_rows;
  return akvq::paged_splits((long)c->B * c->Hkv, max_rows, Hq / c->Hkv, (long)(c->max_len < cap ? c->max_len : cap), {bits, c->G});
}

// Arguments of attention over pages; default_splits: the library's choice for the caller's bound.  a.c.max_rows is 0 where there is nothing to do.
template <typename Splits>
int attention_args(const akvq_paged *c, const akvq_chunk *rows, const void *q, int64_t q_stride, int Hq, const void *k, int64_t k_stride,
                   const void *v, int64_t v_stride, float sm_scale, void *out, int64_t out_stride, float *lse_out, int n_split,
                   void *workspace, size_t workspace_bytes, uint32_t flags, Splits &&default_splits, akvq::PagedAttentionArgs &a) {
  const int st = paged_args(c, rows, a.c);
  if (st != AKVQ_OK) return st;
  if (Hq <= 0 || Hq % c->Hkv != 0) return AKVQ_ERR_INVALID_ARG;
  if (Hq / c->Hkv > 8) return AKVQ_ERR_UNSUPPORTED;
  if ((int64_t)rows->n_rows * Hq >= (1ll << 31)) return AKVQ_ERR_UNSUPPORTED;
  if ((int64_t)a.c.max_rows * (Hq / c->Hkv) > 65535ll * akvq::kPagedManyRows) return AKVQ_ERR_UNSUPPORTED;
  if (flags & ~(uint32_t)(AKVQ_Q_PREROTATED | AKVQ_OUT_ROTATED) || n_split > 1024) return AKVQ_ERR_INVALID_ARG;
  if (a.c.max_rows == 0) return AKVQ_OK;
  if (check_rows(q, q_stride, Hq) != AKVQ_OK || check_rows(k, k_stride, c->Hkv) != AKVQ_OK || check_rows(v, v_stride, c->Hkv) != AKVQ_OK ||
      check_rows(out, out_stride, Hq) != AKVQ_OK)
    return AKVQ_ERR_INVALID_ARG;
  if (lse_out && !aligned(lse_out, 4)) return AKVQ_ERR_INVALID_ARG;
  if (n_split <= 0) n_split = default_splits();  // (of the caller's bound: what its workspace is sized for)
  if (n_split > 1) {
    if (!workspace || !aligned(workspace, 16)) return AKVQ_ERR_INVALID_ARG;
    if (workspace_bytes < akvq_paged_workspace_bytes(rows->n_rows, Hq, n_split)) return AKVQ_ERR_WORKSPACE;
  }
  a.q = static_cast<const uint16_t *>(q); a.k = static_cast<const uint16_t *>(k); a.v = static_cast<const uint16_t *>(v);
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
  a.out = static_cast<uint16_t *>(out); a.lse = lse_out; a.partial = static_cast<float *>(workspace);
  a.Hq = Hq; a.n_split = n_split; a.sm_scale = sm_scale;
  a.q_rotated = (flags & AKVQ_Q_PREROTATED) ? 1 : 0;
  a.out_rotated = (flags & AKVQ_OUT_ROTATED) ? 1 : 0;
  return AKVQ_OK;
}

}  // namespace
