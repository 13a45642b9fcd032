// Checks of what a call over a pool is given, before anything is launched.
#pragma once
#include <cmath>
#include "gear.h"
#include "page_launch.h"

namespace gear {

constexpr int64_t INT_MOST = 0x7FFFFFFF, THREADS_MOST = 0xFFFFFFFF;   // of a launch

inline int check_page_config(const gear_page_config* c, size_t* pool_bytes, PageGeom* g) {
  if (!c) return GEAR_EINVAL;
  if (c->d_h != D || c->n_pages < 1 || c->H_kv < 1 || c->H_kv > 1024) return GEAR_EINVAL;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return GEAR_EINVAL;
  if (c->bits != 16 && c->bits != 8 && c->bits != 4) return GEAR_EINVAL;
  if (c->bits != 16 && c->group != 32 && c->group != 64 && c->group != 128) return GEAR_EINVAL;
  if (c->dtype != GEAR_F16 && c->dtype != GEAR_BF16) return GEAR_EINVAL;
  const int group = c->bits == 16 ? D : c->group;
  g->row_bytes = (uint32_t)(D * c->bits / 8);
  g->block_bytes = (uint32_t)c->page_size * (g->row_bytes + (c->bits == 16 ? 0u : 4u * (uint32_t)(D / group)));
  g->page_bytes = 2ull * (uint64_t)c->H_kv * g->block_bytes;
  g->n_pages = c->n_pages;
  g->shift = __builtin_ctz((unsigned)c->page_size);
  g->gshift = __builtin_ctz((unsigned)group);
  g->H = c->H_kv;
  g->pool = nullptr;
  if (g->page_bytes >= (1ull << 31)) return GEAR_ECAPACITY;
  *pool_bytes = (size_t)g->page_bytes * (size_t)c->n_pages;
  return GEAR_OK;
}

inline bool misaligned(const void* p, uintptr_t by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; }

inline int check_pool(const gear_page_config* cfg, const void* pool, size_t pool_bytes, PageGeom* g) {
  size_t need = 0;
  const int rc = check_page_config(cfg, &need, g);
  if (rc) return rc;
  if (!pool) return GEAR_EINVAL;
  if (misaligned(pool, 16)) return GEAR_EALIGN;
  if (pool_bytes < need) return GEAR_ECAPACITY;
  g->pool = static_cast<const unsigned char*>(pool);
  return GEAR_OK;
}

// Whether rows of these strides lie over one another: within one direction, or one step of two directions in the same place.  (Whatever is laid out one direction
// after the other does not; strides that overlap in other ways are the caller's.)
inline bool rows_overlap(int64_t n_seqs, int64_t seq, int64_t n_rows, int64_t token, int64_t heads, int64_t head) {
  const int64_t count[3] = {n_seqs, n_rows, heads}, stride[3] = {seq, token, head};
  for (int i = 0; i < 3; ++i) {
    if (count[i] <= 1) continue;
    if (stride[i] < D && stride[i] > -D) return true;
    for (int j = 0; j < i; ++j)
      if (count[j] > 1 && (stride[i] == stride[j] || stride[i] == -stride[j])) return true;
  }
  return false;
}
inline int check_rows(const gear_page_rows* r, int64_t n_seqs, int64_t n_rows, int64_t heads, bool written) {
  if (!r->data) return GEAR_EINVAL;
  if (misaligned(r->data, 16) || (n_seqs > 1 && r->seq % 8) || (n_rows > 1 && r->token % 8) || (heads > 1 && r->head % 8)) return GEAR_EALIGN;
  if (written && rows_overlap(n_seqs, r->seq, n_rows, r->token, heads, r->head)) return GEAR_EINVAL;
  return GEAR_OK;
}
inline RowView view_of(const gear_page_rows* r) {
  return r ? RowView{static_cast<unsigned char*>(r->data), r->seq, r->token, r->head} : RowView{nullptr, 0, 0, 0};
}
inline int check_batch(const gear_page_config* cfg, int32_t H_q, const gear_page_batch* b) {
  if (!b || H_q < 1 || H_q % cfg->H_kv) return GEAR_EINVAL;
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_q < 0 || b->max_kv < 0) return GEAR_EINVAL;
  // (all indices of columns, blocks and records' rows are 32-bit numbers)
  if ((int64_t)b->n_tokens * H_q > INT_MOST || (int64_t)b->max_q * H_q > INT_MOST) return GEAR_ECAPACITY;
  if ((int64_t)b->n_seqs * H_q * FEW_COLS_MOST > INT_MOST) return GEAR_ECAPACITY;
  return GEAR_OK;
}
// What gear_page_attn and its kind are given, and what of it goes to the kernels as it is (nothing of it where there are no rows).
inline int check_attn(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_batch* batch, const gear_page_rows* q, int32_t H_q, float scale,
                      const gear_page_rows* out, const void* workspace, PageAttn* to) {
  PageAttn& a = *to;
  int rc = check_pool(cfg, pool, pool_bytes, &a.geom);
  if (rc || (rc = check_batch(cfg, H_q, batch))) return rc;
  const gear_page_batch& b = *batch;
  const float scale_log2 = std::fabs(scale) * 1.44269504088896340736f;
  if (!q || !out || !std::isfinite(scale_log2) || b.table_width < 0) return GEAR_EINVAL;
  if (b.n_seqs == 0 || b.n_tokens == 0 || b.max_q == 0) return GEAR_OK;
  if ((rc = check_rows(q, 1, b.n_tokens, H_q, false)) || (rc = check_rows(out, 1, b.n_tokens, H_q, true))) return rc;
  if (!b.q_start || !b.kv_len || (b.table_width > 0 && !b.page_table)) return GEAR_EINVAL;
  if (misaligned(b.q_start, 4) || misaligned(b.kv_len, 4) || misaligned(b.page_table, 4) || misaligned(workspace, 16)) return GEAR_EALIGN;
  if ((int64_t)b.table_width * cfg->page_size > INT_MOST - 1024) return GEAR_ECAPACITY;
  a.q_start = b.q_start;
  a.kv_len = b.kv_len;
  a.table = b.page_table;
  a.q = view_of(q);
  a.out = view_of(out);
  a.scale_log2 = std::fmax(scale_log2, 1e-37f);   // (a scale of 0: every score comes to less than a step of 2^0)
  a.far = 0x1p23f / a.scale_log2;
  a.flip = scale < 0.0f ? 0x80008000u : 0u;
  a.width = b.table_width;
  a.n_seqs = b.n_seqs;
  a.n_tokens = b.n_tokens;
  a.gq = H_q / cfg->H_kv;
  a.causal = b.causal ? 1 : 0;
  return GEAR_OK;
}

}  // namespace gear
