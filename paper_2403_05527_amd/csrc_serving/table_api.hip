// Entry points of page tables (include/gear.h): arguments are checked here, before anything is launched.
#include "page_checks.h"
#include "serving.h"

using namespace gear;

namespace {

constexpr int PAGES_MOST = 1 << 20, ROWS_MOST = 1 << 18;

int check_table(const gear_page_table* t, int64_t n, PageTable* to) {
  if (!t || n < 0) return GEAR_EINVAL;
  if (t->page_size < 16 || t->page_size > 256 || (t->page_size & (t->page_size - 1))) return GEAR_EINVAL;
  if (t->n_pages < 1 || t->n_rows < 1 || t->width < 1 || !t->table || !t->kv_len || !t->refs) return GEAR_EINVAL;
  if (misaligned(t->table, 4) || misaligned(t->kv_len, 4) || misaligned(t->refs, 16)) return GEAR_EALIGN;
  if (t->n_pages > PAGES_MOST || t->n_rows > ROWS_MOST || (int64_t)t->width * t->page_size > INT_MOST) return GEAR_ECAPACITY;
  *to = PageTable{t->table, t->kv_len, t->refs, t->n_pages, t->n_rows, t->width, __builtin_ctz((unsigned)t->page_size)};
  return GEAR_OK;
}
int check_list(const int32_t* a, const int32_t* b) {
  if (!a || !b) return GEAR_EINVAL;
  return misaligned(a, 4) || misaligned(b, 4) ? GEAR_EALIGN : GEAR_OK;
}

}  // namespace

extern "C" {

int gear_page_extend(const gear_page_table* t, const int32_t* rows, const int32_t* counts, int32_t n, int32_t max_count, int64_t* slots, int32_t* copies,
                     int32_t* refused, void* stream) {
  PageTable p;
  int rc = check_table(t, n, &p);
  if (rc) return rc;
  if (max_count < 0) return GEAR_EINVAL;
  if (n > GEAR_PAGE_LIST_MAX || n * (((int64_t)max_count + SLOT_TOKENS - 1) / SLOT_TOKENS) > THREADS_MOST / SLOT_THREADS) return GEAR_ECAPACITY;
  if (n == 0) return GEAR_OK;
  if ((rc = check_list(rows, counts)) || (rc = check_list(copies, refused))) return rc;
  if (max_count > 0 && !slots) return GEAR_EINVAL;
  if (misaligned(slots, 8)) return GEAR_EALIGN;
  return launch_extend(p, rows, counts, n, max_count, slots, copies, refused, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

int gear_page_truncate(const gear_page_table* t, const int32_t* rows, const int32_t* lens, int32_t n, void* stream) {
  PageTable p;
  int rc = check_table(t, n, &p);
  if (rc) return rc;
  if (n > GEAR_PAGE_LIST_MAX) return GEAR_ECAPACITY;
  if (n == 0) return GEAR_OK;
  if ((rc = check_list(rows, lens))) return rc;
  return launch_truncate(p, rows, lens, n, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

int gear_page_fork(const gear_page_table* t, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  PageTable p;
  int rc = check_table(t, n, &p);
  if (rc) return rc;
  if (n > GEAR_PAGE_LIST_MAX) return GEAR_ECAPACITY;
  if (n == 0) return GEAR_OK;
  if ((rc = check_list(src, dst))) return rc;
  if (((int64_t)p.width + fork_cols(n) - 1) / fork_cols(n) > THREADS_MOST / FORK_THREADS) return GEAR_ECAPACITY;
  return launch_fork(p, src, dst, n, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

int gear_page_compact(const gear_page_table* t, int32_t* moves, int32_t max_moves, int32_t* counts, void* stream) {
  PageTable p;
  int rc = check_table(t, max_moves, &p);
  if (rc) return rc;
  if (!counts || (max_moves > 0 && !moves)) return GEAR_EINVAL;
  if (misaligned(counts, 4) || misaligned(moves, 4)) return GEAR_EALIGN;
  if ((int64_t)p.n_rows * p.width > THREADS_MOST - 1024 || max_moves > PAGES_MOST) return GEAR_ECAPACITY;
  return launch_compact(p, moves, max_moves, counts, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

int gear_page_move(const gear_page_config* cfg, void* pool, size_t pool_bytes, int32_t n_pools, size_t pool_stride, const int32_t* pairs, int32_t n, void* stream) {
  PageGeom g;
  size_t need = 0;
  int rc = check_page_config(cfg, &need, &g);
  if (rc) return rc;
  if (n_pools < 0 || n < 0) return GEAR_EINVAL;
  if (n_pools == 0 || n == 0) return GEAR_OK;
  if (!pool || !pairs || (n_pools > 1 && pool_stride < need)) return GEAR_EINVAL;
  if (misaligned(pool, 16) || (n_pools > 1 && pool_stride % 16) || misaligned(pairs, 4)) return GEAR_EALIGN;
  if (pool_bytes < need || (n_pools > 1 && (pool_bytes - need) / (size_t)(n_pools - 1) < pool_stride)) return GEAR_ECAPACITY;
  const int64_t chunks = ((int64_t)g.page_bytes + MOVE_BYTES - 1) / MOVE_BYTES;
  if (chunks * n > THREADS_MOST / 256 || chunks * n * n_pools > THREADS_MOST / 256) return GEAR_ECAPACITY;
  return launch_move(static_cast<unsigned char*>(pool), g.page_bytes, g.n_pages, n_pools, pool_stride, pairs, n, static_cast<hipStream_t>(stream)) == hipSuccess
             ? GEAR_OK : GEAR_EHIP;
}

}  // extern "C"
