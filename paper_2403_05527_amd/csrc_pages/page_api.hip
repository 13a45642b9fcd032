// Entry points of the paged cache (include/gear.h): arguments are checked here, before anything is launched.
#include <cmath>
#include "page_checks.h"
#include "page_launch.h"

namespace gear {

// The number of equal parts of the key axis that a model finds the fastest, in ns: `blocks` of them undivided on `slots` places, each taking `once` and 2 us
// per `step` tokens, begun or whole; all together no less than `bytes` (the memory's share); with more than one part, a merge whose records (`records` bytes
// per part) are written and read at 5 TB/s.  A quarter of the lesser of the two bounds is added: blocks of unequal length.
// crowded: what a block's time is multiplied by where there are more than CUs (the last to end shares its CU); `merges`: the blocks of the merge, 2.2 ns each.
// filled: parts have a length, not a number, so sequences shorter than max_kv make fewer; but no more than 86 % of the slots count, since blocks that end at once
// leave the XCDs unevenly filled (504 parts on 512 slots: the last dozen began when the first had ended).
int best_parts(int64_t blocks, double filled, int slots, int most_blocks, int max_kv, int least_part, double once, int step, double crowded, double bytes,
                      double records, double merges) {
  const int64_t by_blocks = blocks > 0 ? most_blocks / blocks : 1;
  const int by_keys = max_kv / least_part, most = (int)(by_blocks < by_keys ? by_blocks : by_keys);
  int best = 1;
  double least = 0.0;
  for (int n = 1; n <= most; ++n) {
    const int64_t len = ((int64_t)max_kv + n - 1) / n;
    const double block = (once + 2000.0 * (double)((len + step - 1) / step)) * (blocks * n > GEAR_PAGE_CUS ? crowded : 1.0);
    const double time = std::ceil((n > 1 ? filled / 0.86 : 1.0) * (double)(blocks * n) / slots) * block;
    const double t = (time > bytes ? time + 0.25 * bytes : bytes + 0.25 * time) + (n > 1 ? 4000.0 + 20.0 * n + 2.2 * merges + records * n * 2.0 / 5000.0 : 0.0);
    if (n == 1 || t < least) {
      best = n;
      least = t;
    }
  }
  return best;
}

PagePlan page_plan(int H, int gq, int n_seqs, int n_tokens, int max_q, int max_kv, int bytes_per_key) {
  PagePlan p{};
  const int64_t cols = (int64_t)max_q * gq;
  const bool all_few = cols <= FEW_COLS_MOST;
  // (a batch that is not n_seqs x max_q has shorter sequences, single tokens for instance: one tile of columns is theirs, if it holds one)
  const bool uniform = (int64_t)n_seqs * max_q == n_tokens;
  p.few = all_few || (!uniform && gq <= FEW_COLS_MOST);
  p.many = !all_few;
  p.few_limit = !p.few ? 0 : all_few ? (int)cols : gq <= 16 ? 16 : FEW_COLS_MOST;
  p.few_tiles = p.few_limit <= 16 ? 1 : 2;
  p.few_split = p.many_split = 1;
  // Both in one launch (page_mixed.hip), but where the few columns' bytes take most of the time, and long: there their blocks are better off with eight waves
  // and the chip to themselves.  Estimates in us, at 6 TB/s and 1 PFLOP/s, from the bounds alone.  (One launch and two: 33 sequences of up to 4000 tokens,
  // three of them chunks of up to 700, 110 and 150 us; 20 of up to 1000 tokens, one chunk of 100, 34 and 50; 10 of up to 5908 tokens of 32
  // heads at 16 bits, two chunks of 415, 231 and 194.)
  const double few_us = (double)n_seqs * H * max_kv * bytes_per_key / 6e6, many_us = (double)n_tokens * H * gq * max_kv * 512.0 / 1e9;
  p.one_launch = p.few && p.many && !(few_us > 100.0 && few_us > 2.0 * many_us);
  const double filled = n_seqs >= 4 ? 0.75 : 1.0;
  if (p.few) {
    // A block of eight waves: 4 us (its launch, the first loads, the joining of its waves) and 2 us per step of its waves, 256 tokens; more blocks than CUs take a
    // third longer.  In graphs: 1 x 8 heads x 8192 tokens at 8 bits 10.2 us in 32 parts, 12.4 in 16, 16.0 in 8; x 32768 at 4 bits 15.9 in 32, 19.0 in 43, 18.0 in
    // 55; four rows of 5 sequences of 3000 tokens 15.0 in 6, 240 blocks, 18.0 in 8 and 17.6 in 11.  33 sequences of 600 to 4000 tokens, 264 blocks: 46 undivided, 41
    // and 15 of merging in three parts.
    const int64_t blocks = (int64_t)n_seqs * H;
    // In one launch with blocks of many columns they have four waves, a step is half as long, and nobody waits for them before the others' operations are done
    // (6 sequences of up to 3000 tokens, 32 heads, one of them a chunk of up to 200: 58 us as if alone, 48 so).
    const double bytes_ns = 1000.0 * few_us + (p.one_launch ? 1000.0 * many_us : 0.0), records = (double)blocks * p.few_limit;
    p.few_split = best_parts(blocks, filled, p.few_tiles == 1 ? FEW_SLOTS : FEW_SLOTS / 2, FEW_BLOCKS_MOST, max_kv, FEW_PART, 4000.0, p.one_launch ? FEW_PART / 2 : FEW_PART,
                             p.one_launch ? 1.0 : 1.35, bytes_ns, records * RECORD_BYTES, records);
    if (p.few_split > 1) p.few_rows = (int64_t)n_seqs * H * p.few_limit;
  }
  if (p.many) {
    // A block: 6 us and 2 us per tile of 64 tokens.  Four chunks of 512 tokens behind 4096, 512 blocks: 182 us undivided, and two parts would take 34 for their records
    // alone; three chunks of 483 to 566 behind up to 2900, 416 blocks: 100 us undivided, 140 in two parts.
    const int64_t tiles = uniform ? (cols + MANY_COLS - 1) / MANY_COLS * n_seqs : ((int64_t)n_tokens * gq + MANY_COLS - 1) / MANY_COLS;
    const int64_t rows = (int64_t)n_tokens * H * gq;
    p.many_split = best_parts(tiles * H, filled, MANY_SLOTS, MANY_BLOCKS_MOST, max_kv, MANY_PART, 6000.0, MANY_KEYS, 1.0, 0.0, (double)rows * RECORD_BYTES, 0.0);
    p.many_least = max_kv / p.many_split > MANY_PART ? max_kv / p.many_split : MANY_PART;
    if (p.many_split > 1) p.many_rows = (int64_t)n_tokens * H * gq;
  }
  return p;
}

int64_t page_records_most(int H, int gq, int n_seqs, int n_tokens, int max_q, int max_kv) {
  // rows x parts of either kernel, each bounded by what the slots allow and by what the keys allow
  const int64_t few_cols = (int64_t)max_q * gq < FEW_COLS_MOST ? (int64_t)max_q * gq : FEW_COLS_MOST;
  int64_t few = 0, many = 0;
  if (max_kv / FEW_PART > 1) {
    const int64_t by_keys = (int64_t)n_seqs * H * (max_kv / FEW_PART), blocks = by_keys < FEW_BLOCKS_MOST ? by_keys : FEW_BLOCKS_MOST;
    few = blocks * few_cols;
  }
  if ((int64_t)max_q * gq > FEW_COLS_MOST && max_kv / MANY_PART > 1) {
    const int64_t by_keys = (int64_t)n_tokens * H * gq * (max_kv / MANY_PART), by_slots = (int64_t)MANY_BLOCKS_MOST * MANY_COLS;
    many = by_keys < by_slots ? by_keys : by_slots;
  }
  return few + many;
}

}  // namespace gear

using namespace gear;

namespace {

int copy_rows(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_rows* K, const gear_page_rows* V,
              int32_t n_seqs, int32_t n_rows, const int64_t* slots, bool write, void* stream) {
  PageGeom g;
  int rc = check_pool(cfg, pool, pool_bytes, &g);
  if (rc) return rc;
  if (n_seqs < 0 || n_rows < 0 || (write ? !K || !V : !K && !V)) return GEAR_EINVAL;
  const int64_t total = (int64_t)n_seqs * n_rows;
  if (total == 0) return GEAR_OK;   // (tensors without an entry have no address)
  if (K && (rc = check_rows(K, n_seqs, n_rows, cfg->H_kv, !write))) return rc;
  if (V && (rc = check_rows(V, n_seqs, n_rows, cfg->H_kv, !write))) return rc;
  if (!slots) return GEAR_EINVAL;
  if (misaligned(slots, 8)) return GEAR_EALIGN;
  const int64_t chunks = n_rows == 1 ? ((int64_t)n_seqs + 15) / 16 : (int64_t)n_seqs * (((int64_t)n_rows + 15) / 16);   // of 16 rows, a block for each head, at most
  if (total > INT_MOST - 4096 || chunks * cfg->H_kv > THREADS_MOST / 256) return GEAR_ECAPACITY;
  return launch_page_copy(g, cfg->bits, cfg->dtype == GEAR_BF16, write, view_of(K), view_of(V), slots, n_seqs, n_rows,
                          static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

}  // namespace

extern "C" {

int gear_page_bytes(const gear_page_config* cfg, size_t* pool_bytes) {
  PageGeom g;
  size_t need = 0;
  const int rc = check_page_config(cfg, &need, &g);
  if (rc) return rc;
  if (!pool_bytes) return GEAR_EINVAL;
  *pool_bytes = need;
  return GEAR_OK;
}

int gear_page_write(const gear_page_config* cfg, void* pool, size_t pool_bytes, const gear_page_rows* K, const gear_page_rows* V,
                    int32_t n_seqs, int32_t n_rows, const int64_t* slots, void* stream) {
  return copy_rows(cfg, pool, pool_bytes, K, V, n_seqs, n_rows, slots, true, stream);
}

int gear_page_read(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_rows* K, const gear_page_rows* V,
                   int32_t n_seqs, int32_t n_rows, const int64_t* slots, void* stream) {
  return copy_rows(cfg, pool, pool_bytes, K, V, n_seqs, n_rows, slots, false, stream);
}

int gear_page_attn_bytes(const gear_page_config* cfg, int32_t H_q, const gear_page_batch* batch, size_t* workspace_bytes) {
  PageGeom g;
  size_t need = 0;
  int rc = check_page_config(cfg, &need, &g);
  if (rc || (rc = check_batch(cfg, H_q, batch))) return rc;
  if (!workspace_bytes) return GEAR_EINVAL;
  *workspace_bytes = RECORD_BYTES * (size_t)page_records_most(cfg->H_kv, H_q / cfg->H_kv, batch->n_seqs, batch->n_tokens, batch->max_q, batch->max_kv);
  return GEAR_OK;
}

int gear_page_attn(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_batch* batch, const gear_page_rows* q,
                   int32_t H_q, float scale, const gear_page_rows* out, void* workspace, size_t workspace_bytes, void* stream) {
  PageAttn a{};
  const int rc = check_attn(cfg, pool, pool_bytes, batch, q, H_q, scale, out, workspace, &a);
  if (rc) return rc;
  const gear_page_batch& b = *batch;
  if (b.n_seqs == 0 || b.n_tokens == 0 || b.max_q == 0) return GEAR_OK;
  const int H = cfg->H_kv, gq = H_q / H;
  const int per_key = 2 * (int)(a.geom.block_bytes >> a.geom.shift);
  const PagePlan p = page_plan(H, gq, b.n_seqs, b.n_tokens, b.max_q, b.max_kv, per_key);
  const int64_t few_recs = p.few_rows * p.few_split, many_recs = p.many_rows * p.many_split;
  if (few_recs + many_recs > 0) {
    if (!workspace) return GEAR_EINVAL;
    if (workspace_bytes < RECORD_BYTES * (size_t)(few_recs + many_recs)) return GEAR_ECAPACITY;
  }
  const int64_t tiles = (int64_t)b.n_tokens * gq / MANY_COLS + b.n_seqs;
  if ((int64_t)b.n_seqs * H * p.few_split + tiles * H * p.many_split > THREADS_MOST / 512) return GEAR_ECAPACITY;

  a.few = p.few_limit;
  a.few_cols = p.few_limit;
  a.tiles = (int32_t)tiles;
  // the sums of both kinds, 512 bytes a record (they are stored 16 bytes at a time), then the (maximum, sum) pairs
  float* const sums = static_cast<float*>(workspace);
  float2* const pairs = reinterpret_cast<float2*>(sums + (many_recs + few_recs) * D);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const bool bf = cfg->dtype == GEAR_BF16;
  PageAttn m = a, f = a;
  m.n_split = p.many_split;
  m.least = p.many_least;
  m.rec_o = sums;
  m.rec_ml = pairs;
  f.n_split = p.few_split;
  f.least = FEW_PART;
  f.rec_o = sums + many_recs * D;
  f.rec_ml = pairs + many_recs;
  if (p.one_launch) return launch_page_mixed(m, f, cfg->bits, bf, p.few_tiles, st) == hipSuccess ? GEAR_OK : GEAR_EHIP;
  if (p.many && launch_page_many(m, cfg->bits, bf, st) != hipSuccess) return GEAR_EHIP;
  if (p.few && launch_page_few(f, cfg->bits, bf, p.few_tiles, st) != hipSuccess) return GEAR_EHIP;
  return GEAR_OK;
}

}  // extern "C"
