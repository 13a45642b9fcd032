// Entry points of attention with shared prefixes (include/gear.h): arguments are checked and the work is divided here, before anything is launched.
#include <cmath>
#include "page_checks.h"
#include "shared.h"

namespace gear {

// Records of a call, at most: 512 MB.  A part of the keys has a record for each of its columns, and no axis is divided into more parts than fill the chip once and a half.
constexpr int64_t RECORDS_MOST = (512ll << 20) / (int64_t)RECORD_BYTES, DIVIDED_MOST = (int64_t)MANY_BLOCKS_MOST * MANY_COLS;

static int64_t records_bound(int64_t rows, int max_kv, int max_prefix) {
  const int64_t undivided = 2 * rows, by_blocks = 2 * std::max(rows, DIVIDED_MOST), by_keys = rows * (max_prefix / MANY_PART + max_kv / MANY_PART + 2);
  if (undivided > RECORDS_MOST) return RECORDS_MOST;   // (smaller batches may have as many; this one has none)
  return std::min(RECORDS_MOST, std::min(by_blocks, by_keys));
}

static SharedPlan shared_plan(int H, int gq, const gear_page_batch& b, const gear_page_groups& gr, int bytes_per_key) {
  SharedPlan p{};
  const int64_t rows = (int64_t)b.n_tokens * H * gq;
  // Sequences that have a tile of 128 columns to themselves read a page no more often by themselves than as a group, and need no records for it.
  p.shared = gr.n_groups > 0 && gr.max_prefix >= MANY_KEYS && (int64_t)b.n_tokens * gq < (int64_t)MANY_COLS * b.n_seqs && 2 * rows <= RECORDS_MOST;
  if (!p.shared) return p;
  const int64_t seq_cols = (int64_t)b.max_q * gq, group_cols = std::min((int64_t)gr.max_q, (int64_t)b.n_tokens) * gq, all_cols = (int64_t)b.n_tokens * gq;
  const bool prefix_few = group_cols <= FEW_COLS_MOST;
  const int prefix = std::min(gr.max_prefix, b.max_kv), own = std::max(b.max_kv - prefix, 1);
  const bool uniform = (int64_t)b.n_seqs * b.max_q == b.n_tokens, all_few = seq_cols <= FEW_COLS_MOST;
  const bool few = all_few || (!uniform && gq <= FEW_COLS_MOST), many = !all_few;
  const int few_limit = !few ? 0 : all_few ? (int)seq_cols : gq <= 16 ? 16 : FEW_COLS_MOST;
  p.tiles = few_limit <= 16 && (!prefix_few || group_cols <= 16) ? 1 : 2;
  // parts of the prefixes
  const int64_t tiles = prefix_few ? gr.n_groups : std::max((all_cols + MANY_COLS - 1) / MANY_COLS, (int64_t)gr.n_groups);
  p.prefix.few = prefix_few ? (int)group_cols : 0;
  p.prefix.tiles = (int)(all_cols / MANY_COLS + gr.n_groups);
  const double bytes = (double)gr.n_groups * H * prefix * bytes_per_key / 6e3;   // ns
  p.prefix.n_split = best_parts(tiles * H, 1.0, MANY_SLOTS, MANY_BLOCKS_MOST, prefix, prefix_few ? FEW_PART : MANY_PART, 6000.0, prefix_few ? FEW_PART / 2 : MANY_KEYS, 1.0, bytes,
                                (double)rows * RECORD_BYTES, 0.0);
  while (p.prefix.n_split > 1 && rows * p.prefix.n_split > DIVIDED_MOST) --p.prefix.n_split;
  p.prefix.least = std::max(prefix / p.prefix.n_split, prefix_few ? FEW_PART : MANY_PART);
  // ... and of what lies behind
  p.own_few = SharedKind{1, FEW_PART, few_limit, 0, 0};
  p.own_many = SharedKind{1, MANY_PART, few_limit, (int)(all_cols / MANY_COLS + b.n_seqs), 0};
  if (few) {
    p.own_few.n_split = best_parts((int64_t)b.n_seqs * H, 1.0, FEW_SLOTS, FEW_BLOCKS_MOST, own, FEW_PART, 4000.0, FEW_PART / 2, 1.0, 0.0, (double)rows * RECORD_BYTES, 0.0);
    while (p.own_few.n_split > 1 && rows * p.own_few.n_split > DIVIDED_MOST) --p.own_few.n_split;
  }
  p.own_few.blocks = few ? 1 : 0;
  p.own_many.blocks = many ? 1 : 0;
  p.records = rows * (p.prefix.n_split + std::max(p.own_few.n_split, p.own_many.n_split));
  return p;
}

}  // namespace gear

using namespace gear;

namespace {

int check_groups(const gear_page_groups* g) {
  if (!g || g->n_groups < 0 || g->max_q < 0 || g->max_prefix < 0) return GEAR_EINVAL;
  return GEAR_OK;
}

}  // namespace

extern "C" {

int gear_page_attn_shared_bytes(const gear_page_config* cfg, int32_t H_q, const gear_page_batch* batch, const gear_page_groups* groups, size_t* workspace_bytes) {
  size_t alone = 0;
  int rc = gear_page_attn_bytes(cfg, H_q, batch, &alone);
  if (rc || (rc = check_groups(groups))) return rc;
  if (!workspace_bytes) return GEAR_EINVAL;
  const int64_t most = groups->n_groups == 0 || groups->max_prefix < MANY_KEYS ? 0 : records_bound((int64_t)batch->n_tokens * H_q, batch->max_kv, groups->max_prefix);
  *workspace_bytes = std::max(alone, (size_t)most * RECORD_BYTES);
  return GEAR_OK;
}

int gear_page_attn_shared(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_batch* batch, const gear_page_groups* groups,
                          const gear_page_rows* q, int32_t H_q, float scale, const gear_page_rows* out, void* workspace, size_t workspace_bytes, void* stream) {
  SharedCall c{};
  int rc = check_attn(cfg, pool, pool_bytes, batch, q, H_q, scale, out, workspace, &c.a);
  if (rc || (rc = check_groups(groups))) return rc;
  const gear_page_batch& b = *batch;
  const gear_page_groups& gr = *groups;
  if (b.n_seqs == 0 || b.n_tokens == 0 || b.max_q == 0) return GEAR_OK;
  if (gr.n_groups > 0 && (!gr.group_start || !gr.prefix_len)) return GEAR_EINVAL;
  if (misaligned(gr.group_start, 4) || misaligned(gr.prefix_len, 4)) return GEAR_EALIGN;
  const int H = cfg->H_kv, gq = H_q / H;
  const SharedPlan p = shared_plan(H, gq, b, gr, 2 * (int)(c.a.geom.block_bytes >> c.a.geom.shift));
  if (!p.shared) return gear_page_attn(cfg, pool, pool_bytes, batch, q, H_q, scale, out, workspace, workspace_bytes, stream);
  if (!workspace) return GEAR_EINVAL;
  if (workspace_bytes < RECORD_BYTES * (size_t)p.records) return GEAR_ECAPACITY;
  c.group_start = gr.group_start;
  c.prefix_len = gr.prefix_len;
  c.n_groups = gr.n_groups;
  c.prefix = p.prefix;
  c.own_few = p.own_few;
  c.own_many = p.own_many;
  c.n_records = p.prefix.n_split + std::max(p.own_few.n_split, p.own_many.n_split);
  const int64_t prefix_blocks = (int64_t)H * p.prefix.n_split * (p.prefix.few > 0 ? gr.n_groups : p.prefix.tiles);
  const int64_t few_blocks = (int64_t)H * p.own_few.n_split * b.n_seqs * p.own_few.blocks, many_blocks = (int64_t)H * p.own_many.n_split * p.own_many.tiles * p.own_many.blocks;
  if (prefix_blocks + few_blocks + many_blocks > THREADS_MOST / 512 || (int64_t)b.n_tokens * H_q > THREADS_MOST / 256) return GEAR_ECAPACITY;
  c.prefix.blocks = (int32_t)prefix_blocks;
  c.own_few.blocks = (int32_t)few_blocks;
  c.own_many.blocks = (int32_t)many_blocks;
  c.a.rec_o = static_cast<float*>(workspace);
  c.a.rec_ml = reinterpret_cast<float2*>(c.a.rec_o + p.records * D);
  return launch_page_shared(c, cfg->bits, cfg->dtype == GEAR_BF16, p.tiles, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

}  // extern "C"
