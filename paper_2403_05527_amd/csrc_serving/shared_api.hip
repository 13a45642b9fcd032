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

// Estimates of a call's time, in ns; they choose the parts of the prefixes, and whether they are shared at all.
// Of prefixes in equal parts, `real` blocks in all: a part takes 8 us and, per `step` keys, `alone`, or `beside` where two blocks share a CU.  What lies behind takes `own` by itself, and runs on the
// places that the prefixes' blocks leave until they have ended; the records (`records` bytes) are written and read at 5 TB/s.
struct Shared {
  double prefix;   // until the prefixes' blocks have ended
  double left;     // of the places, for others meanwhile
  double all;
};
static Shared shared_time(double real, int n, int keys, int step, double alone, double beside, double own, double records) {
  const double steps = (double)((((int64_t)keys + n - 1) / n + step - 1) / step), left = real < MANY_SLOTS ? 1.0 - real / MANY_SLOTS : 0.0;
  double block = steps * beside;
  if (real <= GEAR_PAGE_CUS && block > own / left) block = own / left + (steps - own / left / beside) * alone;
  const double prefix = std::ceil(real / MANY_SLOTS) * (8000.0 + block), rest = own - prefix * left;
  return Shared{prefix, left, prefix + (rest > 0.0 ? rest : 0.0) + records * 2.0 / 5000.0};
}
// The number of parts that is the fastest, of `blocks` undivided ones, of which `filled` have keys.  Where much lies behind, the prefixes' blocks are no more than the CUs.
// 64 sequences behind 8192 tokens, bf16, 8 KV heads, 100 to 1000 tokens of their own (37 us by themselves): 76, 50, 47, 54, 52 and 62 us in 4, 8, 12, 16, 24 and 32 parts, and 6 to 12
// of joining; five groups of 1500 to 6001 tokens at 8 bits 47, 32, 34, 37 and 40 in 4, 8, 10, 12 and 24.  Prefixes alone, in 4, 8, 16 and 32 parts: 1024 tokens 13, 11, 11 and 14 us,
// 16384 111, 62, 38 and 31.
static int prefix_parts(double blocks, double filled, int most, int keys, int step, double alone, double beside, double own, double records) {
  int best = 1;
  double least = 0.0;
  for (int n = 1; n <= most; ++n) {
    const double real = blocks * filled * n;
    if (n > 1 && own > 10000.0 && real > GEAR_PAGE_CUS) break;
    const double t = shared_time(real, n, keys, step, alone, beside, own, records * n).all;
    if (n == 1 || t < least) best = n, least = t;
  }
  return best;
}

// What a sequence has behind its prefix is longer than `own` tokens, max_kv less the longest prefix, where it is in no group or in one with a shorter prefix: then it may be all of max_kv,
// which only the device knows.  So parts have a length, and there are as many as bring the longest to half of what the call takes by itself (at ns_per_key), in as many blocks as the chip holds
// twice: most sequences have no more than the usual, and blocks of parts that are not there leave at once, 1000 of them in 2 to 6 us.
// In one part, whatever was there, 16 sequences behind 16000 tokens and one of 16000 by itself took 200 us and take 61, gear_page_attn 120; 8 behind 32000 and 8 of
// 31000 behind 500 686, 227 and 240; 6 behind 32000 and two by themselves 578, 99 and 127; 4 of 7300 behind 1000 and 4 behind 8192 104, 41 and 42.
// Of many columns: two chunks of 64 tokens with 50000 behind 1000 1420, 167 and 160 to 180 us; a chunk of 512 with 30000 beside 15 single tokens 908, 548 and 607;
// 16 questions about 6100 tokens of which one has 30000 more 582, 310 and 405.  With parts of two thirds of these, questions that have no more than 60 tokens 81.7 instead of 79.8.
// (In blocks for eight times what the chip holds: 58 sequences of 7 heads behind 4060 tokens, of which none has more, 36 us instead of 31.)
constexpr int LONGER_LEAST = 1024;
static void divide_longer(SharedKind& k, int own, int max_kv, int64_t blocks, int64_t rows, double by_itself, double ns_per_key) {
  const int parts = k.n_split, enough = std::max(std::max(own / parts, LONGER_LEAST), (int)std::min(0.5 * by_itself / ns_per_key, (double)max_kv));
  k.least = parts > 1 ? own / parts : enough;
  const int64_t wanted = ((int64_t)max_kv + enough / 2) / enough, most = std::min(DIVIDED_MOST / rows, 2 * (int64_t)MANY_SLOTS / std::max(blocks, (int64_t)1));
  k.n_split = (int)std::max((int64_t)parts, std::min(wanted, most));
}

static SharedPlan shared_plan(int H, int gq, const gear_page_batch& b, const gear_page_groups& gr, int bytes_per_key) {
  SharedPlan p{};
  const int64_t rows = (int64_t)b.n_tokens * H * gq, all_cols = (int64_t)b.n_tokens * gq;
  if (gr.n_groups == 0 || gr.max_prefix < MANY_KEYS || 2 * rows > RECORDS_MOST) return p;
  const int64_t seq_cols = (int64_t)b.max_q * gq, group_cols = std::min((int64_t)gr.max_q, (int64_t)b.n_tokens) * gq;
  const bool prefix_few = group_cols <= FEW_COLS_MOST;
  const int prefix = std::min(gr.max_prefix, std::max(b.max_kv, MANY_KEYS)), own = std::max(b.max_kv - prefix, 1);
  const bool uniform = (int64_t)b.n_seqs * b.max_q == b.n_tokens, all_few = seq_cols <= FEW_COLS_MOST;
  const bool few = all_few || (!uniform && gq <= FEW_COLS_MOST), many = !all_few;
  const int few_limit = !few ? 0 : all_few ? (int)seq_cols : gq <= 16 ? 16 : FEW_COLS_MOST;
  p.tiles = few_limit <= 16 && (!prefix_few || group_cols <= 16) ? 1 : 2;
  const double record_bytes = (double)rows * RECORD_BYTES, codes = bytes_per_key < 4 * D ? 1.3 : 1.0;
  // gear_page_attn's time, whose repeated reads of the shared pages the caches serve: 0.04 ns per sequence, KV head and key with few columns (64 sequences of 8300 to 9200 tokens, 8 heads,
  // 174 us, 16 of 2100, 32 heads, 44), 2.36 us per tile of 128 columns and 64 keys on 512 places with many (16 of 6150, 20 to 60 new tokens, 32 query heads over 8: 125 us, shared 97).
  const double keys = (prefix + 0.6 * own) * (double)b.n_seqs * H;
  const double by_itself = all_few ? 7000.0 + 0.04 * (few_limit <= 16 ? 1.0 : 1.4) * keys
                                   : 8000.0 + keys / MANY_KEYS * std::ceil((double)all_cols / b.n_seqs / MANY_COLS) * 2360.0 * codes / MANY_SLOTS;
  // parts of what lies behind the prefixes
  p.own_few = SharedKind{1, FEW_PART, few_limit, 0, 0};
  p.own_many = SharedKind{1, MANY_PART, few_limit, (int)(all_cols / MANY_COLS + b.n_seqs), 0};
  int usual = 1;   // parts of `own` tokens
  if (few) {
    p.own_few.n_split = best_parts((int64_t)b.n_seqs * H, 1.0, FEW_SLOTS, FEW_BLOCKS_MOST, own, FEW_PART, 4000.0, FEW_PART / 2, 1.0, 0.0, record_bytes, 0.0);
    while (p.own_few.n_split > 1 && rows * p.own_few.n_split > DIVIDED_MOST) --p.own_few.n_split;
    usual = std::max(usual, p.own_few.n_split);
    divide_longer(p.own_few, own, b.max_kv, (int64_t)b.n_seqs * H, rows, by_itself, 2000.0 / (FEW_PART / 2));
  }
  if (many) {
    const int64_t blocks = (all_cols + MANY_COLS - 1) / MANY_COLS * H;
    p.own_many.n_split = best_parts(blocks, 1.0, MANY_SLOTS, MANY_BLOCKS_MOST, own, LONGER_LEAST, 6000.0, MANY_KEYS, 1.0, 0.0, record_bytes, 0.0);
    const int64_t places = (int64_t)p.own_many.tiles * H;
    while (p.own_many.n_split > 1 && (rows * p.own_many.n_split > DIVIDED_MOST || places * p.own_many.n_split > 8 * MANY_SLOTS)) --p.own_many.n_split;
    usual = std::max(usual, p.own_many.n_split);
    divide_longer(p.own_many, own, b.max_kv, places, rows, by_itself, 1500.0 * codes / MANY_KEYS);
  }
  // ... and of the prefixes, for each tile of columns
  const int64_t tiles = prefix_few ? gr.n_groups : std::max((all_cols + MANY_COLS - 1) / MANY_COLS, (int64_t)gr.n_groups);
  p.prefix.few = prefix_few ? (int)group_cols : 0;
  p.prefix.tiles = (int)(all_cols / MANY_COLS + gr.n_groups);
  const int least = prefix_few ? FEW_PART : MANY_PART;
  const int64_t by_blocks = MANY_BLOCKS_MOST / std::max(tiles * H, (int64_t)1), by_records = std::max(DIVIDED_MOST / rows, (int64_t)1);
  const int most = (int)std::max((int64_t)1, std::min((int64_t)(prefix / least), std::min(by_blocks, by_records)));
  // As far as the bounds show that there are sequences in no group, those have up to max_kv tokens: their bytes, and the longest part of one, which the chip waits for.  (14 questions about
  // 6100 tokens and two by themselves: 147 us shared, 105 as gear_page_attn.  Fewer parts of the prefix beside what lies behind: 6 sequences behind 32000 and two by themselves 118 -> 99 us, 24 of 8 bits behind
  // 6001 and 8 53 -> 42.)
  const int64_t covered = (int64_t)gr.n_groups * gr.max_q;
  const double outside = covered < b.n_tokens ? (double)(b.n_tokens - covered) * b.n_seqs / b.n_tokens : 0.0;   // sequences
  const double own_ns = 6000.0 + 0.6 * ((b.n_seqs - outside) * own + outside * b.max_kv) * H * bytes_per_key / 4.5e3;
  const int longest = outside > 0.0 ? std::min(b.max_kv, 1 << 29) : 0;   // (sums within 32 bits)
  double part = 0.0;
  if (longest > 0 && few) part = 4000.0 + 2000.0 / (FEW_PART / 2) * parts_of(longest, p.own_few.n_split, p.own_few.least, KEY_STEP).len;
  if (longest > 0 && many) part = std::max(part, 6000.0 + 1500.0 * codes / MANY_KEYS * parts_of(longest, p.own_many.n_split, p.own_many.least, MANY_KEYS).len);
  // (Where they are divided, prefixes are taken to be 0.65 of the longest in the mean from four groups on: five of 1500 to 6001 tokens 39 us, 47 taken to be 6001.  Not where the choice is made, by which
  // 12 sequences behind 4096 tokens would be shared in three groups and not in four, 31.5 us for 23.7.)
  const double blocks = (double)(tiles * H), alone = prefix_few ? 2000.0 : 1500.0 * codes, beside = prefix_few ? 2500.0 : 2360.0 * codes;
  const int step = prefix_few ? FEW_PART / 2 : MANY_KEYS;
  p.prefix.n_split = prefix_parts(blocks, gr.n_groups >= 4 ? 0.65 : 1.0, most, prefix, step, alone, beside, own_ns, record_bytes);
  p.prefix.least = std::max(prefix / p.prefix.n_split, least);
  p.own_few.blocks = few ? 1 : 0;
  p.own_many.blocks = many ? 1 : 0;
  const int n_own = std::max(p.own_few.n_split, p.own_many.n_split);
  p.records = rows * (p.prefix.n_split + n_own);
  p.usual_records = p.prefix.n_split + usual;
  const Shared t = shared_time(blocks * (0.8 + 0.2 / gr.n_groups) * p.prefix.n_split, p.prefix.n_split, prefix, step, alone, beside, own_ns, record_bytes * p.prefix.n_split);
  const double shared = std::max(t.all, (t.left > 0.1 ? 0.0 : t.prefix) + part) + 4000.0 + record_bytes * usual * 2.0 / 5000.0;
  p.shared = gr.always != 0 || shared < by_itself;
  return p;
}

}  // namespace gear

using namespace gear;

namespace {

constexpr int GROUPS_MOST = 1 << 20;

int check_groups(const gear_page_groups* g) {
  if (!g || g->n_groups < 0 || g->max_q < 0 || g->max_prefix < 0 || (g->always != 0 && g->always != 1)) return GEAR_EINVAL;
  return g->n_groups > GROUPS_MOST ? GEAR_ECAPACITY : GEAR_OK;
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
  c.usual_records = p.usual_records;
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
