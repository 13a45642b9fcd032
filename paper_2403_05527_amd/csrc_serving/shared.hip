// Attention of a batch whose sequences share prefixes (include/gear.h).
//
// softmax over [prefix, own] is joined from parts: each part of the keys leaves its maximum, its sum of weights and its weighted sum of Values, and the parts are
// brought to the greatest maximum.  The parts of a prefix take the columns of all the group's new tokens as one sequence's, with the keys that all of them see,
// so a page is read once for 128 columns (32 in the kernel of few); what a sequence has behind the prefix is read as in gear_page_attn.  Both kinds of block run in one launch.
// Bound by the matrix cores and exponentials of the prefix's tiles (questions about 6100 tokens, 2596 columns per KV head: 84 us, matrix cores 0.42 busy), by the bytes of what lies behind (64 sequences
// of 100 to 1000 tokens behind 8192, 188 MB: 50 us), or, where both are small, by a block's chain of loads and joins (16 samples behind 2077 tokens, 32 heads: 13.1 us); and by the records, 520 bytes per
// row and part, which the joining reads back.
// A prefix counts to the last whole 64 tokens that every new token of the group sees, so that no key of it is masked from anyone; what is left of it is read with
// each sequence's own tokens.
#include "page_few.h"
#include "page_many.h"
#include "page_merge.h"
#include "shared.h"

namespace gear {

struct SharedPart : PageAttn {
  const int32_t* group_start;
  const int32_t* prefix_len;
  int32_t n_groups, n_records, first_record;
  int32_t group_cols;   // columns up to which a group has its prefix read; 0: any number
  bool prefix;
};

__device__ __forceinline__ int wave_least(int v) {
  v = min(v, (int)dpp_u<DPP_XOR1>((uint32_t)v));
  v = min(v, (int)dpp_u<DPP_XOR2>((uint32_t)v));
  v = min(v, (int)dpp_u<DPP_HALF_MIRROR>((uint32_t)v));
  v = min(v, (int)dpp_u<DPP_MIRROR>((uint32_t)v));
  uint32_t x = (uint32_t)v, y = x;
  GEAR_LANE_SWAP16(x, y);
  v = min((int)x, (int)y);
  x = y = (uint32_t)v;
  GEAR_LANE_SWAP32(x, y);
  return min((int)x, (int)y);
}
__device__ __forceinline__ int group_bound(const SharedPart& a, int g) { return min(max(a.group_start[g], 0), a.n_seqs); }   // the first sequence of a group, the end of the one before
// The keys that a row count and a length leave before the first new token, which all new tokens see (no new tokens: any number).
__device__ __forceinline__ int keys_before(const SharedPart& a, const SeqSpan& sp) { return sp.nq <= 0 ? INT_MAX : a.causal ? sp.kv - sp.nq : sp.kv; }
__device__ __forceinline__ int whole_tiles(int keys) { return GEAR_WAVE_UNIFORM(max(keys, 0) / MANY_KEYS * MANY_KEYS); }

// A call of up to 64 sequences and 63 groups as a wave has it: sequence i and group i in lane i, so that whatever a block has to know of them is one trip to memory
// (one after the other, which group, its sequences, their lengths, it took 4 us of the 15 of a small call).
struct Lanes {
  SeqSpan sp;    // of sequence i
  int start;     // the first sequence of group i
  int len;       // prefix_len[i]
};
__device__ __forceinline__ bool fits_lanes(const SharedPart& a) { return a.n_seqs <= 64 && a.n_groups < 64; }
__device__ __forceinline__ Lanes load_lanes(const SharedPart& a, int lane) {
  Lanes l;
  l.sp = seq_span(a, min(lane, a.n_seqs - 1));
  l.start = group_bound(a, min(lane, a.n_groups));
  l.len = a.prefix_len[min(lane, a.n_groups - 1)];
  return l;
}
__device__ __forceinline__ SeqSpan lane_span(const Lanes& l, int s) {
  return SeqSpan{__builtin_amdgcn_readlane(l.sp.q0, s), __builtin_amdgcn_readlane(l.sp.nq, s), __builtin_amdgcn_readlane(l.sp.kv, s)};
}
// (a group of more columns than the call's bound shares nothing, and is right all the same)
__device__ __forceinline__ bool too_wide(const SharedPart& a, int rows) { return a.group_cols > 0 && (rows > a.group_cols || rows * a.gq > a.group_cols); }
__device__ __forceinline__ int lane_keys(const SharedPart& a, const Lanes& l, int lane, int g, int s0, int s1) {
  if (s1 <= s0 || too_wide(a, __builtin_amdgcn_readlane(l.sp.q0 + l.sp.nq, s1 - 1) - __builtin_amdgcn_readlane(l.sp.q0, s0))) return 0;
  const int least = wave_least(lane >= s0 && lane < s1 ? keys_before(a, l.sp) : INT_MAX);
  return whole_tiles(min(least, __builtin_amdgcn_readlane(l.len, g)));
}
__device__ __forceinline__ int lane_before(const SharedPart& a, const Lanes& l, int lane, int s) {   // the keys that sequence s shares
  const int g = __popcll(__ballot(lane < a.n_groups && l.start <= s)) - 1;
  if (g < 0) return 0;
  const int s0 = __builtin_amdgcn_readlane(l.start, g), s1 = __builtin_amdgcn_readlane(l.start, g + 1);
  return s < s1 ? lane_keys(a, l, lane, g, s0, s1) : 0;
}

// The same from memory, for any number of them.
__device__ __forceinline__ SeqSpan group_rows(const SharedPart& a, int s0, int s1) {   // a group's columns are those of its sequences, one behind the other (kv: not set)
  SeqSpan r{0, 0, 0};
  if (s1 <= s0) return r;
  r.q0 = max(a.q_start[s0], 0);
  r.nq = min(max(a.q_start[s1], 0), a.n_tokens) - r.q0;
  return r;
}
__device__ __forceinline__ int shared_keys(const SharedPart& a, int g, int s0, int s1) {   // the prefix of group g, as far as it counts
  if (too_wide(a, group_rows(a, s0, s1).nq)) return 0;
  int least = INT_MAX;
  for (int base = s0; base < s1; base += 64) {
    const int s = base + lane_id();
    if (s < s1) least = min(least, keys_before(a, seq_span(a, s)));
  }
  return whole_tiles(min(wave_least(least), a.prefix_len[g]));
}
__device__ __forceinline__ int shared_before(const SharedPart& a, int s) {
  int g = -1;
  for (int base = 0; base < a.n_groups; base += 64) {
    const int i = base + lane_id();
    g += __popcll(__ballot(i < a.n_groups && group_bound(a, i) <= s));
  }
  if (g < 0) return 0;
  const int s0 = group_bound(a, g), s1 = group_bound(a, g + 1);
  return s < s1 ? shared_keys(a, g, s0, s1) : 0;
}
// What lies behind the prefixes, longest first: those that begin when the prefixes' blocks have ended are short.  (Not where all have few columns: four blocks to a CU, they mostly begin at once.)
__device__ __forceinline__ int few_sequence(const SharedPart& a, int i) {
  if (a.group_cols > 0 || !fits_lanes(a)) return i;
  const int lane = lane_id();
  const Lanes l = load_lanes(a, lane);
  int own = lane < a.n_seqs ? l.sp.kv : -1;
  for (int g = 0; g < a.n_groups; ++g) {
    const int s0 = __builtin_amdgcn_readlane(l.start, g), s1 = __builtin_amdgcn_readlane(l.start, g + 1), len = max(__builtin_amdgcn_readlane(l.len, g), 0);
    if (lane >= s0 && lane < s1) own = max(own - len, 0);
  }
  int before = 0;
  for (int j = 0; j < a.n_seqs; ++j) {
    const int other = __builtin_amdgcn_readlane(own, j);
    before += other > own || (other == own && j < lane) ? 1 : 0;
  }
  return GEAR_WAVE_UNIFORM(__ffsll((long long)__ballot(lane < a.n_seqs && before == i)) - 1);
}

// Of what lies behind the prefixes all first parts come first: few sequences have more, and the blocks of parts that are not there leave at the end, without looking for the longest.
__device__ __forceinline__ Place few_place(const SharedPart& a, int at) {
  if (a.prefix) return few_place(static_cast<const PageAttn&>(a), at);
  const int part = a.n_split == 1 ? 0 : at / a.n_seqs, i = at - part * a.n_seqs;
  return Place{part == 0 ? few_sequence(a, i) : i, part};
}
__device__ __forceinline__ Place many_place(const SharedPart& a, int at) {
  if (a.prefix) return many_place(static_cast<const PageAttn&>(a), at);
  const int part = a.n_split == 1 ? 0 : at / a.tiles;
  return Place{at - part * a.tiles, part};
}

__device__ __forceinline__ Span span_of(const SharedPart& a, int s) {
  Span r;
  if (fits_lanes(a)) {
    const int lane = lane_id();
    const Lanes l = load_lanes(a, lane);
    if (!a.prefix) return Span{lane_span(l, s), lane_before(a, l, lane, s), s};
    const int s0 = __builtin_amdgcn_readlane(l.start, s), s1 = __builtin_amdgcn_readlane(l.start, s + 1);
    r = Span{SeqSpan{0, 0, 0}, 0, -1};
    const unsigned long long rows = __ballot(lane >= s0 && lane < s1 && l.sp.nq > 0);
    if (rows != 0ull) {
      r.table_row = GEAR_WAVE_UNIFORM(__ffsll((long long)rows) - 1);   // the first that has new tokens: one without may have been freed
      const SeqSpan first = lane_span(l, s0), last = lane_span(l, s1 - 1);
      r.sp = SeqSpan{first.q0, last.q0 + last.nq - first.q0, lane_keys(a, l, lane, s, s0, s1)};
    }
  } else {
    if (!a.prefix) return Span{seq_span(a, s), shared_before(a, s), s};
    const int s0 = group_bound(a, s), s1 = group_bound(a, s + 1);
    r = Span{group_rows(a, s0, s1), 0, -1};
    for (int base = s0; base < s1 && r.table_row < 0; base += 64) {
      const int i = base + lane_id();
      const unsigned long long rows = __ballot(i < s1 && seq_span(a, min(i, a.n_seqs - 1)).nq > 0);
      if (rows != 0ull) r.table_row = GEAR_WAVE_UNIFORM(base + __ffsll((long long)rows) - 1);
    }
    if (r.table_row >= 0 && r.sp.nq > 0) r.sp.kv = shared_keys(a, s, s0, s1);
  }
  if (r.table_row < 0 || r.sp.kv == 0) r.sp.nq = 0;
  return r;
}
__device__ __forceinline__ bool is_output(const SharedPart& a, const Span& span, int parts) { return !a.prefix && span.begin == 0 && parts == 1; }
__device__ __forceinline__ int64_t many_record(const SharedPart& a, int part, int64_t token, int query_head) {
  return (token * ((int64_t)a.geom.H * a.gq) + query_head) * a.n_records + a.first_record + part;
}
__device__ __forceinline__ int64_t few_record(const SharedPart& a, int, int, int, int part, int64_t token, int query_head) { return many_record(a, part, token, query_head); }

// Column tiles: of sequences as for gear_page_attn, of groups alike.
__device__ __forceinline__ ColTile col_tile(const SharedPart& a, int i, int lane) {
  if (!a.prefix) return col_tile(static_cast<const PageAttn&>(a), i, lane);
  if (a.n_groups <= 64) {   // longest first
    int kv = 0, tiles = 0, before = 0;
    if (fits_lanes(a)) {
      const Lanes l = load_lanes(a, lane);
      const int end = __shfl(l.start, min(lane + 1, 63));   // (lanes from n_groups on have the last group's end)
      const int q0 = __shfl(l.sp.q0, min(l.start, 63)), q1 = __shfl(l.sp.q0 + l.sp.nq, max(end - 1, 0));
      kv = l.len;
      tiles = lane < a.n_groups && end > l.start ? many_tiles(a, SeqSpan{q0, q1 - q0, 0}) : 0;
    } else if (lane < a.n_groups) {
      kv = a.prefix_len[lane];
      tiles = many_tiles(a, group_rows(a, group_bound(a, lane), group_bound(a, lane + 1)));
    }
    for (int j = 0; j < a.n_groups; ++j) {
      const int kv_j = __builtin_amdgcn_readlane(kv, j), n = __builtin_amdgcn_readlane(tiles, j);
      before += kv_j > kv || (kv_j == kv && j < lane) ? n : 0;
    }
    const unsigned long long mine = __ballot(i >= before && i < before + tiles);
    if (mine == 0ull) return ColTile{-1, 0};
    const int s = GEAR_WAVE_UNIFORM(__ffsll((long long)mine) - 1);
    return ColTile{s, (__builtin_amdgcn_readlane(before + tiles, s) - 1 - i) * MANY_COLS};
  }
  // group g has the tiles from (its first row of q) * gq / 128 + g on
  int g = -1;
  for (int base = 0; base < a.n_groups; base += 64) {
    const int j = base + lane;
    g += __popcll(__ballot(j < a.n_groups && ((long long)max(a.q_start[group_bound(a, j < a.n_groups ? j : 0)], 0) * a.gq) / MANY_COLS + j <= i));
  }
  g = GEAR_WAVE_UNIFORM(g);
  if (g < 0) return ColTile{-1, 0};
  const SeqSpan sp = group_rows(a, group_bound(a, g), group_bound(a, g + 1));
  const int local = i - (int)(((long long)sp.q0 * a.gq) / MANY_COLS + g);
  return local >= 0 && local < many_tiles(a, sp) ? ColTile{g, local * MANY_COLS} : ColTile{-1, 0};
}

__device__ __forceinline__ SharedPart part_of(const SharedCall& c, const SharedKind& k, bool prefix) {
  SharedPart p;
  static_cast<PageAttn&>(p) = c.a;
  p.group_start = c.group_start;
  p.prefix_len = c.prefix_len;
  p.n_groups = c.n_groups;
  p.n_records = c.n_records;
  p.first_record = prefix ? 0 : c.prefix.n_split;
  p.group_cols = c.prefix.few;
  p.prefix = prefix;
  p.n_split = k.n_split;
  p.least = k.least;
  p.few = k.few;
  p.tiles = k.tiles;
  return p;
}
// (of a prefix: every row sees all of it, whatever the batch says of its new tokens.  `causal` is left for shared_keys.)
__device__ __forceinline__ int row_sees(const SharedPart& a, const SeqSpan& s, int row) { return a.prefix ? s.kv : row_sees(static_cast<const PageAttn&>(a), s, row); }

constexpr int SHARED_WAVES = MANY_THREADS / 64;

// Blocks of many columns first (as in page_mixed.hip), the prefixes' before the others.
template <int BITS, bool BF, int NC>
__global__ __launch_bounds__(MANY_THREADS, 2) void page_attn_shared_kernel(SharedCall c) {
  GEAR_DYN_LDS(lds);
  int bid = (int)blockIdx.x;
  const int prefix_many = c.prefix.few > 0 ? 0 : c.prefix.blocks, many = prefix_many + c.own_many.blocks;
  if (bid < many) {
    const bool prefix = bid < prefix_many;
    const SharedPart p = part_of(c, prefix ? c.prefix : c.own_many, prefix);
    many_columns<BITS, BF, false>(p, prefix ? bid : bid - prefix_many, lds);
  } else {
    bid -= many;
    const int prefix_few = c.prefix.blocks - prefix_many;
    const bool prefix = bid < prefix_few;
    const SharedPart p = part_of(c, prefix ? c.prefix : c.own_few, prefix);
    few_columns<BITS, BF, NC, SHARED_WAVES>(p, prefix ? bid : bid - prefix_few, lds);
  }
}

// Where no block has many columns: without the registers that those need, four blocks to a CU.
template <int BITS, bool BF, int NC>
__global__ __launch_bounds__(64 * SHARED_WAVES) void page_attn_shared_few_kernel(SharedCall c) {
  GEAR_DYN_LDS(lds);
  const int bid = (int)blockIdx.x;
  const bool prefix = bid < c.prefix.blocks;
  const SharedPart p = part_of(c, prefix ? c.prefix : c.own_few, prefix);
  few_columns<BITS, BF, NC, SHARED_WAVES>(p, prefix ? bid : bid - c.prefix.blocks, lds);
}

// The records of a row become its output: a wave per ROWS query heads of a token, ONCE records of each requested with the lengths, the others by as many.  Bound by its chain of
// loads, 5 us for a wave, so that many rows go four to a wave: 20768 rows of four records, 43 MB, a wave per row 20 us, four rows 14.  (Four waves per row: 11 us instead of 7 on 2048 rows of
// nine.)
template <int ONCE>
struct RowRecords {
  float2 ml[ONCE], v[ONCE];
};
template <int ONCE>
__device__ __forceinline__ void request_row(RowRecords<ONCE>& r, const SharedPart& a, int64_t rec, int i0, int lane) {   // in the row, whether they have been written or not
#pragma unroll
  for (int u = 0; u < ONCE; ++u) {
    const int64_t i = rec + min(i0 + u, a.n_records - 1);
    r.ml[u] = a.rec_ml[i];
    r.v[u] = *reinterpret_cast<const float2*>(a.rec_o + i * D + 2 * lane);
  }
}
template <int ROWS, int ONCE>
__global__ __launch_bounds__(256) void page_merge_shared_kernel(SharedCall c, int bf) {
  const SharedPart a = part_of(c, c.own_many, false);
  const int lane = lane_id(), Hq = a.geom.H * a.gq;
  const unsigned id = (blockIdx.x * 4 + (unsigned)GEAR_WAVE_UNIFORM((int)(threadIdx.x >> 6))) * ROWS;   // (rows: below 2^20)
  const int token = (int)(id / (unsigned)Hq), jq0 = (int)(id - (unsigned)token * (unsigned)Hq);
  if (token >= a.n_tokens) return;
  RowRecords<ONCE> r[ROWS];
#pragma unroll
  for (int j = 0; j < ROWS; ++j) request_row(r[j], a, (int64_t)(id + j) * a.n_records, 0, lane);
  int s = -1;
  for (int base = 0; base < a.n_seqs; base += 64) {
    const int i = base + lane;
    s += __popcll(__ballot(i < a.n_seqs && a.q_start[min(i, a.n_seqs - 1)] <= token));
  }
  if (s < 0) return;
  s = GEAR_WAVE_UNIFORM(s);
  const Span span = span_of(a, s);
  const SeqSpan& sp = span.sp;
  const int row = token - sp.q0, cols = sp.nq * a.gq;
  if (row < 0 || row >= sp.nq) return;
  const bool few = sp.nq <= c.own_few.few && cols <= c.own_few.few;
  if (!few && c.own_many.blocks == 0) return;   // (more new tokens than the call's bound: the rows stay)
  const int before = span.begin == 0 ? 0 : parts_of(span.begin, c.prefix.n_split, c.prefix.least, c.prefix.few > 0 ? KEY_STEP : MANY_KEYS).count;
  // (what rounds to one part is one)
  const SharedKind& kind = few ? c.own_few : c.own_many;
  const int behind = sp.kv - span.begin, first_own = c.prefix.n_split;
  const bool divided = kind.n_split > 1 && behind - kind.least >= kind.least - kind.least / 2;
  if (before == 0 && !divided) return;   // (their one part is their output)
  auto join = [&](RowRecords<ONCE>& r, int j, int end) {   // a row's parts 0 .. before - 1 and first_own .. end - 1
    auto written = [&](int i) { return i < before || (i >= first_own && i < end); };
    const int64_t rec = (int64_t)(id + j) * a.n_records;
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < ONCE; ++u) top = written(u) ? fmaxf(top, r.ml[u].x) : top;
    if (end > ONCE) {
      float more = -INFINITY;
      for (int i = ONCE + lane; i < end; i += 64)
        if (written(i)) more = fmaxf(more, a.rec_ml[rec + i].x);
      top = fmaxf(top, wave_max(more));
    }
    const float from = top == -INFINITY ? 0.0f : top;
    Merged m{0.0f, 0.0f, 0.0f};
    for (int i0 = 0; i0 < end; i0 += ONCE) {
      if (i0 > 0) request_row(r, a, rec, i0, lane);
#pragma unroll
      for (int u = 0; u < ONCE; ++u) {
        const bool there = written(i0 + u);
        const float by = there ? GEAR_EXP2(r.ml[u].x - from) : 0.0f;
        m.sum += there ? r.ml[u].y * by : 0.0f;
        m.x += there ? r.v[u].x * by : 0.0f;
        m.y += there ? r.v[u].y * by : 0.0f;
      }
    }
    store_merged(a, m, token, jq0 + j, lane, bf);
  };
  if (!divided) {   // (by itself: with a count for each row 20768 rows took 15 us instead of 14)
#pragma unroll
    for (int j = 0; j < ROWS; ++j) join(r[j], j, first_own + 1);
    return;
  }
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    int keys = behind;
    if (!few) {   // what the last row of the column's tile sees
      const int col = row * a.gq + (jq0 + j) % a.gq, last = min(col / MANY_COLS * MANY_COLS + MANY_COLS, cols) - 1;
      keys = row_sees(a, sp, last / a.gq) - span.begin;
    }
    const int own = parts_of(keys, kind.n_split, kind.least, few ? KEY_STEP : MANY_KEYS).count;
    if (before > 0 || own > 1) join(r[j], j, first_own + own);
  }
}

template <int BITS, bool BF, int NC>
static hipError_t launch_shared(const SharedCall& c, hipStream_t st) {
  if (c.own_many.blocks == 0 && c.prefix.few > 0) {
    constexpr size_t few = few_lds_bytes<NC, SHARED_WAVES>();   // 33 KB for each column tile
    static std::atomic<uint64_t> raised_few{0};
    const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_attn_shared_few_kernel<BITS, BF, NC>), raised_few, few, LDS_PER_CU);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_attn_shared_few_kernel<BITS, BF, NC>), dim3((unsigned)c.prefix.blocks + (unsigned)c.own_few.blocks), dim3(64 * SHARED_WAVES), few, st, c);
    return hipGetLastError();
  }
  const size_t need = few_lds_bytes<NC, SHARED_WAVES>(), lds = need > (size_t)MANY_LDS ? need : (size_t)MANY_LDS;   // 65 KB with two column tiles
  static std::atomic<uint64_t> raised{0};
  const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_attn_shared_kernel<BITS, BF, NC>), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((page_attn_shared_kernel<BITS, BF, NC>), dim3((unsigned)c.prefix.blocks + (unsigned)c.own_many.blocks + (unsigned)c.own_few.blocks), dim3(MANY_THREADS),
                     lds, st, c);
  return hipGetLastError();
}

#ifndef GEAR_MERGE_ROWS_MANY   // (the CPU stand-in lowers it)
#define GEAR_MERGE_ROWS_MANY 4096
#endif
constexpr int64_t MERGE_ROWS_MANY = GEAR_MERGE_ROWS_MANY;   // rows from which on a wave has four of them

hipError_t launch_page_shared(const SharedCall& c, int bits, bool bf, int tiles, hipStream_t st) {
#define GEAR_SHARED(B) \
  (tiles == 1 ? (bf ? launch_shared<B, true, 1>(c, st) : launch_shared<B, false, 1>(c, st)) : (bf ? launch_shared<B, true, 2>(c, st) : launch_shared<B, false, 2>(c, st)))
  hipError_t e = bits == 16 ? GEAR_SHARED(16) : bits == 8 ? GEAR_SHARED(8) : GEAR_SHARED(4);
#undef GEAR_SHARED
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)c.a.n_tokens * c.a.geom.H * c.a.gq;
  const dim3 blocks((unsigned)((rows + 3) / 4));
  if (rows >= MERGE_ROWS_MANY && c.a.geom.H * c.a.gq % 4 == 0 && c.usual_records <= 4)   // (four rows of a wave are one token's)
    hipLaunchKernelGGL((page_merge_shared_kernel<4, 4>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, st, c, bf ? 1 : 0);
  else if (c.usual_records <= 8) hipLaunchKernelGGL((page_merge_shared_kernel<1, 8>), blocks, dim3(256), 0, st, c, bf ? 1 : 0);
  else hipLaunchKernelGGL((page_merge_shared_kernel<1, 16>), blocks, dim3(256), 0, st, c, bf ? 1 : 0);
  return hipGetLastError();
}

}  // namespace gear
