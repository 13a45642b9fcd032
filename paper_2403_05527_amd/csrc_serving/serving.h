// Host-side launch functions of what stands around the paged cache's reads and writes (include/gear.h): rotary positions, page
// tables, pages moved, prefixes shared.
#pragma once
#include "gear_launch.h"
#include "pages.h"

namespace gear {

// ---- rotary positions
struct Rope {
  const double* freq;   // radians per position of each pair
  int32_t rot;          // channels that turn
  int32_t half;         // rot / 2
  float factor;
  float sign;           // -1: turned back
};
struct RopeRows {
  Rope rope;
  RowView x, out;       // rows that are turned and stored as rows: `heads` of them per token
  RowView k, v;         // rows that go into the pool (k turned)
  PageGeom geom;
  const int64_t* slots;
  const int64_t* positions;
  int32_t n_rows;       // tokens per sequence
  int32_t chunks;       // of 16 tokens per sequence
  int32_t heads, per;   // heads of x, and how many of them a block has
  int32_t kv_per;       // KV heads of a block
  int32_t parts, x_parts;   // blocks per chunk of tokens; of those, the first x_parts have heads of x
};
// bits: 0 where nothing goes into a pool
hipError_t launch_rope(const RopeRows& a, int bits, bool bf, bool interleaved, int n_seqs, hipStream_t st);

// ---- page tables
struct PageTable {
  int32_t* table;
  int32_t* kv_len;
  int32_t* refs;
  int32_t n_pages, n_rows, width, shift;   // shift: log2 of the page size
};
constexpr int SLOT_THREADS = 256, SLOT_TOKENS = 1024;   // where the slots have a launch of their own: a block's
hipError_t launch_extend(const PageTable& t, const int32_t* rows, const int32_t* counts, int n, int most, int64_t* slots, int32_t* copies, int32_t* refused,
                         hipStream_t st);
hipError_t launch_truncate(const PageTable& t, const int32_t* rows, const int32_t* lens, int n, hipStream_t st);
constexpr int FORK_THREADS = 256, FORK_ENTRIES = 8192;   // entries of a block
inline int fork_cols(int n) { return n > FORK_ENTRIES / 64 ? FORK_ENTRIES / n : 64; }   // columns of the table that a block has of n rows
hipError_t launch_fork(const PageTable& t, const int32_t* src, const int32_t* dst, int n, hipStream_t st);
hipError_t launch_compact(const PageTable& t, int32_t* moves, int most, int32_t* counts, hipStream_t st);
constexpr int MOVE_THREADS = 256, MOVE_LOADS = 4, MOVE_BYTES = MOVE_THREADS * MOVE_LOADS * 16;   // a block's share of a page
hipError_t launch_move(unsigned char* pool, uint32_t page_bytes, int n_pages, int n_pools, size_t stride, const int32_t* pairs, int n, hipStream_t st);

}  // namespace gear
