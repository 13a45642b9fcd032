// Attention of a batch whose sequences share prefixes (include/gear.h): what its kernels and their launch agree on.
#pragma once
#include "page_launch.h"

namespace gear {

// One kind of block of a call: the prefixes of groups, for the columns of all their sequences as if they were one's, or what each sequence has behind
// its prefix; with few columns or many (page_few.h, page_many.h).
struct SharedKind {
  int32_t n_split, least, few;   // as in PageAttn
  int32_t tiles;
  int32_t blocks;
};
struct SharedCall {
  PageAttn a;             // n_seqs, q_start, kv_len, table and the rest of the batch; records [token][query head][n_records]
  const int32_t* group_start;
  const int32_t* prefix_len;
  int32_t n_groups;
  int32_t n_records;      // parts of prefixes, then of what lies behind
  int32_t usual_records;  // of most rows (SharedPlan)
  SharedKind prefix, own_many, own_few;   // few > 0 in `prefix`: by the kernel of few columns
};

struct SharedPlan {
  bool shared;            // else the call is gear_page_attn's
  SharedKind prefix, own_many, own_few;   // blocks: not set
  int tiles;              // of 16 columns, of the kernel of few
  int usual_records;      // of a row that has no more behind its prefix than the longest sequence has behind the longest prefix
  int64_t records;
};

hipError_t launch_page_shared(const SharedCall& c, int bits, bool bf, int tiles, hipStream_t st);

}  // namespace gear
