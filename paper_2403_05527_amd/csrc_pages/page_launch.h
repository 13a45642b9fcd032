// Host-side launch functions of the paged cache.
#pragma once
#include "gear_launch.h"
#include "pages.h"

namespace gear {

hipError_t launch_page_copy(const PageGeom& g, int bits, bool bf, bool write, const RowView& k, const RowView& v, const int64_t* slots,
                            int n_seqs, int n_rows, hipStream_t st);

// What a call of gear_page_attn launches: parts of the key axis for sequences of few columns and of many, whether either kind is
// launched, and the records that the parts leave.
struct PagePlan {
  bool few, many, one_launch;
  int few_limit;            // columns up to which a sequence counts as of few
  int few_tiles;            // column tiles of 16 of the few-column kernel (1 or 2)
  int few_split, many_split;
  int many_least;           // tokens of a part, about, where the keys are divided
  int64_t few_rows, many_rows;   // record rows (times the parts), 0 where there is one part
};
PagePlan page_plan(int H, int gq, int n_seqs, int n_tokens, int max_q, int max_kv, int bytes_per_key);   // bytes: of a token in one head
// record rows x parts that no batch within these bounds exceeds
int64_t page_records_most(int H, int gq, int n_seqs, int n_tokens, int max_q, int max_kv);

// the sequences of few columns (tiles: 16 columns each, 1 or 2), those of many, or both, with the joining of their parts
hipError_t launch_page_few(const PageAttn& a, int bits, bool bf, int tiles, hipStream_t st);
hipError_t launch_page_many(const PageAttn& a, int bits, bool bf, hipStream_t st);
hipError_t launch_page_mixed(const PageAttn& many, const PageAttn& few, int bits, bool bf, int tiles, hipStream_t st);
hipError_t merge_page_few(const PageAttn& a, bool bf, hipStream_t st);
hipError_t merge_page_many(const PageAttn& a, bool bf, hipStream_t st);

}  // namespace gear
