// A batch of chunks and single tokens in one launch: the blocks of many columns (page_many.h) first, bound by their operations and of unequal length,
// then those of few (page_few.h), bound by the pages' bytes, which take the places that the first leave.  Three chunks of 483 to 566 tokens among thirty single
// ones, 4 query heads per KV head: 100 and 46 us one after the other.
#include "page_few.h"
#include "page_launch.h"
#include "page_many.h"

namespace gear {

constexpr int MIXED_WAVES = MANY_THREADS / 64;

template <int BITS, bool BF, int NC>
__global__ __launch_bounds__(MANY_THREADS, 2) void page_attn_mixed_kernel(PageAttn many, PageAttn few, int many_blocks) {
  GEAR_DYN_LDS(lds);
  const int bid = (int)blockIdx.x;
  if (bid < many_blocks) many_columns<BITS, BF, false>(many, bid, lds);
  else few_columns<BITS, BF, NC, MIXED_WAVES>(few, bid - many_blocks, lds);
}

template <int BITS, bool BF, int NC>
static hipError_t launch_mixed(const PageAttn& many, const PageAttn& few, hipStream_t st) {
  const size_t need = few_lds_bytes<NC, MIXED_WAVES>(), lds = need > (size_t)MANY_LDS ? need : (size_t)MANY_LDS;   // 65 KB with two column tiles
  static std::atomic<uint64_t> raised{0};
  const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_attn_mixed_kernel<BITS, BF, NC>), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  const int many_blocks = many.geom.H * many.n_split * many.tiles, few_blocks = few.geom.H * few.n_split * few.n_seqs;
  hipLaunchKernelGGL((page_attn_mixed_kernel<BITS, BF, NC>), dim3((unsigned)many_blocks + (unsigned)few_blocks), dim3(MANY_THREADS), lds, st, many, few, many_blocks);
  return hipGetLastError();
}

hipError_t launch_page_mixed(const PageAttn& many, const PageAttn& few, int bits, bool bf, int tiles, hipStream_t st) {
#define GEAR_MIXED(B)                                                                                    \
  (tiles == 1 ? (bf ? launch_mixed<B, true, 1>(many, few, st) : launch_mixed<B, false, 1>(many, few, st)) \
              : (bf ? launch_mixed<B, true, 2>(many, few, st) : launch_mixed<B, false, 2>(many, few, st)))
  const hipError_t e = bits == 16 ? GEAR_MIXED(16) : bits == 8 ? GEAR_MIXED(8) : GEAR_MIXED(4);
#undef GEAR_MIXED
  if (e != hipSuccess) return e;
  const hipError_t e2 = merge_page_many(many, bf, st);
  return e2 != hipSuccess ? e2 : merge_page_few(few, bf, st);
}

}  // namespace gear
