// Attention of few query columns over pages (page_few.h): the launch, and the joining of the parts.
#include "page_few.h"
#include "page_launch.h"
#include "page_merge.h"

namespace gear {

// Eight waves: with four, and twice the blocks, one token behind 32768 took 21 us instead of 18.  (Blocks that share a launch with those of many columns have four:
// page_mixed.hip.)
constexpr int FEW_WAVES = 8;

template <int BITS, bool BF, int NC>
__global__ __launch_bounds__(64 * FEW_WAVES) void page_attn_few_kernel(PageAttn a) {
  GEAR_DYN_LDS(lds);
  few_columns<BITS, BF, NC, FEW_WAVES>(a, (int)blockIdx.x, lds);
}

// The records of a column's parts become its output: one block of four waves per column.
__global__ __launch_bounds__(64 * MERGE_WAVES) void page_merge_few_kernel(PageAttn a, int bf) {
  GEAR_DYN_LDS(lds);
  const PageGeom& g = a.geom;
  const int bid = (int)blockIdx.x, col = bid % a.few_cols, rest = bid / a.few_cols, head = rest % g.H, s = rest / g.H;
  const int lane = lane_id(), wave = (int)(threadIdx.x >> 6);
  const int64_t rec = (((int64_t)s * g.H + head) * a.few_cols + col) * a.n_split;
  FirstRecords first = first_records<MERGE_WAVES>(a, rec, wave, lane);
  const SeqSpan sp = seq_span(a, s);
  const int cols = sp.nq * a.gq;
  if (sp.nq <= 0 || sp.nq > a.few || cols > a.few || col >= cols) return;
  const Parts parts = parts_of(sp.kv, a.n_split, a.least, KEY_STEP);
  if (parts.count <= 1) return;
  const Merged x = merge_records<MERGE_WAVES>(first, a, rec, parts.count, wave, lane, reinterpret_cast<float*>(lds));
  if (wave == 0) store_merged(a, x, sp.q0 + col / a.gq, head * a.gq + col % a.gq, lane, bf);
}

template <int BITS, bool BF, int NC>
static hipError_t launch_few(const PageAttn& a, hipStream_t st) {
  const size_t lds = few_lds_bytes<NC, FEW_WAVES>();   // 65 KB for each column tile
  static std::atomic<uint64_t> raised{0};
  const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_attn_few_kernel<BITS, BF, NC>), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  const unsigned blocks = (unsigned)(a.geom.H * a.n_split) * (unsigned)a.n_seqs;
  hipLaunchKernelGGL((page_attn_few_kernel<BITS, BF, NC>), dim3(blocks), dim3(64 * FEW_WAVES), lds, st, a);
  return hipGetLastError();
}

hipError_t launch_page_few(const PageAttn& a, int bits, bool bf, int tiles, hipStream_t st) {
#define GEAR_FEW(B) \
  (tiles == 1 ? (bf ? launch_few<B, true, 1>(a, st) : launch_few<B, false, 1>(a, st)) : (bf ? launch_few<B, true, 2>(a, st) : launch_few<B, false, 2>(a, st)))
  hipError_t e = bits == 16 ? GEAR_FEW(16) : bits == 8 ? GEAR_FEW(8) : GEAR_FEW(4);
#undef GEAR_FEW
  return e != hipSuccess ? e : merge_page_few(a, bf, st);
}

hipError_t merge_page_few(const PageAttn& a, bool bf, hipStream_t st) {
  if (a.n_split == 1) return hipSuccess;
  const unsigned blocks = (unsigned)(a.geom.H * a.few_cols) * (unsigned)a.n_seqs;
  hipLaunchKernelGGL(page_merge_few_kernel, dim3(blocks), dim3(64 * MERGE_WAVES), (size_t)MERGE_LDS, st, a, bf ? 1 : 0);
  return hipGetLastError();
}

}  // namespace gear
