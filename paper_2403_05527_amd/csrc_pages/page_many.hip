// Attention of many query columns over pages (page_many.h): the launch, and the joining of the parts.
#include "page_launch.h"
#include "page_many.h"
#include "page_merge.h"

namespace gear {

// (two waves per SIMD: the compiler's own choice, 311 registers, leaves one, and a prompt of 8192 tokens takes 1.6 times as long)
template <int BITS, bool BF>
__global__ __launch_bounds__(MANY_THREADS, 2) void page_attn_many_kernel(PageAttn a) {
  GEAR_DYN_LDS(lds);
  many_columns<BITS, BF, true>(a, (int)blockIdx.x, lds);
}

// The records of a row's parts become its output (see page_merge_few_kernel): WAVES waves per token and query head, eight records of each on their way.
template <int WAVES>
__global__ __launch_bounds__(256) void page_merge_many_kernel(PageAttn a, int bf) {
  GEAR_DYN_LDS(lds);
  const PageGeom& g = a.geom;
  const int lane = lane_id(), Hq = g.H * a.gq, wave = (int)(threadIdx.x >> 6), mine = WAVES == 1 ? 0 : wave;
  const int64_t id = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  const int token = (int)(id / Hq), jq = (int)(id - (int64_t)token * Hq), head = jq / a.gq;
  if (token >= a.n_tokens) return;
  FirstRecords first = first_records<WAVES>(a, id * a.n_split, mine, lane);
  int s = -1;
  for (int base = 0; base < a.n_seqs; base += 64) {
    const int i = base + lane;
    s += __popcll(__ballot(i < a.n_seqs && a.q_start[i] <= token));
  }
  if (s < 0) return;
  s = GEAR_WAVE_UNIFORM(s);
  const SeqSpan sp = seq_span(a, s);
  const int row = token - sp.q0, cols = sp.nq * a.gq;
  if (row < 0 || row >= sp.nq || (sp.nq <= a.few && cols <= a.few)) return;
  const int col = row * a.gq + (jq - head * a.gq), last = min(col / MANY_COLS * MANY_COLS + MANY_COLS, cols) - 1;
  const int count = parts_of(row_sees(a, sp, last / a.gq), a.n_split, a.least, MANY_KEYS).count;
  if (count <= 1) return;
  const Merged x = merge_records<WAVES>(first, a, id * a.n_split, count, mine, lane, reinterpret_cast<float*>(lds));
  if (mine == 0) store_merged(a, x, token, jq, lane, bf);
}

template <int BITS, bool BF>
static hipError_t launch_many(const PageAttn& a, hipStream_t st) {
  const unsigned blocks = (unsigned)(a.geom.H * a.n_split) * (unsigned)a.tiles;
  hipLaunchKernelGGL((page_attn_many_kernel<BITS, BF>), dim3(blocks), dim3(MANY_THREADS), (size_t)MANY_LDS, st, a);
  return hipGetLastError();
}

hipError_t launch_page_many(const PageAttn& a, int bits, bool bf, hipStream_t st) {
  const hipError_t e = bits == 16 ? (bf ? launch_many<16, true>(a, st) : launch_many<16, false>(a, st))
                     : bits == 8  ? (bf ? launch_many<8, true>(a, st) : launch_many<8, false>(a, st))
                                  : (bf ? launch_many<4, true>(a, st) : launch_many<4, false>(a, st));
  return e != hipSuccess ? e : merge_page_many(a, bf, st);
}

hipError_t merge_page_many(const PageAttn& a, bool bf, hipStream_t st) {
  if (a.n_split == 1) return hipSuccess;
  const int64_t rows = (int64_t)a.n_tokens * a.geom.H * a.gq;
  if (a.n_split <= 8)
    hipLaunchKernelGGL(page_merge_many_kernel<1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a, bf ? 1 : 0);
  else
    hipLaunchKernelGGL(page_merge_many_kernel<4>, dim3((unsigned)rows), dim3(256), (size_t)MERGE_LDS, st, a, bf ? 1 : 0);
  return hipGetLastError();
}

}  // namespace gear
