// Attention of few query columns over pages (page_few.h): the launch, and the joining of the parts.
#include "page_few.h"
#include "page_launch.h"

namespace gear {

// Eight waves: with four, and twice the blocks, one token behind 32768 took 21 us instead of 18, two tiles of columns 196 instead of 173 in a mixed batch.
constexpr int FEW_WAVES = 8;

template <int BITS, bool BF, int NC>
__global__ __launch_bounds__(64 * FEW_WAVES) void page_attn_few_kernel(PageAttn a) {
  GEAR_DYN_LDS(lds);
  few_columns<BITS, BF, NC, FEW_WAVES>(a, (int)blockIdx.x, lds);
}

// The records of a column's parts become its output: the weight of a part is 2^(its maximum - the greatest).  One block of four waves per
// column; a lane has two channels.
constexpr int MERGE_WAVES = 4;
__global__ __launch_bounds__(64 * MERGE_WAVES) void page_merge_few_kernel(PageAttn a, int bf) {
  GEAR_DYN_LDS(lds);
  const PageGeom& g = a.geom;
  const int bid = (int)blockIdx.x, col = bid % a.few_cols, rest = bid / a.few_cols, head = rest % g.H, s = rest / g.H;
  const SeqSpan sp = seq_span(a, s);
  const int cols = sp.nq * a.gq;
  if (sp.nq <= 0 || sp.nq > a.few || cols > a.few || col >= cols) return;
  const Parts parts = parts_of(sp.kv, a.n_split, a.least, KEY_STEP);
  if (parts.count <= 1) return;
  const int lane = lane_id(), wave = (int)(threadIdx.x >> 6), count = parts.count;
  const int64_t rec = (((int64_t)s * g.H + head) * a.few_cols + col) * a.n_split;
  // A wave's records on their way, eight at a time, with the first maxima; every wave finds the greatest of all.
  float2 ml[8], v[8];
  auto request = [&](int i0) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = rec + min(i0 + MERGE_WAVES * u, count - 1);
      ml[u] = a.rec_ml[i];
      v[u] = *reinterpret_cast<const float2*>(a.rec_o + i * D + 2 * lane);
    }
  };
  request(wave);
  float top = a.rec_ml[rec + min(lane, count - 1)].x;
  for (int i = lane + 64; i < count; i += 64) top = fmaxf(top, a.rec_ml[rec + i].x);
  top = wave_max(top);
  const float from = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f, x = 0.0f, y = 0.0f;
  for (int i0 = wave; i0 < count; i0 += MERGE_WAVES * 8) {
    if (i0 != wave) request(i0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float by = i0 + MERGE_WAVES * u < count ? GEAR_EXP2(ml[u].x - from) : 0.0f;
      sum += ml[u].y * by;
      x += v[u].x * by;
      y += v[u].y * by;
    }
  }
  float* sh = reinterpret_cast<float*>(lds);   // [wave][3][lane]
  sh[(wave * 3 + 0) * 64 + lane] = sum;
  sh[(wave * 3 + 1) * 64 + lane] = x;
  sh[(wave * 3 + 2) * 64 + lane] = y;
  block_lds_sync();
  if (wave != 0) return;
  for (int w = 1; w < MERGE_WAVES; ++w) {
    sum += sh[(w * 3 + 0) * 64 + lane];
    x += sh[(w * 3 + 1) * 64 + lane];
    y += sh[(w * 3 + 2) * 64 + lane];
  }
  const float r = sum > 0.0f ? 1.0f / sum : 0.0f;
  const int row = col / a.gq, j = col - row * a.gq;
  unsigned char* p = a.out.data + 2 * ((int64_t)(sp.q0 + row) * a.out.token + (int64_t)(head * a.gq + j) * a.out.head + 2 * lane);
  *reinterpret_cast<uint32_t*>(p) = bf ? pack2<true>(x * r, y * r) : pack2<false>(x * r, y * r);
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
  hipLaunchKernelGGL(page_merge_few_kernel, dim3(blocks), dim3(64 * MERGE_WAVES), (size_t)MERGE_WAVES * 3 * 64 * 4, st, a, bf ? 1 : 0);
  return hipGetLastError();
}

}  // namespace gear
