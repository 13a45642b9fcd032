// Rows into the pool's slots and back (include/gear.h has the layout and the quantizer's definition).
//
// 16 lanes take one row of one head, eight channels each: one 16-byte access on the 16-bit side and 16, 8 or 4 bytes on the
// pool's, so that a wave's four rows, consecutive tokens of one head, are consecutive in both.  A group's minimum and maximum
// are exchanges among its 4, 8 or 16 lanes.
#include "page_launch.h"
#include "page_piece.h"

namespace gear {

struct PageCopy {
  PageGeom geom;
  RowView k, v;
  const int64_t* slots;
  int32_t n_rows;     // rows per sequence
  int32_t chunks;     // blocks per sequence and head
};

constexpr int COPY_THREADS = 256, COPY_ROWS = COPY_THREADS / 16;
// grid: (head, 16 rows of one sequence), heads next to each other: all but a lane's row and piece is known to the block, whose scalar unit
// works it out (with a sequence per lane, 8 x 4096 tokens of 8 heads took 38.2 us to 4 bits, not 35.8).  A row per 16 lanes: with two or four, whose loads are
// requested together, the writes took 4 and 12 % longer.
template <int BITS, bool BF, bool WRITE, bool PAST>
__global__ __launch_bounds__(COPY_THREADS) void page_copy_kernel(PageCopy a) {
  const PageGeom& g = a.geom;
  const unsigned bid = blockIdx.x, rest = bid / (unsigned)g.H, s = rest / (unsigned)a.chunks;
  const int h = (int)(bid - rest * (unsigned)g.H), c = threadIdx.x & 15, in_chunk = threadIdx.x >> 4;
  const int first = (int)(rest - s * (unsigned)a.chunks) * COPY_ROWS;
  unsigned char* const kp = a.k.data + 2 * ((int64_t)s * a.k.seq + (int64_t)first * a.k.token + h * a.k.head) + 2 * (in_chunk * a.k.token + 8 * c);
  unsigned char* const vp = a.v.data + 2 * ((int64_t)s * a.v.seq + (int64_t)first * a.v.token + h * a.v.head) + 2 * (in_chunk * a.v.token + 8 * c);
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  const bool there = first + in_chunk < a.n_rows;
  if (WRITE && there) {   // (on their way with the slot, a row that is skipped too: 8 x 4096 tokens of 8 heads to 4 bits 42.5 -> 39.6 us)
    k = *reinterpret_cast<const uint4*>(kp);
    v = *reinterpret_cast<const uint4*>(vp);
  }
  const int64_t slot = there ? a.slots[(int64_t)s * a.n_rows + first + in_chunk] : -1;
  const bool live = slot >= 0 && slot < (int64_t)g.n_pages << g.shift;   // the same for the 16 lanes of a row
  const int64_t at = live ? slot : 0;
  const unsigned char* const keys = block_of(g, (int)(at >> g.shift), h, 0);
  const int row = (int)(at & page_mask(g));
  if (!WRITE && live) {
    if (a.k.data) k = load_piece<BITS, BF>(g, keys, row, c);
    if (a.v.data) v = load_piece<BITS, BF>(g, keys + g.block_bytes, row, c);
  }
  if constexpr (WRITE) {
    unsigned char* block = const_cast<unsigned char*>(keys);
    store_piece<BITS, BF>(g, block, row, c, k, live);
    store_piece<BITS, BF>(g, block + g.block_bytes, row, c, v, live);
  } else if (live) {
    if (a.v.data) store16<PAST>(vp, v);   // (the later request first, so that the stores leave together: 16 x 4096 tokens 289 us, not 300)
    if (a.k.data) store16<PAST>(kp, k);
  }
}

template <int BITS, bool BF, bool WRITE>
static hipError_t launch_copy(const PageCopy& a, int n_seqs, hipStream_t st) {
  const int64_t blocks = (int64_t)n_seqs * a.chunks * a.geom.H;
  if (!WRITE && (int64_t)n_seqs * a.n_rows * a.geom.H * ((a.k.data ? 2 * D : 0) + (a.v.data ? 2 * D : 0)) >= PAST_CACHES)
    hipLaunchKernelGGL((page_copy_kernel<BITS, BF, WRITE, !WRITE>), dim3((unsigned)blocks), dim3(COPY_THREADS), 0, st, a);
  else
    hipLaunchKernelGGL((page_copy_kernel<BITS, BF, WRITE, false>), dim3((unsigned)blocks), dim3(COPY_THREADS), 0, st, a);
  return hipGetLastError();
}

static bool one_run(const RowView& r, int64_t n_rows) { return !r.data || r.seq == n_rows * r.token; }

hipError_t launch_page_copy(const PageGeom& g, int bits, bool bf, bool write, const RowView& k, const RowView& v, const int64_t* slots,
                            int n_seqs, int n_rows, hipStream_t st) {
  PageCopy a{g, k, v, slots, n_rows, 1};
  if (n_rows == 1) {   // single tokens, and sequences that follow one another: the rows of one
    a.k.token = k.seq;
    a.v.token = v.seq;
    a.n_rows = n_seqs;
    n_seqs = 1;
  } else if (one_run(k, n_rows) && one_run(v, n_rows)) {
    a.n_rows = n_seqs * n_rows;
    n_seqs = 1;
  }
  a.chunks = (a.n_rows + COPY_ROWS - 1) / COPY_ROWS;
#define GEAR_PAGE_COPY(B)                                                                     \
  return bf ? (write ? launch_copy<B, true, true>(a, n_seqs, st) : launch_copy<B, true, false>(a, n_seqs, st)) \
            : (write ? launch_copy<B, false, true>(a, n_seqs, st) : launch_copy<B, false, false>(a, n_seqs, st))
  if (bits == 16) {   // (copied as they are: the type does not matter)
    return write ? launch_copy<16, false, true>(a, n_seqs, st) : launch_copy<16, false, false>(a, n_seqs, st);
  }
  if (bits == 8) GEAR_PAGE_COPY(8);
  GEAR_PAGE_COPY(4);
#undef GEAR_PAGE_COPY
}

}  // namespace gear
