// Rows into the pool's slots and back (include/gear.h has the layout and the quantizer's definition).
//
// 16 lanes take one row of one head, eight channels each: one 16-byte access on the 16-bit side and 16, 8 or 4 bytes on the
// pool's, so that a wave's four rows, consecutive tokens of one head, are consecutive in both.  A group's minimum and maximum
// are exchanges among its 4, 8 or 16 lanes.
#include "page_launch.h"

namespace gear {

struct PageCopy {
  PageGeom geom;
  RowView k, v;
  const int64_t* slots;
  int32_t n_rows;     // rows per sequence
  int64_t total;      // rows of all sequences, below 2^31
};

template <int CTRL>
__device__ __forceinline__ void lane_min_max(float& mn, float& mx) {
  mn = fminf(mn, dpp_f<CTRL>(mn));
  mx = fmaxf(mx, dpp_f<CTRL>(mx));
}

// One row piece of eight values into its place: `block` the head's Keys or Values in the page, r the row, c the lane's piece (0..15).  Every
// lane of the wave comes here (its row's extremes are exchanged), those with `live` store.
template <int BITS, bool BF>
__device__ __forceinline__ void store_piece(const PageGeom& g, unsigned char* block, int r, int c, const uint4& x, bool live) {
  if constexpr (BITS == 16) {
    if (live) *reinterpret_cast<uint4*>(block + (r * 16 + c) * 16) = x;
  } else {
    constexpr float LEVELS = BITS == 8 ? 255.0f : 15.0f;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = to_f32<BF>(w[e >> 1] >> (16 * (e & 1)) & 0xFFFFu);
    float mn = f[0], mx = f[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      mn = fminf(mn, f[e]);
      mx = fmaxf(mx, f[e]);
    }
    lane_min_max<DPP_XOR1>(mn, mx);
    lane_min_max<DPP_XOR2>(mn, mx);
    if (g.gshift > 5) lane_min_max<DPP_HALF_MIRROR>(mn, mx);
    if (g.gshift > 6) lane_min_max<DPP_MIRROR>(mn, mx);
    // fp32: the differences of 16-bit values are exact unless their exponents lie more than 13 (bf16: 16) apart, and an IEEE
    // quotient of such a difference by a 16-bit scale is rounded across a half only where it lies within 2^-17 of one.
    const float s32 = __fdiv_rn(__fsub_rn(mx, mn), LEVELS);
    const uint32_t sz = (pack2<BF>(s32, 0.0f) & 0xFFFFu) | (pack2<BF>(mn, 0.0f) << 16);
    const float scale = to_f32<BF>(sz & 0xFFFFu), by = scale > 0.0f ? scale : 1.0f, most = scale > 0.0f ? LEVELS : 0.0f;
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = (uint32_t)clamp_f32(rintf(__fdiv_rn(__fsub_rn(f[e], mn), by)), 0.0f, most);
    if constexpr (BITS == 8) {
      const uint2 y = make_uint2(code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24);
      if (live) *reinterpret_cast<uint2*>(block + (r * 16 + c) * 8) = y;
    } else {
      uint32_t y = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) y |= code[e] << (4 * (e >> 1) + 16 * (e & 1));
      if (live) *reinterpret_cast<uint32_t*>(block + (r * 16 + c) * 4) = y;
    }
    if (live && ((c << 3) & ((1 << g.gshift) - 1)) == 0)
      *reinterpret_cast<uint32_t*>(block + words_at(g) + ((((c << 3) >> g.gshift) << g.shift) + r) * 4) = sz;
  }
}

template <int BITS, bool BF>
__device__ __forceinline__ uint4 load_piece(const PageGeom& g, const unsigned char* block, int r, int c) {
  if constexpr (BITS == 16) {
    return *reinterpret_cast<const uint4*>(block + (r * 16 + c) * 16);
  } else {
    const uint32_t sz = *reinterpret_cast<const uint32_t*>(block + words_at(g) + ((((c << 3) >> g.gshift) << g.shift) + r) * 4);
    uint2 w = make_uint2(0, 0);
    if constexpr (BITS == 8) w = *reinterpret_cast<const uint2*>(block + (r * 16 + c) * 8);
    else w.x = *reinterpret_cast<const uint32_t*>(block + (r * 16 + c) * 4);
    return row_run<BITS, BF>(w.x, w.y, pair_scale<BF>(sz, sz), biases());
  }
}

constexpr int COPY_THREADS = 256;

// grid: (head, group of rows); ROWS rows per 16 lanes, whose loads are all requested first.
template <int BITS, bool BF, bool WRITE, int ROWS>
__global__ __launch_bounds__(COPY_THREADS) void page_copy_kernel(PageCopy a) {
  const PageGeom& g = a.geom;
  const int h = (int)(blockIdx.x % (unsigned)g.H), c = threadIdx.x & 15, sub = threadIdx.x >> 4;
  const int64_t first = (int64_t)(blockIdx.x / (unsigned)g.H) * (COPY_THREADS / 16 * ROWS) + sub;
  const int64_t slots = (int64_t)g.n_pages << g.shift;
  bool live[ROWS];              // the same for the 16 lanes of a row
  uint64_t page[ROWS];          // where the head's Keys of the row's page begin
  int row[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int64_t t = first + i * (COPY_THREADS / 16), slot = t < a.total ? a.slots[t] : -1;
    live[i] = slot >= 0 && slot < slots;
    const int64_t at = live[i] ? slot : 0;
    page[i] = (uint64_t)(at >> g.shift) * g.page_bytes + (uint64_t)(2 * h) * g.block_bytes;
    row[i] = (int)(at & page_mask(g));
  }
  int64_t off_k[ROWS], off_v[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const uint32_t t = (uint32_t)(first + i * (COPY_THREADS / 16)), s = t / (uint32_t)a.n_rows, r = t - s * (uint32_t)a.n_rows;
    off_k[i] = 2 * (s * a.k.seq + r * a.k.token + h * a.k.head + 8 * c);
    off_v[i] = 2 * (s * a.v.seq + r * a.v.token + h * a.v.head + 8 * c);
  }
  uint4 k[ROWS], v[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    k[i] = v[i] = make_uint4(0, 0, 0, 0);
    if (!live[i]) continue;
    if constexpr (WRITE) {
      k[i] = *reinterpret_cast<const uint4*>(a.k.data + off_k[i]);
      v[i] = *reinterpret_cast<const uint4*>(a.v.data + off_v[i]);
    } else {
      if (a.k.data) k[i] = load_piece<BITS, BF>(g, g.pool + page[i], row[i], c);
      if (a.v.data) v[i] = load_piece<BITS, BF>(g, g.pool + page[i] + g.block_bytes, row[i], c);
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if constexpr (WRITE) {
      unsigned char* block = const_cast<unsigned char*>(g.pool) + page[i];
      store_piece<BITS, BF>(g, block, row[i], c, k[i], live[i]);
      store_piece<BITS, BF>(g, block + g.block_bytes, row[i], c, v[i], live[i]);
    } else if (live[i]) {
      if (a.k.data) *reinterpret_cast<uint4*>(a.k.data + off_k[i]) = k[i];
      if (a.v.data) *reinterpret_cast<uint4*>(a.v.data + off_v[i]) = v[i];
    }
  }
}

template <int BITS, bool BF, bool WRITE>
static hipError_t launch_copy(const PageCopy& a, hipStream_t st) {
  const int64_t per = COPY_THREADS / 16, blocks = (a.total + per - 1) / per * a.geom.H;
  hipLaunchKernelGGL((page_copy_kernel<BITS, BF, WRITE, 1>), dim3((unsigned)blocks), dim3(COPY_THREADS), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageGeom& g, int bits, bool bf, bool write, const RowView& k, const RowView& v, const int64_t* slots,
                            int n_seqs, int n_rows, hipStream_t st) {
  const PageCopy a{g, k, v, slots, n_rows, (int64_t)n_seqs * n_rows};
#define GEAR_PAGE_COPY(B)                                                                     \
  return bf ? (write ? launch_copy<B, true, true>(a, st) : launch_copy<B, true, false>(a, st)) \
            : (write ? launch_copy<B, false, true>(a, st) : launch_copy<B, false, false>(a, st))
  if (bits == 16) {   // (copied as they are: the type does not matter)
    return write ? launch_copy<16, false, true>(a, st) : launch_copy<16, false, false>(a, st);
  }
  if (bits == 8) GEAR_PAGE_COPY(8);
  GEAR_PAGE_COPY(4);
#undef GEAR_PAGE_COPY
}

}  // namespace gear
