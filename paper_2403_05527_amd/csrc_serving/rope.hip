// Rows turned by their positions, and put into the pool as they come (include/gear.h).
//
// 16 lanes take a row of 128 channels, eight each, and stay with its token: the cosines and sines of a lane's channels are worked out
// once and used for all heads of the block.  The angle t w is reduced in 64 bits, in turns: t w / 2 pi less the nearest whole number, and of that the nearest quarter,
// which leaves an angle of at most pi / 4 in fp32, for which the series of sine and cosine to the powers 9 and 10 are off by
// (pi/4)^11 / 11! = 1.8e-9 and (pi/4)^12 / 12! = 1.2e-10, less than the roundings.
//
// Bound by the bytes: four prompts of 8192 tokens, 32 query heads and 8 KV heads, bf16, 805 MB in 144 us (5.6 TB/s; with one head per block, whose angles take
// as long as its rows, 246); the Keys of 16 x 4096 tokens of 32 heads turned back, 1.07 GB in 183 (5.9 TB/s; 370).  Eight heads' rows requested at once against
// four: 200 -> 183 us there, 151 -> 145 in the first; 16 heads per block 149 in the first, 4 in an 8-bit pool 199 instead of 182.
#include "page_piece.h"
#include "serving.h"

namespace gear {

constexpr int ROPE_THREADS = 256, ROPE_TOKENS = ROPE_THREADS / 16;

// Where the other channel of a pair lies: in the lane's own piece; in the piece of the lane eight on; in a piece a number of lanes on; anywhere.
enum RopePairs { PAIRS_NEXT = 0, PAIRS_LANE8 = 1, PAIRS_LANES = 2, PAIRS_ANY = 3 };

struct Turn {
  float c, s;
};
__device__ __forceinline__ Turn turn_of(double position, double freq, float factor, float sign) {
  const double u = position * (freq * 0.15915494309189533577), whole = u - rint(u), q = rint(4.0 * whole);   // 1 / 2 pi; |whole| <= 1/2, exact
  const float a = (float)((whole - 0.25 * q) * 6.28318530717958647693), b = a * a;
  const float sn = a * __builtin_fmaf(b, __builtin_fmaf(b, __builtin_fmaf(b, __builtin_fmaf(b, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
  const float cs = __builtin_fmaf(
      b, __builtin_fmaf(b, __builtin_fmaf(b, __builtin_fmaf(b, __builtin_fmaf(b, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
  const int k = (int)q & 3;                               // quarters of a turn
  const float c = (k & 1) ? sn : cs, s = (k & 1) ? cs : sn;
  Turn t;
  t.c = factor * ((k == 1 || k == 2) ? -c : c);
  t.s = factor * sign * (k >= 2 ? -s : s);
  return t;
}

// A lane's eight channels: y = c x + s (the other of the pair), s with its sign; `stay`: bit e: channel e is left as it is.
struct LaneTurns {
  float c[8], s[8];
  uint32_t stay;
};
template <int PAIRS>
__device__ __forceinline__ LaneTurns lane_turns(const Rope& r, int c, int64_t position) {
  LaneTurns t;
  t.stay = 0u;
  const double at = (double)position;
  if constexpr (PAIRS == PAIRS_NEXT) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int ch = 8 * c + e;
      if (ch >= r.rot) t.stay |= 3u << e;
      const Turn x = turn_of(at, r.freq[ch < r.rot ? ch >> 1 : 0], r.factor, r.sign);
      t.c[e] = t.c[e + 1] = x.c;
      t.s[e] = -x.s;
      t.s[e + 1] = x.s;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int ch = 8 * c + e;
      if (ch >= r.rot) t.stay |= 1u << e;
      const int p = ch < r.half ? ch : ch - r.half;
      const Turn x = turn_of(at, r.freq[ch < r.rot ? p : 0], r.factor, r.sign);
      t.c[e] = x.c;
      t.s[e] = ch < r.half ? -x.s : x.s;
    }
  }
  return t;
}
// The other channels of the pairs, for a piece `v` of the row at `row` (which is read again only by PAIRS_ANY).
template <int PAIRS>
__device__ __forceinline__ uint4 others(const Rope& r, const uint4& v, const unsigned char* row, int c, bool there) {
  if constexpr (PAIRS == PAIRS_NEXT) {
    return make_uint4(v.x >> 16 | v.x << 16, v.y >> 16 | v.y << 16, v.z >> 16 | v.z << 16, v.w >> 16 | v.w << 16);
  } else if constexpr (PAIRS == PAIRS_LANE8) {
    return make_uint4(dpp_u<DPP_ROR8>(v.x), dpp_u<DPP_ROR8>(v.y), dpp_u<DPP_ROR8>(v.z), dpp_u<DPP_ROR8>(v.w));
  } else if constexpr (PAIRS == PAIRS_LANES) {
    const int by = r.half >> 3, from = c < by ? c + by : c < 2 * by ? c - by : c;
    return make_uint4(__shfl(v.x, from, 16), __shfl(v.y, from, 16), __shfl(v.z, from, 16), __shfl(v.w, from, 16));
  } else {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (there) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int ch = 8 * c + e, o = ch < r.half ? ch + r.half : ch < r.rot ? ch - r.half : ch;
        w[e >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(row + 2 * o) << (16 * (e & 1));
      }
    }
    __builtin_amdgcn_wave_barrier();   // (in place: read before any lane stores)
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
template <bool BF>
__device__ __forceinline__ uint32_t turn_pair(uint32_t x, uint32_t o, const LaneTurns& t, int e) {   // channels e, e + 1
  const float a = to_f32<BF>(x & 0xFFFFu), b = to_f32<BF>(x >> 16), oa = to_f32<BF>(o & 0xFFFFu), ob = to_f32<BF>(o >> 16);
  float ya = __builtin_fmaf(a, t.c[e], oa * t.s[e]), yb = __builtin_fmaf(b, t.c[e + 1], ob * t.s[e + 1]);
  GEAR_IN_VGPR(ya);   // (rounded to fp32 here in every kernel: what gear_page_write_rope stores is what gear_rotate would give)
  GEAR_IN_VGPR(yb);
  const uint32_t y = pack2<BF>(ya, yb);
  const uint32_t m = ((t.stay >> e) & 1u ? 0xFFFFu : 0u) | ((t.stay >> e) & 2u ? 0xFFFF0000u : 0u);
  return (x & m) | (y & ~m);
}
template <bool BF, int PAIRS>
__device__ __forceinline__ uint4 turned(const Rope& r, const LaneTurns& t, const uint4& v, const unsigned char* row, int c, bool there) {
  const uint4 o = others<PAIRS>(r, v, row, c, there);
  return make_uint4(turn_pair<BF>(v.x, o.x, t, 0), turn_pair<BF>(v.y, o.y, t, 2), turn_pair<BF>(v.z, o.z, t, 4), turn_pair<BF>(v.w, o.w, t, 6));
}

// grid: (part of the heads, 16 tokens of one sequence).  BITS: of the pool's rows, 0 where there is none.  A block has up to HEADS heads at a time on their way.
// PAST: `out` is large (PAST_CACHES).  (As a branch at the store it was lost: both stores became one.)
constexpr int HEADS = 8;
template <int BITS, bool BF, int PAIRS, bool PAST>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(RopeRows a) {
  const unsigned bid = blockIdx.x, rest = bid / (unsigned)a.parts, s = rest / (unsigned)a.chunks;
  const int part = (int)(bid - rest * (unsigned)a.parts), c = threadIdx.x & 15, in_chunk = threadIdx.x >> 4;
  const int row = (int)(rest - s * (unsigned)a.chunks) * ROPE_TOKENS + in_chunk;
  const bool there = row < a.n_rows;
  const int64_t at = (int64_t)s * a.n_rows + (there ? row : a.n_rows - 1);
  const int64_t position = a.positions[at];
  if (BITS == 0 || part < a.x_parts) {
    const unsigned char* xp = a.x.data + 2 * ((int64_t)s * a.x.seq + (int64_t)(there ? row : 0) * a.x.token);
    unsigned char* op = a.out.data + 2 * ((int64_t)s * a.out.seq + (int64_t)(there ? row : 0) * a.out.token);
    const int h0 = part * a.per, h1 = min(a.heads, h0 + a.per);
    LaneTurns t;
    for (int h = h0; h < h1; h += HEADS) {
      uint4 v[HEADS];
#pragma unroll
      for (int u = 0; u < HEADS; ++u) {
        v[u] = make_uint4(0, 0, 0, 0);
        if (there && h + u < h1) v[u] = load16_once(xp + 2 * ((h + u) * a.x.head) + 16 * c);
      }
      if (h == h0) t = lane_turns<PAIRS>(a.rope, c, position);   // (behind the first requests)
#pragma unroll
      for (int u = 0; u < HEADS; ++u) {
        if (h + u >= h1) continue;
        const uint4 y = turned<BF, PAIRS>(a.rope, t, v[u], xp + 2 * ((h + u) * a.x.head), c, there);
        unsigned char* to = op + 2 * ((h + u) * a.out.head) + 16 * c;
        if (there) store16<PAST>(to, y);
      }
    }
  } else if constexpr (BITS != 0) {
    const PageGeom& g = a.geom;
    const int64_t slot = there ? a.slots[at] : -1;
    const bool live = slot >= 0 && slot < (int64_t)g.n_pages << g.shift;   // the same for the 16 lanes of a row
    const int64_t to = live ? slot : 0;
    const int in_page = (int)(to & page_mask(g));
    const unsigned char* kp = a.k.data + 2 * ((int64_t)s * a.k.seq + (int64_t)(there ? row : 0) * a.k.token);
    const unsigned char* vp = a.v.data + 2 * ((int64_t)s * a.v.seq + (int64_t)(there ? row : 0) * a.v.token);
    const int h0 = (part - a.x_parts) * a.kv_per, h1 = min(g.H, h0 + a.kv_per);
    LaneTurns t;
    for (int h = h0; h < h1; h += HEADS / 2) {
      uint4 k[HEADS / 2], v[HEADS / 2];
#pragma unroll
      for (int u = 0; u < HEADS / 2; ++u) {
        k[u] = v[u] = make_uint4(0, 0, 0, 0);
        if (there && h + u < h1) {
          k[u] = *reinterpret_cast<const uint4*>(kp + 2 * ((h + u) * a.k.head) + 16 * c);
          v[u] = *reinterpret_cast<const uint4*>(vp + 2 * ((h + u) * a.v.head) + 16 * c);
        }
      }
      if (h == h0) t = lane_turns<PAIRS>(a.rope, c, position);
#pragma unroll
      for (int u = 0; u < HEADS / 2; ++u) {
        if (h + u >= h1) continue;
        unsigned char* block = const_cast<unsigned char*>(block_of(g, (int)(to >> g.shift), h + u, 0));
        store_piece<BITS, BF>(g, block, in_page, c, turned<BF, PAIRS>(a.rope, t, k[u], kp + 2 * ((h + u) * a.k.head), c, there), live);
        store_piece<BITS, BF>(g, block + g.block_bytes, in_page, c, v[u], live);
      }
    }
  }
}

template <int BITS, bool BF, int PAIRS>
static hipError_t launch(const RopeRows& a, int n_seqs, hipStream_t st) {
  const int64_t blocks = (int64_t)n_seqs * a.chunks * a.parts;
  if ((int64_t)n_seqs * a.n_rows * a.heads * 2 * D >= PAST_CACHES) hipLaunchKernelGGL((rope_kernel<BITS, BF, PAIRS, true>), dim3((unsigned)blocks), dim3(ROPE_THREADS), 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<BITS, BF, PAIRS, false>), dim3((unsigned)blocks), dim3(ROPE_THREADS), 0, st, a);
  return hipGetLastError();
}
template <int BITS, bool BF>
static hipError_t launch(const RopeRows& a, bool interleaved, int n_seqs, hipStream_t st) {
  if (interleaved) return launch<BITS, BF, PAIRS_NEXT>(a, n_seqs, st);
  if (a.rope.half == 64) return launch<BITS, BF, PAIRS_LANE8>(a, n_seqs, st);
  if (a.rope.half % 8 == 0) return launch<BITS, BF, PAIRS_LANES>(a, n_seqs, st);
  return launch<BITS, BF, PAIRS_ANY>(a, n_seqs, st);
}

constexpr int ROPE_HEADS_MOST = HEADS;   // of a block
static bool one_run(const RowView& r, int64_t n_rows) { return !r.data || r.seq == n_rows * r.token; }

hipError_t launch_rope(const RopeRows& call, int bits, bool bf, bool interleaved, int n_seqs, hipStream_t st) {
  RopeRows a = call;
  if (a.n_rows == 1) {   // single tokens, and sequences that follow one another: the rows of one
    for (RowView* r : {&a.x, &a.out, &a.k, &a.v}) r->token = r->seq;
    a.n_rows = n_seqs;
    n_seqs = 1;
  } else if (one_run(a.x, a.n_rows) && one_run(a.out, a.n_rows) && one_run(a.k, a.n_rows) && one_run(a.v, a.n_rows)) {
    a.n_rows *= n_seqs;
    n_seqs = 1;
  }
  a.chunks = (a.n_rows + ROPE_TOKENS - 1) / ROPE_TOKENS;
  const int H = bits ? a.geom.H : 0;
  // Heads of a block: one where there are few blocks, as many as leave 8 blocks per CU
  const int64_t rows = (int64_t)n_seqs * a.chunks, per = rows * (a.heads + 2 * H) / (8 * GEAR_CUS);
  a.per = per < 1 ? 1 : per < ROPE_HEADS_MOST ? (int)per : ROPE_HEADS_MOST;
  a.kv_per = (a.per + 1) / 2;
  a.x_parts = (a.heads + a.per - 1) / a.per;
  a.parts = a.x_parts + (H + a.kv_per - 1) / a.kv_per;
  switch (bits) {
    case 0: return bf ? launch<0, true>(a, interleaved, n_seqs, st) : launch<0, false>(a, interleaved, n_seqs, st);
    case 16: return bf ? launch<16, true>(a, interleaved, n_seqs, st) : launch<16, false>(a, interleaved, n_seqs, st);
    case 8: return bf ? launch<8, true>(a, interleaved, n_seqs, st) : launch<8, false>(a, interleaved, n_seqs, st);
    default: return bf ? launch<4, true>(a, interleaved, n_seqs, st) : launch<4, false>(a, interleaved, n_seqs, st);
  }
}

}  // namespace gear
