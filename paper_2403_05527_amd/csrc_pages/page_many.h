// Attention of many query columns over pages: chunks of a prompt, whole prompts.
//
// A block has 128 columns, (new token, query head of the KV head) pairs of one sequence, 32 per wave, and walks over the keys
// 64 at a time.  S^T = K Q^T and O^T = V^T P^T run on the 32x32x16 instruction: a lane has one column and, of each 32 keys, the 16
// whose index has bit 2 equal to its half; both products take the keys in that order, so the weights go from the softmax to the
// second product without leaving the registers, and maximum and sum are one exchange between the halves.  The tile's
// rows lie in LDS as 16-bit values (codes are converted once per block, on their way in): Key operands are 16-byte reads,
// Value operands transposing reads of 4 rows x 16 channels.  A row's sixteen 16-byte pieces are stored at (piece ^ row % 16) for Keys, so
// that the 16 rows which a read serves at a time lie in different banks, and at (piece ^ 4 (row % 4)) for Values, whose reads serve four rows of four
// pieces at a time (with 2 (row % 8): every read twice as long).
// Two tiles: the next one's rows are requested once this one's scores are under way (copied straight into LDS at 16 bits; the
// compiler lets no LDS read pass a copy that is on its way, so a request at the top of the step would be waited for at once).
//
// The maximum that the weights are taken from is raised only when a score exceeds it by more than 8 (in powers of two), so that the 64 accumulators
// are rarely rescaled; it lies 7 (fp16) or 0 below the score that raised it, so that no weight is above 2^15 or 2^8.
//
// A wave that has products to issue goes before one that is in its exponentials (of the two on a SIMD): a prompt of 8192 tokens, 32 heads over 8,
// 547 -> 534 us; chunks of 512 behind 4096, 32 heads, 187 -> 176 us.  Not beside blocks of few columns, whose loads then go out late (33 sequences of
// both kinds: 107 us without, 112 with).
#pragma once
#include "pages.h"

#ifndef GEAR_WAVE_PRIO
#define GEAR_WAVE_PRIO(p) __builtin_amdgcn_s_setprio(p)   // among the waves of a SIMD
#endif

namespace gear {

constexpr int MANY_THREADS = 256;
constexpr float MANY_SLACK = 8.0f;
constexpr int TILE_BYTES = MANY_KEYS * D * 2, MANY_LDS = 4 * TILE_BYTES;

__device__ __forceinline__ uint32_t key_at(uint32_t row, uint32_t piece) { return row * 256 + ((piece ^ (row & 15)) << 4); }
__device__ __forceinline__ uint32_t value_at(uint32_t row, uint32_t piece) { return row * 256 + ((piece ^ ((row & 3) << 2)) << 4); }

// A wave's 16 rows of the next tile on their way: 128 / BITS channels per lane and load.
template <int BITS>
struct Staged {
  static constexpr int PIECE = 128 / BITS, LANES = D / PIECE, ROWS = 64 / LANES, LOADS = 16 / ROWS;
  uint4 k[LOADS], v[LOADS];
  uint32_t ksz[LOADS], vsz[LOADS];
};
// A lane's places in the wave's rows: of a load's piece and of its word, relative to the first row and its words.
template <int BITS>
struct StageOffsets {
  uint32_t piece, word;
};
template <int BITS>
__device__ __forceinline__ StageOffsets<BITS> stage_offsets(const PageGeom& g, int lane) {
  using S = Staged<BITS>;
  const uint32_t piece = lane % S::LANES, row = lane / S::LANES;
  return StageOffsets<BITS>{row * (16 * BITS) + piece * 16, 4 * ((((piece * S::PIECE) >> g.gshift) << g.shift) + row)};
}
template <int BITS>
__device__ __forceinline__ void stage_load(Staged<BITS>& x, const PageGeom& g, const unsigned char* block, uint32_t row0, const StageOffsets<BITS>& o) {
  using S = Staged<BITS>;
  const auto kr = GEAR_BUF_MAKE(block + row0 * (16 * BITS), 16 * (16 * BITS)), vr = GEAR_BUF_MAKE(block + g.block_bytes + row0 * (16 * BITS), 16 * (16 * BITS));
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    x.k[i] = GEAR_BUF_LOAD16(kr, o.piece + i * (S::ROWS * 16 * BITS));
    x.v[i] = GEAR_BUF_LOAD16(vr, o.piece + i * (S::ROWS * 16 * BITS));
  }
  if constexpr (BITS < 16) {
    const uint32_t first = words_at(g) + row0 * 4;
    const auto kw = GEAR_BUF_MAKE(block + first, g.block_bytes - first), vw = GEAR_BUF_MAKE(block + g.block_bytes + first, g.block_bytes - first);
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      x.ksz[i] = GEAR_BUF_LOAD4(kw, o.word + i * (S::ROWS * 4));
      x.vsz[i] = GEAR_BUF_LOAD4(vw, o.word + i * (S::ROWS * 4));
    }
  }
}
template <int BITS, bool BF>
__device__ __forceinline__ uint4 staged_run(const uint4& w, int j, const PairScale& p, const Biases& bs) {   // channels 8 j .. of the lane's piece
  if constexpr (BITS == 16) return w;
  else if constexpr (BITS == 8) return j == 0 ? row_run<8, BF>(w.x, w.y, p, bs) : row_run<8, BF>(w.z, w.w, p, bs);
  else return row_run<4, BF>(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w, 0u, p, bs);
}
// into LDS; `live`: the wave's rows from there on are zeroes as Values, whatever the page holds (their weights are 0)
template <int BITS, bool BF>
__device__ __forceinline__ void stage_store(const Staged<BITS>& x, unsigned char* kt, unsigned char* vt, int wave, int lane, int live, const Biases& bs) {
  using S = Staged<BITS>;
  const uint32_t piece = lane % S::LANES;
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    const uint32_t in_wave = i * S::ROWS + lane / S::LANES, row = 16 * wave + in_wave;
    PairScale pk, pv;
    if constexpr (BITS < 16) {
      pk = pair_scale<BF>(x.ksz[i], x.ksz[i]);
      pv = pair_scale<BF>(x.vsz[i], x.vsz[i]);
    }
    const bool there = (int)in_wave < live;
#pragma unroll
    for (int j = 0; j < S::PIECE / 8; ++j) {
      const uint32_t at = piece * (S::PIECE / 8) + j;
      *reinterpret_cast<uint4*>(kt + key_at(row, at)) = staged_run<BITS, BF>(x.k[i], j, pk, bs);
      uint4 v = staged_run<BITS, BF>(x.v[i], j, pv, bs);
      v.x = there ? v.x : 0u;
      v.y = there ? v.y : 0u;
      v.z = there ? v.z : 0u;
      v.w = there ? v.w : 0u;
      *reinterpret_cast<uint4*>(vt + value_at(row, at)) = v;
    }
  }
}

// Tile `i` of the call's column tiles (s < 0: there is none).
struct ColTile {
  int s, col0;
};
__device__ __forceinline__ int many_tiles(const PageAttn& a, const SeqSpan& sp) {   // of a sequence
  if (sp.nq <= 0 || (sp.nq <= a.few && sp.nq * a.gq <= a.few)) return 0;
  return (sp.nq * a.gq + MANY_COLS - 1) / MANY_COLS;
}
// The tiles that see the most keys come first: sequences by their length, and a sequence's last tiles before its first (with the longest of three
// sequences last, a batch took half as long again).  Each lane counts, for one sequence, the tiles of those that come before it.  More than 64
// sequences: in the order of their numbers, the last first (100 of up to 1767 tokens, a chunk of 700 behind 4000 among them: 152 us where it comes last in the batch, 163 where
// it comes first; three chunks 131 and 145).
__device__ __forceinline__ ColTile col_tile(const PageAttn& a, int i, int lane) {
  if (a.n_seqs <= 64) {
    SeqSpan sp{0, 0, 0};
    if (lane < a.n_seqs) sp = seq_span(a, lane);
    const int tiles = many_tiles(a, sp);
    int before = 0;
    for (int j = 0; j < a.n_seqs; ++j) {
      const int kv = __builtin_amdgcn_readlane(sp.kv, j), n = __builtin_amdgcn_readlane(tiles, j);
      before += kv > sp.kv || (kv == sp.kv && j < lane) ? n : 0;
    }
    const unsigned long long mine = __ballot(i >= before && i < before + tiles);
    if (mine == 0ull) return ColTile{-1, 0};
    const int s = GEAR_WAVE_UNIFORM(__ffsll((long long)mine) - 1);
    return ColTile{s, (__builtin_amdgcn_readlane(before + tiles, s) - 1 - i) * MANY_COLS};
  }
  // sequence s has the tiles from q_start[s] * gq / 128 + s on: room for its own last, partly filled one
  const int tile = a.tiles - 1 - i;
  int s = -1;
  for (int base = 0; base < a.n_seqs; base += 64) {
    const int j = base + lane;
    s += __popcll(__ballot(j < a.n_seqs && ((long long)max(a.q_start[j], 0) * a.gq) / MANY_COLS + j <= tile));
  }
  s = GEAR_WAVE_UNIFORM(s);
  if (s < 0) return ColTile{-1, 0};
  const SeqSpan sp = seq_span(a, s);
  const int local = tile - (int)(((long long)sp.q0 * a.gq) / MANY_COLS + s);
  return local >= 0 && local < many_tiles(a, sp) ? ColTile{s, local * MANY_COLS} : ColTile{-1, 0};
}

// One (column tile, KV head, part) of the call.  lds: [two tiles][Keys, Values][64 rows].  ALONE: no blocks of few columns in the launch.
template <int BITS, bool BF, bool ALONE>
__device__ __forceinline__ void many_columns(const PageAttn& a, int bid, unsigned char* lds) {
  const PageGeom& g = a.geom;
  const int lane = lane_id(), wave = GEAR_WAVE_UNIFORM((int)(threadIdx.x >> 6)), c = lane & 31, half = lane >> 5;
  // heads next to each other: with 8 of them and more, a head's tiles share one XCD's L2
  const int head = bid % g.H, rest = bid / g.H, part = rest % a.n_split;
  const ColTile ct = col_tile(a, rest / a.n_split, lane);
  if (ct.s < 0) return;
  const int s = ct.s, col0 = ct.col0;
  const SeqSpan sp = seq_span(a, s);
  const int cols = sp.nq * a.gq;
  const int last = min(col0 + MANY_COLS, cols) - 1;
  const int keys = row_sees(a, sp, last / a.gq);
  const Parts parts = parts_of(keys, a.n_split, a.least, MANY_KEYS);
  if (part >= parts.count) return;
  const int k0 = part * parts.len, k1 = min(keys, k0 + parts.len);

  const int my = col0 + 32 * wave + c, row = my / a.gq, j = my - row * a.gq;
  const bool mine = my < cols, busy = col0 + 32 * wave < cols;   // `busy`: the wave has columns
  const int sees = mine ? row_sees(a, sp, row) : 0;
  uint4 q[8];   // B operands: channels 16 t + 8 half + 0..7 of the column
#pragma unroll
  for (int t = 0; t < 8; ++t) q[t] = make_uint4(0, 0, 0, 0);
  if (mine) {
    const unsigned char* p = a.q.data + 2 * ((int64_t)(sp.q0 + row) * a.q.token + (int64_t)(head * a.gq + j) * a.q.head + 8 * half);
#pragma unroll
    for (int t = 0; t < 8; ++t) q[t] = signed_query(*reinterpret_cast<const uint4*>(p + 32 * t), a.flip);
  }
  const int all_see = row_sees(a, sp, min(col0 + 32 * wave, cols - 1) / a.gq);   // every column of the wave sees the keys before this one

  PageRow pages = page_row(a, s, k1);
  const Biases bs = biases();
  Staged<BITS> next;                       // codes on their way
  const StageOffsets<BITS> offsets = stage_offsets<BITS>(g, lane);
  // Of the next tile: whether all its keys are there, have pages and lie before k1; where not, the wave's rows that are there, and in bit w whether
  // the keys from 16 w on have a page.
  bool whole = false, whole_next = false;
  int live = 16, have = 15, have_next = 15;
  const int per_tile = MANY_KEYS >> g.shift > 0 ? MANY_KEYS >> g.shift : 1;   // pages
  const unsigned long long all = (1ull << per_tile) - 1ull;
  // (kept short: with the four groups' pages looked up one by one it took 800 of a tile's 3750 cycles)
  auto fetch = [&](int key, unsigned char* to) {
    const int i0 = key >> g.shift;
    if (i0 + 4 > pages.base + 64) load_entries(pages, i0);
    const int at = key + 16 * wave;
    int page = __builtin_amdgcn_readlane(pages.held, (at >> g.shift) - pages.base);
    whole_next = key + MANY_KEYS <= k1 && ((pages.valid >> (i0 - pages.base)) & all) == all;
    live = 16;
    if (!whole_next) {
      have_next = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        have_next |= (__builtin_amdgcn_readlane(pages.held, ((key + 16 * w) >> g.shift) - pages.base) >= 0 && key + 16 * w < k1 ? 1 : 0) << w;
      live = page < 0 ? 0 : min(16, max(0, k1 - at));
      page = max(page, 0);
    }
    const unsigned char* block = block_of(g, page, head, 0);
    const uint32_t row0 = (uint32_t)at & page_mask(g);
    if (BITS == 16 && live == 16) {   // straight into LDS: 16 lanes per row, each the piece that belongs at its place
      const auto kb = GEAR_BUF_MAKE(block + row0 * 256, 16 * 256), vb = GEAR_BUF_MAKE(block + g.block_bytes + row0 * 256, 16 * 256);
      const uint32_t k_at = key_at(lane >> 4, lane & 15), v_at = value_at(lane >> 4, lane & 15);
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // rows 4 i + lane / 16
        GEAR_DMA16(kb, (k_at ^ (64 * i)) + 1024 * i, to + 4096 * wave + 1024 * i);
        GEAR_DMA16(vb, v_at + 1024 * i, to + TILE_BYTES + 4096 * wave + 1024 * i);
      }
    } else {
      stage_load<BITS>(next, g, block, row0, offsets);
      if (BITS == 16) stage_store<BITS, BF>(next, to, to + TILE_BYTES, wave, lane, live, bs);   // (a sequence's last rows)
    }
  };
  floatx16 o[4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  if (k0 < k1) {
    fetch(k0, lds);
    if (BITS < 16) stage_store<BITS, BF>(next, lds, lds + TILE_BYTES, wave, lane, live, bs);
  }
  GEAR_DMA_WAIT();
  GEAR_DMA_BARRIER();
  int buf = 0;
  for (int key = k0; key < k1; key += MANY_KEYS, buf ^= 1) {
    const bool more = key + MANY_KEYS < k1;
    whole = whole_next;
    have = have_next;
    const unsigned char* kt = lds + buf * 2 * TILE_BYTES;
    const unsigned char* vt = kt + TILE_BYTES;
    floatx16 sc[2];
    if (ALONE) GEAR_WAVE_PRIO(2);
    if (busy) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const uint4 ka = *reinterpret_cast<const uint4*>(kt + key_at(32 * b + c, 2 * t + half));
          sc[b] = mfma32<BF>(ka, q[t], sc[b]);
        }
      }
    }
    if (more) fetch(key + MANY_KEYS, lds + (buf ^ 1) * 2 * TILE_BYTES);
    if (busy) {
      // keys 32 b + 8 (i / 4) + 4 half + i % 4 of the tile
      const bool edge = key + MANY_KEYS > all_see || !whole;
      if (edge) {
        int first = key + 4 * half;
        GEAR_PIN_VGPR(first);   // (what depends on it stays in here)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (first + 32 * b + 8 * (i >> 2) + (i & 3) >= sees || (!whole && ((have >> (2 * b + (i >> 3))) & 1) == 0)) sc[b][i] = -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
      top = weights_base<BF>(col_max<false>(top), a.scale_log2, a.far, F16_WEIGHT_LOG2 - MANY_SLACK);
      if (__ballot(top > m + MANY_SLACK) != 0ull) {   // (from -inf on: any score)
        const float now = fmaxf(m, top), by = now == -INFINITY ? 1.0f : GEAR_EXP2(m - now);
        m = now;
        l *= by;
#pragma unroll
        for (int t = 0; t < 4; ++t) o[t] *= by;
      }
      if (ALONE) GEAR_WAVE_PRIO(0);
      const float from = m == -INFINITY ? 0.0f : m;
      uint4 pw[4];   // B operands: keys 16 u + 4 half + 0..3 and + 8
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = GEAR_EXP2(__builtin_fmaf(sc[u >> 1][8 * (u & 1) + i], a.scale_log2, -from));
          l += p[i];
        }
        // rounded to the type for the product (F16_WEIGHT_LOG2); the sum keeps them in fp32
        pw[u] = make_uint4(pack2<BF>(p[0], p[1]), pack2<BF>(p[2], p[3]), pack2<BF>(p[4], p[5]), pack2<BF>(p[6], p[7]));
      }
      if (ALONE) GEAR_WAVE_PRIO(1);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int t = 0; t < 4; ++t) {   // channels 32 t + c
          // lane i of 16: row 4 half + i / 4, channels 32 t + 16 ((lane / 16) % 2) + 4 (i % 4) + 0..3
          const uint32_t r0 = 16 * u + 4 * half + ((lane & 15) >> 2), piece = 4 * t + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          const uint2 lo = GEAR_LDS_READ_TR(vt + value_at(r0, piece) + 8 * (lane & 1));
          const uint2 hi = GEAR_LDS_READ_TR(vt + value_at(r0 + 8, piece) + 8 * (lane & 1));
          o[t] = mfma32<BF>(make_uint4(lo.x, lo.y, hi.x, hi.y), pw[u], o[t]);
        }
      if (ALONE) GEAR_WAVE_PRIO(0);
    }
    if (more) {
      unsigned char* to = lds + (buf ^ 1) * 2 * TILE_BYTES;
      if (BITS < 16) stage_store<BITS, BF>(next, to, to + TILE_BYTES, wave, lane, live, bs);
    }
    GEAR_DMA_WAIT();
    GEAR_DMA_BARRIER();
  }
  if (!busy) return;
  l = col_sum<false>(l);
  if (!mine) return;
  // the lane has channels 32 t + 8 a + 4 half + 0..3 of its column
  const int64_t token = sp.q0 + row;
  if (parts.count == 1) {
    const float r = l > 0.0f ? 1.0f / l : 0.0f;
    unsigned char* p = a.out.data + 2 * (token * a.out.token + (int64_t)(head * a.gq + j) * a.out.head + 4 * half);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<uint2*>(p + 64 * t + 16 * k) =
            make_uint2(pack2<BF>(o[t][4 * k] * r, o[t][4 * k + 1] * r), pack2<BF>(o[t][4 * k + 2] * r, o[t][4 * k + 3] * r));
  } else {
    const int64_t rec = (token * ((int64_t)g.H * a.gq) + head * a.gq + j) * a.n_split + part;
    float* p = a.rec_o + rec * D + 4 * half;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<float4*>(p + 32 * t + 8 * k) = make_float4(o[t][4 * k], o[t][4 * k + 1], o[t][4 * k + 2], o[t][4 * k + 3]);
    if (half == 0) a.rec_ml[rec] = make_float2(m, l);
  }
}

}  // namespace gear
