// Attention of few query columns over pages: single tokens, speculative rows, the tail of a chunk.
//
// A sequence's columns are its (new token, query head of the KV head) pairs; up to 16 or 32 of them share one pass over the
// keys.  A wave takes 32 keys at a time, and works on them without LDS: S^T = K Q^T with the keys as the rows of the 16x16x32
// instruction, straight from 16-byte loads; a lane of the result then holds, for its column, eight keys (four of each 16) --
// exactly the eight that the B operand of O^T = V^T P^T wants from it, if the contraction runs over the keys in that order.  The
// A operand of that product needs, for a channel, the same eight keys: the lane loads eight channels (16 c / b bytes) of its
// eight rows and pairs rows by byte permutations, one per two values, so that product t of eight has channel 8 (l % 16) + t
// in row l % 16, and the lane's results are 32 consecutive channels of its column.
//
// Bound by the pages' bytes at 16 and 8 bits, by the conversions beside them at 4: one token each of 16 sequences of 4096, 32 heads, groups of 64, fp16 181, 101 and
// 63 us at 16, 8 and 4 bits (5.9, 5.7 and 4.8 TB/s), bf16, whose values are rounded in fp32, 187, 106 and 69.
// The keys are divided among the waves of a block and, where the sequences and heads are few, among blocks, whose records
// page_merge_few_kernel joins.
#pragma once
#include "pages.h"

namespace gear {

// 16 keys' rows of one head as loaded.
template <int BITS>
struct KeyRows {
  static constexpr int LOADS = BITS / 4;         // 16-byte pieces of a lane's share of a row (32 channels)
  uint4 w[LOADS];
  uint32_t sz[BITS == 8 ? 2 : 1];
};
// ... the A operand of product t (0..3): channels first_channel(t, l / 16) + 0..7 of key l % 16
template <int BITS>
__device__ __forceinline__ int first_channel(int t, int hh) {
  constexpr int PIECE = 128 / BITS;              // channels of a 16-byte piece: 8, 16, 32
  constexpr int PER = PIECE / 8;                 // products per piece
  return (t / PER) * 4 * PIECE + hh * PIECE + (t % PER) * 8;
}
// A lane's places in 16 rows: Keys of row c = l % 16, Values of rows 4 hh + 0..3, hh = l / 16; relative to the first row and its words.
template <int BITS>
struct LaneOffsets {
  uint32_t key, value, key_word[BITS == 8 ? 2 : 1], value_word;
};
template <int BITS>
__device__ __forceinline__ LaneOffsets<BITS> lane_offsets(const PageGeom& g, int c, int hh) {
  LaneOffsets<BITS> o{};
  o.key = c * (16 * BITS) + hh * 16;
  o.value = 4 * hh * (16 * BITS) + c * BITS;
  if constexpr (BITS < 16) {
#pragma unroll
    for (int u = 0; u < KeyRows<BITS>::LOADS; ++u) o.key_word[u] = 4 * (((uint32_t)(first_channel<BITS>(u * (16 / BITS), hh) >> g.gshift) << g.shift) + c);
    o.value_word = 4 * (((uint32_t)((8 * c) >> g.gshift) << g.shift) + 4 * hh);
  }
  return o;
}
template <int BITS>
__device__ __forceinline__ void load_keys(KeyRows<BITS>& k, const PageGeom& g, const unsigned char* block, uint32_t row0, const LaneOffsets<BITS>& o) {
  const auto rows = GEAR_BUF_MAKE(block + row0 * (16 * BITS), 16 * (16 * BITS));
#pragma unroll
  for (int u = 0; u < KeyRows<BITS>::LOADS; ++u) k.w[u] = GEAR_BUF_LOAD16(rows, o.key + 64 * u);
  if constexpr (BITS < 16) {
    const auto words = GEAR_BUF_MAKE(block + words_at(g) + row0 * 4, g.block_bytes - words_at(g) - row0 * 4);
#pragma unroll
    for (int u = 0; u < KeyRows<BITS>::LOADS; ++u) k.sz[u] = GEAR_BUF_LOAD4(words, o.key_word[u]);
  }
}
template <int BITS, bool BF>
__device__ __forceinline__ uint4 key_operand(const KeyRows<BITS>& k, int t, const Biases& bs) {
  if constexpr (BITS == 16) {
    return k.w[t];
  } else if constexpr (BITS == 8) {
    const uint4& w = k.w[t >> 1];
    const PairScale p = pair_scale<BF>(k.sz[t >> 1], k.sz[t >> 1]);
    return (t & 1) ? row_run<8, BF>(w.z, w.w, p, bs) : row_run<8, BF>(w.x, w.y, p, bs);
  } else {
    const uint4& w = k.w[0];
    const PairScale p = pair_scale<BF>(k.sz[0], k.sz[0]);
    return row_run<4, BF>(t == 0 ? w.x : t == 1 ? w.y : t == 2 ? w.z : w.w, 0u, p, bs);
  }
}
// Eight channels of four consecutive rows.
template <int BITS>
struct ValueRows {
  static constexpr int WORDS = BITS / 4;         // 32-bit words of eight channels: 4, 2, 1
  uint32_t w[4][WORDS];
  uint32_t sz[4];
};
template <int BITS>
__device__ __forceinline__ void load_values(ValueRows<BITS>& v, const PageGeom& g, const unsigned char* block, uint32_t row0, const LaneOffsets<BITS>& o) {
  const auto rows = GEAR_BUF_MAKE(block + row0 * (16 * BITS), 16 * (16 * BITS));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BITS == 16) {
      const uint4 x = GEAR_BUF_LOAD16(rows, o.value + i * 256);
      v.w[i][0] = x.x;
      v.w[i][1] = x.y;
      v.w[i][2] = x.z;
      v.w[i][3] = x.w;
    } else if constexpr (BITS == 8) {
      const uint2 x = GEAR_BUF_LOAD8(rows, o.value + i * 128);
      v.w[i][0] = x.x;
      v.w[i][1] = x.y;
    } else {
      v.w[i][0] = GEAR_BUF_LOAD4(rows, o.value + i * 64);
    }
  }
  if constexpr (BITS < 16) {   // (four rows of a page of 16 and more: 16-byte aligned)
    const auto words = GEAR_BUF_MAKE(block + words_at(g) + row0 * 4, g.block_bytes - words_at(g) - row0 * 4);
    const uint4 x = GEAR_BUF_LOAD16(words, o.value_word);
    v.sz[0] = x.x;
    v.sz[1] = x.y;
    v.sz[2] = x.z;
    v.sz[3] = x.w;
  }
}
template <int BITS>
__device__ __forceinline__ void drop_value(ValueRows<BITS>& v, int i) {   // a row that no column sees: whatever lies there, 0
#pragma unroll
  for (int j = 0; j < ValueRows<BITS>::WORDS; ++j) v.w[i][j] = 0u;
  v.sz[i] = 0u;
}
template <int BITS>
struct KeyBlock {   // 32 keys
  KeyRows<BITS> k[2];
  ValueRows<BITS> v[2];
};

// One (sequence, KV head, part) of the call, NC tiles of 16 columns, WAVES waves.
// lds: the block's states: [wave][column] maxima and sums, [wave][NC][8][lane] partial sums
template <int NC, int WAVES>
constexpr size_t few_lds_bytes() {
  return WAVES * NC * (16 * 2 * 4 + 8 * 64 * 16);
}
template <int BITS, bool BF, int NC, int WAVES, class Attn>
__device__ __forceinline__ void few_columns(const Attn& a, int bid, unsigned char* lds) {
  const PageGeom& g = a.geom;
  const int head = bid % g.H;
  const Place place = few_place(a, bid / g.H);
  const int part = place.part, s = place.i;
  const int lane = lane_id(), wave = GEAR_WAVE_UNIFORM((int)(threadIdx.x >> 6)), c = lane & 15, hh = lane >> 4;
  const Span span = span_of(a, s);
  const SeqSpan& sp = span.sp;
  const int cols = sp.nq * a.gq;
  if (sp.nq <= 0 || sp.nq > a.few || cols > a.few) return;
  const Parts parts = parts_of(sp.kv - span.begin, a.n_split, a.least, KEY_STEP);
  if (part >= parts.count) return;
  const int k0 = span.begin + part * parts.len, k1 = min(sp.kv, k0 + parts.len);

  // The first pages are requested with the queries and looked at behind them (8.5 -> 8.0 us behind 512).
  PageRow pages = page_row(a, span.table_row, k1);
  const int first_entry = (k0 + KEY_STEP * wave) >> g.shift;
  const int32_t entry = k1 > 0 ? pages.table[min(first_entry + lane, (k1 - 1) >> g.shift)] : -1;

  // the columns' query rows, as B operands; what they see
  uint4 q[NC][4];
  int sees[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int col = min(n * 16 + c, cols - 1), row = col / a.gq, j = col - row * a.gq;   // (columns that are not there: the last one's, not stored)
    sees[n] = row_sees(a, sp, row);
    const unsigned char* p = a.q.data + 2 * ((int64_t)(sp.q0 + row) * a.q.token + (int64_t)(head * a.gq + j) * a.q.head);
#pragma unroll
    for (int t = 0; t < 4; ++t) q[n][t] = *reinterpret_cast<const uint4*>(p + 2 * first_channel<BITS>(t, hh));
  }
  const int all_see = row_sees(a, sp, 0);   // every column sees the keys before this one

  floatx4 o[NC][8];
  float m[NC], l[NC];   // (m: weights_base)
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.0f;
#pragma unroll
    for (int t = 0; t < 8; ++t) o[n][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const Biases bs = biases();
  const LaneOffsets<BITS> offsets = lane_offsets<BITS>(g, c, hh);
  auto fetch = [&](KeyBlock<BITS>& x, int key, int p0, int p1) {   // (a key without a page reads page 0, and counts for nothing)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int p = b == 0 ? p0 : p1;
      const unsigned char* block = block_of(g, p < 0 ? 0 : p, head, 0);
      const uint32_t row0 = (uint32_t)(key + 16 * b) & page_mask(g);
      load_keys<BITS>(x.k[b], g, block, row0, offsets);
      load_values<BITS>(x.v[b], g, block + g.block_bytes, row0, offsets);
    }
  };
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int t = 0; t < 4; ++t) q[n][t] = signed_query(q[n][t], a.flip);
  hold_entries(pages, first_entry, entry);
  const int stride = KEY_STEP * WAVES;
  for (int key = k0 + KEY_STEP * wave; key < k1; key += stride) {
    const int p0 = page_of(pages, key), p1 = page_of(pages, key + 16);
    KeyBlock<BITS> x;
    fetch(x, key, p0, p1);
    // scores: keys 4 hh + 0..3 of each 16, column c
    floatx4 score[NC][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int n = 0; n < NC; ++n) score[n][b] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint4 ka = key_operand<BITS, BF>(x.k[b], t, bs);
#pragma unroll
        for (int n = 0; n < NC; ++n) score[n][b] = mfma16<BF>(ka, q[n][t], score[n][b]);
      }
    }
    const bool edge = key + KEY_STEP > all_see || p0 < 0 || p1 < 0;   // some column does not see some of the keys
    if (edge) {
      int first = key + 4 * hh;
      GEAR_PIN_VGPR(first);   // (what depends on it stays in here: as selections on `edge` every step would pay for it)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = first + 16 * b + i;
          const bool there = (b == 0 ? p0 : p1) >= 0;
          if (!there || at >= sp.kv) drop_value<BITS>(x.v[b], i);
#pragma unroll
          for (int n = 0; n < NC; ++n)
            if (!there || at >= sees[n]) score[n][b][i] = -INFINITY;
        }
    }
    uint4 pw[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top = fmaxf(top, score[n][b][i]);
        }
      top = weights_base<BF>(col_max<true>(top), a.scale_log2, a.far, F16_WEIGHT_LOG2);
      if (__ballot(top > m[n]) != 0ull) {
        const float now = fmaxf(m[n], top), by = now == -INFINITY ? 1.0f : GEAR_EXP2(m[n] - now);
        m[n] = now;
        l[n] *= by;
#pragma unroll
        for (int t = 0; t < 8; ++t) o[n][t] *= by;
      }
      const float from = m[n] == -INFINITY ? 0.0f : m[n];
      float p[8];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[4 * b + i] = GEAR_EXP2(__builtin_fmaf(score[n][b][i], a.scale_log2, -from));
          l[n] += p[4 * b + i];
        }
      // rounded to the type for the product (F16_WEIGHT_LOG2); the sum keeps them in fp32
      pw[n] = make_uint4(pack2<BF>(p[0], p[1]), pack2<BF>(p[2], p[3]), pack2<BF>(p[4], p[5]), pack2<BF>(p[6], p[7]));
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      column_words<BITS>(x.v[b].w[0], x.v[b].w[1]);
      column_words<BITS>(x.v[b].w[2], x.v[b].w[3]);
    }
    PairScale ps[4];
    if constexpr (BITS < 16) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        ps[2 * b] = pair_scale<BF>(x.v[b].sz[0], x.v[b].sz[1]);
        ps[2 * b + 1] = pair_scale<BF>(x.v[b].sz[2], x.v[b].sz[3]);
      }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint32_t w[4];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        w[2 * b] = column_pair<BITS, BF>(x.v[b].w[0], x.v[b].w[1], t, ps[2 * b], bs);
        w[2 * b + 1] = column_pair<BITS, BF>(x.v[b].w[2], x.v[b].w[3], t, ps[2 * b + 1], bs);
      }
      const uint4 va = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
      for (int n = 0; n < NC; ++n) o[n][t] = mfma16<BF>(va, pw[n], o[n][t]);
    }
  }

  // the waves' states: every wave brings its own to the common maximum, then sums and stores a share of the channels
  constexpr int waves = WAVES;
  float* top_of = reinterpret_cast<float*>(lds);                   // [wave][NC * 16]
  float* sum_of = top_of + waves * NC * 16;
  float4* part_of = reinterpret_cast<float4*>(sum_of + waves * NC * 16);
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    l[n] = col_sum<true>(l[n]);
    if (hh == 0) {
      top_of[wave * NC * 16 + n * 16 + c] = m[n];
      sum_of[wave * NC * 16 + n * 16 + c] = l[n];
    }
  }
  block_lds_sync();
  float total[NC], top[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    top[n] = -INFINITY;
    for (int w = 0; w < waves; ++w) top[n] = fmaxf(top[n], top_of[w * NC * 16 + n * 16 + c]);
    const float from = top[n] == -INFINITY ? 0.0f : top[n];
    total[n] = 0.0f;
    for (int w = 0; w < waves; ++w) total[n] += sum_of[w * NC * 16 + n * 16 + c] * GEAR_EXP2(top_of[w * NC * 16 + n * 16 + c] - from);
    const float by = GEAR_EXP2(m[n] - from);
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // channels 32 hh + 8 i + 0..7
      part_of[((wave * NC + n) * 8 + 2 * i) * 64 + lane] = make_float4(o[n][0][i] * by, o[n][1][i] * by, o[n][2][i] * by, o[n][3][i] * by);
      part_of[((wave * NC + n) * 8 + 2 * i + 1) * 64 + lane] = make_float4(o[n][4][i] * by, o[n][5][i] * by, o[n][6][i] * by, o[n][7][i] * by);
    }
  }
  block_lds_sync();
  for (int piece = wave; piece < NC * 8; piece += waves) {
    const int n = piece >> 3, k = piece & 7, col = n * 16 + c;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int w = 0; w < waves; ++w) {
      const float4 y = part_of[((w * NC + n) * 8 + k) * 64 + lane];
      x.x += y.x;
      x.y += y.y;
      x.z += y.z;
      x.w += y.w;
    }
    if (col >= cols) continue;
    const float sum = NC == 1 || n == 0 ? total[0] : total[NC - 1];
    const int ch = 32 * hh + 4 * k;
    const int row = col / a.gq, j = col - row * a.gq;
    if (is_output(a, span, parts.count)) {
      const float r = sum > 0.0f ? 1.0f / sum : 0.0f;
      unsigned char* p = a.out.data + 2 * ((int64_t)(sp.q0 + row) * a.out.token + (int64_t)(head * a.gq + j) * a.out.head + ch);
      *reinterpret_cast<uint2*>(p) = make_uint2(pack2<BF>(x.x * r, x.y * r), pack2<BF>(x.z * r, x.w * r));
    } else {
      const int64_t rec = few_record(a, s, head, col, part, sp.q0 + row, head * a.gq + j);
      *reinterpret_cast<float4*>(a.rec_o + rec * D + ch) = x;
      if (ch == 0) a.rec_ml[rec] = make_float2(NC == 1 || n == 0 ? top[0] : top[NC - 1], sum);
    }
  }
}

}  // namespace gear
