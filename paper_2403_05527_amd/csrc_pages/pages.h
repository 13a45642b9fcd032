// Shared by the kernels of the paged cache: the pool's geometry, conversions between codes and values, and the
// matrix instructions in both 16-bit types.
#pragma once
#include "gear_internal.h"

// v_mfma with 16-bit operands and fp32 accumulators (a build that runs the kernels elsewhere may predefine these).
// 16x16x32: A lane l = row l % 16, k = 8 (l / 16) + 0..7; B the same for columns; D lane l = rows 4 (l / 16) + 0..3, column l % 16.
// 32x32x16: A lane l = row l % 32, k = 8 (l / 32) + 0..7; B the same for columns; D lane l, register i = row 8 (i / 4) + 4 (l / 32)
// + i % 4, column l % 32.
#ifndef GEAR_MFMA16_F16
#define GEAR_MFMA16_F16(a, b, c) \
  __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(gear::h8_t, (a)), __builtin_bit_cast(gear::h8_t, (b)), (c), 0, 0, 0)
#define GEAR_MFMA16_BF16(a, b, c) \
  __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(gear::b8_t, (a)), __builtin_bit_cast(gear::b8_t, (b)), (c), 0, 0, 0)
#define GEAR_MFMA32_F16(a, b, c) \
  __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(gear::h8_t, (a)), __builtin_bit_cast(gear::h8_t, (b)), (c), 0, 0, 0)
#define GEAR_MFMA32_BF16(a, b, c) \
  __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(gear::b8_t, (a)), __builtin_bit_cast(gear::b8_t, (b)), (c), 0, 0, 0)
#endif
// ds_read_b64_tr_b16: in each group of 16 lanes, lane i addresses 8 bytes, row i / 4 and columns 4 (i % 4) + 0..3 of a 4 x 16
// matrix of 16-bit values, and gets column i's four rows.
#ifndef GEAR_LDS_READ_TR
#define GEAR_LDS_READ_TR(p) \
  __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) gear::s4_t*)(p)))
#endif
#ifndef GEAR_EXP2
#define GEAR_EXP2(x) __builtin_amdgcn_exp2f(x)
#endif
// two floats as bf16 values (nearest even), the first in the low half: one instruction
#ifndef GEAR_PACK_BF2
#define GEAR_PACK_BF2(a, b) __builtin_bit_cast(uint32_t, (gear::b2_t){(__bf16)(a), (__bf16)(b)})
#endif
// a * b + c on two pairs of fp16 values, each rounded once
#ifndef GEAR_PK_FMA_F16
#define GEAR_PK_FMA_F16(a, b, c)                                                                                            \
  __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(gear::h2_t, (a)), __builtin_bit_cast(gear::h2_t, (b)), \
                                                         __builtin_bit_cast(gear::h2_t, (c))))
#endif

// A constant that is kept in a vector register (an instruction that takes two constants can have one from a scalar register only).
#ifndef GEAR_IN_VGPR
#define GEAR_IN_VGPR(x) asm("" : "+v"(x))
#endif

namespace gear {

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
#ifndef GEAR_NO_BF16_TYPE
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
#endif
typedef short s4_t __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// The pool as the kernels see it.
struct PageGeom {
  const unsigned char* pool;
  uint32_t page_bytes;    // below 2^31
  uint32_t block_bytes;   // Keys or Values of one head in a page
  uint32_t row_bytes;
  int32_t n_pages;
  int32_t shift;          // log2 of the page size
  int32_t gshift;         // log2 of the group size
  int32_t H;
};
__host__ __device__ inline uint32_t page_mask(const PageGeom& g) { return (1u << g.shift) - 1u; }
// where a head's Keys (tensor 0) or Values (1) begin in a page
__device__ __forceinline__ const unsigned char* block_of(const PageGeom& g, int page, int head, int tensor) {
  return g.pool + ((uint64_t)(uint32_t)page * g.page_bytes + (uint32_t)(2 * head + tensor) * g.block_bytes);
}
__host__ __device__ inline uint32_t words_at(const PageGeom& g) { return g.row_bytes << g.shift; }   // the (scale, zero) words in a block

// 16-bit rows with strides in elements
struct RowView {
  unsigned char* data;
  int64_t seq, token, head;
};

// ---- 16-bit values ----------------------------------------------------------
template <bool BF>
__device__ __forceinline__ float to_f32(uint32_t bits16) {
  if constexpr (BF) return __uint_as_float(bits16 << 16);
  else return h2f(bits16 & 0xFFFFu);
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {   // rounded to nearest even, a in the low half
  if constexpr (BF) return GEAR_PACK_BF2(a, b);
  else return pack_h2(a, b);
}
template <bool BF>
__device__ __forceinline__ floatx4 mfma16(const uint4& a, const uint4& b, const floatx4& c) {
  if constexpr (BF) return GEAR_MFMA16_BF16(a, b, c);
  else return GEAR_MFMA16_F16(a, b, c);
}
template <bool BF>
__device__ __forceinline__ floatx16 mfma32(const uint4& a, const uint4& b, const floatx16& c) {
  if constexpr (BF) return GEAR_MFMA32_BF16(a, b, c);
  else return GEAR_MFMA32_F16(a, b, c);
}

// ---- codes to values ----------------------------------------------------------
// Two codes as integers in the halves of a word; fp16 arithmetic has them as 1024 + code or 64 + code (the low mantissa bits of those numbers), bf16 goes
// through fp32.
// (scale, zero) words of the two entries: `sz0` for the low one.  The same word twice where both lie in one group of a row.
struct PairScale {
  uint32_t scale, zero;   // fp16: a pair each
  float s0, z0, s1, z1;   // bf16; the scales times 2^24
};
template <bool BF>
__device__ __forceinline__ PairScale pair_scale(uint32_t sz0, uint32_t sz1) {
  PairScale p;
  if constexpr (BF) {
    p.s0 = __uint_as_float(sz0 << 16) * 16777216.0f;
    p.z0 = __uint_as_float(sz0 & 0xFFFF0000u);
    p.s1 = __uint_as_float(sz1 << 16) * 16777216.0f;
    p.z1 = __uint_as_float(sz1 & 0xFFFF0000u);
  } else {
    p.scale = GEAR_BYTE_PERM(sz1, sz0, 0x05040100u);
    p.zero = GEAR_BYTE_PERM(sz1, sz0, 0x07060302u);
  }
  return p;
}
// 1024 and 64 in both halves, where one instruction puts masked codes into them.
struct Biases {
  uint32_t b1024, b64;
};
__device__ __forceinline__ Biases biases() {
  Biases b{0x64006400u, 0x54005400u};
  GEAR_IN_VGPR(b.b1024);
  GEAR_IN_VGPR(b.b64);
  return b;
}
constexpr uint32_t BYTES_64H = 0x64646464u, F16_NEG_1024 = 0xE400E400u, F16_NEG_64 = 0xD400D400u;
// fp16: value pair of (1024 + code) or (64 + code) pairs.  Both steps are exact but for the one rounding of the fused multiply-add:
// the value that a code stands for.
__device__ __forceinline__ uint32_t value_f16(uint32_t biased, uint32_t neg_bias, const PairScale& p) {
  const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2_t, biased) + __builtin_bit_cast(h2_t, neg_bias));
  return GEAR_PK_FMA_F16(c, p.scale, p.zero);
}
// bf16: value pair of two codes in the halves of a word.  As fp16 numbers those are denormals, code * 2^-24, which one instruction takes into an fp32
// multiply-add (the scales of a pair are 2^24 times theirs): a product and a sum, rounded to fp32 and then to bf16.
__device__ __forceinline__ uint32_t value_bf16(uint32_t codes, float s0, float z0, float s1, float z1) {
  return GEAR_PACK_BF2(__builtin_fmaf(h2f(codes & 0xFFFFu), s0, z0), __builtin_fmaf(h2f(codes >> 16), s1, z1));
}
// Channels 2 i, 2 i + 1 (i = 0..3) of a run of eight along a row: w0, w1 are the run's code words (w1 at 8 bits only).
template <int BITS, bool BF>
__device__ __forceinline__ uint32_t row_pair(uint32_t w0, uint32_t w1, int i, const PairScale& p, const Biases& bs) {
  if constexpr (BITS == 8) {
    const uint32_t w = i < 2 ? w0 : w1;
    if constexpr (BF) {
      return value_bf16(GEAR_BYTE_PERM(0u, w, (i & 1) ? 0x0C030C02u : 0x0C010C00u), p.s0, p.z0, p.s1, p.z1);
    } else {
      return value_f16(GEAR_BYTE_PERM(BYTES_64H, w, (i & 1) ? 0x04030402u : 0x04010400u), F16_NEG_1024, p);
    }
  } else {   // 4 bits: nibble i of each half
    if constexpr (BF) {
      const uint32_t x = i < 2 ? w0 : w0 >> 8;   // (the upper nibble of a byte stays where it is: 16 code, with a 16th of the scale)
      return (i & 1) ? value_bf16(x & 0x00F000F0u, p.s0 * 0.0625f, p.z0, p.s1 * 0.0625f, p.z1) : value_bf16(x & 0x000F000Fu, p.s0, p.z0, p.s1, p.z1);
    } else {
      const uint32_t x = i < 2 ? w0 : w0 >> 8;
      return (i & 1) ? value_f16((x & 0x00F000F0u) | bs.b64, F16_NEG_64, p) : value_f16((x & 0x000F000Fu) | bs.b1024, F16_NEG_1024, p);
    }
  }
}
template <int BITS, bool BF>
__device__ __forceinline__ uint4 row_run(uint32_t w0, uint32_t w1, const PairScale& p, const Biases& bs) {   // eight channels
  return make_uint4(row_pair<BITS, BF>(w0, w1, 0, p, bs), row_pair<BITS, BF>(w0, w1, 1, p, bs), row_pair<BITS, BF>(w0, w1, 2, p, bs),
                    row_pair<BITS, BF>(w0, w1, 3, p, bs));
}
// Two rows' words of eight channels (16 bits: four each; 8: two; 4: one), brought into the order that column_pair takes from them.
// 8 bits: the rows' bytes of two channels in each word (x: channels 0, 1 and 4, 5; y: 2, 3 and 6, 7), the first row's first; 4 bits: the rows'
// even channels in x, the odd ones in y.
template <int BITS>
__device__ __forceinline__ void column_words(uint32_t* x, uint32_t* y) {
#pragma unroll
  for (int j = 0; j < (BITS == 16 ? 0 : BITS / 4); ++j) {
    const uint32_t a = x[j], b = y[j];
    x[j] = GEAR_BYTE_PERM(b, a, BITS == 8 ? 0x05010400u : 0x05040100u);
    y[j] = GEAR_BYTE_PERM(b, a, BITS == 8 ? 0x07030602u : 0x07060302u);
  }
}
// Channel e (a constant, 0..7) of the two rows, the first in the low half.
template <int BITS, bool BF>
__device__ __forceinline__ uint32_t column_pair(const uint32_t* x, const uint32_t* y, int e, const PairScale& p, const Biases& bs) {
  if constexpr (BITS == 16) {
    return GEAR_BYTE_PERM(y[e >> 1], x[e >> 1], (e & 1) ? 0x07060302u : 0x05040100u);
  } else if constexpr (BITS == 8) {
    const uint32_t w = (e & 2) ? y[e >> 2] : x[e >> 2];
    if constexpr (BF) return value_bf16(GEAR_BYTE_PERM(0u, w, (e & 1) ? 0x0C030C02u : 0x0C010C00u), p.s0, p.z0, p.s1, p.z1);
    else return value_f16(GEAR_BYTE_PERM(BYTES_64H, w, (e & 1) ? 0x04030402u : 0x04010400u), F16_NEG_1024, p);
  } else {
    return row_pair<4, BF>((e & 1) ? y[0] : x[0], 0u, e >> 1, p, bs);   // (nibble e / 2 of each half)
  }
}

// ---- attention ------------------------------------------------------------------
struct PageAttn {
  PageGeom geom;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* table;
  RowView q, out;
  float* rec_o;      // [record rows][n_split][128] partial sums
  float2* rec_ml;    // [record rows][n_split] (what the weights' exponents are taken from, sum of weights), in units of log2
  float scale_log2;  // |scale| * log2(e), above 0: scores are compared before they are scaled, and -inf times it is -inf
  float far;         // 2^23 / scale_log2
  uint32_t flip;     // 0x80008000 where the scale is negative: the queries change sign instead
  int32_t width;     // entries of a sequence's row of the table
  int32_t n_seqs, n_tokens, gq, causal;
  int32_t n_split;   // parts of the key axis, at most
  int32_t least;     // tokens that make a part
  int32_t few;       // columns (new tokens x gq) up to which page_attn_few_kernel has a sequence; 0: page_attn_many_kernel has them all
  int32_t few_cols;  // record rows per sequence and head there
  int32_t tiles;     // column tiles of page_attn_many_kernel, at most
};
constexpr int KEY_STEP = 32, MANY_COLS = 128, MANY_KEYS = 64;
// The weights' rounding to the type for the product with V: half a step, 2^-11 (fp16) or 2^-8 (bf16) of each, as the outputs'.  fp16 numbers below 2^-14 have
// fewer bits, and below 2^-25 none: the weights are held times 2^15 for the greatest that there can be, so that a long tail of small ones counts in the product with V
// as it counts in their sum (held up to 1, 131072 weights of 2^-26 beside one of 1 were 2^-9 of the sum and nothing of the product).
constexpr float F16_WEIGHT_LOG2 = 15.0f;
constexpr int FEW_PART = 256, MANY_PART = 128;   // tokens of a part, at least (of few columns: one step of a block's waves)

// The key axis of `keys` tokens in at most n_split equal parts of about `least` tokens and more, multiples of `unit`: tokens of a part, and how many
// there are (at least one).
struct Parts {
  int len, count;
};
__host__ __device__ inline Parts parts_of(int keys, int n_split, int least, int unit) {
  int n = (keys + least / 2) / least;
  n = n < 1 ? 1 : (n > n_split ? n_split : n);
  const int len = ((keys + n - 1) / n + unit - 1) / unit * unit;
  return Parts{len, len > 0 ? (keys + len - 1) / len : 1};
}
struct SeqSpan {
  int q0, nq, kv;
};
__device__ __forceinline__ SeqSpan seq_span(const PageAttn& a, int s) {   // nothing outside the arrays, whatever the device holds
  const int q0 = a.q_start[s], q1 = a.q_start[s + 1], kv = a.kv_len[s];
  SeqSpan r;
  r.q0 = max(q0, 0);
  r.nq = min(max(q1, 0), a.n_tokens) - r.q0;   // (both at least 0: below 2^31 apart)
  r.kv = (int)min((long long)max(kv, 0), (long long)a.width << a.geom.shift);
  return r;
}
// tokens that row `row` (of the sequence's nq) sees
__device__ __forceinline__ int row_sees(const PageAttn& a, const SeqSpan& s, int row) {
  return a.causal ? max(0, min(s.kv, s.kv - s.nq + row + 1)) : s.kv;
}

// A sequence's row of the page table as a wave reads it: 64 entries at a time, one per lane, so that a step waits for the table once per 64
// pages and not for each.
struct PageRow {
  const int32_t* table;
  int32_t base, held, n_pages, shift, end;   // `end`: no key from there on is asked for
  unsigned long long valid;                  // bit i: entry base + i is a page
};
__device__ __forceinline__ PageRow page_row(const PageAttn& a, int s, int end) {
  return PageRow{a.table + (int64_t)s * a.width, -64, 0, a.geom.n_pages, a.geom.shift, end, 0ull};
}
__device__ __forceinline__ void hold_entries(PageRow& r, int i, int32_t entry) {   // the lane's entry, i + its number
  r.base = i;
  r.held = entry >= 0 && entry < r.n_pages ? entry : -1;
  r.valid = __ballot(r.held >= 0);
}
__device__ __forceinline__ void load_entries(PageRow& r, int i) {   // from entry i on, which is one of a key before `end`; behind the last: that one
  const int at = i + lane_id(), last = (r.end - 1) >> r.shift;
  hold_entries(r, i, r.table[at <= last ? at : last]);
}
// The page of a key (the same in all lanes of the wave); -1: none.  Keys are asked for in ascending order.
__device__ __forceinline__ int page_of(PageRow& r, int key) {
  if (key >= r.end) return -1;
  const int i = key >> r.shift;
  if (i >= r.base + 64) load_entries(r, i);
  return __builtin_amdgcn_readlane(r.held, i - r.base);
}
__device__ __forceinline__ uint4 signed_query(const uint4& q, uint32_t flip) { return make_uint4(q.x ^ flip, q.y ^ flip, q.z ^ flip, q.w ^ flip); }
// What the exponents of a column's weights are taken from, whose greatest score is `top`, times `scale`: `below` less than that in fp16.  Not from `far`, 2^23, on, where the
// base is a whole number and the greatest weight off by as many powers of two as it is rounded by: half a step is 1 from 2^24 on, and fp16 ends at 2^16.
template <bool BF>
__device__ __forceinline__ float weights_base(float top, float scale, float far, float below) {
  return __builtin_fmaf(top, scale, !BF && fabsf(top) < far ? -below : 0.0f);
}
// Greatest value / sum over the lanes of a column, l % 16 (Q16) or l % 32.
template <bool Q16>
__device__ __forceinline__ float col_max(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  GEAR_LANE_SWAP32(a, b);
  v = fmaxf(__uint_as_float(a), __uint_as_float(b));
  if constexpr (Q16) {
    a = b = __float_as_uint(v);
    GEAR_LANE_SWAP16(a, b);
    v = fmaxf(__uint_as_float(a), __uint_as_float(b));
  }
  return v;
}
template <bool Q16>
__device__ __forceinline__ float col_sum(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  GEAR_LANE_SWAP32(a, b);
  v = __uint_as_float(a) + __uint_as_float(b);
  if constexpr (Q16) {
    a = b = __float_as_uint(v);
    GEAR_LANE_SWAP16(a, b);
    v = __uint_as_float(a) + __uint_as_float(b);
  }
  return v;
}

}  // namespace gear
