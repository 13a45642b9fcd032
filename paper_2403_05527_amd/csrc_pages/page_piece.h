// Eight channels of one row into the pool and back: 16 lanes take a row (include/gear.h has the layout and the quantizer's definition).
#pragma once
#include "pages.h"

namespace gear {

typedef short i16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t min_i16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2_t, a), __builtin_bit_cast(i16x2_t, b)));
}
__device__ __forceinline__ uint32_t max_i16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2_t, a), __builtin_bit_cast(i16x2_t, b)));
}
// Two 16-bit floating numbers as signed integers of the same order, and back.
__device__ __forceinline__ uint32_t ordered(uint32_t x) {
  return x ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2_t, x) >> 15) & 0x7FFF7FFFu);
}
template <int CTRL>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) { return max_i16x2(x, dpp_u<CTRL>(x)); }

// One row piece of eight values into its place: `block` the head's Keys or Values in the page, r the row, c the lane's piece (0..15).  Every
// lane of the wave comes here (its row's extremes are exchanged), those with `live` store.
template <int BITS, bool BF>
__device__ __forceinline__ void store_piece(const PageGeom& g, unsigned char* block, int r, int c, const uint4& v, bool live) {
  if constexpr (BITS == 16) {
    if (live) *reinterpret_cast<uint4*>(block + (r * 16 + c) * 16) = v;
  } else {
    constexpr float LEVELS = BITS == 8 ? 255.0f : 15.0f;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    auto value = [](uint32_t pair, int e) { return to_f32<BF>(pair >> (16 * (e & 1)) & 0xFFFFu); };
    // extremes: two values at a time as signed 16-bit integers of the same order (negative ones with their other bits turned around)
    uint32_t lo = ordered(w[0]), hi = lo;
#pragma unroll
    for (int j = 1; j < 4; ++j) {
      const uint32_t k = ordered(w[j]);
      lo = min_i16x2(lo, k);
      hi = max_i16x2(hi, k);
    }
    lo = min_i16x2(lo, lo >> 16 | lo << 16);
    hi = max_i16x2(hi, hi >> 16 | hi << 16);
    uint32_t ext = (hi & 0xFFFFu) | (~lo & 0xFFFF0000u);   // (the greatest complement is that of the least)
    ext = lanes_max<DPP_XOR1>(ext);
    ext = lanes_max<DPP_XOR2>(ext);
    if (g.gshift > 5) ext = lanes_max<DPP_HALF_MIRROR>(ext);
    if (g.gshift > 6) ext = lanes_max<DPP_MIRROR>(ext);
    ext = ordered(ext ^ 0xFFFF0000u);
    const uint32_t zero = ext >> 16;
    const float mn = to_f32<BF>(zero), mx = to_f32<BF>(ext & 0xFFFFu);
    // (a quotient as below; 1 / 255 and 1 / 15 are constants)
    const float range = __fsub_rn(mx, mn), by = __fmul_rn(range, 1.0f / LEVELS);
    float s32 = __builtin_fmaf(__builtin_fmaf(-by, LEVELS, range), 1.0f / LEVELS, by);
    GEAR_IN_VGPR(s32);   // (rounded here: else the last step and the rounding to fp16 become one instruction, which rounds another number once)
    const uint32_t sz = (pack2<BF>(s32, 0.0f) & 0xFFFFu) | zero << 16;
    const float scale = to_f32<BF>(sz & 0xFFFFu);
    uint32_t code[8];
    // (x - zero) / scale as IEEE division in fp32 gives it, in a product and two fused steps: with a correctly rounded reciprocal the last one rounds
    // the exact quotient, which by a scale of 11 bits or 8 is never rounded to a half that it is not.  The difference is exact unless the exponents lie more than
    // 12 (bf16: 15) apart; one that is not, and is rounded to a half of the scale, gets the even code (include/gear.h).  Then the nearest integer is the sum with
    // 1.5 * 2^23, whose last bits are the code.  (Dividing: 8 x 4096 tokens of 8 heads to 4 bits 58 us.)
    // A scale is off by 2^-11 (fp16) or 2^-8 (bf16) of it, more where it is denormal: only of these and of 8-bit codes in bf16 may a quotient come to more than half
    // a step past the last code.
    const float inv = scale > 0.0f ? recip_of_half(scale) : 0.0f;
    float one = 1.0f;
    GEAR_IN_VGPR(one);   // (with it, an fp16 value's conversion and the difference are one instruction, rounded once as the difference is)
    if (scale >= (BF ? 0x1p-100f : 0x1p-14f) || !(scale > 0.0f)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = value(w[e >> 1], e), d = BF ? __fsub_rn(x, mn) : __builtin_fmaf(x, one, -mn), t = __fmul_rn(d, inv), q = __builtin_fmaf(__builtin_fmaf(-t, scale, d), inv, t);
        code[e] = __float_as_uint(__fadd_rn(BF && BITS == 8 ? fminf(q, LEVELS) : q, 12582912.0f));
      }
    } else {   // (bf16: the reciprocal, or the remainder above, would leave fp32's range)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t pair = w[e >> 1];
        GEAR_PIN_VGPR(pair);   // (converted in here: above, one conversion for both ways would take the place of the fused difference)
        code[e] = __float_as_uint(__fadd_rn(fminf(__fdiv_rn(__fsub_rn(value(pair, e), mn), scale), LEVELS), 12582912.0f));
      }
    }
    if constexpr (BITS == 8) {
      auto bytes = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return GEAR_BYTE_PERM(GEAR_BYTE_PERM(d, c, 0x0C0C0400u), GEAR_BYTE_PERM(b, a, 0x0C0C0400u), 0x05040100u); };
      if (live) *reinterpret_cast<uint2*>(block + (r * 16 + c) * 8) = make_uint2(bytes(code[0], code[1], code[2], code[3]), bytes(code[4], code[5], code[6], code[7]));
    } else {
      // (the sums' other bits, from bit 22 on, are shifted further up)
      auto nibbles = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return ((((((d << 4) + c) << 4) + b) << 4) + a); };
      if (live)
        *reinterpret_cast<uint32_t*>(block + (r * 16 + c) * 4) =
            GEAR_BYTE_PERM(nibbles(code[1], code[3], code[5], code[7]), nibbles(code[0], code[2], code[4], code[6]), 0x05040100u);
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

#ifndef GEAR_PAGE_PAST_CACHES   // (the CPU stand-in lowers it)
#define GEAR_PAGE_PAST_CACHES (64ll << 20)
#endif
constexpr int64_t PAST_CACHES = GEAR_PAGE_PAST_CACHES;   // bytes that are brought back

// What is brought back and is large is stored past the caches, which keep what they held: behind the write of the same rows (8 x 4096 tokens of 8 heads, 128 MiB, 4
// bits) both take 60 us, and 69 into the caches; 7 x 1777 tokens of 40 heads, 255 MB, 79 -> 47; 16 x 4096 of 32, 1.07 GB, 314 -> 289.  A kernel that reads the rows at once
// would find part of less than 256 MB there, and pays for it.  In us, 8 KV heads, groups of 64, into the caches and past them: the read by itself, and with a maximum
// over each tensor behind it:
//   MiB               64                 128                192                256                512
//   fp16 at 8 bits    15 14, 57 66       26 25, 89 108      60 37, 142 155     82 49, 220 223     160 148, 437 421
//   bf16 at 4 bits    14 13, 57 67       24 22, 89 108      40 32, 136 151     87 46, 217 228     164 79, 453 432
//   fp16 at 16 bits   18 18, 60 69       35 34, 98 117      77 49, 168 173     103 64, 240 243    199 196, 471 471
template <bool PAST>
__device__ __forceinline__ void store16(unsigned char* p, const uint4& v) {
#ifdef GEAR_NO_NONTEMPORAL
  *reinterpret_cast<uint4*>(p) = v;
#else
  if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(p));
  else *reinterpret_cast<uint4*>(p) = v;
#endif
}
// (rows that are read once need no place in the caches: 2 us of 184 where 8-bit pages are written)
__device__ __forceinline__ uint4 load16_once(const unsigned char* p) {
#ifdef GEAR_NO_NONTEMPORAL
  return *reinterpret_cast<const uint4*>(p);
#else
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
#endif
}

}  // namespace gear
