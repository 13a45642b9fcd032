// The records that the parts of a key axis leave become one row: the weight of a part is 2^(its maximum - the greatest).
#pragma once
#include "pages.h"

namespace gear {

constexpr int MERGE_WAVES = 4, MERGE_LDS = MERGE_WAVES * 3 * 64 * 4;

struct Merged {   // a lane's two channels, and the sum of the weights
  float sum, x, y;
};
// Eight records of a wave on their way.
struct Records {
  float2 ml[8], v[8];
};
template <int WAVES>
__device__ __forceinline__ void request_records(Records& r, const PageAttn& a, int64_t rec, int i0, int lane) {   // in the row, whatever lies behind its parts
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int64_t i = rec + min(i0 + WAVES * u, a.n_split - 1);
    r.ml[u] = a.rec_ml[i];
    r.v[u] = *reinterpret_cast<const float2*>(a.rec_o + i * D + 2 * lane);
  }
}
// What a wave asks for before it knows how many parts there are (the lengths are on their way then, too): its first records, and a maximum per lane.
struct FirstRecords {
  Records r;
  float top;
};
template <int WAVES>
__device__ __forceinline__ FirstRecords first_records(const PageAttn& a, int64_t rec, int wave, int lane) {
  FirstRecords f;
  request_records<WAVES>(f.r, a, rec, wave, lane);
  f.top = a.rec_ml[rec + min(lane, a.n_split - 1)].x;
  return f;
}
// WAVES waves take the records of `count` parts from `rec` on in turn; wave 0 has the result.  lds: [wave][3][lane].
template <int WAVES>
__device__ __forceinline__ Merged merge_records(FirstRecords& f, const PageAttn& a, int64_t rec, int count, int wave, int lane, float* lds) {
  float top = lane < count ? f.top : -INFINITY;   // (of all parts: each wave looks through them by itself)
  for (int i = lane + 64; i < count; i += 64) top = fmaxf(top, a.rec_ml[rec + i].x);
  top = wave_max(top);
  const float from = top == -INFINITY ? 0.0f : top;
  Merged m{0.0f, 0.0f, 0.0f};
  for (int i0 = wave; i0 < count; i0 += WAVES * 8) {
    if (i0 != wave) request_records<WAVES>(f.r, a, rec, i0, lane);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool there = i0 + WAVES * u < count;
      const float by = there ? GEAR_EXP2(f.r.ml[u].x - from) : 0.0f;
      m.sum += there ? f.r.ml[u].y * by : 0.0f;
      m.x += there ? f.r.v[u].x * by : 0.0f;
      m.y += there ? f.r.v[u].y * by : 0.0f;
    }
  }
  if constexpr (WAVES > 1) {
    lds[(wave * 3 + 0) * 64 + lane] = m.sum;
    lds[(wave * 3 + 1) * 64 + lane] = m.x;
    lds[(wave * 3 + 2) * 64 + lane] = m.y;
    block_lds_sync();
    if (wave == 0)
      for (int w = 1; w < WAVES; ++w) {
        m.sum += lds[(w * 3 + 0) * 64 + lane];
        m.x += lds[(w * 3 + 1) * 64 + lane];
        m.y += lds[(w * 3 + 2) * 64 + lane];
      }
  }
  return m;
}
__device__ __forceinline__ void store_merged(const PageAttn& a, const Merged& m, int token, int head, int lane, int bf) {
  const float r = m.sum > 0.0f ? 1.0f / m.sum : 0.0f;
  unsigned char* p = a.out.data + 2 * ((int64_t)token * a.out.token + (int64_t)head * a.out.head + 2 * lane);
  *reinterpret_cast<uint32_t*>(p) = bf ? pack2<true>(m.x * r, m.y * r) : pack2<false>(m.x * r, m.y * r);
}

}  // namespace gear
