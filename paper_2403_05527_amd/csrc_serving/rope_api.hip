// Entry points of rotary positions (include/gear.h): arguments are checked here, before anything is launched.
#include <cmath>
#include "page_checks.h"
#include "serving.h"

using namespace gear;

namespace {

int check_rope(const gear_rope* r, Rope* to) {
  if (!r || r->rot_dim < 2 || r->rot_dim > D || r->rot_dim % 2) return GEAR_EINVAL;
  if ((r->interleaved != 0 && r->interleaved != 1) || (r->inverse != 0 && r->inverse != 1) || !std::isfinite(r->factor) || !r->freq) return GEAR_EINVAL;
  if (misaligned(r->freq, 8)) return GEAR_EALIGN;
  *to = Rope{r->freq, r->rot_dim, r->rot_dim / 2, r->factor, r->inverse ? -1.0f : 1.0f};
  return GEAR_OK;
}
// rows that are turned into themselves, or into others (which may not lie over one another)
int check_turned(const gear_page_rows* x, const gear_page_rows* out, int64_t n_seqs, int64_t n_rows, int64_t heads) {
  const int rc = check_rows(x, n_seqs, n_rows, heads, false);
  if (rc) return rc;
  if (out->data == x->data && ((n_seqs > 1 && out->seq != x->seq) || (n_rows > 1 && out->token != x->token) || (heads > 1 && out->head != x->head))) return GEAR_EINVAL;
  return check_rows(out, n_seqs, n_rows, heads, true);
}
// 16 rows a block, a block for each head, at most
bool too_many_blocks(int64_t n_seqs, int64_t n_rows, int64_t heads) {
  const int64_t chunks = n_rows == 1 ? (n_seqs + 15) / 16 : n_seqs * ((n_rows + 15) / 16);
  return n_seqs * n_rows > INT_MOST - 4096 || chunks * heads > THREADS_MOST / 256;
}

}  // namespace

extern "C" {

int gear_rope_freq(int scaling, int32_t rot_dim, double base, double scale, double trained_len, double low, double high, double* freq) {
  if (rot_dim < 2 || rot_dim > D || rot_dim % 2 || !freq) return GEAR_EINVAL;
  if (!(base > 0.0) || !(scale > 0.0) || !std::isfinite(base) || !std::isfinite(scale)) return GEAR_EINVAL;
  if (scaling < GEAR_ROPE_PLAIN || scaling > GEAR_ROPE_TURNS) return GEAR_EINVAL;
  if (scaling == GEAR_ROPE_BASE && rot_dim == 2) return GEAR_EINVAL;   // (one pair, whose frequency is 1 whatever the base)
  if (scaling == GEAR_ROPE_TURNS && (!(trained_len > 0.0) || !std::isfinite(trained_len) || !(low >= 0.0) || !(high > low) || !std::isfinite(high))) return GEAR_EINVAL;
  const double b = scaling == GEAR_ROPE_BASE ? base * std::pow(scale, rot_dim / (rot_dim - 2.0)) : base;
  for (int p = 0; p < rot_dim / 2; ++p) {
    double w = std::pow(b, -2.0 * p / rot_dim);
    if (scaling == GEAR_ROPE_LINEAR) w /= scale;
    if (scaling == GEAR_ROPE_TURNS) {
      const double k = (trained_len * w / 6.28318530717958647693 - low) / (high - low), keep = k < 0.0 ? 0.0 : k > 1.0 ? 1.0 : k;
      w *= keep + (1.0 - keep) / scale;
    }
    freq[p] = w;
  }
  return GEAR_OK;
}

int gear_rotate(const gear_rope* rope, int dtype, const gear_page_rows* x, const gear_page_rows* out, int32_t n_seqs, int32_t n_rows, int32_t heads,
                const int64_t* positions, void* stream) {
  RopeRows a{};
  int rc = check_rope(rope, &a.rope);
  if (rc) return rc;
  if ((dtype != GEAR_F16 && dtype != GEAR_BF16) || !x || !out || n_seqs < 0 || n_rows < 0 || heads < 0) return GEAR_EINVAL;
  if (n_seqs == 0 || n_rows == 0 || heads == 0) return GEAR_OK;   // (tensors without an entry have no address)
  if ((rc = check_turned(x, out, n_seqs, n_rows, heads))) return rc;
  if (!positions) return GEAR_EINVAL;
  if (misaligned(positions, 8)) return GEAR_EALIGN;
  if (too_many_blocks(n_seqs, n_rows, heads)) return GEAR_ECAPACITY;
  a.x = view_of(x);
  a.out = view_of(out);
  a.k = a.v = view_of(nullptr);
  a.positions = positions;
  a.n_rows = n_rows;
  a.heads = heads;
  return launch_rope(a, 0, dtype == GEAR_BF16, rope->interleaved != 0, n_seqs, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

int gear_page_write_rope(const gear_page_config* cfg, void* pool, size_t pool_bytes, const gear_rope* rope, const gear_page_rows* K, const gear_page_rows* V,
                         const gear_page_rows* q, const gear_page_rows* q_out, int32_t H_q, int32_t n_seqs, int32_t n_rows, const int64_t* slots,
                         const int64_t* positions, void* stream) {
  RopeRows a{};
  int rc = check_pool(cfg, pool, pool_bytes, &a.geom);
  if (rc || (rc = check_rope(rope, &a.rope))) return rc;
  if (!K || !V || n_seqs < 0 || n_rows < 0 || H_q < 0 || !q != !q_out || !q != (H_q == 0)) return GEAR_EINVAL;
  if (n_seqs == 0 || n_rows == 0) return GEAR_OK;
  if ((rc = check_rows(K, n_seqs, n_rows, cfg->H_kv, false)) || (rc = check_rows(V, n_seqs, n_rows, cfg->H_kv, false))) return rc;
  if (q && (rc = check_turned(q, q_out, n_seqs, n_rows, H_q))) return rc;
  if (!slots || !positions) return GEAR_EINVAL;
  if (misaligned(slots, 8) || misaligned(positions, 8)) return GEAR_EALIGN;
  if (too_many_blocks(n_seqs, n_rows, (int64_t)H_q + cfg->H_kv)) return GEAR_ECAPACITY;
  a.x = view_of(q);
  a.out = view_of(q_out);
  a.k = view_of(K);
  a.v = view_of(V);
  a.slots = slots;
  a.positions = positions;
  a.n_rows = n_rows;
  a.heads = H_q;
  return launch_rope(a, cfg->bits, cfg->dtype == GEAR_BF16, rope->interleaved != 0, n_seqs, static_cast<hipStream_t>(stream)) == hipSuccess ? GEAR_OK : GEAR_EHIP;
}

}  // extern "C"
