// How gear_page_attn_shared divides calls on the device's 256 CUs: the entry points, with launches that print what they are given.  Each line of standard input is a call: KV heads, query heads per
// KV head, bits, n_seqs, n_tokens, max_q, max_kv, n_groups, max_q of a group, max_prefix, always.
#include "page_api.hip"
#include "shared_api.hip"
#include <cstdio>

__attribute__((section("simt_lds"), used)) static unsigned char lds_section[16];
namespace gear {
hipError_t launch_page_shared(const SharedCall& c, int, bool, int, hipStream_t) {
  printf("shared %d %d %d %d", c.prefix.n_split, c.prefix.least, c.prefix.few, c.prefix.blocks);
  for (const SharedKind& k : {c.own_few, c.own_many}) printf(" %d %d %d %d", k.n_split, k.least, k.few, k.blocks);
  printf(" %d\n", c.n_records);
  return hipSuccess;
}
hipError_t launch_page_few(const PageAttn&, int, bool, int, hipStream_t) { return puts("plain"), hipSuccess; }
hipError_t launch_page_many(const PageAttn&, int, bool, hipStream_t) { return puts("plain"), hipSuccess; }
hipError_t launch_page_mixed(const PageAttn&, const PageAttn&, int, bool, int, hipStream_t) { return puts("plain"), hipSuccess; }
hipError_t launch_page_copy(const PageGeom&, int, bool, bool, const RowView&, const RowView&, const int64_t*, int, int, hipStream_t) { return hipSuccess; }
}  // namespace gear

int main() {
  void* const fake = (void*)0x10000000;   // never dereferenced
  int H, gq, bits;
  gear_page_batch b{};
  gear_page_groups g{};
  while (scanf("%d %d %d %d %d %d %d %d %d %d %d", &H, &gq, &bits, &b.n_seqs, &b.n_tokens, &b.max_q, &b.max_kv, &g.n_groups, &g.max_q, &g.max_prefix, &g.always) == 11) {
    const gear_page_config cfg{64, 64, H, 128, bits, 64, GEAR_BF16};
    const gear_page_rows rows{fake, 0, (int64_t)H * gq * 128, 128};
    b.table_width = (b.max_kv + 63) / 64;
    b.causal = 1;
    b.q_start = b.kv_len = b.page_table = g.group_start = g.prefix_len = (const int32_t*)fake;
    size_t bytes = 0;
    int rc = gear_page_attn_shared_bytes(&cfg, H * gq, &b, &g, &bytes);
    if (!rc) rc = gear_page_attn_shared(&cfg, fake, (size_t)1 << 40, &b, &g, &rows, H * gq, 0.1f, &rows, fake, bytes, nullptr);
    if (rc) printf("refused %d\n", rc);
    fflush(stdout);
  }
  return 0;
}
