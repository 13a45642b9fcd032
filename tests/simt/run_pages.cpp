// Runs the paged cache's entry points on the CPU stand-in.  argv[1]: a folder with
//   meta.txt   n_pages page_size H_kv bits group dtype H_q scale causal table_width | n_seqs n_rows (of slots) | n_tokens max_q max_kv
//   pool.bin, K.bin V.bin slots.bin (n_rows > 0: written, then read back to K_back.bin V_back.bin), q.bin q_start.bin kv_len.bin
//   table.bin (n_tokens > 0: out.bin, from out_before.bin), pool_after.bin
// Every buffer is a heap block of exactly its size.
#include <hip/hip_runtime.h>
#include <fstream>
#include <iostream>
#include <string>
#include <vector>
#include "gear.h"

// (the kernels here have dynamically sized LDS only; the runtime wants the section of the other kind to be there)
__attribute__((section("simt_lds"), used)) static unsigned char lds_section[16];
static std::string dir;
struct Block {
  unsigned char* p = nullptr;
  size_t n = 0;
  explicit Block(size_t bytes) : n(bytes) { p = bytes ? (unsigned char*)aligned_alloc(16, (bytes + 15) / 16 * 16) : nullptr; }
  explicit Block(const char* name) {
    std::ifstream f(dir + "/" + name, std::ios::binary | std::ios::ate);
    n = f ? (size_t)f.tellg() : 0;
    p = n ? (unsigned char*)aligned_alloc(16, (n + 15) / 16 * 16) : nullptr;
    f.seekg(0);
    f.read((char*)p, (long)n);
  }
  ~Block() { free(p); }
  void save(const char* name) { std::ofstream(dir + "/" + name, std::ios::binary).write((char*)p, (long)n); }
};
static void tell(const char* kernel, dim3 grid, dim3 block, size_t lds) {
  fprintf(stderr, "launch %s grid %u block %u lds %zu\n", kernel[0] == '(' ? kernel + 1 : kernel, grid.x, block.x, lds);
}
#define CHECK(x)                                                  \
  do {                                                            \
    const int rc = (x);                                           \
    if (rc) { fprintf(stderr, "%s: %d\n", #x, rc); return 1; }    \
  } while (0)

int main(int, char** argv) {
  dir = argv[1];
  simt::observer = tell;
  std::ifstream f(dir + "/meta.txt");
  gear_page_config c{};
  gear_page_batch b{};
  int H_q, n_seqs, n_rows;
  float scale;
  f >> c.n_pages >> c.page_size >> c.H_kv >> c.bits >> c.group >> c.dtype >> H_q >> scale >> b.causal >> b.table_width >> n_seqs >> n_rows >> b.n_tokens >> b.max_q >> b.max_kv;
  c.d_h = 128;
  b.n_seqs = n_seqs;
  Block pool("pool.bin");
  size_t need = 0;
  CHECK(gear_page_bytes(&c, &need));
  if (need != pool.n) { fprintf(stderr, "pool bytes %zu, %zu wanted\n", pool.n, need); return 1; }
  if (n_rows > 0) {
    Block K("K.bin"), V("V.bin"), slots("slots.bin"), kb("K_before.bin"), vb("V_before.bin");
    const gear_page_rows in_k{K.p, (int64_t)n_rows * c.H_kv * 128, c.H_kv * 128, 128}, in_v{V.p, (int64_t)n_rows * c.H_kv * 128, c.H_kv * 128, 128};
    CHECK(gear_page_write(&c, pool.p, pool.n, &in_k, &in_v, n_seqs, n_rows, (const int64_t*)slots.p, nullptr));
    // back as [n_seqs][heads][rows]
    const gear_page_rows out_k{kb.p, (int64_t)n_rows * c.H_kv * 128, 128, (int64_t)n_rows * 128}, out_v{vb.p, (int64_t)n_rows * c.H_kv * 128, 128, (int64_t)n_rows * 128};
    CHECK(gear_page_read(&c, pool.p, pool.n, &out_k, nullptr, n_seqs, n_rows, (const int64_t*)slots.p, nullptr));
    CHECK(gear_page_read(&c, pool.p, pool.n, nullptr, &out_v, n_seqs, n_rows, (const int64_t*)slots.p, nullptr));
    kb.save("K_back.bin");
    vb.save("V_back.bin");
    pool.save("pool_after.bin");
  }
  if (b.n_tokens > 0) {
    Block q("q.bin"), q_start("q_start.bin"), kv_len("kv_len.bin"), table("table.bin"), out("out_before.bin");
    b.q_start = (const int32_t*)q_start.p;
    b.kv_len = (const int32_t*)kv_len.p;
    b.page_table = (const int32_t*)table.p;
    size_t bytes = 0;
    CHECK(gear_page_attn_bytes(&c, H_q, &b, &bytes));
    Block ws(bytes);
    if (bytes) memset(ws.p, 0xFF, bytes);
    const gear_page_rows qr{q.p, 0, (int64_t)H_q * 128, 128}, orow{out.p, 0, (int64_t)H_q * 128, 128};
    CHECK(gear_page_attn(&c, pool.p, pool.n, &b, &qr, H_q, scale, &orow, ws.p, ws.n, nullptr));
    out.save("out.bin");
    size_t words = 0;   // a record: 130 words, none of which is the filling
    for (size_t i = 0; i + 4 <= ws.n; i += 4) words += memcmp(ws.p + i, "\xFF\xFF\xFF\xFF", 4) != 0;
    fprintf(stderr, "records %zu of %zu\n", words / 130, ws.n / 520);
  }
  return 0;
}
