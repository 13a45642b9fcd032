// Runs the calls that a text file names on the CPU stand-in.  argv[1]: a folder with calls.txt and a NAME.bin for every `load NAME`.
// Every buffer is a heap block of exactly its size; `save NAME` writes it to NAME.out.
#include <fstream>
#include <iostream>
#include <map>
#include <sstream>
#include <string>
#include <vector>
#include "gear.h"

__attribute__((section("simt_lds"), used)) static unsigned char lds_section[16];
static std::string dir;
struct Block {
  unsigned char* p = nullptr;
  size_t n = 0;
};
static std::map<std::string, Block> blocks;
static std::map<std::string, gear_page_rows> rows;
static void tell(const char* kernel, dim3 grid, dim3 block, size_t lds) {
  fprintf(stderr, "launch %s grid %u block %u lds %zu\n", kernel[0] == '(' ? kernel + 1 : kernel, grid.x, block.x, lds);
}
template <class T>
static T* at(std::istream& f) {
  std::string name;
  f >> name;
  if (name == "-") return nullptr;
  if (!blocks.count(name)) { fprintf(stderr, "no block %s\n", name.c_str()); exit(2); }
  return (T*)blocks[name].p;
}
static const gear_page_rows* view(std::istream& f) {
  std::string name;
  f >> name;
  return name == "-" ? nullptr : &rows.at(name);
}

int main(int, char** argv) {
  dir = argv[1];
  simt::observer = tell;
  std::ifstream calls(dir + "/calls.txt");
  gear_page_config c{};
  gear_rope rope{};
  gear_page_table table{};
  std::string line;
  while (std::getline(calls, line)) {
    std::istringstream f(line);
    std::string op;
    f >> op;
    int rc = 0;
    if (op == "load") {
      std::string name;
      f >> name;
      std::ifstream in(dir + "/" + name + ".bin", std::ios::binary | std::ios::ate);
      Block b;
      b.n = (size_t)in.tellg();
      b.p = b.n ? (unsigned char*)aligned_alloc(16, (b.n + 15) / 16 * 16) : nullptr;
      in.seekg(0);
      in.read((char*)b.p, (long)b.n);
      if (b.n % 16) {   // (exactly its size)
        unsigned char* exact = nullptr;
        if (posix_memalign((void**)&exact, 16, b.n)) return 2;
        memcpy(exact, b.p, b.n);
        free(b.p);
        b.p = exact;
      }
      blocks[name] = b;
    } else if (op == "save") {
      std::string name;
      f >> name;
      std::ofstream(dir + "/" + name + ".out", std::ios::binary).write((char*)blocks[name].p, (long)blocks[name].n);
    } else if (op == "config") {
      f >> c.n_pages >> c.page_size >> c.H_kv >> c.bits >> c.group >> c.dtype;
      c.d_h = 128;
    } else if (op == "rope") {
      f >> rope.rot_dim >> rope.interleaved >> rope.inverse >> rope.factor;
      rope.freq = at<double>(f);
    } else if (op == "rows") {
      std::string name;
      f >> name;
      gear_page_rows r{};
      r.data = at<void>(f);
      int64_t offset;
      f >> offset >> r.seq >> r.token >> r.head;
      r.data = (unsigned char*)r.data + 2 * offset;
      rows[name] = r;
    } else if (op == "rotate") {
      int dtype, n_seqs, n_rows, heads;
      f >> dtype;
      const gear_page_rows *x = view(f), *out = view(f);
      f >> n_seqs >> n_rows >> heads;
      rc = gear_rotate(&rope, dtype, x, out, n_seqs, n_rows, heads, at<int64_t>(f), nullptr);
    } else if (op == "write" || op == "write_rope") {
      std::string pool;
      f >> pool;
      const gear_page_rows *K = view(f), *V = view(f);
      int n_seqs, n_rows, H_q = 0;
      if (op == "write") {
        f >> n_seqs >> n_rows;
        rc = gear_page_write(&c, blocks[pool].p, blocks[pool].n, K, V, n_seqs, n_rows, at<int64_t>(f), nullptr);
      } else {
        const gear_page_rows *q = view(f), *q_out = view(f);
        f >> H_q >> n_seqs >> n_rows;
        const int64_t* slots = at<int64_t>(f);
        rc = gear_page_write_rope(&c, blocks[pool].p, blocks[pool].n, &rope, K, V, q, q_out, H_q, n_seqs, n_rows, slots, at<int64_t>(f), nullptr);
      }
    } else if (op == "table") {
      table.table = at<int32_t>(f);
      table.kv_len = at<int32_t>(f);
      table.refs = at<int32_t>(f);
      f >> table.n_pages >> table.page_size >> table.n_rows >> table.width;
    } else if (op == "extend") {
      const int32_t *r = at<int32_t>(f), *n = at<int32_t>(f);
      int count, most;
      f >> count >> most;
      int64_t* slots = at<int64_t>(f);
      int32_t* copies = at<int32_t>(f);
      rc = gear_page_extend(&table, r, n, count, most, slots, copies, at<int32_t>(f), nullptr);
    } else if (op == "truncate" || op == "fork") {
      const int32_t *a = at<int32_t>(f), *b = at<int32_t>(f);
      int count;
      f >> count;
      rc = op == "fork" ? gear_page_fork(&table, a, b, count, nullptr) : gear_page_truncate(&table, a, b, count, nullptr);
    } else if (op == "compact") {
      int32_t* moves = at<int32_t>(f);
      int most;
      f >> most;
      rc = gear_page_compact(&table, moves, most, at<int32_t>(f), nullptr);
    } else if (op == "move") {
      std::string pool;
      int n_pools, n;
      size_t stride;
      f >> pool >> n_pools >> stride;
      const int32_t* pairs = at<int32_t>(f);
      f >> n;
      rc = gear_page_move(&c, blocks[pool].p, blocks[pool].n, n_pools, stride, pairs, n, nullptr);
    } else if (op == "shared") {
      std::string pool;
      gear_page_batch b{};
      gear_page_groups g{};
      int H_q;
      float scale;
      f >> pool >> H_q >> scale >> b.causal >> b.n_seqs >> b.n_tokens >> b.max_q >> b.max_kv >> b.table_width;
      b.q_start = at<int32_t>(f);
      b.kv_len = at<int32_t>(f);
      b.page_table = at<int32_t>(f);
      f >> g.n_groups >> g.max_q >> g.max_prefix;
      g.always = 1;
      g.group_start = at<int32_t>(f);
      g.prefix_len = at<int32_t>(f);
      const gear_page_rows *q = view(f), *out = view(f);
      size_t bytes = 0;
      rc = gear_page_attn_shared_bytes(&c, H_q, &b, &g, &bytes);
      unsigned char* ws = bytes ? (unsigned char*)malloc(bytes) : nullptr;
      if (bytes) memset(ws, 0xFF, bytes);
      if (!rc) rc = gear_page_attn_shared(&c, blocks[pool].p, blocks[pool].n, &b, &g, q, H_q, scale, out, ws, bytes, nullptr);
      free(ws);
    } else if (!op.empty()) {
      fprintf(stderr, "unknown: %s\n", op.c_str());
      return 2;
    }
    if (rc) {
      fprintf(stderr, "%s: %d\n", line.c_str(), rc);
      return 1;
    }
  }
  return 0;
}
