// Page tables on the device (include/gear.h): which pages a sequence has, and how often each is named.
//
// All of it is integers, and no result depends on the order in which blocks or lanes work: free pages are ranked by a prefix count over refs
// and given out by rank; what is added up in any order is counts; what could be claimed twice is exchanged for -1 or goes to the first of the list.
#include "page_piece.h"
#include "serving.h"

namespace gear {

constexpr int LIST_MOST = GEAR_PAGE_LIST_MAX, TABLE_THREADS = 1024, TABLE_WAVES = TABLE_THREADS / 64;

__device__ __forceinline__ int64_t entry_at(const PageTable& t, int row, int64_t i) { return (int64_t)row * t.width + i; }
__device__ __forceinline__ bool is_page(const PageTable& t, int p) { return p >= 0 && p < t.n_pages; }
// Whether any thread of the block has `x`.  `flag`: an LDS word of the call's own.
__device__ __forceinline__ bool block_any(bool x, int* flag) {
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
  if (x) *flag = 1;
  __syncthreads();
  const bool any = *flag != 0;
  __syncthreads();   // (the next call clears it)
  return any;
}
template <typename T>
__device__ __forceinline__ T wave_prefix(T v) {   // of lanes 0 .. own
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(v, o);
    if (lane_id() >= o) v += u;
  }
  return v;
}
// Marks the rows of a list in a bit per row of the table; true where entry i's row is one that an earlier entry names.  `seen`: LDS, (n_rows + 31) / 32 words; `list`: LIST_MOST.
__device__ __forceinline__ bool named_before(const PageTable& t, int i, int n, int row, bool valid, uint32_t* seen, int* list, int* flag) {
  for (int w = threadIdx.x; w < (t.n_rows + 31) / 32; w += blockDim.x) seen[w] = 0u;
  __syncthreads();
  bool twice = false;
  if (valid) twice = (atomicOr(&seen[row >> 5], 1u << (row & 31)) >> (row & 31) & 1u) != 0u;
  if (i < n) list[i] = valid ? row : -1;
  if (!block_any(twice, flag)) return false;
  bool before = false;
  if (valid)
    for (int j = 0; j < i; ++j) before = before || list[j] == row;
  return before;
}

// ---- pages for new tokens
// Pages per thread and step of the walk over refs: SCAN_LOADS times four.
constexpr int SCAN_LOADS = 4, SCAN_STEP = TABLE_THREADS * 4 * SCAN_LOADS;
// The slots of a granted row's tokens (LINES of threads by row).
__device__ __forceinline__ int64_t slot_of(const PageTable& t, int row, int64_t pos) {
  const int p = t.table[entry_at(t, row, pos >> t.shift)];
  return p < 0 ? -1 : ((int64_t)p << t.shift) + (pos & ((1 << t.shift) - 1));
}

struct ExtendLds {
  int flag, list[LIST_MOST], page[LIST_MOST];
  long long upto[LIST_MOST];       // pages that entries 0 .. i ask for
  long long wave_sum[TABLE_WAVES];
  int first[LIST_MOST], code[LIST_MOST], kv[LIST_MOST];
  int found[2][TABLE_WAVES * SCAN_LOADS];
};

// One block: entry i of the list is thread i's.  Bound by its chain of loads, barriers and ranks: 7.7 us for a token each of 64 sequences among 36000 pages, 16 for 512 pages each of 32
// among 49152 and those of 100 others (16384 pages a step).
__global__ __launch_bounds__(TABLE_THREADS) void page_extend_kernel(PageTable t, const int32_t* rows, const int32_t* counts, int n, int most, int64_t* slots,
                                                                    int32_t* copies, int32_t* refused, int with_slots) {
  GEAR_DYN_LDS(lds);
  ExtendLds& x = *reinterpret_cast<ExtendLds*>(lds);
  uint32_t* seen = reinterpret_cast<uint32_t*>(lds + sizeof(ExtendLds));
  const int i = (int)threadIdx.x, lane = lane_id(), wave = i >> 6, page_tokens = 1 << t.shift;
  const int row = i < n ? rows[i] : -1, count = i < n ? counts[i] : 0;
  bool ok = row >= 0 && row < t.n_rows;
  const int kv = ok ? t.kv_len[row] : 0;
  const bool twice = named_before(t, i, n, row, ok, seen, x.list, &x.flag);
  ok = ok && !twice && count >= 0 && count <= most && kv >= 0 && (int64_t)kv + count <= (int64_t)t.width << t.shift;
  // the entry that the first new token goes into, if it holds a page with tokens already
  const int first = kv >> t.shift;
  const bool partly = ok && count > 0 && (kv & (page_tokens - 1)) != 0;
  int held = partly ? t.table[entry_at(t, row, first)] : -1;
  held = is_page(t, held) ? held : -1;
  const int named = held >= 0 ? t.refs[held] : 0;
  const bool shared = named > 1;
  int before = 0, last = -1;   // of the entries before this one, those whose tokens go into the same page: how many, and the last
  if (block_any(shared, &x.flag)) {
    if (i < n) x.page[i] = shared ? held : -1;
    __syncthreads();
    if (shared)
      for (int j = 0; j < i; ++j)
        if (x.page[j] == held) {
          ++before;
          last = j;
        }
  }
  const bool copy = shared && named - before > 1, keeps = held >= 0 && !copy;
  const int64_t need = ok && count > 0 ? (int64_t)(((int64_t)kv + count - 1) >> t.shift) - first + 1 - (keeps ? 1 : 0) : 0;
  long long upto = wave_prefix((long long)need);
  if (lane == 63) x.wave_sum[wave] = upto;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < TABLE_WAVES; ++w) {
    if (w < wave) upto += x.wave_sum[w];
    total += x.wave_sum[w];
  }
  x.upto[i] = upto;
  x.first[i] = first + (keeps ? 1 : 0);
  x.list[i] = row;
  __syncthreads();

  // free pages by rank, while any are asked for
  long long free_pages = 0;
  for (int base = 0, step = 0; free_pages < total && base < t.n_pages; base += SCAN_STEP, ++step) {
    uint32_t mine[SCAN_LOADS];   // bit e: page base + 4 (u THREADS + i) + e is free
    int below[SCAN_LOADS];
    int4 r[SCAN_LOADS];
#pragma unroll
    for (int u = 0; u < SCAN_LOADS; ++u) {
      const int p = base + 4 * (u * TABLE_THREADS + i);
      r[u] = make_int4(1, 1, 1, 1);
      if (p + 4 <= t.n_pages) {
        r[u] = *reinterpret_cast<const int4*>(t.refs + p);
      } else if (p < t.n_pages) {
        r[u].x = t.refs[p];
        if (p + 1 < t.n_pages) r[u].y = t.refs[p + 1];
        if (p + 2 < t.n_pages) r[u].z = t.refs[p + 2];
      }
    }
    int* found = x.found[step & 1];
#pragma unroll
    for (int u = 0; u < SCAN_LOADS; ++u) {
      mine[u] = (r[u].x == 0 ? 1u : 0u) | (r[u].y == 0 ? 2u : 0u) | (r[u].z == 0 ? 4u : 0u) | (r[u].w == 0 ? 8u : 0u);
      const unsigned long long under = (1ull << lane) - 1ull;
      int all = 0;
      below[u] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned long long b = __ballot((mine[u] >> e & 1u) != 0u);
        below[u] += __popcll(b & under);
        all += __popcll(b);
      }
      if (lane == 0) found[u * TABLE_WAVES + wave] = all;
    }
    __syncthreads();
    static_assert(TABLE_WAVES * SCAN_LOADS == 64, "a wave has a lane for each");
    const int sum = wave_prefix(found[lane]);
#pragma unroll
    for (int u = 0; u < SCAN_LOADS; ++u) {
      const int at = u * TABLE_WAVES + wave;
      long long k = free_pages + below[u] + (at > 0 ? __shfl(sum, at - 1) : 0);
      if (mine[u] == 0u || k >= total) continue;
      // page k goes to the first entry of the list that asks for more than k with those before it: looked for once, the thread's next pages are its, or the next's
      // (a search for each page: 32 prompts of 8192 tokens 18.8 us instead of 16.0)
      int lo = 0, hi = n - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (x.upto[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      for (int e = 0; e < 4; ++e) {
        if ((mine[u] >> e & 1u) == 0u || k >= total) continue;
        while (x.upto[lo] <= k) ++lo;
        const int p = base + 4 * (u * TABLE_THREADS + i) + e;
        t.table[entry_at(t, x.list[lo], x.first[lo] + (k - (lo > 0 ? x.upto[lo - 1] : 0)))] = p;
        t.refs[p] = 1;
        ++k;
      }
    }
    free_pages += __shfl(sum, 63);
  }
  __syncthreads();

  // who gets what was asked for: no entry whose pages, with those before it, are more than there are; nor one that counted on an earlier one's copy
  int code = ok ? 0 : 1;
  if (ok && need > 0 && upto > free_pages) code = 2;
  x.code[i] = code;
  __syncthreads();
  if (code == 0 && keeps && shared && last >= 0 && x.code[last] == 2) code = 2;
  if (code == 2 && need > 0) {   // what it was given goes back
    const long long from = upto - need, got = free_pages - from;
    for (long long k = 0; k < need && k < got; ++k) {
      const int64_t at = entry_at(t, row, x.first[i] + k);
      const int p = t.table[at];
      t.refs[p] = 0;
      t.table[at] = copy && k == 0 ? held : -1;
    }
  }
  if (i < n) {
    refused[i] = code;
    const bool copied = code == 0 && copy;
    copies[2 * i] = copied ? held : -1;
    copies[2 * i + 1] = copied ? t.table[entry_at(t, row, first)] : -1;
    if (copied) atomicSub(&t.refs[held], 1);
    if (code == 0 && count > 0) t.kv_len[row] = kv + count;
  }
  if (!with_slots) return;
  x.page[i] = code == 0 ? count : 0;   // tokens granted
  x.kv[i] = kv;
  __syncthreads();
  for (int64_t k = i; k < (int64_t)n * most; k += TABLE_THREADS) {
    const int e = (int)(k / most), j = (int)(k - (int64_t)e * most);
    slots[k] = j < x.page[e] ? slot_of(t, x.list[e], (int64_t)x.kv[e] + j) : -1;
  }
}

// Many slots, behind the kernel above: a block per entry of the list and 1024 of its tokens.
__global__ __launch_bounds__(SLOT_THREADS) void page_slots_kernel(PageTable t, const int32_t* rows, const int32_t* counts, int most, int chunks, const int32_t* refused,
                                                                  int64_t* slots) {
  const int e = (int)(blockIdx.x / (unsigned)chunks), j0 = (int)(blockIdx.x - (unsigned)e * (unsigned)chunks) * SLOT_TOKENS;
  const int count = refused[e] == 0 ? counts[e] : 0, row = count > 0 ? rows[e] : 0;
  const int64_t kv = count > 0 ? (int64_t)t.kv_len[row] - count : 0;
  for (int64_t j = (int64_t)j0 + (int)threadIdx.x; j < min((int64_t)most, (int64_t)j0 + SLOT_TOKENS); j += SLOT_THREADS)
    slots[(int64_t)e * most + j] = j < count ? slot_of(t, row, kv + j) : -1;
}

// ---- tokens dropped: a block per entry of the list (3 us for 64 sequences, latency)
constexpr int DROP_THREADS = 256;
__global__ __launch_bounds__(DROP_THREADS) void page_truncate_kernel(PageTable t, const int32_t* rows, const int32_t* lens) {
  const int row = rows[blockIdx.x], len = max(lens[blockIdx.x], 0);
  if (row < 0 || row >= t.n_rows) return;
  __shared__ int kv_of_row;   // (read once: where the row is named twice, the other block changes it)
  if (threadIdx.x == 0) kv_of_row = t.kv_len[row];
  __syncthreads();
  const int kv = kv_of_row;
  if (kv <= len) return;
  const int64_t page_tokens = (int64_t)1 << t.shift;
  const int64_t e0 = (len + page_tokens - 1) >> t.shift, e1 = min((int64_t)t.width, (kv + page_tokens - 1) >> t.shift);
  // (an entry goes to whoever takes it first: a row that is named twice loses each of its pages once)
  for (int64_t e = e0 + (int)threadIdx.x; e < e1; e += DROP_THREADS) {
    const int p = atomicExch(&t.table[entry_at(t, row, e)], -1);
    if (is_page(t, p)) atomicSub(&t.refs[p], 1);
  }
  if (threadIdx.x == 0) atomicMin(&t.kv_len[row], len);
}

// ---- rows copied: a block per FORK_ENTRIES / n columns of the table, all of whose sources it reads before it writes (5.3 us for 16 copies of 257 entries, latency)
__global__ __launch_bounds__(FORK_THREADS) void page_fork_kernel(PageTable t, const int32_t* src, const int32_t* dst, int n, int cols) {
  GEAR_DYN_LDS(lds);
  int* from = reinterpret_cast<int*>(lds);          // [LIST_MOST] source row, -1: nothing to do
  int* to = from + LIST_MOST;
  int* len = to + LIST_MOST;
  int* flag = len + LIST_MOST;
  int* held = flag + 4;                             // [FORK_ENTRIES]
  uint32_t* seen = reinterpret_cast<uint32_t*>(held + FORK_ENTRIES);
  for (int w = threadIdx.x; w < (t.n_rows + 31) / 32; w += FORK_THREADS) seen[w] = 0u;
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += FORK_THREADS) {
    const int s = src[i], d = dst[i];
    const bool ok = s >= 0 && s < t.n_rows && d >= 0 && d < t.n_rows;
    from[i] = ok ? s : -1;
    to[i] = ok ? d : -1;
    len[i] = ok && blockIdx.x == 0 ? t.kv_len[s] : 0;
    if (ok && (atomicOr(&seen[d >> 5], 1u << (d & 31)) >> (d & 31) & 1u) != 0u) *flag = 1;
  }
  __syncthreads();
  if (*flag != 0) {   // a destination twice: the first counts
    for (int i = threadIdx.x; i < n; i += FORK_THREADS)
      for (int j = 0; j < i; ++j)
        if (to[i] >= 0 && to[j] == to[i]) from[i] = -1;
    __syncthreads();
  }
  const int64_t c0 = (int64_t)blockIdx.x * cols;
  const int mine = (int)min((int64_t)cols, t.width - c0);
  for (int k = threadIdx.x; k < n * mine; k += FORK_THREADS) {
    const int i = k / mine, e = k - i * mine;
    held[k] = from[i] >= 0 ? t.table[entry_at(t, from[i], c0 + e)] : -1;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < n * mine; k += FORK_THREADS) {
    const int i = k / mine, e = k - i * mine;
    if (from[i] < 0) continue;
    const int p = held[k], was = atomicExch(&t.table[entry_at(t, to[i], c0 + e)], p);
    if (p == was) continue;
    if (is_page(t, p)) atomicAdd(&t.refs[p], 1);
    if (is_page(t, was)) atomicSub(&t.refs[was], 1);
  }
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < n; i += FORK_THREADS)
      if (from[i] >= 0) t.kv_len[to[i]] = len[i];
}

// ---- pages in use brought to the front
// Which pages are in use is read once, into a bit per page in LDS: 11 us for 10200 pages of which 2500 move, in one block, latency (14 with three walks over refs).
struct CompactLds {
  int sum[TABLE_WAVES];
  uint32_t used[];
};
__device__ __forceinline__ int block_sum(int v, int* sum) {
  v = wave_prefix(v);
  if (lane_id() == 63) sum[threadIdx.x >> 6] = v;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < TABLE_WAVES; ++w) all += sum[w];
  __syncthreads();
  return all;
}
// Set bits of `words` words (word(w), looked at from word 0 on, each from its low bit up, or with BACK from its high bit down): take(k, w, bit) for the first `most`, ranked by k.  How many there were of them.
template <bool BACK, class Word, class F>
__device__ __forceinline__ int ranked_bits(int words, int most, int* sum, Word word, F take) {
  int count = 0;
  for (int base = 0; base < words && count < most; base += TABLE_THREADS) {
    const int w = base + (int)threadIdx.x;
    uint32_t bits = w < words ? word(w) : 0u;
    const int mine = __popc(bits), upto = wave_prefix(mine);
    if (lane_id() == 63) sum[threadIdx.x >> 6] = upto;
    __syncthreads();
    int k = count + upto - mine, all = 0;
    for (int v = 0; v < TABLE_WAVES; ++v) {
      if (v < (int)(threadIdx.x >> 6)) k += sum[v];
      all += sum[v];
    }
    for (; bits != 0u && k < most; ++k) {
      const int bit = BACK ? 31 - __clz((int)bits) : __ffs((int)bits) - 1;
      take(k, w, bit);
      bits &= ~(1u << bit);
    }
    count += all;
    __syncthreads();
  }
  return min(count, most);
}
__global__ __launch_bounds__(TABLE_THREADS) void page_compact_kernel(PageTable t, int32_t* moves, int most, int32_t* counts) {
  GEAR_DYN_LDS(lds);
  CompactLds& x = *reinterpret_cast<CompactLds*>(lds);
  const int lane = lane_id(), words = (t.n_pages + 31) / 32;
  int used = 0;
  constexpr int LOADS = 8;
  for (int base = 0; base < t.n_pages; base += TABLE_THREADS * LOADS) {
    int r[LOADS];
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int p = base + u * TABLE_THREADS + (int)threadIdx.x;
      r[u] = p < t.n_pages ? t.refs[p] : 0;
    }
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int w = (base + u * TABLE_THREADS + (int)threadIdx.x) / 64 * 2;   // 64 pages of a wave: two words
      const unsigned long long b = __ballot(r[u] > 0);
      if (lane < 2 && w + lane < words) {
        const uint32_t bits = (uint32_t)(b >> (32 * lane));
        x.used[w + lane] = bits;
        used += __popc(bits);
      }
    }
  }
  const int live = block_sum(used, x.sum);
  // bits of word w from page `live` on
  auto from_live = [&](int w) { return w * 32 >= live ? 0xFFFFFFFFu : w * 32 + 32 <= live ? 0u : 0xFFFFFFFFu << (live & 31); };
  const int n = ranked_bits<false>((live + 31) / 32, most, x.sum, [&](int w) { return ~x.used[w] & ~from_live(w); }, [&](int k, int w, int bit) { moves[2 * (int64_t)k + 1] = 32 * w + bit; });
  const int first = live / 32;
  ranked_bits<true>(words - first, n, x.sum, [&](int i) { return x.used[words - 1 - i] & from_live(words - 1 - i); },
                    [&](int k, int i, int bit) { moves[2 * (int64_t)k] = 32 * (words - 1 - i) + bit; });
  __syncthreads();
  for (int k = (int)threadIdx.x; k < n; k += TABLE_THREADS) {
    const int from = moves[2 * (int64_t)k], to = moves[2 * (int64_t)k + 1];
    t.refs[to] = t.refs[from];
    t.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    counts[0] = live;
    counts[1] = n;
  }
}
// Entries that name a moved page, and the end of the list of moves.
constexpr int REMAP_THREADS = 256;
__global__ __launch_bounds__(REMAP_THREADS) void page_remap_kernel(PageTable t, int32_t* moves, int most, const int32_t* counts) {
  const int live = counts[0], n = counts[1];
  const int64_t entries = (int64_t)t.n_rows * t.width, at = (int64_t)blockIdx.x * REMAP_THREADS + threadIdx.x;
  if (at < most && at >= n) moves[2 * at] = moves[2 * at + 1] = -1;
  if (at >= entries || n == 0) return;
  const int p = t.table[at];
  if (p < live || p >= t.n_pages) return;
  int lo = 0, hi = n;   // moves[.][0] falls
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (moves[2 * (int64_t)mid] > p) lo = mid + 1;
    else hi = mid;
  }
  if (lo < n && moves[2 * (int64_t)lo] == p) t.table[at] = moves[2 * (int64_t)lo + 1];
}

// ---- pages' bytes: a block per MOVE_BYTES of a pair in one pool.  Past the caches: 16 copies of a page of 256 KB in four pools 5.3 us, and 19.7 where the
// kernel's end waits for the caches to write them back; 2200 pages of 256 KB, 1.3 GB in all, 248 us (5.3 TB/s) and 269.
__global__ __launch_bounds__(MOVE_THREADS) void page_move_kernel(unsigned char* pool, uint32_t page_bytes, int n_pages, uint64_t stride, const int32_t* pairs, int n, int chunks) {
  const unsigned bid = blockIdx.x, rest = bid / (unsigned)chunks, layer = rest / (unsigned)n, i = rest - layer * (unsigned)n;
  const int from = pairs[2 * (int64_t)i], to = pairs[2 * (int64_t)i + 1];
  if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) return;
  const uint32_t at = (bid - rest * (unsigned)chunks) * (uint32_t)MOVE_BYTES + threadIdx.x * 16;
  const unsigned char* a = pool + layer * stride + (uint64_t)(uint32_t)from * page_bytes + at;
  unsigned char* b = pool + layer * stride + (uint64_t)(uint32_t)to * page_bytes + at;
  uint4 v[MOVE_LOADS];
#pragma unroll
  for (int u = 0; u < MOVE_LOADS; ++u)
    if (at + u * (MOVE_THREADS * 16) < page_bytes) v[u] = load16_once(a + u * (MOVE_THREADS * 16));
#pragma unroll
  for (int u = 0; u < MOVE_LOADS; ++u)
    if (at + u * (MOVE_THREADS * 16) < page_bytes) store16<true>(b + u * (MOVE_THREADS * 16), v[u]);
}

// ---- launches
static size_t seen_bytes(const PageTable& t) { return (size_t)(t.n_rows + 31) / 32 * 4; }

// Slots that the extending block writes itself; more go to a launch of their own.
constexpr int64_t SLOTS_IN_BLOCK = 16384;

hipError_t launch_extend(const PageTable& t, const int32_t* rows, const int32_t* counts, int n, int most, int64_t* slots, int32_t* copies, int32_t* refused,
                         hipStream_t st) {
  const size_t lds = sizeof(ExtendLds) + seen_bytes(t);   // up to 65 KB
  static std::atomic<uint64_t> raised{0};
  hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_extend_kernel), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  const bool with_slots = (int64_t)n * most <= SLOTS_IN_BLOCK;
  hipLaunchKernelGGL(page_extend_kernel, dim3(1), dim3(TABLE_THREADS), lds, st, t, rows, counts, n, most, slots, copies, refused, with_slots ? 1 : 0);
  e = hipGetLastError();
  if (e != hipSuccess || with_slots) return e;
  const int chunks = (int)(((int64_t)most + SLOT_TOKENS - 1) / SLOT_TOKENS);
  hipLaunchKernelGGL(page_slots_kernel, dim3((unsigned)n * (unsigned)chunks), dim3(SLOT_THREADS), 0, st, t, rows, counts, most, chunks, refused, slots);
  return hipGetLastError();
}
hipError_t launch_truncate(const PageTable& t, const int32_t* rows, const int32_t* lens, int n, hipStream_t st) {
  hipLaunchKernelGGL(page_truncate_kernel, dim3((unsigned)n), dim3(DROP_THREADS), 0, st, t, rows, lens);
  return hipGetLastError();
}
hipError_t launch_fork(const PageTable& t, const int32_t* src, const int32_t* dst, int n, hipStream_t st) {
  const size_t lds = (3 * LIST_MOST + 4 + FORK_ENTRIES) * 4 + seen_bytes(t);   // up to 77 KB
  static std::atomic<uint64_t> raised{0};
  const hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_fork_kernel), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  const int cols = fork_cols(n);
  hipLaunchKernelGGL(page_fork_kernel, dim3((unsigned)((t.width + cols - 1) / cols)), dim3(FORK_THREADS), lds, st, t, src, dst, n, cols);
  return hipGetLastError();
}
hipError_t launch_compact(const PageTable& t, int32_t* moves, int most, int32_t* counts, hipStream_t st) {
  const size_t lds = sizeof(CompactLds) + (size_t)(t.n_pages + 31) / 32 * 4;   // up to 128 KB
  static std::atomic<uint64_t> raised{0};
  hipError_t e = raise_dynamic_lds(reinterpret_cast<const void*>(page_compact_kernel), raised, lds, LDS_PER_CU);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(page_compact_kernel, dim3(1), dim3(TABLE_THREADS), lds, st, t, moves, most, counts);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t entries = std::max((int64_t)t.n_rows * t.width, (int64_t)most);
  hipLaunchKernelGGL(page_remap_kernel, dim3((unsigned)((entries + REMAP_THREADS - 1) / REMAP_THREADS)), dim3(REMAP_THREADS), 0, st, t, moves, most, counts);
  return hipGetLastError();
}
hipError_t launch_move(unsigned char* pool, uint32_t page_bytes, int n_pages, int n_pools, size_t stride, const int32_t* pairs, int n, hipStream_t st) {
  const int chunks = (int)((page_bytes + MOVE_BYTES - 1) / MOVE_BYTES);
  const unsigned blocks = (unsigned)chunks * (unsigned)n * (unsigned)n_pools;
  hipLaunchKernelGGL(page_move_kernel, dim3(blocks), dim3(MOVE_THREADS), 0, st, pool, page_bytes, n_pages, (uint64_t)stride, pairs, n, chunks);
  return hipGetLastError();
}

}  // namespace gear
