/*
 * gear.h -- C ABI of libgear: GEAR KV-cache compression (arXiv 2403.05527) and
 * the single-query attention read of the compressed cache, for AMD MI355X
 * (gfx950).  Plain C: pointers and sizes only, no C++ or torch types.
 *
 * Conventions (all entry points)
 *  - "device" pointers are HIP device memory of the current device, "host"
 *    pointers ordinary host memory.  Every buffer is allocated and freed by
 *    the caller; the library allocates nothing and keeps no global state.
 *  - Work is enqueued on the caller's hipStream_t (passed as void*, NULL = the
 *    default stream); no call synchronises with the host.  Inputs may be
 *    released once the stream has passed the call.
 *  - d_h (head dimension) must be 128.  Tensors are fp16, contiguous,
 *    [B, H, tokens, d_h] unless stated otherwise.  Inputs must be finite.
 *  - Return value: GEAR_OK (0) or a negative gear_status.  Arguments are
 *    validated on the host before anything is launched, so a failed call
 *    leaves the cache untouched.
 *  - A gear_cache is a small host-side descriptor owned by the caller.  It
 *    records what the device arena holds (segments, ranks, token counts) so
 *    that capacity and shape errors are caught without reading device memory.
 *    Calls on one gear_cache must be issued in stream order by one thread.
 */
#ifndef GEAR_H
#define GEAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum gear_status {
  GEAR_OK = 0,
  GEAR_EINVAL = -1,    /* bad / unsupported parameter, or NULL pointer            */
  GEAR_ECAPACITY = -2, /* arena, workspace, segment or chunk capacity exceeded     */
  GEAR_EALIGN = -3,    /* a pointer is not 16-byte aligned                         */
  GEAR_EHIP = -4       /* a HIP runtime call failed (launch error)                 */
} gear_status;

#define GEAR_MAX_CHUNKS 256
/* Size of the library's built-in scratch array (gear_decode_attn_static). */
#define GEAR_STATIC_SCRATCH_BYTES (32u << 20)

/* Hyper-parameters of Algorithm 1 of the paper plus the capacities of one
 * layer's cache. */
typedef struct gear_config {
  int32_t B;             /* batch                                                  */
  int32_t H_kv;          /* KV heads                                               */
  int32_t H_q;           /* query heads, multiple of H_kv, H_q/H_kv <= 8           */
  int32_t d_h;           /* head dimension, must be 128                            */
  int32_t bits;          /* b in {2, 4}  (Eq. 2)                                   */
  int32_t group;         /* g in {32, 64, 128}: Keys g tokens of one channel,      */
                         /* Values g channels of one token.  0: the coarse         */
                         /* per-vector grouping of the paper's background section  */
                         /* ("KCVT"): one group per Key channel over the tokens of */
                         /* a call, one per Value token over all H_kv*d_h channels */
  int32_t outlier_ppm;   /* s of Filter_s (Eq. 4) in parts per million of a        */
                         /* vector; 20000 = 2 %, 0 = GEAR-L (no sparse term)       */
  int32_t n_buf_cap;     /* n_b: streaming-buffer capacity, 1..255                 */
  int32_t n_prefill_max; /* capacity of the first (prefill) segment, <= 32768      */
  int32_t n_chunks_max;  /* number of flushed buffers that can be appended, <= 256 */
  int32_t rank_max;      /* largest rank any compress call will use, 0..8          */
  int32_t flags;         /* GEAR_FLAG_* bits, 0 = the method as the paper states it */
} gear_config;

/* Filter_s ranks each KV head's d_h channels of a Value token on their own (vector
 * length d_h, count ceil(s d_h) per head) instead of the token's row over all heads
 * (Eq. 4 read with X = V in R^{n x d}).  Every head is then independent of the others. */
#define GEAR_FLAG_V_FILTER_PER_HEAD 1

/* Host-side descriptor of one cache.  Filled by gear_cache_init, advanced by
 * gear_compress.  Treat the fields as read-only. */
typedef struct gear_cache {
  gear_config cfg;
  void*    arena;                        /* device                                 */
  uint64_t arena_bytes;
  int32_t  n_prefill;                    /* tokens in segment 0 (0 = none yet)     */
  int32_t  rank_prefill;
  int32_t  n_chunks;                     /* appended chunk segments                */
  int32_t  n_total;                      /* tokens in all segments                 */
  uint8_t  chunk_n[GEAR_MAX_CHUNKS];     /* tokens of chunk j                      */
  uint8_t  chunk_rank[GEAR_MAX_CHUNKS];  /* rank of chunk j                        */
} gear_cache;

/* Sizes the caller must provide for `cfg`: the device arena that holds the
 * compressed cache and a device workspace shared by gear_compress and
 * gear_decode_attn (scratch; contents need not survive between calls). */
int gear_cache_bytes(const gear_config* cfg, size_t* arena_bytes, size_t* workspace_bytes);

/* Binds a device arena (>= arena_bytes, 256-byte aligned) to `cache` (host,
 * out) and marks it empty.  Nothing is launched. */
int gear_cache_init(const gear_config* cfg, void* arena, size_t arena_bytes, gear_cache* cache);

/* Forgets every segment (the arena memory is reused). */
int gear_cache_reset(gear_cache* cache);

/*
 * Compress one segment of n tokens and append it (Algorithm 1: the prefill body
 * on the first call, the decoding-phase body on a flushed buffer afterwards):
 *   S = Filter_s(X)  (Eq. 4: per Key channel over the n tokens of this call,
 *                     per Value token over all H_kv*d_h channels; ties go to
 *                     the lower index),
 *   D = Quant_b(X - S) (Eq. 2 / Eq. 5, scale and zero-point stored in fp16),
 *   R = X - D - S, and per (batch, head) A, B = SVDSolver_rank(R) (Eq. 6,
 *   Algorithm 2 with `iters` rounds, start matrix init_B).
 * K, V      : device fp16 [B, H_kv, n, d_h].
 * n         : first call: 1..n_prefill_max; later calls: 1..n_buf_cap.
 * rank      : 0..rank_max (0 = no low-rank term); iters >= 1.
 * init_B    : device fp32 [2 (K,V), B, H_kv, d_h, rank], the start matrices B0 of
 *             Algorithm 2 (its random initialisation, taken as an input so that runs are
 *             reproducible), or NULL: the library then draws the same array on the
 *             device from `seed`: entry i (row-major) is ((z >> 40) - 2^23) / 2^23 with
 *             z = mix(seed + (i + 1) * 0x9E3779B97F4A7C15), mix(z): z ^= z >> 30,
 *             z *= 0xBF58476D1CE4E5B9, z ^= z >> 27, z *= 0x94D049BB133111EB,
 *             z ^= z >> 31 (64-bit arithmetic): uniform on a 24-bit grid in [-1, 1).
 * seed      : used only when init_B is NULL and rank > 0.
 * workspace : device, >= workspace_bytes of gear_cache_bytes.
 */
int gear_compress(gear_cache* cache, const void* K, const void* V, int32_t n, int32_t rank,
                  int32_t iters, const float* init_B, uint64_t seed, void* workspace,
                  size_t workspace_bytes, void* stream);

/*
 * gear_compress with the error-reduction (low-rank) term on the n_lowrank most recent tokens of
 * the call only: the ablation of Sec. 4.3 that recovers the quantization error of the p % most
 * recent prefill tokens (n_lowrank = ceil(p n / 100)).  SVDSolver runs on the residual rows of
 * those tokens; the earlier tokens get A = 0, i.e. Filter and Quant only.  n_lowrank = n is
 * gear_compress; n_lowrank = 0 stores the segment with rank 0.  (The other ablation of that
 * section, error reduction on the prefill tokens only -- "GEAR-L Prefill" --, needs no entry
 * point of its own: compress the flushed buffers with rank = 0.)
 */
int gear_compress_recent(gear_cache* cache, const void* K, const void* V, int32_t n, int32_t rank,
                         int32_t iters, const float* init_B, uint64_t seed, int32_t n_lowrank,
                         void* workspace, size_t workspace_bytes, void* stream);

/* X-hat = D + A B^T + S for every stored token (Algorithm 1, "replace X with
 * D + L + S"), rounded to fp16.  K_out, V_out: device fp16
 * [B, H_kv, n_total, d_h]; either may be NULL. */
int gear_decompress(const gear_cache* cache, void* K_out, void* V_out, void* stream);

/*
 * Single-query attention (Eq. 1) over the compressed cache followed by the
 * first n_buf rows of the fp16 streaming buffer, never materialising K-hat or
 * V-hat: softmax(q K^T / sqrt(d_h)) V per query head; query head i reads KV
 * head i / (H_q / H_kv).
 * q         : device fp16 [B, H_q, 1, d_h].
 * K_buf,V_buf: device fp16 [B, H_kv, n_buf_cap, d_h]; may be NULL when n_buf == 0.
 * n_buf     : 0..n_buf_cap; n_buf == 0 with an empty cache is GEAR_EINVAL.
 * out       : device fp16 [B, H_q, 1, d_h].
 * Value range: the products q[c] * scale_K(group, c) and p * scale_V (p <= 1) are fed to
 *             the matrix cores as fp16 numbers times at most 16, so finite outputs need
 *             |q[c] * scale_K| < 4094 and scale_V < 4094 for every entry (scale = (max - min)
 *             / (2^b - 1) of a group: K and V entries of magnitude up to ~1000 with |q| up to
 *             ~10 are inside).  Inputs beyond that are not detected: the outputs of the heads
 *             concerned are then inf or NaN and the call still returns GEAR_OK.
 */
int gear_decode_attn(const gear_cache* cache, const void* q, const void* K_buf, const void* V_buf,
                     int32_t n_buf, void* out, void* workspace, size_t workspace_bytes,
                     void* stream);

/*
 * The same read for q_len query rows per head (chunked prefill, speculative decoding): the
 * packed codes are unpacked once and feed all rows' products.  The q_len newest tokens are the
 * last q_len of the n_buf buffer rows.  Every query attends to the whole compressed cache;
 * with causal != 0 query row j (0-based) attends to the buffer rows 0 .. n_buf - q_len + j
 * (Eq. 1 with the usual causal mask among the new tokens), otherwise to all n_buf rows.
 * q, out    : device fp16 [B, H_q, q_len, d_h].
 * q_len     : a power of two with q_len * (H_q / H_kv) <= 8 (longer blocks: several calls);
 *             causal needs n_buf >= q_len.  Otherwise GEAR_EINVAL.
 * workspace : the workspace of gear_cache_bytes; GEAR_ECAPACITY if the records of q_len rows do
 *             not fit into it (they do whenever rank_max > 0 and n_prefill_max > 256; behind a
 *             shorter prompt it depends on the number of appended segments).
 */
int gear_decode_attn_mq(const gear_cache* cache, const void* q, int32_t q_len, int32_t causal,
                        const void* K_buf, const void* V_buf, int32_t n_buf, void* out,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * gear_decode_attn for callers that cannot allocate device memory or bring a
 * workspace along: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same computation, same kernels and same results as
 * gear_decode_attn; the partial softmax records of the split blocks go to a
 * fixed array of GEAR_STATIC_SCRATCH_BYTES (32 MiB) that is part of the library
 * and that every GPU the library runs on holds until the process ends.  The call
 * allocates and frees nothing.
 *  - The records take B * H_q * (ceil(n_prefill / 512) + ceil(pieces / 4) + 1) * 520
 *    bytes (pieces = n_chunks, or 2 * n_chunks when n_buf_cap > 128); a cache
 *    that needs more than the array returns GEAR_ECAPACITY and launches nothing.
 *  - All calls on one GPU share that GPU's array: two calls that may overlap on
 *    one GPU (different streams, different threads) race and must be ordered
 *    by the caller.  Nothing has to be cleared between calls: every record a
 *    call reads it has written itself.
 */
int gear_decode_attn_static(const gear_cache* cache, const void* q, const void* K_buf, const void* V_buf,
                            int32_t n_buf, void* out, void* stream);

/*
 * Canonical views of the stored components (the physical arena layout is
 * private); used to check the library against an independent implementation.
 * which: 0 = Keys, 1 = Values.
 *  codes_u8 : device u8  [B, H_kv, n_total, d_h], one integer code per entry.
 *  scale/zero: device fp16; Keys [B, H_kv, NG, d_h] with NG = sum over segments
 *             of ceil(n_seg / g) (segments in append order); Values
 *             [B, H_kv, n_total, d_h / g].
 *  mask_u8  : device u8  [B, H_kv, n_total, d_h], 1 on the support of S.
 *  values   : device fp16 same shape, S itself (0 off the support).
 *  A_f16    : device fp16 [B, H_kv, n_seg, rank_seg]; B_f16: [B, H_kv, d_h, rank_seg].
 */
int gear_export_codes(const gear_cache* cache, int which, void* codes_u8, void* scale_f16,
                      void* zero_f16, void* stream);
int gear_export_sparse(const gear_cache* cache, int which, void* mask_u8, void* values_f16,
                       void* stream);
int gear_export_lowrank(const gear_cache* cache, int which, int seg, void* A_f16, void* B_f16,
                        void* stream);

/*
 * The sparse matrix S of Filter_s (Eq. 4) in the coordinate form the paper's Sec. 3.1
 * describes (index vectors plus one value vector), over all stored segments:
 *  nnz           : host, out.  Fixed by Eq. 4: every Key channel of a segment of n tokens
 *                  holds ceil(s n) entries, every Value token ceil(s H_kv d_h); the call
 *                  computes it on the host, so a first call with lin_index_i64 ==
 *                  value_f16 == NULL (nothing launched) tells the caller what to allocate.
 *  lin_index_i64 : device int64 [nnz], the linear index ((b * H_kv + h) * n_total + t) * d_h + c
 *                  of every entry, ascending (the two index vectors of the coordinate
 *                  form are index / d_h and index % d_h).
 *  value_f16     : device fp16 [nnz], the entries (bit copies of the input) in the same order.
 *  workspace     : device scratch, >= 4 * B * H_kv * n_total + 4 * ceil(B * H_kv * n_total / 1024)
 *                  + 512 bytes (the workspace of gear_cache_bytes is large enough); GEAR_ECAPACITY
 *                  otherwise.
 */
int gear_export_sparse_coo(const gear_cache* cache, int which, int64_t* nnz, void* lin_index_i64,
                           void* value_f16, void* workspace, size_t workspace_bytes, void* stream);

/*
 * ---- Paged cache --------------------------------------------------------------------------------
 * K and V of one layer in fixed-size pages that sequences take as they grow: rows are written (and
 * quantized) as they arrive, one token at a time or a whole prompt, and attention reads them through a
 * page table.  It is the cache a prompt is prefilled with, chunk by chunk, before gear_compress takes
 * its rows, the one a decompressed session continues in, and, with codes of 8 or 4 bits, the per-token
 * grouping (one group = g channels of one token, for Keys and Values alike) that needs no buffer.
 *
 * Pool layout (public: a page can be copied, shared or sent as bytes).  Page p starts at p * page_bytes;
 * inside it KV head h's Keys at 2 h * block_bytes and Values at (2 h + 1) * block_bytes.  A block holds
 * page_size rows of 16 bits (a row's 128 values as they are), or of b-bit codes (16 b bytes per row):
 *   8 bits: byte c of the row is channel c's code;
 *   4 bits: channel 8 w + e is word w's bits 4 (e / 2) + 16 (e % 2) and the three above;
 * and behind the code rows (scale, zero) words u32 [128 / group][page_size], scale in the low half, both
 * of the cache's type.  A code stands for the value  scale * code + zero,  rounded to fp16 once, or to fp32 and then to bf16, with
 *   zero = min x,  scale = (max x - min x) / (2^b - 1) rounded to the cache's type (the quotient in fp32),
 *   code = the integer nearest to (x - zero) / scale, halves to even, at most 2^b - 1; 0 where scale is 0.  The difference x - zero is
 *   rounded to fp32 first: where one of the two is so small beside the other (below 2^-12 of it in fp16, 2^-15 in bf16) that fp32 does
 *   not hold it, and what it is rounded to is an odd half of the scale, the code is the even one of two that are all but equally near,
 * over the group's entries x (Eq. 2).  Slot i is row i % page_size of page i / page_size.
 */
typedef enum gear_dtype { GEAR_F16 = 0, GEAR_BF16 = 1 } gear_dtype;

typedef struct gear_page_config {
  int32_t n_pages;    /* pages of the pool, >= 1                                            */
  int32_t page_size;  /* tokens per page: 16, 32, 64, 128 or 256                            */
  int32_t H_kv;       /* KV heads, 1..1024                                                  */
  int32_t d_h;        /* head dimension, must be 128                                        */
  int32_t bits;       /* 16 (stored as they are), 8 or 4                                    */
  int32_t group;      /* g in {32, 64, 128} channels per (scale, zero); not used at 16 bits */
  int32_t dtype;      /* gear_dtype of rows, queries and outputs                            */
} gear_page_config;

/* 16-bit values [n_seqs][tokens][heads][128], the 128 contiguous; strides in elements.  Rows that a call writes must not overlap
 * (GEAR_EINVAL where two sequences, tokens or heads in a row do, or two strides are the same); rows that it reads may. */
typedef struct gear_page_rows {
  void*   data;       /* device, 16-byte aligned; strides multiples of 8 */
  int64_t seq;
  int64_t token;
  int64_t head;
} gear_page_rows;

/* Which tokens a call of gear_page_attn is about.  The lengths are read on the device, so a captured
 * call follows them; the int fields bound them and size the launch. */
typedef struct gear_page_batch {
  int32_t n_seqs;
  int32_t n_tokens;             /* rows of q and out (those outside every sequence are not touched)   */
  int32_t max_q;                /* no sequence has more new tokens (the rows of one that has may stay)  */
  int32_t max_kv;               /* about the longest sequence: what the work is divided by            */
  int32_t table_width;          /* entries of a sequence's row of page_table                          */
  int32_t causal;               /* 0: every row sees all kv_len tokens                                */
  const int32_t* q_start;       /* device [n_seqs + 1], ascending: sequence s has rows q_start[s] ..   */
  const int32_t* kv_len;        /* device [n_seqs]: tokens in the cache, the new ones included         */
  const int32_t* page_table;    /* device [n_seqs][table_width]: tokens page_size i .. are in page [i] */
} gear_page_batch;

/* Bytes of a pool.  GEAR_ECAPACITY if a page has 2 GiB or more. */
int gear_page_bytes(const gear_page_config* cfg, size_t* pool_bytes);

/*
 * Writes row (s, t, h) of K and V into slot slots[s * n_rows + t] of head h, for all s < n_seqs, t < n_rows.
 * slots     : device int64.  A slot outside 0 .. n_pages * page_size - 1 (-1: padding) is skipped.  A slot
 *             should be named once: of one that is named twice the bytes may come from either row.
 * Values must be finite and, where they are quantized, below 2^16 - 128 (fp16; a code of one beyond may stand
 * for an infinity) or 2^100 (bf16) in magnitude.
 */
int gear_page_write(const gear_page_config* cfg, void* pool, size_t pool_bytes, const gear_page_rows* K,
                    const gear_page_rows* V, int32_t n_seqs, int32_t n_rows, const int64_t* slots, void* stream);

/* The reverse: the values that slot slots[s * n_rows + t] stands for into row (s, t, h) of K and V (either may
 * be NULL).  Rows whose slot is outside the pool are left as they are.  With seq, token and head strides
 * of a [B, H_kv, n, 128] tensor the rows come as gear_compress takes them. */
int gear_page_read(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_rows* K,
                   const gear_page_rows* V, int32_t n_seqs, int32_t n_rows, const int64_t* slots, void* stream);

/* Workspace of gear_page_attn for H_q query heads and every batch with at most these n_seqs, n_tokens, max_q and
 * max_kv (0 where no axis is divided).  Only the int fields of `batch` are read. */
int gear_page_attn_bytes(const gear_page_config* cfg, int32_t H_q, const gear_page_batch* batch, size_t* workspace_bytes);

/*
 * Attention of each sequence's new tokens over its pages, which hold them already: with n = q_start[s + 1] -
 * q_start[s], row i (0-based) of sequence s is its token kv_len[s] - n + i and sees the tokens up to and with
 * itself (causal) or all kv_len[s]:
 *     out = softmax(scale * q K^T) V  over the values the pages' rows stand for;
 * query head j reads KV head j / (H_q / H_kv).  Any mix of single tokens, a few rows and whole chunks.  A row that
 * sees nothing is 0.  Scores, softmax statistics and sums are held in fp32; the weights are rounded to the
 * cache's type for the product with V (fp16: by half a step of 2^-10 of each down to 2^-21 of a row's greatest, by 2^-32 of that below).  A Value that is not finite makes NaN of rows of its sequence that are masked from it, too
 * (their weight for it is 0); what lies in slots past kv_len does not matter.
 * q, out    : rows [n_tokens][H_q][128] (seq strides not used), dtype of cfg.
 * H_q       : a multiple of H_kv.
 * page_table: entries outside 0 .. n_pages - 1 are not followed: their tokens are not seen.  kv_len is
 *             taken as table_width * page_size where it is more.
 * workspace : device, >= the bytes of gear_page_attn_bytes, 16-byte aligned; NULL where those are 0.  Nothing in
 *             it need survive, but calls that may run at the same time need one each.
 */
int gear_page_attn(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_batch* batch,
                   const gear_page_rows* q, int32_t H_q, float scale, const gear_page_rows* out, void* workspace,
                   size_t workspace_bytes, void* stream);

/*
 * ---- Rotary positions ---------------------------------------------------------------------------
 * Channels 0 .. rot_dim - 1 of a row at position t are turned pair by pair, the others stay as they are:
 *     y_a = f (x_a cos(t w_p) - x_b sin(t w_p)),   y_b = f (x_a sin(t w_p) + x_b cos(t w_p)),
 * pair p < rot_dim / 2 being channels a = p, b = p + rot_dim / 2, or a = 2 p, b = 2 p + 1 (interleaved).  Angles are formed and
 * reduced in 64 bits (|t w_p| below 2^31: the cosine and sine are off by less than 2^-20, and 2^-22 below 2^24), the turn is fp32, rounded once.
 */
typedef struct gear_rope {
  int32_t rot_dim;       /* even, 2..128                                                          */
  int32_t interleaved;   /* which channels are a pair: 0 or 1                                     */
  int32_t inverse;       /* 1: by -t w_p, which takes a turn back (and, times f, is its gradient) */
  float factor;          /* f, finite; 1 in the plain form                                        */
  const double* freq;    /* device [rot_dim / 2]: w_p in radians per position                     */
} gear_rope;

/* How the frequencies base^(-2 p / rot_dim) are brought to longer contexts. */
typedef enum gear_rope_scaling {
  GEAR_ROPE_PLAIN = 0,    /* not at all                                                                                */
  GEAR_ROPE_LINEAR = 1,   /* w / scale (positions interpolated)                                                        */
  GEAR_ROPE_BASE = 2,     /* base * scale^(rot_dim / (rot_dim - 2)) in place of base: the slowest pair is w / scale    */
  GEAR_ROPE_TURNS = 3     /* by the turns u = trained_len * w / (2 pi) a pair makes over the trained length: w / scale  */
                          /* up to `low` turns, w from `high` on, and w (k + (1 - k) / scale), k = (u - low) / (high - low) */
                          /* between (the ramp in the paper on YaRN, whose f is 0.1 ln(scale) + 1; models whose ramp goes by the number of the */
                          /* pair, between rounded bounds, have other frequencies: any may be given to gear_rope)             */
} gear_rope_scaling;

/* Fills host freq [rot_dim / 2].  base and scale are above 0; trained_len, low and high (0 <= low < high) count for GEAR_ROPE_TURNS only. */
int gear_rope_freq(int scaling, int32_t rot_dim, double base, double scale, double trained_len, double low, double high, double* freq);

/* Turns rows [n_seqs][n_rows][heads][128] of x into out; row (s, t) stands at positions[s * n_rows + t].
 * dtype     : a gear_dtype.
 * out       : the same rows as x (in place), or rows that do not overlap them.
 * positions : device int64, any sign. */
int gear_rotate(const gear_rope* rope, int dtype, const gear_page_rows* x, const gear_page_rows* out, int32_t n_seqs, int32_t n_rows,
                int32_t heads, const int64_t* positions, void* stream);

/* A step's rows into the cache in one launch: gear_rotate of q (H_q heads, into q_out) and K, rounded to the cache's type, and gear_page_write of
 * the turned K and of V, bit for bit.  Queries are turned whatever their row's slot is.
 * q, q_out  : NULL both (and H_q 0) where only K and V are given; in place as in gear_rotate. */
int gear_page_write_rope(const gear_page_config* cfg, void* pool, size_t pool_bytes, const gear_rope* rope, const gear_page_rows* K,
                         const gear_page_rows* V, const gear_page_rows* q, const gear_page_rows* q_out, int32_t H_q, int32_t n_seqs,
                         int32_t n_rows, const int64_t* slots, const int64_t* positions, void* stream);

/*
 * ---- Page tables --------------------------------------------------------------------------------
 * Which pages a sequence has, kept on the device: a step that takes pages, forks sequences or drops tokens needs no host in between and can be
 * captured.  One table serves all layers, whose pools have the same pages.  A table begins with every entry -1 and every kv_len and count
 * 0, and is changed by these calls only; then refs[p] is the number of entries that name page p, and entries from ceil(kv_len / page_size) on
 * are -1.  Results do not depend on the order in which the device works: pages are taken lowest number first, in the order of the list.
 * Rows outside 0 .. n_rows - 1 in a list are passed over.  The calls on one table must be ordered on one stream.
 */
typedef struct gear_page_table {
  int32_t n_pages;     /* pages of a pool, 1 .. 2^20                       */
  int32_t page_size;   /* tokens per page: 16, 32, 64, 128 or 256          */
  int32_t n_rows;      /* sequences, 1 .. 2^18                             */
  int32_t width;       /* entries of a row, width * page_size below 2^31   */
  int32_t* table;      /* device [n_rows][width]                           */
  int32_t* kv_len;     /* device [n_rows]                                  */
  int32_t* refs;       /* device [n_pages], 16-byte aligned                */
} gear_page_table;

#define GEAR_PAGE_LIST_MAX 1024   /* entries of a list of rows */

/*
 * Room for counts[i] more tokens of row rows[i], i = 0 .. n - 1 one after the other: pages are taken for them, and where the first of them
 * goes into a partly filled page that other entries name, too, the row gets a page of its own in its place.
 * max_count : columns of slots; a row that asks for more is refused.
 * slots     : device int64 [n][max_count]: the new tokens' slots, as gear_page_write takes them; -1 behind a row's last.
 * copies    : device int32 [n][2]: (page, the page in its place), as gear_page_move takes them, or (-1, -1).
 * refused   : device int32 [n]: 0; 1 where the row is none, is named before in the list, has no room in its width, or the count is
 *             negative or above max_count; 2 where too few pages are free for it (what those before it asked for counts as taken), or
 *             where it would have had a shared page to itself if one before it had not been refused a page in its place.  A refused row is left as
 *             it is, its slots are -1.
 */
int gear_page_extend(const gear_page_table* t, const int32_t* rows, const int32_t* counts, int32_t n, int32_t max_count, int64_t* slots,
                     int32_t* copies, int32_t* refused, void* stream);

/* Row rows[i] keeps its first lens[i] tokens (0: the row is freed); pages that no entry names any more are free.  A row that has fewer is left
 * as it is; one that is named twice keeps the fewer. */
int gear_page_truncate(const gear_page_table* t, const int32_t* rows, const int32_t* lens, int32_t n, void* stream);

/* Row dst[i] becomes what row src[i] was before the call, i = 0 .. n - 1: parallel samples of a prompt, beams in another order.  What dst[i]
 * held is dropped.  A row that is named twice in dst gets the first of its sources. */
int gear_page_fork(const gear_page_table* t, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

/* The highest pages in use change to the lowest free numbers, until those in use are the first ones or max_moves have moved.
 * moves  : device int32 [max_moves][2]: (from, to) for gear_page_move, from falling, to rising; (-1, -1) behind the last.
 * counts : device int32 [2]: pages in use, moves. */
int gear_page_compact(const gear_page_table* t, int32_t* moves, int32_t max_moves, int32_t* counts, void* stream);

/* Copies page pairs[i][0] over page pairs[i][1] in each of n_pools pools, which lie pool_stride bytes (a multiple of 16) apart.  Pairs with a page
 * outside 0 .. n_pages - 1 are passed over.  A page that is written should be written once and not be read by another pair: of one that
 * is, the bytes may come from either, or be those of before or after.
 * pool_bytes : from `pool` to the end of the last. */
int gear_page_move(const gear_page_config* cfg, void* pool, size_t pool_bytes, int32_t n_pools, size_t pool_stride, const int32_t* pairs,
                   int32_t n, void* stream);

/*
 * ---- Attention with shared prefixes -------------------------------------------------------------
 * gear_page_attn for a batch whose sequences share their first tokens in groups: samples of one prompt, requests behind one system
 * prompt, questions about one document.  The shared tokens' pages are read once for all new tokens of a group, instead of once for each sequence, and the two
 * parts of a row's softmax are joined.  The same batch, and up to the order of sums the same result, as gear_page_attn.
 */
typedef struct gear_page_groups {
  int32_t n_groups;             /* up to 2^20                                                          */
  int32_t max_q;                /* no group has more rows of q (one that has may share nothing; its rows are right) */
  int32_t max_prefix;           /* about the longest prefix: what the work is divided by               */
  int32_t always;               /* 0: prefixes are shared where that is estimated to be faster, else the call is gear_page_attn's (rows of q beyond */
                                /* n_groups * max_q are taken to be those of sequences in no group, of up to max_kv tokens);                       */
                                /* 1: always (but where a workspace of 512 MB would not do)            */
  const int32_t* group_start;   /* device [n_groups + 1], ascending: group i has sequences group_start[i] .. */
  const int32_t* prefix_len;    /* device [n_groups]: the first tokens that are the same in all of them; they are read through the row
                                 * of the page table of the group's first sequence that has new tokens.  Where the sequences part within a page, each may have its own copy. */
} gear_page_groups;

/* Workspace of gear_page_attn_shared for H_q query heads and every batch and groups with at most these n_seqs, n_tokens, max_q and max_kv, n_groups, max_q and
 * max_prefix (it serves gear_page_attn for them, too).  Only the int fields are read. */
int gear_page_attn_shared_bytes(const gear_page_config* cfg, int32_t H_q, const gear_page_batch* batch, const gear_page_groups* groups,
                                size_t* workspace_bytes);

/* Sequences outside every group share nothing.  A prefix counts as far as all rows of its group's new tokens see it.  The other arguments are
 * those of gear_page_attn. */
int gear_page_attn_shared(const gear_page_config* cfg, const void* pool, size_t pool_bytes, const gear_page_batch* batch,
                          const gear_page_groups* groups, const gear_page_rows* q, int32_t H_q, float scale, const gear_page_rows* out,
                          void* workspace, size_t workspace_bytes, void* stream);

const char* gear_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* GEAR_H */
