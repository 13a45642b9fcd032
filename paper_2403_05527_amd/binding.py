"""ctypes binding of libgear (include/gear.h).  Argument marshalling only: every
step of the path runs in the HIP library; torch supplies device memory and the
current stream.  There is no CPU fallback: a missing library is an error."""
import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgear.so")

GEAR_MAX_CHUNKS = 256
GEAR_STATIC_SCRATCH_BYTES = 32 << 20
GEAR_OK, GEAR_EINVAL, GEAR_ECAPACITY, GEAR_EALIGN, GEAR_EHIP = 0, -1, -2, -3, -4

EXPORTED = [
    "gear_cache_bytes", "gear_cache_init", "gear_cache_reset", "gear_compress", "gear_compress_recent", "gear_decompress",
    "gear_decode_attn", "gear_decode_attn_mq", "gear_decode_attn_static", "gear_export_codes", "gear_export_sparse", "gear_export_sparse_coo", "gear_export_lowrank", "gear_strerror",
    "gear_page_bytes", "gear_page_write", "gear_page_read", "gear_page_attn_bytes", "gear_page_attn",
    "gear_rope_freq", "gear_rotate", "gear_page_write_rope",
    "gear_page_extend", "gear_page_truncate", "gear_page_fork", "gear_page_compact", "gear_page_move",
    "gear_page_attn_shared_bytes", "gear_page_attn_shared",
]


class gear_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "B", "H_kv", "H_q", "d_h", "bits", "group", "outlier_ppm", "n_buf_cap", "n_prefill_max",
        "n_chunks_max", "rank_max", "flags")]


class gear_cache(ctypes.Structure):
    _fields_ = [
        ("cfg", gear_config),
        ("arena", ctypes.c_void_p),
        ("arena_bytes", ctypes.c_uint64),
        ("n_prefill", ctypes.c_int32),
        ("rank_prefill", ctypes.c_int32),
        ("n_chunks", ctypes.c_int32),
        ("n_total", ctypes.c_int32),
        ("chunk_n", ctypes.c_uint8 * GEAR_MAX_CHUNKS),
        ("chunk_rank", ctypes.c_uint8 * GEAR_MAX_CHUNKS),
    ]


class gear_page_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "H_kv", "d_h", "bits", "group", "dtype")]


class gear_page_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class gear_page_batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_tokens", "max_q", "max_kv", "table_width", "causal")] + \
               [(n, ctypes.c_void_p) for n in ("q_start", "kv_len", "page_table")]


class gear_rope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rot_dim", "interleaved", "inverse")] + [("factor", ctypes.c_float), ("freq", ctypes.c_void_p)]


class gear_page_table(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_rows", "width")] + [(n, ctypes.c_void_p) for n in ("table", "kv_len", "refs")]


class gear_page_groups(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_groups", "max_q", "max_prefix", "always")] + [(n, ctypes.c_void_p) for n in ("group_start", "prefix_len")]


GEAR_PAGE_LIST_MAX = 1024
GEAR_ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "turns": 3}
GEAR_DTYPES = {torch.float16: 0, torch.bfloat16: 1}


class GearError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (what, strerror(status), status))


_lib = None


def load_library():
    """Loads libgear.so built in-tree (python -m paper_2403_05527_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libgear.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp, cachep = ctypes.POINTER(gear_config), ctypes.POINTER(gear_cache)
    lib.gear_cache_bytes.argtypes = [cfgp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.gear_cache_init.argtypes = [cfgp, vp, sz, cachep]
    lib.gear_cache_reset.argtypes = [cachep]
    lib.gear_compress.argtypes = [cachep, vp, vp, i32, i32, i32, vp, ctypes.c_uint64, vp, sz, vp]
    lib.gear_compress_recent.argtypes = [cachep, vp, vp, i32, i32, i32, vp, ctypes.c_uint64, i32, vp, sz, vp]
    lib.gear_decompress.argtypes = [cachep, vp, vp, vp]
    lib.gear_decode_attn.argtypes = [cachep, vp, vp, vp, i32, vp, vp, sz, vp]
    lib.gear_decode_attn_mq.argtypes = [cachep, vp, i32, i32, vp, vp, i32, vp, vp, sz, vp]
    lib.gear_decode_attn_static.argtypes = [cachep, vp, vp, vp, i32, vp, vp]
    lib.gear_export_codes.argtypes = [cachep, ctypes.c_int, vp, vp, vp, vp]
    lib.gear_export_sparse.argtypes = [cachep, ctypes.c_int, vp, vp, vp]
    lib.gear_export_sparse_coo.argtypes = [cachep, ctypes.c_int, ctypes.POINTER(ctypes.c_int64), vp, vp, vp, sz, vp]
    lib.gear_export_lowrank.argtypes = [cachep, ctypes.c_int, ctypes.c_int, vp, vp, vp]
    pcfg, rows, batch = (ctypes.POINTER(t) for t in (gear_page_config, gear_page_rows, gear_page_batch))
    lib.gear_page_bytes.argtypes = [pcfg, ctypes.POINTER(sz)]
    lib.gear_page_write.argtypes = [pcfg, vp, sz, rows, rows, i32, i32, vp, vp]
    lib.gear_page_read.argtypes = [pcfg, vp, sz, rows, rows, i32, i32, vp, vp]
    lib.gear_page_attn_bytes.argtypes = [pcfg, i32, batch, ctypes.POINTER(sz)]
    lib.gear_page_attn.argtypes = [pcfg, vp, sz, batch, rows, i32, ctypes.c_float, rows, vp, sz, vp]
    rope, table, groups, f64 = ctypes.POINTER(gear_rope), ctypes.POINTER(gear_page_table), ctypes.POINTER(gear_page_groups), ctypes.c_double
    lib.gear_rope_freq.argtypes = [ctypes.c_int, i32, f64, f64, f64, f64, f64, ctypes.POINTER(f64)]
    lib.gear_rotate.argtypes = [rope, ctypes.c_int, rows, rows, i32, i32, i32, vp, vp]
    lib.gear_page_write_rope.argtypes = [pcfg, vp, sz, rope, rows, rows, rows, rows, i32, i32, i32, vp, vp, vp]
    lib.gear_page_extend.argtypes = [table, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.gear_page_truncate.argtypes = [table, vp, vp, i32, vp]
    lib.gear_page_fork.argtypes = [table, vp, vp, i32, vp]
    lib.gear_page_compact.argtypes = [table, vp, i32, vp, vp]
    lib.gear_page_move.argtypes = [pcfg, vp, sz, i32, sz, vp, i32, vp]
    lib.gear_page_attn_shared_bytes.argtypes = [pcfg, i32, batch, groups, ctypes.POINTER(sz)]
    lib.gear_page_attn_shared.argtypes = [pcfg, vp, sz, batch, groups, rows, i32, ctypes.c_float, rows, vp, sz, vp]
    lib.gear_strerror.argtypes = [ctypes.c_int]
    lib.gear_strerror.restype = ctypes.c_char_p
    for name in EXPORTED:
        if name != "gear_strerror":
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(status):
    return load_library().gear_strerror(int(status)).decode()


def _check(status, what):
    if status != GEAR_OK:
        raise GearError(status, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


# The handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object for it, 2.7 us of the 10 that a
# read's call took on the host (the kernel of a small read takes 8); torch's own generated code asks for the handle alone.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _bytes(t):
    return t.numel() * t.element_size()


GEAR_FLAG_V_FILTER_PER_HEAD = 1


def make_config(B, H_kv, H_q, bits, group, outlier_ppm, n_buf_cap, n_prefill_max, n_chunks_max, rank_max,
                d_h=128, flags=0):
    return gear_config(B, H_kv, H_q, d_h, bits, group, outlier_ppm, n_buf_cap, n_prefill_max, n_chunks_max,
                       rank_max, flags)


# ---- thin wrappers with the C names ---------------------------------------
def gear_cache_bytes(cfg):
    a, w = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().gear_cache_bytes(ctypes.byref(cfg), ctypes.byref(a), ctypes.byref(w)), "gear_cache_bytes")
    return a.value, w.value


def gear_cache_init(cfg, arena):
    cache = gear_cache()
    _check(load_library().gear_cache_init(ctypes.byref(cfg), _ptr(arena), _bytes(arena),
                                          ctypes.byref(cache)), "gear_cache_init")
    return cache


def gear_cache_reset(cache):
    _check(load_library().gear_cache_reset(ctypes.byref(cache)), "gear_cache_reset")


def gear_compress(cache, K, V, rank, iters, init_B, workspace, seed=0):
    n = K.shape[2]
    _check(load_library().gear_compress(ctypes.byref(cache), _ptr(K), _ptr(V), n, rank, iters, _ptr(init_B),
                                        seed, _ptr(workspace), _bytes(workspace), _stream()),
           "gear_compress")


def gear_compress_recent(cache, K, V, rank, iters, init_B, n_lowrank, workspace, seed=0):
    n = K.shape[2]
    _check(load_library().gear_compress_recent(ctypes.byref(cache), _ptr(K), _ptr(V), n, rank, iters, _ptr(init_B),
                                               seed, n_lowrank, _ptr(workspace),
                                               _bytes(workspace), _stream()),
           "gear_compress_recent")


def gear_decompress(cache, K_out, V_out):
    _check(load_library().gear_decompress(ctypes.byref(cache), _ptr(K_out), _ptr(V_out), _stream()),
           "gear_decompress")


def gear_decode_attn(cache, q, K_buf, V_buf, n_buf, out, workspace):
    _check(load_library().gear_decode_attn(ctypes.byref(cache), _ptr(q), _ptr(K_buf), _ptr(V_buf), n_buf, _ptr(out),
                                           _ptr(workspace), _bytes(workspace), _stream()),
           "gear_decode_attn")


def gear_decode_attn_mq(cache, q, causal, K_buf, V_buf, n_buf, out, workspace):
    _check(load_library().gear_decode_attn_mq(ctypes.byref(cache), _ptr(q), q.shape[2], 1 if causal else 0, _ptr(K_buf),
                                              _ptr(V_buf), n_buf, _ptr(out), _ptr(workspace),
                                              _bytes(workspace), _stream()),
           "gear_decode_attn_mq")


def gear_decode_attn_static(cache, q, K_buf, V_buf, n_buf, out):
    _check(load_library().gear_decode_attn_static(ctypes.byref(cache), _ptr(q), _ptr(K_buf), _ptr(V_buf), n_buf,
                                                  _ptr(out), _stream()), "gear_decode_attn_static")


def gear_export_codes(cache, which, codes, scale, zero):
    _check(load_library().gear_export_codes(ctypes.byref(cache), which, _ptr(codes), _ptr(scale), _ptr(zero),
                                            _stream()), "gear_export_codes")


def gear_export_sparse(cache, which, mask, values):
    _check(load_library().gear_export_sparse(ctypes.byref(cache), which, _ptr(mask), _ptr(values), _stream()),
           "gear_export_sparse")


def gear_export_sparse_coo(cache, which, lin_index, values, workspace):
    """Returns nnz; with lin_index = values = None only the count is computed (nothing is launched)."""
    nnz = ctypes.c_int64(0)
    wb = 0 if workspace is None else _bytes(workspace)
    _check(load_library().gear_export_sparse_coo(ctypes.byref(cache), which, ctypes.byref(nnz), _ptr(lin_index),
                                                 _ptr(values), _ptr(workspace), wb, _stream()), "gear_export_sparse_coo")
    return nnz.value


def gear_export_lowrank(cache, which, seg, A, Bf):
    _check(load_library().gear_export_lowrank(ctypes.byref(cache), which, seg, _ptr(A), _ptr(Bf), _stream()),
           "gear_export_lowrank")


# ---- the paged cache: rows are tensors [n_seqs, tokens, heads, 128] (or [tokens, heads, 128]) of the pool's type, of any
# strides that the C ABI takes; a view of [n_seqs, heads, tokens, 128] is x.transpose(1, 2).  What is about to be read as
# something that it is not (another type, device or shape) is refused here, with ValueError, since the library sees pointers only.
def make_page_config(n_pages, page_size, H_kv, bits, group=128, dtype=torch.float16, d_h=128):
    return gear_page_config(n_pages, page_size, H_kv, d_h, bits, group, GEAR_DTYPES[dtype])


def _page_device():
    """The current GPU's index; where none is in use yet, one that no tensor lies on."""
    if not torch.cuda.is_initialized():
        return -2
    return torch.cuda.current_device() if _device is None else _device()


# (One pass over what a call is given, 1 us a tensor: a decode step's kernels take 6 to 10.)
def _page_rows(t, cfg, heads, device, what):
    """(the view, sequences, tokens) of a tensor of rows."""
    shape, stride = t.shape, t.stride()
    n = len(shape)
    if n not in (3, 4) or shape[-1] != cfg.d_h or shape[-2] != heads:
        raise ValueError("%s is [n_seqs, tokens, %d, %d] or without the first: got %s" % (what, heads, cfg.d_h, tuple(shape)))
    if GEAR_DTYPES.get(t.dtype) != cfg.dtype or stride[-1] != 1:
        raise ValueError("%s: another type than the pool's, or a row that is not contiguous" % what)
    if t.get_device() != device:
        raise ValueError("%s lies on %s, not on the current GPU" % (what, t.device))
    if n == 3:
        return gear_page_rows(t.data_ptr(), 0, stride[0], stride[1]), 1, shape[0]
    return gear_page_rows(t.data_ptr(), stride[0], stride[1], stride[2]), shape[0], shape[1]


def _page_index(t, dtype, n, device, what):
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s is a contiguous %s tensor of %d entries: got %s %s" % (what, dtype, n, t.dtype, tuple(t.shape)))
    if t.get_device() != device:
        raise ValueError("%s lies on %s, not on the current GPU" % (what, t.device))
    return t.data_ptr()


def _page_bytes(t, device, what):
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError("%s is one contiguous tensor on the current GPU: got one on %s" % (what, t.device))
    return t.data_ptr(), t.nbytes


def gear_page_bytes(cfg):
    n = ctypes.c_size_t(0)
    _check(load_library().gear_page_bytes(ctypes.byref(cfg), ctypes.byref(n)), "gear_page_bytes")
    return n.value


def _page_copy(name, cfg, pool, K, V, slots):
    device = _page_device()
    k = None if K is None else _page_rows(K, cfg, cfg.H_kv, device, "K")
    v = None if V is None else _page_rows(V, cfg, cfg.H_kv, device, "V")
    if k is None and v is None:
        raise ValueError("neither K nor V is given")
    if k and v and k[1:] != v[1:]:
        raise ValueError("K and V differ in their rows: %s and %s" % (tuple(K.shape), tuple(V.shape)))
    _, n_seqs, n_rows = k or v
    p, n = _page_bytes(pool, device, "the pool")
    _check(getattr(load_library(), name)(cfg, p, n, k and k[0], v and v[0], n_seqs, n_rows,
                                         _page_index(slots, torch.int64, n_seqs * n_rows, device, "slots"), _stream()), name)


def gear_page_write(cfg, pool, K, V, slots):
    _page_copy("gear_page_write", cfg, pool, K, V, slots)


def gear_page_read(cfg, pool, K_out, V_out, slots):
    _page_copy("gear_page_read", cfg, pool, K_out, V_out, slots)


def make_page_batch(q_start, kv_len, page_table, n_tokens, max_q, max_kv, causal=True):
    """The batch of a gear_page_attn call (one serves all layers of a step): int32 tensors q_start [n_seqs + 1], kv_len [n_seqs],
    page_table [n_seqs, width].  It keeps them alive."""
    n, width = page_table.shape
    d = _page_device()
    b = gear_page_batch(n, n_tokens, max_q, max_kv, width, 1 if causal else 0, _page_index(q_start, torch.int32, n + 1, d, "q_start"),
                        _page_index(kv_len, torch.int32, n, d, "kv_len"), _page_index(page_table, torch.int32, n * width, d, "page_table"))
    b.tensors, b.device = (q_start, kv_len, page_table), d
    return b


def gear_page_attn_bytes(cfg, H_q, batch):
    n = ctypes.c_size_t(0)
    _check(load_library().gear_page_attn_bytes(ctypes.byref(cfg), H_q, ctypes.byref(batch), ctypes.byref(n)), "gear_page_attn_bytes")
    return n.value


def _attn_arguments(cfg, pool, batch, q, out, workspace):
    device = _page_device()
    if getattr(batch, "device", device) != device:
        raise ValueError("the batch's lengths and page table lie on cuda:%d, not on the current GPU" % batch.device)
    H_q = q.shape[-2]
    a, seqs, n = _page_rows(q, cfg, H_q, device, "q")
    b, seqs_out, n_out = _page_rows(out, cfg, H_q, device, "out")
    if not seqs * n == seqs_out * n_out == n == n_out == batch.n_tokens:
        raise ValueError("q and out are [%d, H_q, %d]: got %s and %s" % (batch.n_tokens, cfg.d_h, tuple(q.shape), tuple(out.shape)))
    p, size = _page_bytes(pool, device, "the pool")
    w, w_size = (None, 0) if workspace is None else _page_bytes(workspace, device, "the workspace")
    return p, size, a, b, H_q, w, w_size


def gear_page_attn(cfg, pool, batch, q, out, scale, workspace):
    p, size, a, b, H_q, w, w_size = _attn_arguments(cfg, pool, batch, q, out, workspace)
    _check(load_library().gear_page_attn(cfg, p, size, batch, a, H_q, scale, b, w, w_size, _stream()), "gear_page_attn")


# ---- rotary positions
class _RowsOf(ctypes.Structure):   # what _page_rows asks of a configuration
    _fields_ = [("d_h", ctypes.c_int32), ("dtype", ctypes.c_int32)]


def gear_rope_freq(rot_dim=128, base=10000.0, scaling="plain", scale=1.0, trained_len=0.0, low=1.0, high=4.0):
    """The frequencies as a float64 tensor on the host, radians per position and pair."""
    freq = torch.empty(max(0, rot_dim // 2), dtype=torch.float64)
    _check(load_library().gear_rope_freq(GEAR_ROPE_SCALINGS[scaling], rot_dim, base, scale, trained_len, low, high,
                                         ctypes.cast(freq.data_ptr(), ctypes.POINTER(ctypes.c_double))), "gear_rope_freq")
    return freq


def make_rope(freq, interleaved=False, inverse=False, factor=1.0):
    """The rotation of one model's rows (one serves all layers): float64 frequencies on the GPU, which it keeps alive."""
    d = _page_device()
    r = gear_rope(2 * freq.numel(), 1 if interleaved else 0, 1 if inverse else 0, factor, _page_index(freq, torch.float64, freq.numel(), d, "freq"))
    r.tensors, r.device = freq, d
    return r


def _rope_device(rope, device):
    if getattr(rope, "device", device) != device:
        raise ValueError("the frequencies lie on cuda:%d, not on the current GPU" % rope.device)


def gear_rotate(rope, x, out, positions):
    """x, out: [n_seqs, tokens, heads, 128], or without the first; out may be x."""
    device = _page_device()
    _rope_device(rope, device)
    if x.dtype not in GEAR_DTYPES or x.shape != out.shape:
        raise ValueError("x and out are fp16 or bf16 rows of one shape: got %s %s and %s" % (x.dtype, tuple(x.shape), tuple(out.shape)))
    kind, heads = _RowsOf(128, GEAR_DTYPES[x.dtype]), x.shape[-2] if x.dim() > 1 else 0
    a, n_seqs, n_rows = _page_rows(x, kind, heads, device, "x")
    b = _page_rows(out, kind, heads, device, "out")[0]
    _check(load_library().gear_rotate(rope, kind.dtype, a, b, n_seqs, n_rows, heads,
                                      _page_index(positions, torch.int64, n_seqs * n_rows, device, "positions"), _stream()), "gear_rotate")


def gear_page_write_rope(cfg, pool, rope, K, V, slots, positions, q=None, q_out=None):
    """Rows as gear_page_write takes them, and a position for each; q_out may be q."""
    device = _page_device()
    _rope_device(rope, device)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    k, n_seqs, n_rows = _page_rows(K, cfg, cfg.H_kv, device, "K")
    v = _page_rows(V, cfg, cfg.H_kv, device, "V")
    if v[1:] != (n_seqs, n_rows):
        raise ValueError("K and V differ in their rows: %s and %s" % (tuple(K.shape), tuple(V.shape)))
    a = b = None
    H_q = 0
    if q is not None:
        H_q = q.shape[-2]
        a, b = _page_rows(q, cfg, H_q, device, "q"), _page_rows(q_out, cfg, H_q, device, "q_out")
        if not H_q or a[1:] != (n_seqs, n_rows) or b[1:] != (n_seqs, n_rows):
            raise ValueError("q, q_out and K differ in their rows: %s, %s and %s" % (tuple(q.shape), tuple(q_out.shape), tuple(K.shape)))
    p, size = _page_bytes(pool, device, "the pool")
    n = n_seqs * n_rows
    _check(load_library().gear_page_write_rope(cfg, p, size, rope, k, v[0], a and a[0], b and b[0], H_q, n_seqs, n_rows,
                                               _page_index(slots, torch.int64, n, device, "slots"),
                                               _page_index(positions, torch.int64, n, device, "positions"), _stream()), "gear_page_write_rope")


# ---- page tables
def make_page_table(table, kv_len, refs, page_size):
    """int32 tensors table [n_rows, width], kv_len [n_rows], refs [n_pages], which it keeps alive."""
    n_rows, width = table.shape
    d = _page_device()
    t = gear_page_table(refs.numel(), page_size, n_rows, width, _page_index(table, torch.int32, n_rows * width, d, "table"),
                        _page_index(kv_len, torch.int32, n_rows, d, "kv_len"), _page_index(refs, torch.int32, refs.numel(), d, "refs"))
    t.tensors, t.device = (table, kv_len, refs), d
    return t


def _table_device(t):
    device = _page_device()
    if getattr(t, "device", device) != device:
        raise ValueError("the page table lies on cuda:%d, not on the current GPU" % t.device)
    return device


def gear_page_extend(t, rows, counts, slots, copies, refused):
    """slots: int64 [n, max_count]; copies int32 [n, 2]; refused int32 [n]."""
    d, n, shape = _table_device(t), rows.numel(), slots.shape
    if len(shape) != 2 or shape[0] != n:
        raise ValueError("slots is [%d, max_count]: got %s" % (n, tuple(shape)))
    _check(load_library().gear_page_extend(t, _page_index(rows, torch.int32, n, d, "rows"), _page_index(counts, torch.int32, n, d, "counts"), n, shape[1],
                                           _page_index(slots, torch.int64, n * shape[1], d, "slots"), _page_index(copies, torch.int32, 2 * n, d, "copies"),
                                           _page_index(refused, torch.int32, n, d, "refused"), _stream()), "gear_page_extend")


def gear_page_truncate(t, rows, lens):
    d, n = _table_device(t), rows.numel()
    _check(load_library().gear_page_truncate(t, _page_index(rows, torch.int32, n, d, "rows"), _page_index(lens, torch.int32, n, d, "lens"), n, _stream()),
           "gear_page_truncate")


def gear_page_fork(t, src, dst):
    d, n = _table_device(t), src.numel()
    _check(load_library().gear_page_fork(t, _page_index(src, torch.int32, n, d, "src"), _page_index(dst, torch.int32, n, d, "dst"), n, _stream()), "gear_page_fork")


def gear_page_compact(t, moves, counts):
    """moves: int32 [max_moves, 2]; counts int32 [2]: pages in use, moves."""
    d = _table_device(t)
    if moves.dim() != 2 or moves.shape[1] != 2:
        raise ValueError("moves is [max_moves, 2]: got %s" % (tuple(moves.shape),))
    _check(load_library().gear_page_compact(t, _page_index(moves, torch.int32, moves.numel(), d, "moves"), moves.shape[0],
                                            _page_index(counts, torch.int32, 2, d, "counts"), _stream()), "gear_page_compact")


def gear_page_move(cfg, pool, pairs):
    """pool: the bytes of one pool, or [n_pools, bytes] with rows of one stride (a layer's pool each); pairs: int32 [n, 2]."""
    device = _page_device()
    if pool.get_device() != device or pool.dim() not in (1, 2) or pool.stride(-1) != 1:
        raise ValueError("the pool is contiguous bytes on the current GPU, or rows of them: got %s on %s" % (tuple(pool.shape), pool.device))
    if pairs.dim() != 2 or pairs.shape[1] != 2:
        raise ValueError("pairs is [n, 2]: got %s" % (tuple(pairs.shape),))
    es = pool.element_size()
    n_pools, stride = (1, 0) if pool.dim() == 1 else (pool.shape[0], pool.stride(0) * es)
    size = pool.shape[-1] * es + max(0, n_pools - 1) * stride
    _check(load_library().gear_page_move(cfg, pool.data_ptr(), size, n_pools, stride, _page_index(pairs, torch.int32, pairs.numel(), device, "pairs"),
                                         pairs.shape[0], _stream()), "gear_page_move")


# ---- attention with shared prefixes
def make_page_groups(group_start, prefix_len, max_q, max_prefix, always=False):
    """The groups of a batch: int32 tensors group_start [n_groups + 1], prefix_len [n_groups], which it keeps alive."""
    n = prefix_len.numel()
    d = _page_device()
    g = gear_page_groups(n, max_q, max_prefix, 1 if always else 0, _page_index(group_start, torch.int32, n + 1, d, "group_start"),
                         _page_index(prefix_len, torch.int32, n, d, "prefix_len"))
    g.tensors, g.device = (group_start, prefix_len), d
    return g


def gear_page_attn_shared_bytes(cfg, H_q, batch, groups):
    n = ctypes.c_size_t(0)
    _check(load_library().gear_page_attn_shared_bytes(ctypes.byref(cfg), H_q, ctypes.byref(batch), ctypes.byref(groups), ctypes.byref(n)),
           "gear_page_attn_shared_bytes")
    return n.value


def gear_page_attn_shared(cfg, pool, batch, groups, q, out, scale, workspace):
    p, size, a, b, H_q, w, w_size = _attn_arguments(cfg, pool, batch, q, out, workspace)
    if getattr(groups, "device", _page_device()) != _page_device():
        raise ValueError("the groups lie on cuda:%d, not on the current GPU" % groups.device)
    _check(load_library().gear_page_attn_shared(cfg, p, size, batch, groups, a, H_q, scale, b, w, w_size, _stream()), "gear_page_attn_shared")


# ---- convenience owner of the device buffers -------------------------------
class GearCache:
    """Allocates the arena and workspace with torch and forwards to the C ABI."""

    def __init__(self, cfg, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        a, w = gear_cache_bytes(cfg)
        self.arena_bytes, self.workspace_bytes = a, w
        self.arena = torch.empty(a, dtype=torch.uint8, device=self.device)
        self.workspace = torch.empty(w, dtype=torch.uint8, device=self.device)
        self.cache = gear_cache_init(cfg, self.arena)

    @property
    def n_total(self):
        return self.cache.n_total

    def n_groups_total(self):
        g = self.cfg.group
        if g == 0:                                  # per-vector groups: one Key group per segment
            return (1 if self.cache.n_prefill > 0 else 0) + self.cache.n_chunks
        ng = -(-self.cache.n_prefill // g)
        for j in range(self.cache.n_chunks):
            ng += -(-self.cache.chunk_n[j] // g)
        return ng

    def reset(self):
        gear_cache_reset(self.cache)

    def compress(self, K, V, rank, iters=3, init_B=None, seed=0, n_lowrank=None):
        if n_lowrank is None:
            gear_compress(self.cache, K, V, rank, iters, init_B, self.workspace, seed)
        else:
            gear_compress_recent(self.cache, K, V, rank, iters, init_B, n_lowrank, self.workspace, seed)

    def decompress(self):
        c = self.cfg
        shape = (c.B, c.H_kv, self.n_total, c.d_h)
        K = torch.empty(shape, dtype=torch.float16, device=self.device)
        V = torch.empty(shape, dtype=torch.float16, device=self.device)
        gear_decompress(self.cache, K, V)
        return K, V

    def decode_attn(self, q, K_buf=None, V_buf=None, n_buf=0, out=None):
        if out is None:
            out = torch.empty_like(q)
        gear_decode_attn(self.cache, q, K_buf, V_buf, n_buf, out, self.workspace)
        return out

    def decode_attn_mq(self, q, K_buf, V_buf, n_buf, causal=True, out=None):
        if out is None:
            out = torch.empty_like(q)
        gear_decode_attn_mq(self.cache, q, causal, K_buf, V_buf, n_buf, out, self.workspace)
        return out

    def export_codes(self, which):
        c = self.cfg
        codes = torch.empty((c.B, c.H_kv, self.n_total, c.d_h), dtype=torch.uint8, device=self.device)
        if which == 0:
            shape = (c.B, c.H_kv, self.n_groups_total(), c.d_h)
        else:
            shape = (c.B, c.H_kv, self.n_total, c.d_h // (c.group or c.d_h))
        scale = torch.empty(shape, dtype=torch.float16, device=self.device)
        zero = torch.empty(shape, dtype=torch.float16, device=self.device)
        gear_export_codes(self.cache, which, codes, scale, zero)
        return codes, scale, zero

    def export_sparse(self, which):
        c = self.cfg
        shape = (c.B, c.H_kv, self.n_total, c.d_h)
        mask = torch.empty(shape, dtype=torch.uint8, device=self.device)
        vals = torch.empty(shape, dtype=torch.float16, device=self.device)
        gear_export_sparse(self.cache, which, mask, vals)
        return mask, vals

    def export_sparse_coo(self, which):
        nnz = gear_export_sparse_coo(self.cache, which, None, None, None)
        lin = torch.empty(max(nnz, 1), dtype=torch.int64, device=self.device)
        vals = torch.empty(max(nnz, 1), dtype=torch.float16, device=self.device)
        gear_export_sparse_coo(self.cache, which, lin, vals, self.workspace)
        return lin[:nnz], vals[:nnz]

    def export_lowrank(self, which, seg):
        c = self.cfg
        n = self.cache.n_prefill if seg == 0 else self.cache.chunk_n[seg - 1]
        r = self.cache.rank_prefill if seg == 0 else self.cache.chunk_rank[seg - 1]
        A = torch.empty((c.B, c.H_kv, n, r), dtype=torch.float16, device=self.device)
        Bf = torch.empty((c.B, c.H_kv, c.d_h, r), dtype=torch.float16, device=self.device)
        if r > 0:
            gear_export_lowrank(self.cache, which, seg, A, Bf)
        return A, Bf


class PagePool:
    """Allocates a pool of pages, and the workspace of its reads as they need it; forwards to the C ABI."""

    def __init__(self, cfg, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        self.pool = torch.zeros(gear_page_bytes(cfg), dtype=torch.uint8, device=self.device)

    def write(self, K, V, slots):
        gear_page_write(self.cfg, self.pool, K, V, slots)

    def write_rope(self, rope, K, V, slots, positions, q=None, q_out=None):
        """Turned Keys and Values into their slots; the turned queries, if there are any."""
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        gear_page_write_rope(self.cfg, self.pool, rope, K, V, slots, positions, q, q_out)
        return q_out

    def move(self, pairs):
        gear_page_move(self.cfg, self.pool, pairs)

    def read(self, slots, heads_first=False):
        """K, V of slots [n_seqs, tokens] as [n_seqs, tokens, H_kv, 128], or [n_seqs, H_kv, tokens, 128]: what GearCache.compress takes.
        Rows whose slot is outside the pool are 0."""
        c, (n, m) = self.cfg, slots.shape
        dt = {v: k for k, v in GEAR_DTYPES.items()}[c.dtype]
        shape = (n, c.H_kv, m, c.d_h) if heads_first else (n, m, c.H_kv, c.d_h)
        K, V = (torch.zeros(shape, dtype=dt, device=self.device) for _ in range(2))
        gear_page_read(c, self.pool, K.transpose(1, 2) if heads_first else K, V.transpose(1, 2) if heads_first else V, slots)
        return K, V

    def workspace_for(self, H_q, batch):
        """A workspace for this batch and all smaller ones (None where none is needed)."""
        n = gear_page_attn_bytes(self.cfg, H_q, batch)
        return torch.empty(n, dtype=torch.uint8, device=self.device) if n else None

    def attn(self, q, batch, scale=None, out=None, workspace=None):
        if out is None:
            out = torch.empty_like(q)
        if workspace is None:
            workspace = self.workspace_for(q.shape[-2], batch)
        gear_page_attn(self.cfg, self.pool, batch, q, out, self.cfg.d_h ** -0.5 if scale is None else scale, workspace)
        return out

    def attn_shared(self, q, batch, groups, scale=None, out=None, workspace=None):
        if out is None:
            out = torch.empty_like(q)
        if workspace is None:
            n = gear_page_attn_shared_bytes(self.cfg, q.shape[-2], batch, groups)
            workspace = torch.empty(n, dtype=torch.uint8, device=self.device) if n else None
        gear_page_attn_shared(self.cfg, self.pool, batch, groups, q, out, self.cfg.d_h ** -0.5 if scale is None else scale, workspace)
        return out


class PageTable:
    """Allocates a page table; forwards to the C ABI.  One serves the pools of all layers."""

    def __init__(self, n_pages, page_size, n_rows, width, device="cuda:0"):
        self.device = torch.device(device)
        self.page_size = page_size
        self.table = torch.full((n_rows, width), -1, dtype=torch.int32, device=self.device)
        self.kv_len = torch.zeros(n_rows, dtype=torch.int32, device=self.device)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
        self.c = make_page_table(self.table, self.kv_len, self.refs, page_size)

    def _new(self, *shape, dtype=torch.int32):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def extend(self, rows, counts, max_count):
        """(slots [n, max_count], copies [n, 2], refused [n]) of counts[i] more tokens in row rows[i]."""
        n = rows.numel()
        slots, copies, refused = self._new(n, max_count, dtype=torch.int64), self._new(n, 2), self._new(n)
        gear_page_extend(self.c, rows, counts, slots, copies, refused)
        return slots, copies, refused

    def truncate(self, rows, lens):
        gear_page_truncate(self.c, rows, lens)

    def fork(self, src, dst):
        gear_page_fork(self.c, src, dst)

    def compact(self, max_moves):
        """(moves [max_moves, 2], counts [2]: pages in use, moves)."""
        moves, counts = self._new(max_moves, 2), self._new(2)
        gear_page_compact(self.c, moves, counts)
        return moves, counts
