"""The entry points around the paged cache (rotary positions, page tables, shared prefixes) refuse on the host what they cannot do (no GPU: nothing
is launched), and the frequencies, which are formed there."""
import ctypes
import math
import os

import pytest
import torch

from paper_2403_05527_amd import binding as gb

FAKE = 0x10000000            # never dereferenced: validation fails first, or there is nothing to do
INVAL, ALIGN, CAP, OK = gb.GEAR_EINVAL, gb.GEAR_EALIGN, gb.GEAR_ECAPACITY, gb.GEAR_OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2403_05527_amd.build import build_library
        build_library(verbose=False)
    return gb.load_library()


def changed(s, **kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def config(**kw):
    return changed(gb.make_page_config(10, 32, 4, 8, 64), **kw)


def rope(**kw):
    return changed(gb.gear_rope(128, 0, 0, 1.0, FAKE), **kw)


def rows(data=FAKE, seq=1 << 16, token=1024, head=128):
    return gb.gear_page_rows(data, seq, token, head)


def table(**kw):
    return changed(gb.gear_page_table(100, 16, 8, 20, FAKE, FAKE, FAKE), **kw)


def batch(**kw):
    return changed(gb.gear_page_batch(3, 7, 4, 100, 4, 1, FAKE, FAKE, FAKE), **kw)


def groups(**kw):
    return changed(gb.gear_page_groups(2, 7, 80, 1, FAKE, FAKE), **kw)


def test_struct_sizes_match_header():
    assert ctypes.sizeof(gb.gear_rope) == 4 * 4 + 8
    assert ctypes.sizeof(gb.gear_page_table) == 4 * 4 + 3 * 8
    assert ctypes.sizeof(gb.gear_page_groups) == 4 * 4 + 2 * 8


def test_frequencies(lib):
    """To a rounding or two of 64 bits of the formulas (2^-50 of them: a power's error is at most 2^-52, a product's 2^-53)."""
    near = lambda a, b: all(abs(x - y) <= 2.0 ** -50 * abs(y) for x, y in zip(a.tolist(), b))  # noqa: E731
    plain = [10000.0 ** (-2 * p / 96) for p in range(48)]
    assert near(gb.gear_rope_freq(96), plain)
    assert near(gb.gear_rope_freq(96, scaling="linear", scale=4.0), [w / 4 for w in plain])
    based = gb.gear_rope_freq(96, scaling="base", scale=4.0)
    assert based[0] == 1.0 and abs(based[-1] - plain[-1] / 4) < 2.0 ** -48 * plain[-1]        # the slowest pair, by the scale; the fastest as it was
    got = gb.gear_rope_freq(128, 500000.0, "turns", 8.0, 8192, 1.0, 4.0).tolist()
    want = []
    for p in range(64):
        w = 500000.0 ** (-2 * p / 128)
        u = 8192 * w / (2 * math.pi)
        k = min(1.0, max(0.0, (u - 1) / 3))
        want.append(w * (k + (1 - k) / 8))
    assert near(torch.tensor(got, dtype=torch.float64), want)
    assert any(8192 * w / (2 * math.pi) > 4 for w in want) and any(8192 * w * 8 / (2 * math.pi) < 1 for w in want)
    assert gb.gear_rope_freq(2).tolist() == [1.0]


def test_frequencies_are_checked(lib):
    def call(scaling=0, rot=64, base=1e4, scale=2.0, length=100.0, low=1.0, high=4.0, to=(ctypes.c_double * 64)()):
        return lib.gear_rope_freq(scaling, rot, base, scale, length, low, high, to)
    nan, inf = float("nan"), float("inf")
    assert call() == OK and call(rot=0) == INVAL and call(rot=63) == INVAL and call(rot=130) == INVAL and call(rot=-2) == INVAL and call(to=None) == INVAL
    assert call(base=0.0) == INVAL and call(base=nan) == INVAL and call(base=inf) == INVAL and call(scale=0.0) == INVAL and call(scale=-1.0) == INVAL and call(scale=nan) == INVAL
    assert call(scaling=4) == INVAL and call(scaling=-1) == INVAL and call(scaling=2, rot=2) == INVAL and call(scaling=2, rot=4) == OK
    assert call(length=0.0) == OK and call(scaling=3, length=0.0) == INVAL and call(scaling=3, length=inf) == INVAL
    assert call(scaling=3, low=4.0) == INVAL and call(scaling=3, low=-1.0) == INVAL and call(scaling=3, high=nan) == INVAL and call(scaling=3, high=inf) == INVAL
    with pytest.raises(KeyError):
        gb.gear_rope_freq(64, scaling="other")
    with pytest.raises(gb.GearError):
        gb.gear_rope_freq(63)


BAD_ROPES = [dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=3), dict(rot_dim=130), dict(interleaved=2), dict(interleaved=-1), dict(inverse=2), dict(factor=float("nan")),
             dict(factor=float("inf")), dict(freq=None)]


def test_turns_are_checked(lib):
    def call(r=rope(), dtype=0, x=rows(), out=rows(FAKE * 2), n_seqs=2, n_rows=3, heads=4, positions=FAKE):
        return lib.gear_rotate(r and ctypes.byref(r), dtype, x and ctypes.byref(x), out and ctypes.byref(out), n_seqs, n_rows, heads, positions, None)
    assert call(r=None) == INVAL and call(x=None) == INVAL and call(out=None) == INVAL and call(dtype=2) == INVAL and call(dtype=-1) == INVAL
    for kw in BAD_ROPES:
        assert call(r=rope(**kw)) == INVAL, kw
    assert call(r=rope(freq=FAKE + 4)) == ALIGN and call(x=rows(FAKE + 8)) == ALIGN and call(out=rows(FAKE + 2)) == ALIGN and call(positions=FAKE + 4) == ALIGN
    assert call(x=rows(token=1028)) == ALIGN and call(out=rows(FAKE * 2, head=132)) == ALIGN and call(x=rows(seq=4)) == ALIGN
    assert call(positions=None) == INVAL and call(x=rows(None)) == INVAL and call(out=rows(None)) == INVAL
    assert call(n_seqs=-1) == INVAL and call(n_rows=-1) == INVAL and call(heads=-1) == INVAL
    assert call(out=rows(FAKE * 2, token=0)) == INVAL and call(out=rows(FAKE * 2, head=0)) == INVAL      # rows in one place
    assert call(out=rows(token=512)) == INVAL and call(out=rows(head=256)) == INVAL                     # in place, with other strides
    assert call(n_seqs=1 << 20, n_rows=1 << 12) == CAP
    none = rows(None)
    assert call(n_seqs=0, x=none, out=none, positions=None) == OK and call(n_rows=0, x=none) == OK and call(heads=0, out=none) == OK


def test_turned_writes_are_checked(lib):
    cfg, n = config(), gb.gear_page_bytes(config())

    def call(cfg=cfg, pool=FAKE, nbytes=n, r=rope(), K=rows(), V=rows(), q=rows(), q_out=rows(), H_q=8, n_seqs=2, n_rows=3, slots=FAKE, positions=FAKE):
        ref = lambda x: x and ctypes.byref(x)  # noqa: E731
        return lib.gear_page_write_rope(ref(cfg), pool, nbytes, ref(r), ref(K), ref(V), ref(q), ref(q_out), H_q, n_seqs, n_rows, slots, positions, None)
    assert call(cfg=None) == INVAL and call(cfg=config(bits=3)) == INVAL and call(pool=None) == INVAL and call(r=None) == INVAL
    for kw in BAD_ROPES:
        assert call(r=rope(**kw)) == INVAL, kw
    assert call(K=None) == INVAL and call(V=None) == INVAL and call(K=rows(None)) == INVAL and call(slots=None) == INVAL and call(positions=None) == INVAL
    assert call(q=None) == INVAL and call(q_out=None) == INVAL and call(q=None, q_out=None) == INVAL and call(H_q=0) == INVAL and call(H_q=-1) == INVAL
    assert call(n_seqs=-1) == INVAL and call(n_rows=-1) == INVAL and call(q_out=rows(FAKE * 2, token=0)) == INVAL and call(q_out=rows(token=2048)) == INVAL
    assert call(pool=FAKE + 8) == ALIGN and call(K=rows(FAKE + 8)) == ALIGN and call(V=rows(token=1025)) == ALIGN and call(q=rows(FAKE + 2)) == ALIGN
    assert call(slots=FAKE + 4) == ALIGN and call(positions=FAKE + 4) == ALIGN
    assert call(nbytes=n - 1) == CAP and call(n_seqs=1 << 20, n_rows=1 << 12) == CAP
    assert call(n_seqs=0, K=rows(None), slots=None) == OK and call(n_rows=0) == OK
    assert call(n_rows=0, q=None, q_out=None, H_q=0) == OK


def test_tables_are_checked(lib):
    def extend(t=table(), r=FAKE, c=FAKE, n=4, most=5, slots=FAKE, copies=FAKE, refused=FAKE):
        return lib.gear_page_extend(t and ctypes.byref(t), r, c, n, most, slots, copies, refused, None)

    def truncate(t=table(), r=FAKE, c=FAKE, n=4):
        return lib.gear_page_truncate(t and ctypes.byref(t), r, c, n, None)

    def fork(t=table(), r=FAKE, c=FAKE, n=4):
        return lib.gear_page_fork(t and ctypes.byref(t), r, c, n, None)

    def compact(t=table(), moves=FAKE, n=4, counts=FAKE):
        return lib.gear_page_compact(t and ctypes.byref(t), moves, n, counts, None)
    for call in (extend, truncate, fork, compact):
        assert call(t=None) == INVAL and call(n=-1) == INVAL
        for kw in (dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(n_pages=0), dict(n_rows=0), dict(width=0), dict(table=None),
                   dict(kv_len=None), dict(refs=None), dict(n_pages=-1), dict(n_rows=-1), dict(width=-1)):
            assert call(t=table(**kw)) == INVAL, kw
        for kw in (dict(table=FAKE + 2), dict(kv_len=FAKE + 1), dict(refs=FAKE + 4)):
            assert call(t=table(**kw)) == ALIGN, kw
        for kw in (dict(n_pages=(1 << 20) + 1), dict(n_rows=(1 << 18) + 1), dict(width=1 << 27)):
            assert call(t=table(**kw)) == CAP, kw
    for call in (extend, truncate, fork):
        assert call(r=None) == INVAL and call(c=None) == INVAL and call(r=FAKE + 2) == ALIGN and call(c=FAKE + 1) == ALIGN
        assert call(n=gb.GEAR_PAGE_LIST_MAX + 1) == CAP and call(n=0) == OK and call(n=0, r=None, c=None) == OK
    assert extend(most=-1) == INVAL and extend(slots=None) == INVAL and extend(copies=None) == INVAL and extend(refused=None) == INVAL
    assert extend(slots=FAKE + 4) == ALIGN and extend(copies=FAKE + 2) == ALIGN and extend(refused=FAKE + 2) == ALIGN
    assert extend(n=1024, most=(1 << 31) - 1) == CAP
    assert compact(counts=None) == INVAL and compact(moves=None) == INVAL and compact(moves=FAKE + 2) == ALIGN and compact(counts=FAKE + 2) == ALIGN
    assert compact(t=table(n_rows=1 << 18, width=1 << 14)) == CAP


def test_moves_are_checked(lib):
    cfg, n = config(), gb.gear_page_bytes(config())

    def call(cfg=cfg, pool=FAKE, nbytes=n, n_pools=1, stride=0, pairs=FAKE, k=3):
        return lib.gear_page_move(cfg and ctypes.byref(cfg), pool, nbytes, n_pools, stride, pairs, k, None)
    assert call(cfg=None) == INVAL and call(cfg=config(bits=2)) == INVAL and call(pool=None) == INVAL and call(pairs=None) == INVAL
    assert call(n_pools=-1) == INVAL and call(k=-1) == INVAL and call(n_pools=2, stride=n - 16, nbytes=4 * n) == INVAL
    assert call(pool=FAKE + 8) == ALIGN and call(pairs=FAKE + 2) == ALIGN and call(n_pools=2, stride=n + 8, nbytes=4 * n) == ALIGN
    assert call(nbytes=n - 1) == CAP and call(n_pools=3, stride=n, nbytes=3 * n - 1) == CAP and call(n_pools=2, stride=1 << 62, nbytes=4 * n) == CAP
    assert call(n_pools=1 << 20, stride=n, nbytes=n << 20, k=1 << 10) == CAP
    assert call(k=0, pairs=None) == OK and call(n_pools=0) == OK


def test_shared_attention_is_checked(lib):
    cfg, n = config(), gb.gear_page_bytes(config())

    def call(cfg=cfg, pool=FAKE, nbytes=n, b=batch(), g=groups(), q=rows(), H_q=8, scale=0.1, out=rows(), ws=None, wn=0):
        ref = lambda x: x and ctypes.byref(x)  # noqa: E731
        return lib.gear_page_attn_shared(ref(cfg), pool, nbytes, ref(b), ref(g), ref(q), H_q, scale, ref(out), ws, wn, None)
    assert call(cfg=None) == INVAL and call(cfg=config(group=7)) == INVAL and call(pool=None) == INVAL and call(b=None) == INVAL and call(g=None) == INVAL
    assert call(q=None) == INVAL and call(out=None) == INVAL and call(H_q=6) == INVAL and call(scale=float("nan")) == INVAL
    for kw in (dict(n_seqs=-1), dict(n_tokens=-1), dict(max_q=-1), dict(max_kv=-1), dict(table_width=-1), dict(q_start=None), dict(kv_len=None), dict(page_table=None)):
        assert call(b=batch(**kw)) == INVAL, kw
    for kw in (dict(n_groups=-1), dict(max_q=-1), dict(max_prefix=-1), dict(always=2), dict(always=-1), dict(group_start=None), dict(prefix_len=None)):
        assert call(g=groups(**kw)) == INVAL, kw
    for kw in (dict(group_start=FAKE + 2), dict(prefix_len=FAKE + 1)):
        assert call(g=groups(**kw)) == ALIGN, kw
    assert call(out=rows(token=0)) == INVAL and call(q=rows(FAKE + 2)) == ALIGN and call(ws=FAKE + 8, wn=1 << 30) == ALIGN and call(nbytes=n - 1) == CAP
    assert call(g=groups(n_groups=(1 << 20) + 1)) == CAP
    assert call(b=batch(n_seqs=1 << 25)) == CAP and call(b=batch(table_width=1 << 27)) == CAP
    need = gb.gear_page_attn_shared_bytes(cfg, 8, batch(), groups())
    assert need > 0 and call() == INVAL and call(ws=FAKE, wn=16) == CAP          # records of the parts need a workspace
    assert call(b=batch(n_seqs=0)) == OK and call(b=batch(n_tokens=0)) == OK and call(b=batch(max_q=0)) == OK
    assert lib.gear_page_attn_shared_bytes(ctypes.byref(cfg), 8, ctypes.byref(batch()), None, ctypes.byref(ctypes.c_size_t())) == INVAL
    assert lib.gear_page_attn_shared_bytes(ctypes.byref(cfg), 8, ctypes.byref(batch()), ctypes.byref(groups()), None) == INVAL


def test_a_workspace_serves_all_smaller_batches(lib):
    sizes = {}
    for seqs in (1, 3, 40, 600):
        for max_q in (1, 5, 33, 700):
            for kv in (1, 300, 5000, 100000):
                for prefix in (0, 64, 200, 4000):
                    for g in (0, 1, 30):
                        b = batch(n_seqs=seqs, n_tokens=seqs * max_q, max_q=max_q, max_kv=kv)
                        sizes[seqs, max_q, kv, prefix, g] = gb.gear_page_attn_shared_bytes(config(), 8, b, groups(n_groups=g, max_q=seqs * max_q, max_prefix=prefix))
    for small, v in sizes.items():
        assert all(v <= w for large, w in sizes.items() if all(a <= b for a, b in zip(small, large)))
    assert max(sizes.values()) <= 512 << 20


def test_the_binding_refuses_what_the_library_cannot_see(monkeypatch):
    monkeypatch.setattr(gb, "_page_device", lambda: -1)        # (where a CPU tensor's get_device() says it is)
    cfg = gb.make_page_config(4, 16, 2, 8, 64)
    pool, x = torch.zeros(gb.gear_page_bytes(cfg), dtype=torch.uint8), torch.zeros(3, 2, 128, dtype=torch.float16)
    i64, i32 = torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        gb.make_rope(torch.ones(64))                           # not float64
    r = gb.make_rope(torch.ones(64, dtype=torch.float64))
    for a, b, p in ((x.float(), x.float(), i64), (x, x[:2], i64), (x[..., :64], x[..., :64], i64), (x, x, i32), (x, x, i64[:2]), (x, x.bfloat16(), i64)):
        with pytest.raises(ValueError):
            gb.gear_rotate(r, a, b, p)
    for kw in (dict(K=x.bfloat16()), dict(V=x[:2]), dict(K=x[:, :1]), dict(slots=i32), dict(positions=i64[:1]), dict(q=x), dict(q=x, q_out=x[:2]), dict(q=x[:, :0], q_out=x[:, :0])):
        with pytest.raises(ValueError):
            gb.gear_page_write_rope(cfg, pool, r, **dict(dict(K=x, V=x, slots=i64, positions=i64), **kw))
    with pytest.raises(ValueError):
        gb.make_page_table(torch.zeros(2, 3), i32[:2], i32, 16)
    t = gb.make_page_table(torch.zeros(2, 3, dtype=torch.int32), i32[:2], i32, 16)
    pair = torch.zeros(3, 2, dtype=torch.int32)
    for a in ((i64, i32, torch.zeros(3, 1, dtype=torch.int64), pair, i32), (i32, i32[:2], torch.zeros(3, 1, dtype=torch.int64), pair, i32), (i32, i32, i64, pair, i32),
              (i32, i32, torch.zeros(2, 1, dtype=torch.int64), pair, i32), (i32, i32, torch.zeros(3, 1, dtype=torch.int32), pair, i32), (i32, i32, torch.zeros(3, 1, dtype=torch.int64), pair[:2], i32)):
        with pytest.raises(ValueError):
            gb.gear_page_extend(t, *a)
    for f in (gb.gear_page_truncate, gb.gear_page_fork):
        with pytest.raises(ValueError):
            f(t, i32, i32[:2])
    for a in ((i32, i32[:2]), (pair, i32), (pair.long(), i32[:2])):
        with pytest.raises(ValueError):
            gb.gear_page_compact(t, *a)
    for a in ((pool, i32), (pool, pair.long()), (pool.view(4, -1).t(), pair)):
        with pytest.raises(ValueError):
            gb.gear_page_move(cfg, *a)
    with pytest.raises(ValueError):
        gb.make_page_groups(i32[:2], i32, 1, 1)
    monkeypatch.setattr(gb, "_page_device", lambda: 1)         # what was made on another GPU
    b = changed(gb.gear_page_batch(1, 3, 3, 3, 1, 1, FAKE, FAKE, FAKE), device=1)
    for f in (lambda: gb.gear_rotate(r, x, x, i64), lambda: gb.gear_page_write_rope(cfg, pool, r, x, x, i64, i64), lambda: gb.gear_page_truncate(t, i32, i32),
              lambda: gb.gear_page_attn_shared(cfg, pool, b, changed(groups(), device=-1), x, x, 0.1, None)):
        with pytest.raises(ValueError):
            f()
