"""The paged cache's entry points refuse on the host what they cannot do (no GPU: nothing is launched)."""
import ctypes
import os

import pytest
import torch

from paper_2403_05527_amd import binding as gb

FAKE = 0x10000000            # never dereferenced: validation fails first, or there is nothing to do


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2403_05527_amd.build import build_library
        build_library(verbose=False)
    return gb.load_library()


def good(**kw):
    c = gb.make_page_config(10, 32, 4, 8, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_struct_sizes_match_header():
    assert ctypes.sizeof(gb.gear_page_config) == 7 * 4
    assert ctypes.sizeof(gb.gear_page_rows) == 32
    assert ctypes.sizeof(gb.gear_page_batch) == 6 * 4 + 3 * 8


def test_pool_bytes_and_invalid_configs(lib):
    assert gb.gear_page_bytes(good()) == 10 * 4 * 2 * 32 * (128 + 8)
    assert gb.gear_page_bytes(good(bits=4, group=32)) == 10 * 4 * 2 * 32 * (64 + 16)
    assert gb.gear_page_bytes(good(bits=16, group=0)) == 10 * 4 * 2 * 32 * 256
    for kw in (dict(n_pages=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(H_kv=0), dict(H_kv=1025), dict(d_h=64), dict(bits=2),
               dict(bits=5), dict(group=16), dict(group=256), dict(group=0), dict(dtype=2), dict(dtype=-1)):
        with pytest.raises(gb.GearError) as e:
            gb.gear_page_bytes(good(**kw))
        assert e.value.status == gb.GEAR_EINVAL, kw
    assert lib.gear_page_bytes(None, ctypes.byref(ctypes.c_size_t())) == gb.GEAR_EINVAL
    assert lib.gear_page_bytes(ctypes.byref(good()), None) == gb.GEAR_EINVAL
    # 1024 heads x 256 tokens x 2 x 256 bytes is 128 MiB a page: the widest there is
    assert gb.gear_page_bytes(good(H_kv=1024, page_size=256, bits=16, n_pages=100000)) == 100000 << 27


def rows(data=FAKE, seq=1 << 16, token=512, head=128):
    return gb.gear_page_rows(data, seq, token, head)


@pytest.mark.parametrize("name", ["gear_page_write", "gear_page_read"])
def test_copies_are_checked(lib, name):
    cfg, n = good(), gb.gear_page_bytes(good())

    def call(cfg=cfg, pool=FAKE, nbytes=n, K=rows(), V=rows(), n_seqs=2, n_rows=3, slots=FAKE):
        return getattr(lib, name)(cfg and ctypes.byref(cfg), pool, nbytes, K and ctypes.byref(K), V and ctypes.byref(V), n_seqs, n_rows, slots, None)
    inval, align, cap = gb.GEAR_EINVAL, gb.GEAR_EALIGN, gb.GEAR_ECAPACITY
    assert call(cfg=None) == inval and call(cfg=good(bits=3)) == inval and call(pool=None) == inval
    assert call(K=None, V=None) == inval and call(slots=None) == inval
    assert call(n_seqs=-1) == inval and call(n_rows=-1) == inval
    assert call(K=rows(data=None)) == inval
    assert call(pool=FAKE + 8) == align and call(slots=FAKE + 4) == align
    assert call(K=rows(data=FAKE + 8)) == align and call(V=rows(token=516)) == align and call(V=rows(head=132)) == align and call(K=rows(seq=4)) == align
    assert call(nbytes=n - 1) == cap and call(n_seqs=1 << 20, n_rows=1 << 12) == cap
    assert call(n_seqs=0) == gb.GEAR_OK and call(n_rows=0, slots=None) == gb.GEAR_OK
    if name == "gear_page_write":
        assert call(K=None) == inval and call(V=None) == inval
    else:   # two rows in one place
        assert call(K=rows(token=0)) == inval and call(V=rows(head=0)) == inval and call(V=rows(seq=0)) == inval


@pytest.mark.parametrize("name", ["gear_page_write", "gear_page_read"])
def test_copies_of_no_rows(lib, name):
    """A tensor without an entry has no address."""
    cfg, none, one = good(), rows(data=None), rows()
    for n_seqs, n_rows in ((0, 3), (3, 0), (0, 0)):
        assert getattr(lib, name)(ctypes.byref(cfg), FAKE, gb.gear_page_bytes(cfg), ctypes.byref(none), ctypes.byref(one), n_seqs, n_rows, None, None) == gb.GEAR_OK


def batch(**kw):
    b = gb.gear_page_batch(3, 7, 4, 100, 4, 1, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def test_attention_is_checked(lib):
    cfg, n = good(), gb.gear_page_bytes(good())

    def call(cfg=cfg, pool=FAKE, nbytes=n, b=batch(), q=rows(), H_q=8, scale=0.1, out=rows(), ws=None, wn=0):
        return lib.gear_page_attn(cfg and ctypes.byref(cfg), pool, nbytes, b and ctypes.byref(b), q and ctypes.byref(q), H_q, scale,
                                  out and ctypes.byref(out), ws, wn, None)
    inval, align, cap = gb.GEAR_EINVAL, gb.GEAR_EALIGN, gb.GEAR_ECAPACITY
    assert call(cfg=None) == inval and call(cfg=good(group=7)) == inval and call(pool=None) == inval and call(b=None) == inval
    assert call(q=None) == inval and call(out=None) == inval and call(q=rows(data=None)) == inval
    assert call(H_q=0) == inval and call(H_q=6) == inval and call(H_q=-4) == inval
    assert call(scale=float("nan")) == inval and call(scale=float("inf")) == inval
    for kw in (dict(n_seqs=-1), dict(n_tokens=-1), dict(max_q=-1), dict(max_kv=-1), dict(table_width=-1), dict(q_start=None), dict(kv_len=None),
               dict(page_table=None)):
        assert call(b=batch(**kw)) == inval, kw
    assert call(out=rows(token=0)) == inval and call(out=rows(head=0)) == inval
    assert call(pool=FAKE + 8) == align and call(q=rows(data=FAKE + 2)) == align and call(q=rows(token=513)) == align and call(out=rows(head=4)) == align
    for kw in (dict(q_start=FAKE + 2), dict(kv_len=FAKE + 1), dict(page_table=FAKE + 3)):
        assert call(b=batch(**kw)) == align, kw
    assert call(ws=FAKE + 8, wn=1 << 30) == align
    assert call(nbytes=n - 1) == cap
    assert call(b=batch(n_tokens=1 << 30)) == cap and call(b=batch(n_seqs=1 << 25)) == cap and call(b=batch(table_width=1 << 27)) == cap
    # divided keys need a workspace
    long = batch(n_seqs=1, n_tokens=1, max_q=1, max_kv=8192)
    need = gb.gear_page_attn_bytes(cfg, 8, long)
    assert need > 0 and call(b=long) == inval and call(b=long, ws=FAKE, wn=16) == cap
    # nothing to do
    assert call(b=batch(n_seqs=0)) == gb.GEAR_OK and call(b=batch(n_tokens=0)) == gb.GEAR_OK and call(b=batch(max_q=0)) == gb.GEAR_OK


def test_attention_of_no_rows_and_scales_past_fp32(lib):
    cfg, n, none = good(), gb.gear_page_bytes(good()), rows(data=None)

    def call(b, q, out, scale):
        return lib.gear_page_attn(ctypes.byref(cfg), FAKE, n, ctypes.byref(b), ctypes.byref(q), 8, scale, ctypes.byref(out), None, 0, None)
    assert call(batch(n_tokens=0), none, none, 0.1) == gb.GEAR_OK
    assert call(batch(n_tokens=0), none, none, 3e38) == gb.GEAR_EINVAL      # log2(e) times it is infinite
    assert call(batch(n_tokens=0), none, none, -3e38) == gb.GEAR_EINVAL and call(batch(n_tokens=0), none, none, -2e38) == gb.GEAR_OK


def test_a_workspace_serves_all_smaller_batches(lib):
    """The bytes grow with every bound, so what suffices for the largest batch suffices for each."""
    sizes = {}
    for H_q, H in ((4, 4), (8, 4), (40, 1)):
        for seqs in (1, 3, 40, 600):
            for max_q in (1, 5, 33, 700):
                for kv in (1, 300, 512, 5000, 100000):
                    b = batch(n_seqs=seqs, n_tokens=seqs * max_q, max_q=max_q, max_kv=kv)
                    sizes[H_q, H, seqs, max_q, kv] = gb.gear_page_attn_bytes(good(H_kv=H), H_q, b)
    for (a, h, s, m, k), v in sizes.items():
        assert all(v <= w for (a2, h2, s2, m2, k2), w in sizes.items() if (a2, h2) == (a, h) and s2 >= s and m2 >= m and k2 >= k)
    assert max(sizes.values()) < 64 << 20        # bounded by what the chip holds at once, not by the batch


def test_the_binding_refuses_what_the_library_cannot_see():
    cfg = gb.make_page_config(4, 16, 2, 8, 64)
    pool = torch.zeros(gb.gear_page_bytes(cfg), dtype=torch.uint8)
    x, slots = torch.zeros(3, 2, 128, dtype=torch.float16), torch.zeros(3, dtype=torch.int64)
    bad = [(x.float(), x, slots), (x.bfloat16(), x, slots), (x[:, :1], x, slots), (x[..., :64], x, slots), (x.expand(2, 2, 3, 2, 128), x, slots),
           (x, x, slots),                                                # not on a GPU
           (x.transpose(1, 2).contiguous().transpose(1, 2), x, slots)]   # rows that are not contiguous
    for K, V, s in bad:
        with pytest.raises(ValueError):
            gb.gear_page_write(cfg, pool, K, V, s)
    with pytest.raises(ValueError):
        gb.gear_page_read(cfg, pool, None, None, slots)
    with pytest.raises(KeyError):
        gb.make_page_config(4, 16, 2, 8, 64, torch.float32)
    i = torch.zeros(3, dtype=torch.int32)
    for a in ((i.long(), i[:2], i.view(1, 3)), (i[:1], i[:2], i.view(1, 3)), (i[:2], i[:1], i.view(1, 3))):
        with pytest.raises(ValueError):
            gb.make_page_batch(*a, 1, 1, 1)


def test_a_batch_of_another_gpu_is_refused(monkeypatch):
    """The tensors of a batch are looked at when it is made; the call may come with another GPU current."""
    cfg = gb.make_page_config(4, 16, 2, 8, 64)
    pool, x, i = torch.zeros(gb.gear_page_bytes(cfg), dtype=torch.uint8), torch.zeros(1, 2, 128, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    monkeypatch.setattr(gb, "_page_device", lambda: -1)        # (where a CPU tensor's get_device() says it is)
    b = gb.make_page_batch(i, i[:1], i.view(1, 2), 1, 1, 16)
    monkeypatch.setattr(gb, "_page_device", lambda: 1)
    with pytest.raises(ValueError, match="batch"):
        gb.gear_page_attn(cfg, pool, b, x, x, 0.1, None)
