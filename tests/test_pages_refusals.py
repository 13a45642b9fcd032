"""Rows that the paged cache's calls write must not share a place: refused on the host where the strides alone show it (no GPU: nothing is launched)."""
import ctypes
import os

import pytest

from paper_2403_05527_amd import binding as gb

FAKE = 0x10000000            # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2403_05527_amd.build import build_library
        build_library(verbose=False)
    return gb.load_library()


SHARED = [dict(token=64), dict(head=120), dict(seq=8), dict(token=-64), dict(token=128, head=128), dict(seq=512, token=512), dict(seq=256, head=256), dict(head=-8)]
BAD = dict(data=FAKE + 2)    # a call that is not refused for its strides ends here, with GEAR_EALIGN


def rows(data=FAKE, seq=1 << 16, token=512, head=128):
    return gb.gear_page_rows(data, seq, token, head)


@pytest.mark.parametrize("kw", SHARED)
def test_rows_that_share_a_place(kw, lib):
    cfg = gb.make_page_config(10, 32, 4, 8, 64)
    size = gb.gear_page_bytes(cfg)

    def read(K, V, n_seqs=2, n_rows=3):
        return lib.gear_page_read(ctypes.byref(cfg), FAKE, size, ctypes.byref(K), ctypes.byref(V), n_seqs, n_rows, FAKE, None)
    assert read(rows(**kw), rows()) == gb.GEAR_EINVAL and read(rows(), rows(**kw)) == gb.GEAR_EINVAL
    # rows that are only read may
    K = rows(**kw)
    assert lib.gear_page_write(ctypes.byref(cfg), FAKE, size, ctypes.byref(K), ctypes.byref(rows(**BAD)), 2, 3, FAKE, None) == gb.GEAR_EALIGN
    if "seq" not in kw:
        b = gb.gear_page_batch(1, 7, 7, 100, 4, 1, FAKE, FAKE, FAKE)

        def attn(q, out):
            return lib.gear_page_attn(ctypes.byref(cfg), FAKE, size, ctypes.byref(b), ctypes.byref(q), 8, 0.1, ctypes.byref(out), None, 0, None)
        assert attn(rows(), rows(**kw)) == gb.GEAR_EINVAL
        assert attn(rows(**kw), rows(**BAD)) == gb.GEAR_EALIGN


@pytest.mark.parametrize("kw", [dict(), dict(seq=3 * 128, token=9 * 128 * 4, head=128), dict(token=128, head=3 * 128), dict(token=-512), dict(seq=128, token=256, head=6 * 128)])
def test_rows_of_their_own(kw, lib):
    cfg = gb.make_page_config(10, 32, 4, 8, 64)
    K = rows(**kw)
    assert lib.gear_page_read(ctypes.byref(cfg), FAKE, gb.gear_page_bytes(cfg), ctypes.byref(K), ctypes.byref(rows(**BAD)), 2, 3, FAKE, None) == gb.GEAR_EALIGN


def test_strides_of_one_row_do_not_matter(lib):
    cfg = gb.make_page_config(10, 32, 1, 8, 64)
    K = rows(seq=0, token=3, head=1)
    assert lib.gear_page_read(ctypes.byref(cfg), FAKE, gb.gear_page_bytes(cfg), ctypes.byref(K), ctypes.byref(rows(**BAD)), 1, 1, FAKE, None) == gb.GEAR_EALIGN
