"""Calls on a page table that would need more threads than a launch has are refused on the host (no GPU: nothing is launched)."""
import ctypes
import os

from paper_2403_05527_amd import binding as gb

FAKE = 0x10000000


def test_forks_of_more_threads_than_a_launch_has():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2403_05527_amd.build import build_library
        build_library(verbose=False)
    lib = gb.load_library()
    for width in ((1 << 27) - 7, (1 << 27) - 1):            # 8 columns to a block of 256 threads
        t = gb.gear_page_table(100, 16, 1, width, FAKE, FAKE, FAKE)
        for n in (911, 1024):
            assert lib.gear_page_fork(ctypes.byref(t), FAKE, FAKE, n, None) == gb.GEAR_ECAPACITY
