"""The paged cache's attention on the CPU stand-in (tests/simt/) with the plans that it makes for the 256 CUs of the device, so that axes are
divided and their parts joined: under the address sanitizer, 16-byte stores looked at for their alignment, on buffers of exactly their size, against the definition in 64 bits."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

from tests import page_util as pg
from tests.test_cpu_emulation_pages import BF16, CSRC, F16, PAGES, ROOT, SIMT, SOURCES, Case, find_clang, make_inputs


@pytest.fixture(scope="module")
def emulator(tmp_path_factory):
    cxx = find_clang()
    if cxx is None:
        pytest.skip("no clang++ to build the CPU emulation")
    out = tmp_path_factory.mktemp("simt_parts")
    flags = ["-std=c++17", "-O1", "-gline-tables-only", "-fsanitize=address", "-DSIMT_ALIGNED_STORES", "-fno-omit-frame-pointer", "-pthread",
             "-DGEAR_PAGE_CUS=256", "-I", SIMT, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", PAGES]
    procs = []
    for s in SOURCES + ["simt_rt", "run_pages"]:
        src = ["-x", "c++", "-c", os.path.join(PAGES, s + ".hip")] if s in SOURCES else ["-c", os.path.join(SIMT, s + ".cpp")]
        procs.append((str(out / (s + ".o")), subprocess.Popen([cxx] + src + ["-o", str(out / (s + ".o"))] + flags, stderr=subprocess.PIPE, text=True)))
    for _, p in procs:
        err = p.communicate()[1]
        assert p.returncode == 0, err[-3000:]
    exe = str(out / "run_pages")
    r = subprocess.run([cxx] + [o for o, _ in procs] + ["-o", exe] + flags, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


def launches(err):
    """{kernel with its template arguments: blocks}"""
    return {k: int(n) for k, n in re.findall(r"^launch (\w+(?:<[^>]*>)?)\)? grid (\d+)", err, re.M)}


# name -> (case, kernels that have to be among the launches, records that are written)
PARTS = {c.name: (c, kernels, records) for c, kernels, records in [
    # 34 columns in 5 parts, 175 records in the workspace, and one in 3: an odd number of records lies before those of the few columns
    (Case("both_odd", F16, 16, 128, 16, 1, 1, [(34, 800), (1, 790)]), ["page_attn_mixed_kernel", "page_merge_many_kernel<1>", "page_merge_few_kernel"], 34 * 5 + 3),
]}


@pytest.fixture(scope="module")
def runs(request, emulator, tmp_path_factory):
    def one(c):
        d = str(tmp_path_factory.mktemp(c.name))
        s = make_inputs(c, d)
        return d, s, subprocess.run([emulator, d], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    names = {i.callspec.params["name"] for i in request.session.items if getattr(i, "originalname", "") == "test_parts_are_joined"}
    pool = ThreadPoolExecutor(3)
    return {n: pool.submit(one, PARTS[n][0]) for n in PARTS if n in names}


def check(c, d, s, r):
    assert r.returncode == 0 and "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]
    got = torch.from_numpy(np.fromfile(os.path.join(d, "out.bin"), np.uint8)).view(c.dtype).view(s["out"].shape).double()
    want, bound = pg.attend(s["q"], s["K"], s["V"], s["q_start"], s["kv"], s["table"], c.scale, c.causal)
    dead = torch.isnan(want)
    assert bool((got[dead] == 77.0).all())
    assert bool(((got - want).abs() <= bound)[~dead].all()), float(((got - want).abs() / bound)[~dead].max())


@pytest.mark.parametrize("name", list(PARTS))
def test_parts_are_joined(runs, name):
    c, kernels, records = PARTS[name]
    d, s, r = runs[name].result()
    check(c, d, s, r)
    ran = launches(r.stderr)
    for k in kernels:
        assert any(x.startswith(k) for x in ran), (k, ran)
    assert int(re.search(r"^records (\d+) of", r.stderr, re.M).group(1)) == records, r.stderr[-500:]


LEAST, MOST = -2 ** 31, 2 ** 31 - 1
STARTS = [   # q_start of sequences that a case has, where it does not ascend: rows that nobody has are left alone, and nothing outside the arrays is read
    ([(40, 800)], 200, [200, LEAST], "none"),                            # a difference that leaves 32 bits
    ([(40, 800)], 200, [MOST, LEAST], "none"),
    ([(40, 800)], 200, [300, 299], "none"),
    ([(40, 90), (1, 800)], 150, [190, LEAST, LEAST], "none"),
    ([(40, 90), (1, 40)], 150, [LEAST, MOST, 0], "any"),                 # the first has all rows
    ([(1 + 33 * (i == 5), 40) for i in range(66)], 150, [LEAST if i % 2 else 150 + i for i in range(67)], "any"),
]


@pytest.mark.parametrize("i", range(len(STARTS)))
def test_starts_that_do_not_ascend(i, emulator, tmp_path):
    seqs, pad, starts, rows = STARTS[i]
    c = Case("starts", F16, 8, 64, 16, 1, 1, seqs, pad=pad)
    s = make_inputs(c, str(tmp_path))
    torch.tensor(starts, dtype=torch.int32).numpy().tofile(str(tmp_path / "q_start.bin"))
    r = subprocess.run([emulator, str(tmp_path)], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]
    got = torch.from_numpy(np.fromfile(str(tmp_path / "out.bin"), np.uint8)).view(F16).view(s["out"].shape)
    assert rows == "any" or bool((got == 77.0).all())
