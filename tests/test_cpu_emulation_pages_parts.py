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
