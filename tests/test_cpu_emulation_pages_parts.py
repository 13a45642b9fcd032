"""The paged cache's attention on the CPU stand-in (tests/simt/) with the plans that it makes for the 256 CUs of the device, so that axes are
divided and their parts joined: under the address sanitizer, 16-byte stores looked at for their alignment, on buffers of exactly their size, against the definition in 64 bits."""
import math
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
    """{kernel as the launch names it: blocks}"""
    return {k: int(n) for k, n in re.findall(r"^launch (\w+(?:<[^>]*>)?)\)? grid (\d+)", err, re.M)}


# name -> (case, kernels that have to be among the launches, records that are written)
PARTS = {c.name: (c, kernels, records) for c, kernels, records in [
    # 34 columns in 5 parts, 175 records in the workspace, and one in 3: an odd number of records lies before those of the few columns
    (Case("both_odd", F16, 16, 128, 16, 1, 1, [(34, 800), (1, 790)]), ["page_attn_mixed_kernel", "page_merge_many_kernel<1>", "page_merge_few_kernel"], 34 * 5 + 3),
    # 9 parts, and 5
    (Case("both_four_waves", BF16, 8, 64, 16, 1, 1, [(34, 1700), (1, 1690)]), ["page_attn_mixed_kernel", "page_merge_many_kernel<4>", "page_merge_few_kernel"], 34 * 9 + 5),
    (Case("few", F16, 8, 128, 16, 1, 2, [(1, 1100), (1, 30)], bad=True), ["page_attn_few_kernel", "page_merge_few_kernel"], 2 * 3),
    (Case("few_two_tiles", F16, 4, 32, 16, 1, 10, [(2, 1100), (1, 600)]), ["page_attn_few_kernel", "page_merge_few_kernel"], 20 * 3 + 10 * 2),
    # more records than the four waves of a merge ask for at a time (32), and than a wave's lanes look at (64)
    (Case("few_34_parts", F16, 4, 128, 256, 1, 1, [(1, 17000)]), ["page_attn_few_kernel", "page_merge_few_kernel"], 34),
    (Case("few_65_parts", F16, 4, 128, 256, 1, 1, [(1, 33000)]), ["page_attn_few_kernel", "page_merge_few_kernel"], 65),
    (Case("many_68_parts", F16, 16, 128, 256, 1, 1, [(33, 13000)]), ["page_attn_many_kernel", "page_merge_many_kernel<4>"], 33 * 68),
    # the joining looks for a row's sequence among more than a wave has lanes
    (Case("many_of_66", F16, 8, 128, 16, 1, 1, [(34, 1500) if i == 64 else (1, 17 + i % 3) for i in range(66)]), ["page_attn_mixed_kernel", "page_merge_many_kernel<1>"], 34 * 8),
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


# a part's pages are more than a wave's lanes hold at a time (64): tables of 94 entries, some of no page, one part
ENTRIES = [(n, form) for n in (1, 40) for form in ((F16, 16, 128), (F16, 4, 32), (BF16, 8, 64))]


@pytest.mark.parametrize("n,form", ENTRIES)
def test_pages_past_the_first_look(n, form, emulator, tmp_path):
    dtype, bits, group = form
    c = Case("entries", dtype, bits, group, 16, 1, 1, [(n, 1500), (n, 1040)], max_kv=1)
    s = make_inputs(c, str(tmp_path))
    for i, page in ((3, -1), (64, -7), (70, 10 ** 6), (71, s["pool"].shape[0]), (93, -1)):
        s["table"][0][i] = page
    torch.tensor(s["table"], dtype=torch.int32).numpy().tofile(str(tmp_path / "table.bin"))
    r = subprocess.run([emulator, str(tmp_path)], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    check(c, str(tmp_path), s, r)
    assert len(launches(r.stderr)) == 1, r.stderr


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


def run_with(emulator, path, c, s, scale):
    """The case with s's Keys, Values and queries, 16 bits, one head, and this scale: [rows, 128] in 64 bits."""
    c.scale = scale
    meta = (path / "meta.txt").read_text().split()
    meta[7] = repr(scale)
    (path / "meta.txt").write_text(" ".join(meta) + "\n")
    blocks = torch.stack([pg.pack(x, 16, 128, c.dtype) for x in (s["K"], s["V"])], 2)
    for name, t in (("pool.bin", blocks), ("q.bin", s["q"])):
        t.contiguous().view(torch.uint8).numpy().tofile(str(path / name))
    r = subprocess.run([emulator, str(path)], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    check(c, str(path), s, r)
    assert [k.split("<")[0] for k in launches(r.stderr)] == ["page_attn_few_kernel" if len(s["q"]) == 1 else "page_attn_many_kernel"], r.stderr
    return torch.from_numpy(np.fromfile(str(path / "out.bin"), np.uint8)).view(c.dtype).view(s["out"].shape)[:, 0].double()


@pytest.mark.parametrize("n", [1, 36])
def test_a_flat_tail_counts(n, emulator, tmp_path):
    """Many weights that are each far below a row's greatest, in the sum of Values as in the sum of weights: one token, and a chunk."""
    kv, page = 1536, 16
    c = Case("tail", F16, 16, 128, page, 1, 1, [(n, kv)], max_kv=1)     # (one part)
    s = make_inputs(c, str(tmp_path))
    scale = pg.sink_and_tail(s["K"], s["V"], s["q"], s["table"][0], kv, page)
    got = run_with(emulator, tmp_path, c, s, scale)
    want, bound = pg.tail_bound(s["q"], s["K"], s["V"], s["table"][0], kv, 0, n, scale, page)
    assert float(want.min()) > 2.0 ** -20         # 1500 of 2^-26, each with a Value of 1/2 and more, beside 8 of 1
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [1, 36])
@pytest.mark.parametrize("log2", [15.3, 22.97, 23.02, 24.3, 25.7, 27.4])
def test_equal_scores_of_any_size(log2, n, dtype, emulator, tmp_path):
    """All scores equal, from 2^15 to 2^27 steps of the exponent: the mean of the Values, however the base of the weights is rounded."""
    kv, page = 70, 16
    c = Case("equal", dtype, 16, 128, page, 1, 1, [(n, kv)], causal=False)
    s = make_inputs(c, str(tmp_path))
    s["K"][:], s["q"][:] = 512.0, 512.0                                 # (sums of products are exact)
    got = run_with(emulator, tmp_path, c, s, 2.0 ** (log2 - 25) * math.log(2.0))
    at = torch.arange(kv)
    v = s["V"][torch.tensor(s["table"][0])[at // page], 0, at % page].double()
    # one weight for all tokens, but rounded before the product and not before the sum; 70 terms in fp32
    eps, most = torch.finfo(dtype).eps / 2, v.abs().mean(0)
    bound = most * (eps + 80 * 2.0 ** -23)
    assert bool(((got - v.mean(0)).abs() <= bound + (v.mean(0).abs() + bound) * eps + 2.0 ** -25).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_codes_and_values_at_ties(bits, dtype, emulator, tmp_path):
    """The codes of a difference that fp32 does not hold, and the values of a sum that it does not hold: as stated.  And the pool's bytes, of slots that were
    named and of such that were not."""
    x, codes = pg.rows_at_ties(bits, dtype)
    if bits == 4 and dtype == BF16:
        x = torch.cat((torch.tensor([-2.0 ** -30, 15.125, 3.015625] + [0.5] * 29, dtype=torch.float64).repeat(1, 4).to(dtype), x))
    n, page = len(x), 16
    c = Case("ties", dtype, bits, 32, page, 1, 1, [(0, n)], write=True)
    s = make_inputs(c, str(tmp_path))
    new = torch.stack((x, -x.flip(0)))                                   # Keys; Values
    for name, t in zip(("K.bin", "V.bin"), new):
        t.contiguous().view(torch.uint8).numpy().tofile(str(tmp_path / name))
    r = subprocess.run([emulator, str(tmp_path)], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and "Sanitizer" not in r.stderr, r.stderr[-4000:]
    code, scale, zero = pg.quantise_fp32(new, bits, 32, dtype)
    assert [(int(code[0, i, 2]), int(pg.quantise(x, bits, 32, dtype)[0][i, 2])) for i in range(n - len(codes), n)] == codes
    values = pg.values_fp32(code, scale, zero, 32, dtype)
    if bits == 4 and dtype == BF16:
        assert values[0, 0, 2] == 3.03125 and pg.stored_values(code, scale, zero, 32, dtype)[0, 0, 2] == 3.015625
    slots = s["slots"][0]
    live = (slots >= 0) & (slots < s["pool"].shape[0] * page)
    assert int(live.sum()) == n - 2
    for name, v in zip(("K_back.bin", "V_back.bin"), values):
        got = torch.from_numpy(np.fromfile(str(tmp_path / name), np.uint8)).view(dtype).view(n, 128)
        assert torch.equal(got[live].view(torch.int16), v[live].contiguous().view(torch.int16))
    rb, want = 128 * bits // 8, s["pool"].clone()                        # [pages, 1, 2, bytes]
    block = pg.block_of_codes(code[:, :, None], scale[:, :, None], zero[:, :, None], bits)      # a block of one row each
    for i, slot in enumerate(slots.tolist()):
        if live[i]:
            p, row = slot // page, slot % page
            want[p, 0, :, row * rb:(row + 1) * rb] = block[:, i, :rb]
            want[p, 0, :, page * rb:].view(2, 4, page, 4)[:, :, row] = block[:, i, rb:].view(2, 4, 4)
    after = torch.from_numpy(np.fromfile(str(tmp_path / "pool_after.bin"), np.uint8)).view(want.shape)
    assert torch.equal(after, want)


def test_bytes_of_the_tensors_that_are_read(emulator, tmp_path):
    """Rows are stored past the caches from a number of bytes on (32 KB in the stand-in), of Keys and Values together where both are brought back: each of
    the two reads here brings back one, of 79 rows and 20 KB, or of 128 and 32."""
    for rows, past in ((79, False), (128, True)):
        d = tmp_path / str(rows)
        d.mkdir()
        make_inputs(Case("past", F16, 8, 64, 16, 1, 1, [(0, rows)], write=True), str(d))
        r = subprocess.run([emulator, str(d)], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
        assert r.returncode == 0, r.stderr[-2000:]
        reads = re.findall(r"^launch page_copy_kernel<BITS, BF, WRITE, (\S+)>", r.stderr, re.M)
        assert reads == ["false"] + ["!WRITE" if past else "false"] * 2, r.stderr[-2000:]
