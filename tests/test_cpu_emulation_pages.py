"""The paged cache's kernels and entry points, compiled as plain C++ against the CPU stand-in for the HIP device environment in
tests/simt/ and run under the address sanitizer on buffers of exactly their size, against the definition in 64 bits."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

from tests import page_util as pg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIMT = os.path.join(ROOT, "tests", "simt")
CSRC = os.path.join(ROOT, "paper_2403_05527_amd", "csrc")
PAGES = os.path.join(ROOT, "paper_2403_05527_amd", "csrc_pages")
SOURCES = ["page_api", "page_copy", "page_few", "page_many", "page_mixed"]


def find_clang():
    for c in ("/opt/rocm/llvm/bin/clang++", shutil.which("clang++")):
        if c and os.path.exists(c):
            return c
    return None


@pytest.fixture(scope="module")
def emulator(tmp_path_factory):
    cxx = find_clang()
    if cxx is None:
        pytest.skip("no clang++ to build the CPU emulation")
    out = tmp_path_factory.mktemp("simt_pages")
    flags = ["-std=c++17", "-O1", "-gline-tables-only", "-fsanitize=address", "-fno-omit-frame-pointer", "-pthread",
             "-I", SIMT, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", PAGES]
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


class Case:
    """Sequences of (new tokens, tokens in all); odd: pages out of range in the table, garbage in every slot that no sequence has."""

    def __init__(self, name, dtype, bits, group, page, H, gq, seqs, causal=True, scale=None, max_kv=None, pad=0, bad=False, write=False, slots=None):
        self.__dict__.update(locals())
        self.scale = 128 ** -0.5 if scale is None else scale


F16, BF16 = torch.float16, torch.bfloat16
CASES = [
    Case("one", F16, 16, 128, 16, 2, 1, [(1, 1)]),
    Case("few_f16", F16, 16, 128, 16, 2, 2, [(1, 77), (1, 0), (1, 200)], bad=True),
    Case("few_8", F16, 8, 64, 32, 1, 4, [(3, 45), (0, 20), (2, 33)], pad=2),
    Case("few_4", F16, 4, 32, 16, 3, 1, [(1, 97)], bad=True),
    Case("few_bf16", BF16, 16, 128, 64, 1, 5, [(6, 90)]),
    Case("few_bf16_8_two_tiles", BF16, 8, 32, 16, 1, 8, [(4, 70), (1, 130)], bad=True),
    Case("few_bf16_4", BF16, 4, 128, 16, 1, 3, [(2, 50)], causal=False),
    Case("few_split", F16, 8, 128, 16, 1, 2, [(1, 1100), (1, 30)], max_kv=1100),
    Case("empty_rows", F16, 16, 128, 16, 1, 2, [(9, 4), (1, 0)]),
    Case("many_f16", F16, 16, 128, 16, 1, 2, [(40, 140), (33, 33)], bad=True),
    Case("many_8", F16, 8, 32, 16, 1, 1, [(150, 150)], pad=3),
    Case("many_4", F16, 4, 64, 32, 1, 4, [(35, 100)], causal=False),
    Case("many_bf16", BF16, 16, 128, 128, 1, 3, [(50, 70)]),
    Case("many_bf16_8", BF16, 8, 128, 16, 2, 1, [(40, 75)]),
    Case("many_bf16_4", BF16, 4, 32, 16, 1, 1, [(34, 131)], bad=True),
    Case("many_split", F16, 16, 128, 64, 1, 1, [(36, 1100)], max_kv=1100),
    Case("mixed", F16, 8, 64, 16, 1, 4, [(1, 60), (50, 90), (0, 0), (3, 30)], pad=1),
    Case("mixed_two_launches", F16, 16, 128, 16, 1, 2, [(1, 60), (33, 90), (2, 30)], max_kv=1000000),
    Case("mixed_two_tiles", BF16, 4, 64, 16, 1, 20, [(1, 40), (3, 50)], bad=True),
    Case("merge_many_parts", F16, 4, 32, 16, 1, 1, [(33, 1300)], max_kv=1300),
    Case("many_sequences", F16, 8, 128, 16, 1, 1, [(1 + 33 * (i == 5), 17 + i % 3 + 33 * (i == 5)) for i in range(66)]),
    Case("empty_many", F16, 16, 128, 16, 1, 1, [(70, 20)]),
    Case("negative_scale", BF16, 16, 128, 16, 1, 2, [(1, 40), (40, 60)], scale=-0.05),
    Case("write_f16", F16, 16, 128, 16, 2, 1, [(0, 19)], write=True),
    Case("write_8_32", F16, 8, 32, 16, 2, 1, [(0, 19), (0, 19)], write=True),
    Case("write_8_64", BF16, 8, 64, 32, 1, 1, [(0, 33)], write=True),
    Case("write_8_128", F16, 8, 128, 16, 1, 1, [(0, 16)], write=True),
    Case("write_4_32", BF16, 4, 32, 16, 1, 1, [(0, 40)], write=True),
    Case("write_4_64", F16, 4, 64, 64, 3, 1, [(0, 1)], write=True),
    Case("write_4_128", F16, 4, 128, 16, 1, 1, [(0, 17)], write=True),
]
BY_NAME = {c.name: c for c in CASES}


def rows_of(gen, shape, dtype):
    x = torch.randn(shape, generator=gen, dtype=torch.float64)
    x[..., 3] *= 12.0
    x.view(-1, 128)[9::17] = 0.25   # (rows of equal values: scale 0)
    return x.to(dtype)


def make_inputs(c, d):
    gen = torch.Generator().manual_seed(len(c.name) + 7 * c.bits)
    width = max(1, max(-(-kv // c.page) for _, kv in c.seqs))
    S, used = len(c.seqs), len(c.seqs) * width
    n_pages = used + 1
    table = torch.randperm(n_pages, generator=gen)[:used].to(torch.int32).view(S, width)
    K, V = (rows_of(gen, (n_pages, c.H, c.page, 128), c.dtype) for _ in range(2))
    pool = torch.stack([pg.pack(x, c.bits, c.group, c.dtype) for x in (K, V)], 2)                 # [pages, H, 2, bytes]
    K, V = (pg.unpack(pool[:, :, w].contiguous(), c.bits, c.group, c.dtype, c.page) for w in (0, 1))
    q_start = [c.pad]
    for n, _ in c.seqs:
        q_start.append(q_start[-1] + n)
    T = q_start[-1] + c.pad
    q = torch.randn((T, c.H * c.gq, 128), generator=gen).to(c.dtype)
    kv = [n for _, n in c.seqs]
    shown = table.clone()
    if c.bad:
        # slots that no sequence has hold NaN patterns and infinities; one page of the longest sequence is out of range
        held = torch.zeros(n_pages, c.page, dtype=torch.bool)
        for s, (_, n) in enumerate(c.seqs):
            for p in range(n):
                held[table[s, p // c.page], p % c.page] = True
        raw = pool.numpy()
        rb = 128 * c.bits // 8
        for p in range(n_pages):
            for r in range(c.page):
                if not held[p, r]:
                    raw[p, :, :, r * rb:(r + 1) * rb] = 0xFF
                    words = raw[p, :, :, c.page * rb:].reshape(c.H, 2, -1, c.page, 4) if c.bits < 16 else None
                    if words is not None:
                        words[:, :, :, r] = np.frombuffer(np.uint16([0x7C00, 0xFFFF]).tobytes(), np.uint8)
                        raw[p, :, :, c.page * rb:] = words.reshape(c.H, 2, -1)
        longest = max(range(S), key=lambda i: kv[i])
        if kv[longest] > 2 * c.page:
            shown[longest, 1] = n_pages if c.gq % 2 else -1
    total = c.seqs[0][1]
    max_q = max(n for n, _ in c.seqs)
    T = 0 if c.write else T
    w = lambda name, t: t.contiguous().view(torch.uint8).numpy().tofile(os.path.join(d, name)) if t.numel() else open(os.path.join(d, name), "wb").close()  # noqa: E731
    w("pool.bin", pool)
    out = torch.full(q.shape, 77.0, dtype=c.dtype)
    for name, t in (("q.bin", q), ("q_start.bin", torch.tensor(q_start, dtype=torch.int32)), ("kv_len.bin", torch.tensor(kv, dtype=torch.int32)),
                    ("table.bin", shown), ("out_before.bin", out)):
        w(name, t)
    new = back = slots = None
    if c.write:
        new = [rows_of(gen, (S, total, c.H, 128), c.dtype) for _ in range(2)]
        pos = torch.arange(total)
        slots = table.long()[:, pos // c.page] * c.page + pos % c.page
        if total > 1:
            slots[0, 1] = -1
            slots[-1, -1] = n_pages * c.page
        back = torch.full((S, c.H, total, 128), 55.0, dtype=c.dtype)
        for name, t in (("K.bin", new[0]), ("V.bin", new[1]), ("slots.bin", slots), ("K_before.bin", back), ("V_before.bin", back)):
            w(name, t)
    with open(os.path.join(d, "meta.txt"), "w") as f:
        f.write(" ".join(str(x) for x in [n_pages, c.page, c.H, c.bits, c.group, pg.DTYPES.index(c.dtype), c.H * c.gq, c.scale, int(c.causal), width, S,
                                          total if c.write else 0, T, max_q, c.max_kv or max(kv)]) + "\n")
    return dict(pool=pool, K=K, V=V, q=q, q_start=q_start, kv=kv, table=shown.tolist(), out=out, new=new, slots=slots, back=back)


LAUNCHED = set()


@pytest.fixture(scope="module")
def runs(request, emulator, tmp_path_factory):
    def one(c):
        d = str(tmp_path_factory.mktemp(c.name))
        s = make_inputs(c, d)
        return d, s, subprocess.run([emulator, d], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    names = {i.callspec.params["name"] for i in request.session.items if getattr(i, "originalname", "") == "test_pages_under_address_sanitizer"}
    pool = ThreadPoolExecutor(3)
    return {n: pool.submit(one, BY_NAME[n]) for n in BY_NAME if n in names}


@pytest.mark.parametrize("name", list(BY_NAME))
def test_pages_under_address_sanitizer(runs, name):
    c = BY_NAME[name]
    d, s, r = runs[name].result()
    assert r.returncode == 0 and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    LAUNCHED.update(re.findall(r"^launch (\w+)", r.stderr, re.M))
    load = lambda f, like: torch.from_numpy(np.fromfile(os.path.join(d, f), np.uint8)).view(like.dtype).view(like.shape)  # noqa: E731
    if c.write:
        S, total = s["slots"].shape
        slots = s["slots"]
        live = (slots >= 0) & (slots < s["pool"].shape[0] * c.page)
        for f, x in (("K_back.bin", s["new"][0]), ("V_back.bin", s["new"][1])):
            got = load(f, s["back"])
            want = torch.where(live[:, None, :, None], pg.expected(x, c.bits, c.group, c.dtype).transpose(1, 2), s["back"])
            assert torch.equal(got.view(torch.int16), want.contiguous().view(torch.int16))
        after = load("pool_after.bin", s["pool"])
        touched = torch.zeros(s["pool"].shape[0], c.page, dtype=torch.bool)
        touched.view(-1)[slots[live]] = True
        for w in (0, 1):   # every slot that was not named is as it was, and the pool is what the layout says
            now, was = (pg.unpack(t[:, :, w].contiguous(), c.bits, c.group, c.dtype, c.page) for t in (after, s["pool"]))
            same = now.view(torch.int16) == was.view(torch.int16)
            assert bool(same.all(-1).transpose(1, 2)[~touched].all())
        return
    got = load("out.bin", s["out"]).double()
    want, bound = pg.attend(s["q"], s["K"], s["V"], s["q_start"], s["kv"], s["table"], c.scale, c.causal)
    dead = torch.isnan(want)
    assert bool((got[dead] == 77.0).all())
    assert bool(((got - want).abs() <= bound)[~dead].all()), float(((got - want).abs() / bound)[~dead].max())


def test_every_kernel_ran(request):
    if sum(getattr(i, "originalname", "") == "test_pages_under_address_sanitizer" for i in request.session.items) < len(CASES):
        pytest.skip("not all cases were selected")
    kernels = set()
    for f in sorted(os.listdir(PAGES)):
        with open(os.path.join(PAGES, f)) as src:
            kernels |= set(re.findall(r"__global__(?:\s+__launch_bounds__\((?:[^()]|\([^()]*\))*\))?\s+void\s+(\w+)\(", src.read()))
    assert len(kernels) >= 5 and kernels <= LAUNCHED, kernels - LAUNCHED
