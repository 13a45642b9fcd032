"""Rotary positions, page tables and shared prefixes, compiled as plain C++ against the CPU stand-in for the HIP device environment in
tests/simt/ and run under the address sanitizer on buffers of exactly their size, against the definitions."""
import os
import random
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import page_util as pg
from tests import serving_util as sv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIMT = os.path.join(ROOT, "tests", "simt")
CSRC, PAGES, SERVING = (os.path.join(ROOT, "paper_2403_05527_amd", d) for d in ("csrc", "csrc_pages", "csrc_serving"))
SOURCES = [(PAGES, s) for s in ("page_api", "page_copy", "page_few", "page_many", "page_mixed")] + \
          [(SERVING, s) for s in ("rope_api", "rope", "table_api", "table", "shared_api", "shared")]
F16, BF16 = torch.float16, torch.bfloat16
LAUNCHED = set()


@pytest.fixture(scope="module")
def emulator(tmp_path_factory):
    cxx = next((c for c in ("/opt/rocm/llvm/bin/clang++", shutil.which("clang++")) if c and os.path.exists(c)), None)
    if cxx is None:
        pytest.skip("no clang++ to build the CPU emulation")
    out = tmp_path_factory.mktemp("simt_serving")
    flags = ["-std=c++17", "-O1", "-gline-tables-only", "-fsanitize=address", "-fno-omit-frame-pointer", "-pthread", "-include", os.path.join(SIMT, "serving_env.h"),
             "-I", SIMT, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", PAGES, "-I", SERVING]
    procs = []
    for folder, s in SOURCES + [(SIMT, "simt_rt"), (SIMT, "run_serving")]:
        src = ["-c", os.path.join(folder, s + ".cpp")] if folder == SIMT else ["-x", "c++", "-c", os.path.join(folder, s + ".hip")]
        procs.append((str(out / (s + ".o")), subprocess.Popen([cxx] + src + ["-o", str(out / (s + ".o"))] + flags, stderr=subprocess.PIPE, text=True)))
    for _, p in procs:
        err = p.communicate()[1]
        assert p.returncode == 0, err[-3000:]
    exe = str(out / "run_serving")
    r = subprocess.run([cxx] + [o for o, _ in procs] + ["-o", exe] + flags, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


def run(emulator, d, blocks, calls, results):
    """The blocks after the calls: {name: tensor like the one that went in}."""
    for name, t in blocks.items():
        with open(os.path.join(d, name + ".bin"), "wb") as f:
            if t.numel():
                f.write(t.contiguous().view(torch.uint8).numpy().tobytes())
    with open(os.path.join(d, "calls.txt"), "w") as f:
        f.write("\n".join(["load " + n for n in blocks] + calls + ["save " + n for n in results]) + "\n")
    r = subprocess.run([emulator, d], capture_output=True, text=True, timeout=900, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    LAUNCHED.update(re.findall(r"^launch (\w+)", r.stderr, re.M))
    return {n: torch.from_numpy(np.fromfile(os.path.join(d, n + ".out"), np.uint8)).view(blocks[n].dtype).view(blocks[n].shape) for n in results}


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


# rot, interleaved, inverse, factor, dtype, sequences, tokens, heads, heads first, in place
TURNS = [(128, 0, 0, 1.0, F16, 2, 19, 2, True, False), (128, 1, 1, 1.0, BF16, 1, 17, 3, False, True), (64, 0, 0, 1.2, F16, 3, 1, 2, False, True),
         (50, 0, 1, 1.0, F16, 1, 5, 2, False, True), (50, 1, 0, 0.5, BF16, 1, 5, 1, True, False), (2, 0, 0, 1.0, F16, 1, 3, 1, False, False)]


@pytest.mark.parametrize("case", range(len(TURNS)))
def test_rows_are_turned(emulator, tmp_path, case):
    rot, inter, inv, factor, dtype, S, n, H, first, in_place = TURNS[case]
    gen = torch.Generator().manual_seed(case)
    x = torch.randn(S, n, H, 128, generator=gen).to(dtype)
    pos = torch.randint(-9, 1 << 20, (S, n), generator=gen)
    freq = sv.frequencies(rot)
    held = x.transpose(1, 2).contiguous() if first else x.clone()
    strides = "%d 128 %d" % (n * H * 128, n * 128) if first else "%d %d 128" % (n * H * 128, H * 128)
    blocks = dict(x=held, out=torch.full_like(held, 7.0), pos=pos, freq=freq)
    calls = ["rope %d %d %d %r freq" % (rot, inter, inv, factor), "rows a x 0 " + strides, "rows b %s 0 %s" % ("x" if in_place else "out", strides),
             "rotate %d a b %d %d %d pos" % (pg.DTYPES.index(dtype), S, n, H)]
    got = run(emulator, str(tmp_path), blocks, calls, ["x" if in_place else "out"])["x" if in_place else "out"]
    got = got.transpose(1, 2) if first else got
    y, bound = sv.rotate(x, pos, freq, inter, inv, torch.tensor(factor, dtype=torch.float32).item())
    assert sv.is_close(got, y, bound) <= 1.0
    assert same_bits(got[..., rot:], x[..., rot:])


WRITES = [(F16, 16, 128, 16, 2, 2, 2, 19, 128, 0), (BF16, 8, 32, 16, 1, 3, 1, 17, 64, 0), (F16, 8, 64, 32, 2, 1, 3, 1, 128, 1), (F16, 4, 128, 16, 1, 0, 1, 18, 50, 0),
          (BF16, 4, 32, 16, 3, 1, 1, 4, 128, 0)]


@pytest.mark.parametrize("case", range(len(WRITES)))
def test_turned_rows_are_written(emulator, tmp_path, case):
    """Bit for bit what gear_rotate and gear_page_write make of them."""
    dtype, bits, group, page, H, gq, S, n, rot, inter = WRITES[case]
    gen = torch.Generator().manual_seed(case + 40)
    n_pages, Hq = S * (-(-n // page)) + 2, H * gq
    qkv = torch.randn(S, n, Hq + 2 * H, 128, generator=gen).to(dtype)
    pos = torch.randint(0, 100000, (S, n), generator=gen)
    slots = torch.randperm(n_pages * page, generator=gen)[:S * n].view(S, n)
    if S * n > 2:
        slots[0, 0], slots[-1, -1] = -1, n_pages * page
    pool = torch.randint(0, 255, (n_pages * H * 2 * pg.block_bytes(bits, group, page),), generator=gen, dtype=torch.int32).to(torch.uint8)
    q_out = torch.full((S, n, max(Hq, 1), 128), 3.0, dtype=dtype)
    turned = torch.zeros(S, n, H, 128, dtype=dtype)
    blocks = dict(qkv=qkv, pool=pool, pool2=pool.clone(), q_out=q_out, q_out2=q_out.clone(), turned=turned, pos=pos, slots=slots, freq=sv.frequencies(rot))
    w = (Hq + 2 * H) * 128
    part = lambda name, h: "rows %s qkv %d %d %d 128" % (name, h * 128, n * w, w)  # noqa: E731
    whole = lambda name, b, h: "rows %s %s 0 %d %d 128" % (name, b, n * h * 128, h * 128)  # noqa: E731
    calls = ["config %d %d %d %d %d %d" % (n_pages, page, H, bits, group, pg.DTYPES.index(dtype)), "rope %d %d 0 1.0 freq" % (rot, inter),
             part("q", 0), part("K", Hq), part("V", Hq + H), whole("o", "q_out", Hq), whole("o2", "q_out2", Hq), whole("t", "turned", H),
             "write_rope pool K V %s %d %d %d slots pos" % ("q o" if Hq else "- -", Hq, S, n),
             "rotate %d K t %d %d %d pos" % (pg.DTYPES.index(dtype), S, n, H), "write pool2 t V %d %d slots" % (S, n)]
    if Hq:
        calls.append("rotate %d q o2 %d %d %d pos" % (pg.DTYPES.index(dtype), S, n, Hq))
    got = run(emulator, str(tmp_path), blocks, calls, ["pool", "pool2", "q_out", "q_out2", "turned"])
    assert torch.equal(got["pool"], got["pool2"]) and same_bits(got["q_out"], got["q_out2"])
    y, bound = sv.rotate(qkv[:, :, Hq:Hq + H], pos, blocks["freq"], inter)
    assert sv.is_close(got["turned"], y, bound) <= 1.0


def script(seed, page, n_pages, n_rows, width, steps, most=70, rows_of_list=None):
    """A model's table after random calls, and the calls."""
    r, t, blocks, calls, checks = random.Random(seed), sv.Table(n_pages, page, n_rows, width), {}, [], []
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    blocks.update(table=i32(t.table), kv=i32(t.kv), refs=i32(t.refs))
    calls.append("table table kv refs %d %d %d %d" % (n_pages, page, n_rows, width))
    for k in range(steps):
        op = r.choice(("extend", "extend", "extend", "truncate", "fork", "compact"))
        n = r.randint(1, rows_of_list or n_rows + 2)
        a, b = [[r.randint(-1, n_rows) for _ in range(n)] for _ in range(2)]
        A, B, C, E, F = ("%s%d" % (x, k) for x in "abcef")
        if op == "compact":
            m = r.choice((n_pages, 2, 0))
            blocks[A], blocks[B] = torch.full((m, 2), 9, dtype=torch.int32), i32([0, 0])
            calls.append("compact %s %d %s" % (A if m else "-", m, B))
            want = t.compact(m)
            checks += [(A, want[0])] * (m > 0) + [(B, want[1])]
        elif op == "extend":
            m = r.choice((1, 1, most))
            counts = [r.choice((1, 1, m, r.randint(0, m), -1, m + 1)) for _ in range(n)]
            blocks[A], blocks[B] = i32(a), i32(counts)
            blocks[C], blocks[E], blocks[F] = torch.full((n, m), 9), torch.full((n, 2), 9, dtype=torch.int32), torch.full((n,), 9, dtype=torch.int32)
            calls.append("extend %s %s %d %d %s %s %s" % (A, B, n, m, C, E, F))
            checks += list(zip((C, E, F), t.extend(a, counts, m)))
        elif op == "fork":
            blocks[A], blocks[B] = i32(a), i32(b)
            calls.append("fork %s %s %d" % (A, B, n))
            t.fork(a, b)
        else:
            lens = [r.choice((0, r.randint(0, width * page), -3)) for _ in range(n)]
            blocks[A], blocks[B] = i32(a), i32(lens)
            calls.append("truncate %s %s %d" % (A, B, n))
            t.truncate(a, lens)
        assert t.consistent()
    return t, blocks, calls, checks


@pytest.mark.parametrize("seed", range(6))
def test_tables_follow_the_definition(emulator, tmp_path, seed):
    page, n_pages, n_rows, width = [(16, 40, 6, 9), (16, 13, 5, 6), (32, 30, 4, 40), (16, 5000, 3, 7), (64, 9, 3, 3), (16, 7, 9, 2)][seed]
    t, blocks, calls, checks = script(seed, page, n_pages, n_rows, width, 10)
    got = run(emulator, str(tmp_path), blocks, calls, ["table", "kv", "refs"] + [n for n, _ in checks])
    for name, want in checks + [("table", t.table), ("kv", t.kv), ("refs", t.refs)]:
        assert got[name].tolist() == want, name


def test_many_slots_have_a_launch_of_their_own(emulator, tmp_path):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    t = sv.Table(700, 16, 3, 400)
    blocks = dict(table=i32(t.table), kv=i32(t.kv), refs=i32(t.refs), rows=i32([2, 0, 5]), counts=i32([5000, 6001, 1]), slots=torch.full((3, 6001), 9),
                  copies=torch.full((3, 2), 9, dtype=torch.int32), refused=i32([9, 9, 9]))
    want = t.extend([2, 0, 5], [5000, 6001, 1], 6001)
    got = run(emulator, str(tmp_path), blocks, ["table table kv refs 700 16 3 400", "extend rows counts 3 6001 slots copies refused"], ["slots", "copies", "refused", "table"])
    for name, w in zip(("slots", "copies", "refused", "table"), want + (t.table,)):
        assert got[name].tolist() == w, name


def test_pages_are_moved(emulator, tmp_path):
    gen = torch.Generator().manual_seed(3)
    for k, (bits, group, page, H, n_pools, gap) in enumerate([(16, 128, 32, 3, 2, 48), (4, 64, 16, 1, 1, 0), (8, 32, 16, 2, 3, 0)]):
        n_pages, size = 6, H * 2 * pg.block_bytes(bits, group, page)
        stride = n_pages * size + gap
        pool = torch.randint(0, 255, ((n_pools - 1) * stride + n_pages * size,), generator=gen, dtype=torch.int32).to(torch.uint8)
        pairs = torch.tensor([[5, 0], [-1, -1], [3, 1], [6, 2], [2, 6], [4, 4]], dtype=torch.int32)
        d = tmp_path / str(k)
        d.mkdir()
        got = run(emulator, str(d), dict(pool=pool, pairs=pairs), ["config %d %d %d %d %d 0" % (n_pages, page, H, bits, group),
                                                                   "move pool %d %d pairs 6" % (n_pools, stride)], ["pool"])["pool"]
        want = pool.clone()
        for i in range(n_pools):
            p = want[i * stride:i * stride + n_pages * size].view(n_pages, size)
            p[0], p[1] = p[5].clone(), p[3].clone()
        assert torch.equal(got, want)


# dtype, bits, group, page, H, gq, groups (shared tokens, sequences (new tokens, own tokens)), causal, padding rows, other bounds
SHARED = {
    "few_columns": (F16, 16, 128, 16, 2, 2, [(100, [(1, 5), (1, 40), (1, 1)])], 1, 0, {}),
    "many_columns": (BF16, 16, 128, 16, 1, 8, [(200, [(1, 9)] * 6), (70, [(1, 33)])], 1, 2, {}),
    "codes_8": (F16, 8, 64, 32, 1, 4, [(0, [(1, 20)]), (150, [(2, 30)] * 5), (64, [(1, 1)] * 2)], 1, 0, {}),
    "codes_4_two_tiles": (F16, 4, 32, 16, 1, 4, [(130, [(5, 6)] * 4), (0, [(6, 90)])], 0, 1, {}),
    "many_behind": (F16, 16, 128, 16, 1, 4, [(150, [(9, 12), (20, 40), (9, 9)])], 1, 0, {}),
    "mixed_behind": (BF16, 8, 128, 16, 1, 2, [(130, [(1, 12), (40, 50), (1, 9), (1, 60)] + [(1, 3)] * 6)], 1, 0, {}),
    "prefix_no_one_sees": (F16, 16, 128, 16, 1, 2, [(90, [(1, 5), (1, 9)])], 1, 0, dict(prefix=[200])),
    "divided": (F16, 16, 128, 16, 1, 4, [(1100, [(1, 300), (1, 20)])], 1, 0, {}),
    "divided_many": (F16, 4, 64, 16, 1, 4, [(900, [(1, 30)] * 9)], 1, 0, {}),
    "many_groups": (F16, 16, 128, 16, 1, 1, [(64 + g % 3, [(1, 2 + g % 4)] * (1 + (g % 2))) for g in range(66)], 1, 0, {}),
    "many_groups_many_columns": (BF16, 16, 128, 16, 1, 17, [(64 + g % 3, [(1, 2 + g % 4)] * (1 + (g % 2))) for g in range(66)], 1, 0, {}),
    "merge_of_many_parts": (F16, 8, 32, 16, 1, 1, [(2600, [(1, 30)] * 3)], 1, 0, {}),
}


@pytest.mark.parametrize("name", list(SHARED))
def test_shared_prefixes(emulator, tmp_path, name):
    dtype, bits, group, page, H, gq, groups, causal, pad, other = SHARED[name]
    gen = torch.Generator().manual_seed(len(name))
    n_pages = sum(-(-(s + o) // page) + 1 for s, seqs in groups for _, o in seqs) + 1
    q_start, kv, table, group_start, prefix, copies = sv.shared_table(page, groups, n_pages, gen)
    prefix = other.get("prefix", prefix)
    x = torch.randn(2, n_pages, H, page, 128, generator=gen)
    x[..., 3] *= 6.0
    pool = torch.stack([pg.pack(t.to(dtype), bits, group, dtype) for t in x], 2)
    for a, b in copies:
        pool[b] = pool[a]
    K, V = (pg.unpack(pool[:, :, w].contiguous(), bits, group, dtype, page) for w in (0, 1))
    T = q_start[-1] + pad
    q = torch.randn(T, H * gq, 128, generator=gen).to(dtype)
    out = torch.full(q.shape, 77.0, dtype=dtype)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    blocks = dict(pool=pool, q=q, out=out, q_start=i32(q_start), kv=i32(kv), table=table, group_start=i32(group_start), prefix=i32(prefix))
    most = max(q_start[b] - q_start[a] for a, b in zip(group_start, group_start[1:]))
    calls = ["config %d %d %d %d %d %d" % (n_pages, page, H, bits, group, pg.DTYPES.index(dtype)), "rows q q 0 0 %d 128" % (H * gq * 128), "rows o out 0 0 %d 128" % (H * gq * 128),
             "shared pool %d %r %d %d %d %d %d %d q_start kv table %d %d %d group_start prefix q o" % (
                 H * gq, 128 ** -0.5, causal, len(kv), T, max(b - a for a, b in zip(q_start, q_start[1:])), max(kv), table.shape[1], len(prefix), most, max(prefix))]
    got = run(emulator, str(tmp_path), blocks, calls, ["out"])["out"].double()
    want, bound = pg.attend(q, K, V, q_start, kv, table.tolist(), 128 ** -0.5, causal)
    dead = torch.isnan(want)
    assert bool((got[dead] == 77.0).all())
    assert sv.is_close(got[~dead], want[~dead], bound[~dead]) <= 1.0


def test_every_kernel_ran(request):
    names = {"test_rows_are_turned": len(TURNS), "test_turned_rows_are_written": len(WRITES), "test_tables_follow_the_definition": 6, "test_many_slots_have_a_launch_of_their_own": 1,
             "test_pages_are_moved": 1, "test_shared_prefixes": len(SHARED)}
    for n, count in names.items():
        if sum(getattr(i, "originalname", i.name) == n and "serving" in str(i.fspath) for i in request.session.items) < count:
            pytest.skip("not all cases were selected")
    kernels = set()
    for f in sorted(os.listdir(SERVING)):
        with open(os.path.join(SERVING, f)) as src:
            kernels |= set(re.findall(r"__global__(?:\s+__launch_bounds__\((?:[^()]|\([^()]*\))*\))?\s+void\s+(\w+)\(", src.read()))
    assert len(kernels) >= 8 and kernels <= LAUNCHED, kernels - LAUNCHED
