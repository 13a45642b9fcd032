"""How gear_page_attn_shared divides its work and when it shares: the entry points compiled for the host with the device's 256 CUs, and launches that print
what they are given (tests/simt/plan_shared.cpp).  Which sequence has how many keys is known on the device alone: what a batch's blocks are is worked out here."""
import os
import subprocess

import pytest

from tests.test_cpu_emulation_pages import CSRC, PAGES, ROOT, SIMT, find_clang

SERVING = os.path.join(ROOT, "paper_2403_05527_amd", "csrc_serving")


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    cxx = find_clang()
    if cxx is None:
        pytest.skip("no clang++ for the host build")
    exe = str(tmp_path_factory.mktemp("plan") / "plan_shared")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-DGEAR_PAGE_CUS=256", "-pthread", "-include", os.path.join(SIMT, "serving_env.h"), "-I", SIMT, "-I", os.path.join(ROOT, "include"),
                        "-I", CSRC, "-I", PAGES, "-I", SERVING, os.path.join(SIMT, "plan_shared.cpp"), os.path.join(SIMT, "simt_rt.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


def sequences(*groups):
    """(shared tokens, [(new tokens, own tokens) of every sequence]); None shared: in no group."""
    return groups


def call(H, gq, bits, groups, always=1):
    seqs = [(n, (shared or 0) + own) for shared, g in groups for n, own in g]
    real = [(shared, sum(n for n, _ in g)) for shared, g in groups if shared is not None]
    return (H, gq, bits, len(seqs), sum(n for n, _ in seqs), max(n for n, _ in seqs), max(k for _, k in seqs), len(real), max(n for _, n in real), max(s for s, _ in real), always)


def plans(planner, calls):
    r = subprocess.run([planner], input="\n".join(" ".join(map(str, c)) for c in calls) + "\n", capture_output=True, text=True, timeout=60)
    lines = r.stdout.split("\n")[:-1]
    assert r.returncode == 0 and len(lines) == len(calls), (r.stdout, r.stderr)
    out = []
    for line in lines:
        w = line.split()
        out.append((w[0], None) if w[0] != "shared" else (w[0], dict(zip(("prefix", "few", "many"), [dict(zip(("n_split", "least", "few", "blocks"), map(int, w[i:i + 4]))) for i in (1, 5, 9)]),
                                                                     records=int(w[13]))))
    return out


def part_length(keys, kind, unit):
    n = min(max((keys + kind["least"] // 2) // kind["least"], 1), kind["n_split"])
    return -(-(-(-keys // n)) // unit) * unit


def behind(groups):
    """(new tokens, keys behind the prefix as it counts) of every sequence."""
    for shared, g in groups:
        counts = min([(shared or 0)] + [(shared or 0) + own - n for n, own in g]) // 64 * 64
        for n, own in g:
            yield n, (shared or 0) + own - counts


def longest(plan, gq, groups):
    """The longest block behind the prefixes in us: 2 us per 128 keys with few columns, 1.5 per 64 with many (what the kernels' blocks take that have a CU to themselves)."""
    few, many = plan["few"], plan["many"]
    most = 0.0
    for n, keys in behind(groups):
        if few["few"] and n <= few["few"] and n * gq <= few["few"]:
            most = max(most, 2.0 * -(-part_length(keys, few, 32) // 128))
        else:
            most = max(most, 1.5 * -(-part_length(keys, many, 64) // 64))
    return most


# batches, and what gear_page_attn took for them, us (8 KV heads, 4 query heads each, bf16, pages of 64)
FEW = {
    "one by itself": (sequences((16000, [(1, 20)] * 16), (None, [(1, 16000)])), 121),
    "a short prefix": (sequences((32000, [(1, 100)] * 8), (500, [(1, 31000)] * 8)), 241),
    "two by themselves": (sequences((32000, [(1, 100)] * 6), (None, [(1, 32000)] * 2)), 127),
    "unequal prefixes": (sequences((1000, [(1, 7300)] * 4), (8192, [(1, 100)] * 4)), 43),
    "half by themselves": (sequences((8200, [(1, 100)] * 8), (None, [(1, 8300)] * 8)), 66),
    "one of 64": (sequences((8192, [(1, 550)] * 63), (None, [(1, 9000)])), 169),
    "a few tokens each": (sequences((4000, [(5, 200)] * 12), (None, [(5, 4000)] * 4)), 47),
}

MANY = {
    "two chunks": (sequences((1000, [(64, 50000)] * 2)), 180),
    "a chunk beside single tokens": (sequences((2000, [(512, 30000)] + [(1, 30000)] * 15)), 620),
    "a long question": (sequences((6100, [(40, 60)] * 15 + [(40, 30000)])), 407),
}


@pytest.mark.parametrize("name", list(FEW) + list(MANY))
def test_what_lies_behind_is_divided_by_its_own_length(planner, name):
    """No block behind the prefixes takes longer than gear_page_attn for the whole batch, whichever sequence the longest is."""
    groups, plain = FEW.get(name) or MANY[name]
    (kind, plan), = plans(planner, [call(8, 4, 16, groups)])
    assert kind == "shared"
    assert longest(plan, 4, groups) <= plain, plan


# batches, and us shared and not
CHOICE = {
    "samples": (32, 1, 16, sequences((2077, [(1, 64)] * 16)), 18, 47),
    "a system prompt": (8, 4, 16, sequences((8192, [(1, 550)] * 64)), 48, 165),
    "unequal groups": (8, 4, 8, sequences(*[(p, [(1, 700)] * 10) for p in (1500, 6001, 3000, 5200, 2222)]), 39, 83),
    "questions": (8, 4, 16, sequences((6100, [(n, n) for n in range(20, 61, 3)])), 90, 127),
    "one by itself": (8, 4, 16, sequences((16000, [(1, 20)] * 16), (None, [(1, 16000)])), 62, 120),
    "two by themselves": (8, 4, 16, sequences((32000, [(1, 100)] * 6), (None, [(1, 32000)] * 2)), 99, 127),
    "one of 64 by itself": (8, 4, 16, sequences((8192, [(1, 550)] * 63), (None, [(1, 9000)])), 88, 168),
    "eight of 32 by themselves": (8, 4, 8, sequences((6001, [(1, 400)] * 24), (None, [(1, 6000)] * 8)), 42, 53),
    "three groups of one length": (8, 4, 16, sequences(*[(4096, [(1, 200)] * 4)] * 3), 22, 31),
    "four": (8, 4, 16, sequences(*[(4096, [(1, 200)] * 3)] * 4), 24, 32),
    "three of 24": (8, 4, 16, sequences(*[(2048, [(1, 200)] * 8)] * 3), 21, 28),
    "four of 24": (8, 4, 16, sequences(*[(2048, [(1, 200)] * 6)] * 4), 22, 28),
    "eight of 24": (8, 4, 16, sequences(*[(2048, [(1, 200)] * 3)] * 8), 24, 28),
    "questions by themselves": (8, 4, 16, sequences((6100, [(40, 60)] * 14), (None, [(40, 6000)] * 2)), 147, 105),
    "a question by itself": (8, 4, 16, sequences((6100, [(40, 900)] * 15), (None, [(40, 6500)])), 155, 112),
}


@pytest.mark.parametrize("name", list(CHOICE))
def test_prefixes_are_shared_where_that_is_faster(planner, name):
    H, gq, bits, groups, shared, plain = CHOICE[name]
    (kind, _), = plans(planner, [call(H, gq, bits, groups, always=0)])
    assert kind == ("shared" if shared < plain else "plain")


def test_usual_batches_keep_their_parts(planner):
    """Where nobody has more behind the prefix than the longest sequence has behind the longest prefix, one part each, as blocks that begin at once."""
    usual = [(32, 1, 16, sequences((2077, [(1, 64)] * 16))), (8, 4, 16, sequences((8192, [(1, 1000)] * 64))), (8, 4, 8, sequences(*[(p, [(1, 700)] * 10) for p in (1500, 6001, 3000, 5200, 2222)]))]
    usual += [(8, 4, 16, sequences((6100, [(n, n) for n in range(20, 60, 3)])))]
    for H, gq, bits, groups in usual:
        (kind, plan), = plans(planner, [call(H, gq, bits, groups)])
        which, unit = ("few", 32) if all(n * gq <= 32 for n, _ in behind(groups)) else ("many", 64)
        assert kind == "shared" and all(part_length(keys, plan[which], unit) >= keys for _, keys in behind(groups))


def test_blocks_and_records_stay_bounded(planner):
    calls = [(H, gq, 16, seqs, seqs * q, q, kv, 1, seqs * q, prefix, 1)
             for H, gq in ((1, 1), (8, 4), (32, 1), (8, 8)) for seqs in (1, 3, 64, 900, 30000) for q in (1, 4, 40, 700) for kv in (1, 1500, 40000, 2 ** 30) for prefix in (64, 1000, 39000) if seqs * q < 50000]
    calls += [(8, 4, 16, 400000, 40, 40, 40000, 1, 40, prefix, 1) for prefix in (64, 39000)]                # all but a few without new tokens
    for c, (kind, plan) in zip(calls, plans(planner, calls)):
        H, gq, _, seqs, tokens = c[:5]
        assert kind in ("shared", "plain")
        if plan:
            rows = tokens * H * gq
            assert rows * plan["records"] <= 2 * max(rows, 768 * 128) and plan["few"]["blocks"] <= max(seqs * H, 1024) and plan["many"]["blocks"] <= max((tokens * gq // 128 + seqs) * H, 4096), (c, plan)
