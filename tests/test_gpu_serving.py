"""Rotary positions, page tables and shared prefixes on the GPU, through the binding, against their definitions (tests/serving_util.py,
tests/page_util.py): whole numbers and moved bytes bit for bit, the others to the bound that the declared precisions give."""
import random

import pytest
import torch

from paper_2403_05527_amd import binding as gb
from tests import page_util as pg
from tests import serving_util as sv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16).cpu(), b.contiguous().view(torch.int16).cpu())


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- rotary positions
ROTS = [(128, False), (128, True), (64, False), (96, True), (48, False), (50, False), (50, True), (2, False), (126, False)]


@pytest.mark.parametrize("dtype", (F16, BF16))
@pytest.mark.parametrize("rot,inter", ROTS)
def test_rows_are_turned(rot, inter, dtype):
    gen = torch.Generator().manual_seed(rot)
    freq = sv.frequencies(rot)
    for S, n, H in ((1, 1, 1), (3, 1, 5), (2, 33, 3), (5, 16, 1), (1, 300, 8)):
        x = torch.randn(S, n, H, 128, generator=gen).to(dtype)
        pos = torch.randint(-1000, 1 << 23, (S, n), generator=gen)
        for inverse, factor in ((False, 1.0), (True, 1.25)):
            y, bound = sv.rotate(x, pos, freq, inter, inverse, factor)
            r = gb.make_rope(freq.to(DEV), inter, inverse, factor)
            got = torch.empty(x.shape, dtype=dtype, device=DEV)
            gb.gear_rotate(r, x.to(DEV), got, pos.to(DEV))
            assert sv.is_close(got.cpu(), y, bound) <= 1.0
            assert same_bits(got[..., rot:], x[..., rot:])
            # heads first, out of wider rows, into itself: the same bits
            wide = torch.randn(S, n, H + 3, 128, generator=gen).to(dtype).to(DEV)
            wide[:, :, 2:2 + H] = x.to(DEV)
            before = wide.clone()
            gb.gear_rotate(r, wide[:, :, 2:2 + H], wide[:, :, 2:2 + H], pos.to(DEV))
            assert same_bits(wide[:, :, 2:2 + H], got) and same_bits(wide[:, :, :2], before[:, :, :2]) and same_bits(wide[:, :, 2 + H:], before[:, :, 2 + H:])
            first = torch.empty(S, H, n, 128, dtype=dtype, device=DEV)
            gb.gear_rotate(r, x.to(DEV), first.transpose(1, 2), pos.to(DEV))
            assert same_bits(first.transpose(1, 2), got)


def test_far_positions_turn_as_their_angles_say():
    """|t w| up to 2^31: a cosine or sine is off by 2^-20 (2.5 roundings in 64 bits of 2^28.4 turns are 2^-20.6 rad, and the 2^-22.5 of nearer positions)."""
    freq = torch.ones(64, dtype=torch.float64) * torch.linspace(0.5, 1.0, 64, dtype=torch.float64)
    pos = torch.tensor([[(1 << 31) - 1, -(1 << 31), (1 << 30) + 12345, 1 << 24]])
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(1, 4, 2, 128, generator=gen).to(F16)
    out = torch.empty(x.shape, dtype=F16, device=DEV)
    gb.gear_rotate(gb.make_rope(freq.to(DEV)), x.to(DEV), out, pos.to(DEV))
    y, bound = sv.rotate(x, pos, freq)
    a = x.double().abs()
    far = (a[..., :64] + a[..., 64:]) * 2.0 ** -20
    assert sv.is_close(out.cpu(), y, bound + 1.001 * torch.cat((far, far), -1)) <= 1.0


@pytest.mark.parametrize("inter", (False, True))
def test_the_inverse_is_the_gradient(inter):
    """Of the sum of g y over the rows: by the formula's autograd in 64 bits, and by differences (which are exact of a linear function)."""
    gen = torch.Generator().manual_seed(5)
    freq, pos = sv.frequencies(64), torch.randint(0, 5000, (2, 7), generator=gen)
    x = torch.randn(2, 7, 3, 128, generator=gen, dtype=torch.float64, requires_grad=True)
    g = torch.randn(2, 7, 3, 128, generator=gen).to(F16)
    i, j = (torch.arange(0, 64, 2), torch.arange(1, 64, 2)) if inter else (torch.arange(32), torch.arange(32, 64))
    t = pos.double()[..., None, None] * freq
    a, b = x[..., i], x[..., j]
    turned = x.clone()
    turned[..., i], turned[..., j] = 1.5 * (a * t.cos() - b * t.sin()), 1.5 * (a * t.sin() + b * t.cos())
    (turned * g.double()).sum().backward()
    got = torch.empty(g.shape, dtype=F16, device=DEV)
    gb.gear_rotate(gb.make_rope(freq.to(DEV), inter, True, 1.5), g.to(DEV), got, pos.to(DEV))
    _, bound = sv.rotate(g, pos, freq, inter, True, 1.5)
    bound[..., 64:] = 0.0
    assert sv.is_close(got.cpu(), x.grad, bound + 2.0 ** -40) <= 1.0
    d = torch.zeros(x.shape, dtype=torch.float64)
    d[1, 3, 2, 5] = 1.0
    up, b_up = sv.rotate(d.to(F16), pos, freq, inter, False, 1.5)
    assert abs(float((up * g.double()).sum()) - float(got[1, 3, 2, 5])) <= float(bound[1, 3, 2, 5]) + 2.0 ** -40


FORMS = [(F16, 16, 128), (BF16, 16, 128), (F16, 8, 128), (BF16, 8, 32), (F16, 4, 64), (BF16, 4, 128)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "%s-%d-%d" % (str(f[0])[6:], f[1], f[2]))
@pytest.mark.parametrize("rot,inter", [(128, False), (128, True), (64, False), (50, False)])
def test_turned_rows_are_written(form, rot, inter):
    """Bit for bit what gear_rotate and gear_page_write make of them."""
    dtype, bits, group = form
    gen = torch.Generator().manual_seed(bits)
    r = gb.make_rope(sv.frequencies(rot).to(DEV), inter)
    for S, n, H, gq, page in ((1, 1, 1, 1, 16), (17, 1, 8, 4, 16), (3, 37, 2, 3, 32), (1, 200, 5, 0, 64)):
        n_pages, Hq = S * (-(-n // page)) + 3, H * gq
        cfg = gb.make_page_config(n_pages, page, H, bits, group, dtype)
        qkv = torch.randn(S, n, Hq + 2 * H, 128, generator=gen).to(dtype).to(DEV)
        pos = torch.randint(0, 1 << 20, (S, n), generator=gen).to(DEV)
        slots = torch.randperm(n_pages * page, generator=gen)[:S * n].view(S, n)
        if S * n > 2:
            slots[0, 0], slots[-1, -1] = -1, n_pages * page
        slots = slots.to(DEV)
        a = torch.randint(0, 255, (gb.gear_page_bytes(cfg),), generator=gen, dtype=torch.int32).to(torch.uint8).to(DEV)
        b = a.clone()
        q, K, V = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        out, want = (torch.empty(S, n, Hq, 128, dtype=dtype, device=DEV) for _ in range(2))
        turned = torch.empty(S, n, H, 128, dtype=dtype, device=DEV)
        gb.gear_page_write_rope(cfg, a, r, K, V, slots, pos, *((q, out) if gq else ()))
        gb.gear_rotate(r, K, turned, pos)
        gb.gear_page_write(cfg, b, turned, V, slots)
        if gq:
            gb.gear_rotate(r, q, want, pos)
            assert same_bits(out, want)
        assert torch.equal(a, b)


# ---- page tables
def same_table(t, model):
    return t.table.tolist() == model.table and t.kv_len.tolist() == model.kv and t.refs.tolist() == model.refs


def random_calls(t, model, r, steps, most, longest):
    n_rows, width = len(model.kv), model.width
    for k in range(steps):
        op = r.choice(("extend", "extend", "extend", "truncate", "fork", "compact"))
        n = r.randint(1, longest)
        a, b = [[r.randint(-1, n_rows) for _ in range(n)] for _ in range(2)]
        if r.random() < 0.5:
            a = r.sample(range(n_rows), min(n, n_rows))
            n = len(a)
            b = [r.randint(0, n_rows - 1) for _ in a]
        if op == "compact":
            m = r.choice((len(model.refs), 3))
            got = [x.tolist() for x in t.compact(m)]
            assert got == list(model.compact(m))
        elif op == "extend":
            m = r.choice((1, 1, most))
            counts = [r.choice((1, 1, m, r.randint(0, m), -1, m + 1)) for _ in a]
            got = [x.tolist() for x in t.extend(i32(a), i32(counts), m)]
            assert got == list(model.extend(a, counts, m)), (k, a, counts)
        elif op == "fork":
            t.fork(i32(a), i32(b))
            model.fork(a, b)
        else:
            lens = [r.choice((0, r.randint(0, width * model.page), -3)) for _ in a]
            t.truncate(i32(a), i32(lens))
            model.truncate(a, lens)
        assert model.consistent() and same_table(t, model), (k, op)


@pytest.mark.parametrize("shape", [(16, 40, 6, 9, 70, 8), (16, 13, 5, 6, 40, 7), (32, 300, 64, 40, 100, 64), (16, 20000, 30, 50, 700, 30), (256, 50, 9, 3, 500, 9), (16, 700, 400, 4, 3, 1024)])
def test_tables_follow_the_definition(shape):
    page, n_pages, n_rows, width, most, longest = shape
    for seed in range(3):
        random_calls(gb.PageTable(n_pages, page, n_rows, width), sv.Table(n_pages, page, n_rows, width), random.Random(seed), 25, most, longest)


def test_a_large_pool_and_a_full_list():
    """1024 rows in one call, 300001 pages of which the first 290000 are taken, and prompts whose slots have a launch of their own."""
    n_pages, page, n_rows, width = 300001, 16, 1025, 600
    t = gb.PageTable(n_pages, page, n_rows, width)
    t.refs[:290000] = 1
    rows = torch.randperm(1024, generator=torch.Generator().manual_seed(1))
    slots, copies, refused = t.extend(rows.to(torch.int32).to(DEV), i32([33] * 1024), 40)
    want = 290000 + 3 * torch.arange(1024)[:, None] + torch.arange(40) // 16
    want = torch.where(torch.arange(40) < 33, want * page + torch.arange(40) % 16, -1)
    assert torch.equal(slots.cpu(), want) and int(refused.abs().sum()) == 0 and int((copies + 1).abs().sum()) == 0
    assert int(t.refs[290000:].sum()) == 3 * 1024
    # one more row: the free pages end
    slots, _, refused = t.extend(i32([1024, 1024, 0]), i32([9000, 1, 1]), 9000)
    assert refused.tolist() == [0, 1, 0] and int(slots[0, 8999]) == (290000 + 3 * 1024 + 562) * 16 + 7 and int(slots[1].max()) == -1
    _, _, refused = t.extend(i32([1, 2, 3]), i32([32, (600 - 3) * 16, 15]), 600 * 16)
    assert refused.tolist() == [0, 0, 0]
    moves, counts = t.compact(4)
    assert counts.tolist() == [int((t.refs > 0).sum()), 0] and int((moves + 1).abs().sum()) == 0


def test_the_largest_pool_is_compacted():
    """2^20 pages (a bit each in the 160 KB of LDS), those in use at its end."""
    n_pages = 1 << 20
    t = gb.PageTable(n_pages, 16, 3, 400)
    t.refs[:n_pages - 1000] = 1                              # (as if other tables had them, so that the rows get the last)
    _, _, refused = t.extend(i32([2, 0]), i32([300 * 16, 5]), 300 * 16)
    t.refs[:n_pages - 1000] = 0
    t.refs[7] = 1                                            # one that is in its place, and one that is not named
    before = t.table.clone()
    moves, counts = t.compact(1000)
    assert refused.tolist() == [0, 0] and counts.tolist() == [302, 301]
    high = torch.arange(n_pages - 1000 + 300, n_pages - 1000 - 1, -1, device=DEV)
    low = torch.tensor([p for p in range(302) if p != 7], device=DEV)
    assert torch.equal(moves[:301].long(), torch.stack((high, low), 1)) and bool((moves[301:] == -1).all())
    goes = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    goes[high] = low.to(torch.int32)
    assert torch.equal(t.table, torch.where(before >= 0, goes[before.clamp(min=0).long()], -1))
    assert torch.equal(t.refs, (torch.arange(n_pages, device=DEV) < 302).to(torch.int32))


def test_running_out_of_pages_changes_nothing_of_the_refused():
    t, m = gb.PageTable(8, 16, 6, 8), sv.Table(8, 16, 6, 8)
    for a, n in (([0], [20]), ([1, 2], [40, 40]), ([3], [1])):
        assert [x.tolist() for x in t.extend(i32(a), i32(n), 40)] == list(m.extend(a, n, 40))
    t.fork(i32([0, 0, 0]), i32([1, 4, 5]))
    m.fork([0, 0, 0], [1, 4, 5])
    assert same_table(t, m)
    # four rows write into one partly filled page, with fewer pages free than copies are needed: the last does not get the page of those that were refused
    a, n = [0, 1, 2, 4, 5], [1, 1, 30, 1, 1]
    assert [x.tolist() for x in t.extend(i32(a), i32(n), 30)] == list(m.extend(a, n, 30)) and same_table(t, m) and m.consistent()


@pytest.mark.parametrize("bits,group,page,H,layers", [(16, 128, 16, 32, 3), (8, 64, 64, 3, 1), (4, 128, 256, 1, 2), (16, 128, 128, 8, 1)])
def test_pages_are_moved(bits, group, page, H, layers):
    n_pages = 40
    cfg = gb.make_page_config(n_pages, page, H, bits, group)
    size = gb.gear_page_bytes(cfg)
    pool = torch.randint(0, 255, (layers, size + 32), dtype=torch.uint8, device=DEV)
    want = pool.clone()
    order = torch.randperm(n_pages)
    pairs = torch.stack((order[:13], order[13:26]), 1).to(torch.int32)
    pages = want[:, :size].view(layers, n_pages, -1)
    pages[:, order[13:26].to(DEV)] = pages[:, order[:13].to(DEV)]
    bad = torch.tensor([[-1, -1], [0, n_pages], [-5, 3], [n_pages, 1], [2, 2]], dtype=torch.int32)
    gb.gear_page_move(cfg, pool[:, :size], torch.cat((bad, pairs, bad)).to(DEV))
    assert torch.equal(pool, want)
    gb.gear_page_move(cfg, pool[0], torch.empty(0, 2, dtype=torch.int32, device=DEV))
    assert torch.equal(pool, want)


# ---- shared prefixes
class Batch:
    """A pool and a batch whose sequences share prefixes: groups of (shared tokens, sequences of (new tokens, own tokens))."""

    def __init__(self, dtype, bits, group, page, H, gq, groups, pad=0, seed=0, wider=0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.page, self.gq = dtype, page, gq
        n_pages = sum(-(-(s + o) // page) + 1 for s, seqs in groups for _, o in seqs) + 2
        self.q_start, self.kv, self.table, self.group_start, self.prefix, copies = sv.shared_table(page, groups, n_pages, gen)
        if wider:
            self.table = torch.cat((self.table, torch.full((len(self.kv), wider), -1, dtype=torch.int32)), 1)
        self.cfg = gb.make_page_config(n_pages, page, H, bits, group, dtype)
        x = torch.randn(2, n_pages, H, page, 128, generator=gen)
        x[..., 3] *= 6.0
        self.blocks = torch.stack([pg.pack(t.to(dtype), bits, group, dtype) for t in x], 2)
        for a, b in copies:
            self.blocks[b] = self.blocks[a]
        self.K, self.V = (pg.unpack(self.blocks[:, :, w].contiguous(), bits, group, dtype, page) for w in (0, 1))
        self.pool = self.blocks.reshape(-1).to(DEV)
        self.T = self.q_start[-1] + pad
        self.q = torch.randn(self.T, H * gq, 128, generator=gen).to(dtype)

    def made(self, causal=True, prefix=None, table=None, max_prefix=None, always=True):
        most = max(self.q_start[b] - self.q_start[a] for a, b in zip(self.group_start, self.group_start[1:]))
        prefix = self.prefix if prefix is None else prefix
        b = gb.make_page_batch(i32(self.q_start), i32(self.kv), (self.table if table is None else table).to(DEV), self.T,
                               max(b - a for a, b in zip(self.q_start, self.q_start[1:])), max(self.kv), causal)
        return b, gb.make_page_groups(i32(self.group_start), i32(prefix), most, max(prefix) if max_prefix is None else max_prefix, always)

    def run(self, q=None, out=None, scale=128 ** -0.5, made=None, **kw):
        b, g = made or self.made(**kw)
        q = self.q.to(DEV) if q is None else q
        if out is None:
            out = torch.full(q.shape, 77.0, dtype=q.dtype, device=DEV)
        n = gb.gear_page_attn_shared_bytes(self.cfg, q.shape[1], b, g)
        gb.gear_page_attn_shared(self.cfg, self.pool, b, g, q, out, scale, torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None)
        return out

    def check(self, out, scale=128 ** -0.5, causal=True, table=None):
        want, bound = pg.attend(self.q, self.K, self.V, self.q_start, self.kv, (self.table if table is None else table).tolist(), scale, causal)
        dead = torch.isnan(want)
        got = out.cpu().double()
        assert bool((got[dead] == 77.0).all())
        worst = sv.is_close(got[~dead], want[~dead], bound[~dead])
        assert worst <= 1.0, worst


GROUPS = [
    (16, 2, 2, [(100, [(1, 5), (1, 40), (1, 1)])], 0),                                     # few columns
    (16, 1, 8, [(200, [(1, 9)] * 6), (70, [(1, 33)])], 2),
    (32, 3, 4, [(0, [(1, 20)]), (1000, [(2, 30)] * 9), (64, [(1, 1)] * 2), (63, [(1, 2)])], 1),
    (64, 2, 4, [(5000, [(1, 1 + 17 * i) for i in range(40)])], 0),                          # divided
    (16, 1, 4, [(900, [(9, 12), (20, 40), (9, 9), (31, 200)])], 0),                         # many columns behind
    (16, 1, 2, [(700, [(1, 12), (40, 50), (1, 900), (1, 60)] + [(1, 3)] * 20)], 1),         # both
    (128, 1, 20, [(300, [(1, 5)] * 3), (2000, [(1, 100), (0, 4), (1, 7)])], 0),              # a sequence without new tokens
    (16, 1, 3, [(64 + g % 3, [(1, 2 + g % 4)] * (1 + (g % 2))) for g in range(70)], 0),      # more groups than a wave has lanes
    (16, 1, 17, [(64 + g, [(1, 2 + g % 4)] * (2 + (g % 3))) for g in range(66)], 0),
    (256, 1, 1, [(2048, [(1, 300)] * 130), (1, [(1, 5)] * 3)], 3),                           # more sequences
    (16, 2, 4, [(130, [(40, 45)] * 16)], 0),                                                 # many rows to join
    (16, 4, 1, [(129, [(300, 300), (1, 1)])], 0),                                            # a prompt: by itself
]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "%s-%d-%d" % (str(f[0])[6:], f[1], f[2]))
@pytest.mark.parametrize("shape", range(len(GROUPS)))
def test_shared_prefixes(form, shape):
    dtype, bits, group = form
    page, H, gq, groups, pad = GROUPS[shape]
    c = Batch(dtype, bits, group, page, H, gq, groups, pad, seed=shape)
    for causal in (True, False):
        c.check(c.run(causal=causal), causal=causal)
    c.check(c.run(always=False))


@pytest.mark.parametrize("form", [FORMS[0], FORMS[3], FORMS[4]], ids=lambda f: "%s-%d-%d" % (str(f[0])[6:], f[1], f[2]))
def test_prefixes_that_are_not_what_the_call_says(form):
    """Longer than what every new token sees, negative, past the table; bounds that are not met; a page of the prefix that is none."""
    dtype, bits, group = form
    c = Batch(dtype, bits, group, 16, 2, 4, [(400, [(1, 30), (1, 1), (2, 9)] * 3), (150, [(1, 5)] * 2)], seed=9)
    whole = c.run()
    c.check(whole)
    for prefix in ([1 << 30, 1 << 30], [-5, 0], [64, 63], [400, -1]):
        shown = list(prefix)
        if prefix[0] > 400:   # (what is not the same in all of them may not count: here none has a token more in whole 64s)
            shown = [c.prefix[0] + 40, c.prefix[1] + 5]
        c.check(c.run(prefix=shown, max_prefix=400))
    c.check(c.run(max_prefix=64))
    c.check(c.run(max_prefix=1 << 20))
    gone = c.table.clone()
    for row, p in zip(c.table.tolist(), gone):
        if row[2] == c.table[0, 2]:
            p[2] = c.cfg.n_pages + 7
    c.check(c.run(table=gone), table=gone)


@pytest.mark.parametrize("more", (0, 70))
def test_the_first_sequence_of_a_group_may_be_an_empty_place(more):
    """A row of the batch that has been freed: no tokens, no pages, no new ones; the prefix is read through the others' rows."""
    c = Batch(F16, 16, 128, 16, 2, 4, [(200, [(0, 4), (1, 5), (2, 9), (0, 3)]), (0, [(0, 0)]), (300, [(0, 1), (0, 1)])] + [(0, [(1, 3)])] * more, seed=13)
    for s in (0, 5, 6):
        c.table[s], c.kv[s] = -1, 0
    c.check(c.run())


def test_more_rows_than_the_call_says():
    """A group of more rows than its bound is right all the same; a sequence of more new tokens than the batch's bound may stay as it was, and the others are right."""
    c = Batch(F16, 16, 128, 16, 2, 4, [(300, [(1, 30)] * 6), (200, [(2, 9)] * 2)], seed=11)
    b, g = c.made()
    g.max_q = 2
    c.check(c.run(made=(b, g)))
    c = Batch(F16, 16, 128, 16, 2, 4, [(300, [(1, 30), (20, 30), (1, 1)]), (200, [(2, 9)] * 2)], seed=12)
    b, g = c.made()
    b.max_q = 2
    out = c.run(made=(b, g)).cpu()
    whole = c.run().cpu()
    c.check(whole)
    late = torch.zeros(c.T, dtype=torch.bool)
    late[1:21] = True
    assert bool((out[late] == 77.0).all()) or sv.is_close(out[late], whole[late].double(), torch.full_like(whole[late], 0.02).double()) <= 1.0
    want, bound = pg.attend(c.q, c.K, c.V, c.q_start, c.kv, c.table.tolist(), 128 ** -0.5, True)
    assert sv.is_close(out[~late], want[~late], bound[~late]) <= 1.0


def test_slots_without_a_token_may_hold_anything():
    c = Batch(F16, 16, 128, 16, 2, 4, [(150, [(1, 30), (1, 1), (2, 9)] * 3), (70, [(1, 5)] * 2)], seed=4)
    held = torch.zeros(c.cfg.n_pages, 16, dtype=torch.bool)
    for s, n in enumerate(c.kv):
        for t in range(n):
            held[c.table[s, t // 16], t % 16] = True
    rows = c.blocks.view(torch.int16).view(c.cfg.n_pages, 2, 2, 16, 128)
    rows.copy_(torch.where(held[:, None, None, :, None], rows, torch.tensor(0x7FFF, dtype=torch.int16)))
    c.pool = c.blocks.reshape(-1).to(DEV)
    c.check(c.run())


def test_views_scales_and_repeats():
    c = Batch(BF16, 8, 64, 32, 2, 4, [(700, [(1, 30)] * 12)], pad=1, seed=2)
    qkv = torch.zeros(c.T, 12, 128, dtype=BF16, device=DEV)
    qkv[:, :8] = c.q.to(DEV)
    wide = torch.full((c.T, 3, 8, 128), 77.0, dtype=BF16, device=DEV)
    for scale in (128 ** -0.5, -0.03, 0.0):
        wide.fill_(77.0)
        c.check(c.run(qkv[:, :8], wide[:, 1], scale=scale), scale=scale)
        assert bool((wide[:, 0] == 77.0).all()) and bool((wide[:, 2] == 77.0).all())
    first = c.run()
    for _ in range(5):
        assert same_bits(c.run(), first)


def test_groups_that_share_nothing_are_the_plain_call():
    c = Batch(F16, 16, 128, 16, 2, 2, [(0, [(1, 300), (3, 50), (40, 90)])], seed=3)
    b, g = c.made()
    plain = torch.full(c.q.shape, 77.0, dtype=F16, device=DEV)
    n = gb.gear_page_attn_bytes(c.cfg, 4, b)
    gb.gear_page_attn(c.cfg, c.pool, b, c.q.to(DEV), plain, 128 ** -0.5, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
    assert same_bits(c.run(), plain)
    none = gb.make_page_groups(i32([0]), i32([]), 0, 0)
    assert same_bits(c.run(made=(b, none)), plain)


# ---- together
class Served:
    """A layer's pool, its page table and a model of both: rows of every sequence as they were written."""

    def __init__(self, dtype=F16, H=2, gq=4, page=16, n_pages=400, n_rows=24, width=40):
        self.cfg = gb.make_page_config(n_pages, page, H, 16, 128, dtype)
        self.pool, self.t = gb.PagePool(self.cfg), gb.PageTable(n_pages, page, n_rows, width)
        self.rope = gb.make_rope(sv.frequencies(128).to(DEV))
        self.H, self.gq, self.dtype, self.page = H, gq, dtype, page
        self.gen = torch.Generator(device=DEV).manual_seed(0)
        self.rows = [torch.empty(0, 2, H, 128, dtype=dtype, device=DEV) for _ in range(n_rows)]

    def append(self, rows, n):
        """n new tokens of each row: (turned queries, the batch's q_start)."""
        start = self.t.kv_len[i32(rows).long()].long()
        slots, copies, refused = self.t.extend(i32(rows), i32([n] * len(rows)), n)
        self.pool.move(copies)
        qkv = torch.randn(len(rows), n, self.H * (self.gq + 2), 128, device=DEV, generator=self.gen).to(self.dtype)
        Hq = self.H * self.gq
        pos = start[:, None] + torch.arange(n, device=DEV)
        q = self.pool.write_rope(self.rope, qkv[:, :, Hq:Hq + self.H], qkv[:, :, Hq + self.H:], slots, pos, qkv[:, :, :Hq])
        assert int(refused.abs().sum()) == 0
        K = torch.empty(len(rows), n, self.H, 128, dtype=self.dtype, device=DEV)
        gb.gear_rotate(self.rope, qkv[:, :, Hq:Hq + self.H], K, pos)
        for i, r in enumerate(rows):
            self.rows[r] = torch.cat((self.rows[r], torch.stack((K[i], qkv[i, :, Hq + self.H:]), 1)))
        return q.reshape(len(rows) * n, Hq, 128)

    def check(self, rows, n, q, out):
        got, want = out.cpu().double(), torch.empty(out.shape, dtype=torch.float64)
        bound = torch.empty_like(want)
        for i, r in enumerate(rows):
            x = self.rows[r].cpu()
            kv = x.shape[0]
            pages = -(-kv // self.page)
            x = torch.cat((x, torch.zeros(pages * self.page - kv, 2, self.H, 128, dtype=x.dtype))).view(pages, self.page, 2, self.H, 128).permute(2, 0, 3, 1, 4)
            want[i * n:(i + 1) * n], bound[i * n:(i + 1) * n] = pg.attend(q[i * n:(i + 1) * n].cpu(), x[0], x[1], [0, n], [kv], [list(range(pages))], 128 ** -0.5, True)
        worst = sv.is_close(got, want, bound)
        assert worst <= 1.0, worst

    def attend(self, rows, n, q, groups):
        at = i32(rows).long()
        b = gb.make_page_batch(i32([n * i for i in range(len(rows) + 1)]), self.t.kv_len[at], self.t.table[at].contiguous(), n * len(rows), n, max(len(self.rows[r]) for r in rows))
        start, prefix = groups
        g = gb.make_page_groups(i32(start), i32(prefix), n * max(b - a for a, b in zip(start, start[1:])), max(prefix), always=True)
        return self.pool.attn_shared(q, b, g)


def test_a_server_s_life():
    """Prompts in, forked, extended a token at a time over their shared pages, some dropped, the pool compacted, more tokens, and a sequence handed to gear_compress."""
    s = Served()
    for r, n in ((0, 150), (1, 333)):
        q = s.append([r], n)
        s.check([r], n, q, s.attend([r], n, q, ([0, 1], [0])))
    kids = [[2, 3, 4, 5, 6], [7, 8, 9]]
    for parent, rows in zip((0, 1), kids):
        s.t.fork(i32([parent] * len(rows)), i32(rows))
        for r in rows:
            s.rows[r] = s.rows[parent]
    rows, groups = kids[0] + kids[1], ([0, 5, 8], [150, 333])
    for n in (1, 1, 3, 1):
        q = s.append(rows, n)
        s.check(rows, n, q, s.attend(rows, n, q, groups))
    # one beam takes another's place, some rows and the second prompt end, one falls back by two tokens
    s.t.fork(i32([3, 2, 9]), i32([2, 3, 7]))
    s.rows[2], s.rows[3], s.rows[7] = s.rows[3], s.rows[2], s.rows[9]
    s.t.truncate(i32([4, 1, 8, 5]), i32([0, 0, 0, len(s.rows[5]) - 2]))
    s.rows[4] = s.rows[1] = s.rows[8] = s.rows[0][:0]
    s.rows[5] = s.rows[5][:-2]
    moves, counts = s.t.compact(400)
    s.pool.move(moves)
    live = int((s.t.refs > 0).sum())
    assert counts.tolist()[0] == live and int(counts[1]) > 0 and bool((s.t.refs[:live] > 0).all()) and int(s.t.table.max()) == live - 1
    rows, groups = [2, 3, 5, 6, 7, 9], ([0, 4, 6], [150, 333])
    for n in (2, 1):
        q = s.append(rows, n)
        s.check(rows, n, q, s.attend(rows, n, q, groups))
    # back out of the pages, bit for bit, and into the compressor
    n = len(s.rows[9])
    pos = torch.arange(n, device=DEV)
    slots = s.t.table[9].long()[pos // 16] * 16 + pos % 16
    K, V = s.pool.read(slots[None], heads_first=True)
    assert same_bits(K[0].transpose(0, 1), s.rows[9][:, 0]) and same_bits(V[0].transpose(0, 1), s.rows[9][:, 1])
    cache = gb.GearCache(gb.make_config(1, 2, 8, 4, 64, 20000, 20, 512, 1, 4))
    cache.compress(K, V, 4, seed=1)
    Kc, _ = cache.decompress()
    assert float((Kc.float() - K.float()).norm() / K.float().norm()) < 0.1
    s.t.truncate(i32(list(range(24))), i32([0] * 24))
    assert int(s.t.refs.abs().sum()) == 0 and int((s.t.table + 1).abs().sum()) == 0 and int(s.t.kv_len.sum()) == 0


def test_a_step_is_captured_and_replayed():
    """Fork, extend, copy, write, attend and truncate as one graph, replayed with eager work in between: each replay is the eager step on the state it finds."""
    def state():
        s = Served(n_pages=300)
        s.append([0], 130)
        return s

    s, e = state(), state()
    kids = list(range(1, 7))
    src, dst, counts, zero = i32([0] * 6), i32(kids), i32([2] * 6), i32([0] * 6)
    slots, copies, refused = torch.empty(6, 2, dtype=torch.int64, device=DEV), torch.empty(6, 2, dtype=torch.int32, device=DEV), torch.empty(6, dtype=torch.int32, device=DEV)
    qkv = torch.randn(6, 2, 12, 128, device=DEV).to(F16)
    q_out, out = torch.empty(6, 2, 8, 128, dtype=F16, device=DEV), torch.empty(12, 8, 128, dtype=F16, device=DEV)
    pos = 130 + torch.arange(2, device=DEV).repeat(6, 1)
    q_start, start, prefix = i32([2 * i for i in range(7)]), i32([0, 6]), i32([130])
    ws = torch.empty(8 << 20, dtype=torch.uint8, device=DEV)

    def step(s, out):
        gb.gear_page_fork(s.t.c, src, dst)
        gb.gear_page_extend(s.t.c, dst, counts, slots, copies, refused)
        gb.gear_page_move(s.cfg, s.pool.pool, copies)
        gb.gear_page_write_rope(s.cfg, s.pool.pool, s.rope, qkv[:, :, 8:10], qkv[:, :, 10:], slots, pos, qkv[:, :, :8], q_out)
        b = gb.make_page_batch(q_start, s.t.kv_len[1:7], s.t.table[1:7], 12, 2, 400)
        gb.gear_page_attn_shared(s.cfg, s.pool.pool, b, gb.make_page_groups(start, prefix, 12, 130, always=True), q_out.view(12, 8, 128), out, 128 ** -0.5, ws)
        gb.gear_page_truncate(s.t.c, dst, zero)
        return b

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        keep = step(s, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        keep = step(s, out)   # noqa: F841
    for k in range(4):
        qkv.normal_()
        if k:   # the prompt grows, and another sequence takes pages
            for x in (s, e):
                x.t.extend(i32([0, 9]), i32([3, 20]), 20)
        out.fill_(5.0)
        graph.replay()
        got, table, refs = out.clone(), s.t.table.clone(), s.t.refs.clone()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        e.pool.pool.copy_(s.pool.pool)
        step(e, want)
        assert same_bits(got, want) and torch.equal(table, e.t.table) and torch.equal(refs, e.t.refs)


def test_calls_on_another_stream():
    c = Batch(F16, 16, 128, 16, 2, 4, [(500, [(1, 30)] * 12)], seed=6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = c.run()
    s.synchronize()
    c.check(out)
