"""The paged cache's attention on the GPU where weights, scores and parts are out of the ordinary, against the definition in 64 bits
(tests/page_util.py)."""
import math

import pytest
import torch

from paper_2403_05527_amd import binding as gb
from tests import page_util as pg
from tests.test_gpu_pages import BF16, DEV, F16, Cache, attn

pytestmark = pytest.mark.gpu


def pool_of(c, bits=16, group=128):
    c.pool = torch.stack([pg.pack(x, bits, group, c.q.dtype) for x in (c.K, c.V)], 2).reshape(-1).to(DEV)


@pytest.mark.parametrize("max_kv", [1, None])
@pytest.mark.parametrize("n,kv", [(1, 1536), (1, 20000), (40, 1536), (40, 20000)])
def test_a_flat_tail_counts(n, kv, max_kv):
    """Many weights that are each far below a row's greatest, in the sum of Values as in the sum of weights."""
    c = Cache(F16, 16, 128, 16, 1, 1, [(n, kv)], seed=21)
    scale = pg.sink_and_tail(c.K, c.V, c.q, c.table[0].tolist(), kv, 16)
    pool_of(c)
    got = attn(c, scale=scale, max_kv=max_kv)[:, 0].cpu().double()
    want, bound = pg.tail_bound(c.q, c.K, c.V, c.table[0].tolist(), kv, 0, n, scale, 16)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("log2", [15.3, 22.97, 23.02, 24.3, 25.7, 27.4])
def test_equal_scores_of_any_size(log2, n, dtype):
    """All scores equal, from 2^15 to 2^27 steps of the exponent: the mean of the Values, however the base of the weights is rounded."""
    kv = 700
    c = Cache(dtype, 16, 128, 16, 1, 1, [(n, kv)], seed=22)
    c.K[:], c.q[:] = 512.0, 512.0                                       # (sums of products are exact)
    pool_of(c)
    at = torch.arange(kv)
    v = c.V[c.table[0].long()[at // 16], 0, at % 16].double()
    eps, most = torch.finfo(dtype).eps / 2, v.abs().mean(0)
    bound = most * (eps + (kv + 10) * 2.0 ** -23)                       # a weight rounded before the product, kv terms in fp32
    for max_kv in (1, 100000):
        got = attn(c, scale=2.0 ** (log2 - 25) * math.log(2.0), causal=False, max_kv=max_kv)[:, 0].cpu().double()
        assert bool(((got - v.mean(0)).abs() <= bound + (v.mean(0).abs() + bound) * eps + 2.0 ** -25).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_codes_and_values_at_ties(bits, dtype):
    """The codes of a difference that fp32 does not hold, and the values of a sum that it does not hold: as stated."""
    x, _ = pg.rows_at_ties(bits, dtype)
    if bits == 4 and dtype == BF16:
        x = torch.cat((torch.tensor([-2.0 ** -30, 15.125, 3.015625] + [0.5] * 29, dtype=torch.float64).repeat(1, 4).to(dtype), x))
    n, page = len(x), 64
    new = torch.stack((x, -x.flip(0)))                                   # Keys; Values
    pool = gb.PagePool(gb.make_page_config(1, page, 1, bits, 32, dtype), DEV)
    slots = torch.arange(n, device=DEV)
    pool.write(new[0][:, None].to(DEV), new[1][:, None].to(DEV), slots)
    code, scale, zero = pg.quantise_fp32(torch.cat((new, torch.zeros(2, page - n, 128, dtype=dtype)), 1), bits, 32, dtype)
    assert torch.equal(pool.pool.cpu(), pg.block_of_codes(code, scale, zero, bits).reshape(-1))
    values = pg.values_fp32(code, scale, zero, 32, dtype)[:, :n]
    for got, v in zip(pool.read(slots[None]), values):
        assert torch.equal(got[0, :, 0].cpu().view(torch.int16), v.contiguous().view(torch.int16))
    # a token that sees one key alone gets its Value (a score of 0: its weight is a power of two)
    b = gb.make_page_batch(*(torch.tensor(t, dtype=torch.int32, device=DEV) for t in ((0, 1), (1,), ((0,),))), 1, 1, page)
    for i in range(0, n, 5):
        one = gb.PagePool(pool.cfg, DEV)
        one.write(new[0][i:i + 1, None].to(DEV), new[1][i:i + 1, None].to(DEV), slots[:1])
        out = one.attn(torch.zeros(1, 1, 128, dtype=dtype, device=DEV), b)
        assert torch.equal(out.cpu().view(torch.int16).view(-1), values[1, i].contiguous().view(torch.int16))


def test_a_bf16_sum_goes_through_fp32():
    """8-bit codes whose value is half a bf16 step but for what fp32 does not hold."""
    page = 16
    code = torch.full((2, page, 128), 3)
    scale = torch.full((2, page, 4), 1.0078125).to(BF16)
    zero = torch.full((2, page, 4), -2.0 ** -30).to(BF16)
    pool = gb.PagePool(gb.make_page_config(1, page, 1, 8, 32, BF16), DEV)
    pool.pool.copy_(pg.block_of_codes(code, scale, zero, 8).reshape(-1))
    K, V = pool.read(torch.arange(page, device=DEV)[None])
    assert bool((K == 3.03125).all()) and bool((V == 3.03125).all())     # (once: 3.015625)


LONG = [   # page, H, gq, sequences (new tokens, tokens), padding rows
    (16, 1, 1, [(34, 800), (1, 790)], 0),                                 # an odd number of records before those of the few columns
    (16, 1, 1, [(301, 9000), (2, 8999)], 1),
    (16, 1, 1, [(1, 9000)], 0),                                           # more parts than a merge's waves ask for at a time (32) ...
    (32, 1, 3, [(1, 40000)], 0),                                          # ... than a wave's lanes look at (64)
    (64, 1, 2, [(20, 14000)], 0),                                         # the same of many columns
    (16, 1, 1, [(34, 1500) if i == 64 else (1, 17 + i % 3) for i in range(66)], 0),   # the joining looks for a row among more than 64 sequences
    (16, 2, 2, [(1 + (i % 30 == 7) * 50, 40 + 7 * i) for i in range(130)], 2),
]


@pytest.mark.parametrize("dtype,bits,group", [(F16, 16, 128), (BF16, 8, 64), (F16, 4, 32)])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_many_parts(i, dtype, bits, group):
    page, H, gq, seqs, pad = LONG[i]
    c = Cache(dtype, bits, group, page, H, gq, seqs, seed=30 + i, pad=pad)
    c.check(attn(c), before=77.0)


@pytest.mark.parametrize("dtype,bits,group", [(F16, 16, 128), (BF16, 8, 64), (F16, 4, 32)])
@pytest.mark.parametrize("n", [1, 40])
def test_pages_past_the_first_look(n, dtype, bits, group):
    """A part's pages are more than a wave's lanes hold at a time (64): tables of 313 entries, some of no page, in one part and as the call divides them."""
    c = Cache(dtype, bits, group, 16, 2, 1, [(n, 5000), (n, 1040)], seed=40)
    table = c.table.clone()
    for e, page in ((3, -1), (64, -7), (70, 10 ** 6), (71, c.cfg.n_pages), (200, -1), (312, -1)):
        table[0, e] = page
    for max_kv in (1, None):
        c.check(attn(c, table=table, max_kv=max_kv), table=table)


STARTS = [(200, -2 ** 31), (2 ** 31 - 1, -2 ** 31), (300, 299)]


@pytest.mark.parametrize("starts", STARTS)
def test_starts_that_do_not_ascend(starts):
    """Rows that nobody has are left alone, and nothing outside the arrays is read."""
    for seqs in ([(40, 800)], [(40, 800)] * 70):
        c = Cache(F16, 8, 64, 16, 1, 1, seqs, seed=50, pad=200)
        b = c.batch()
        b.tensors[0].copy_(torch.tensor([starts[k % 2] for k in range(len(seqs) + 1)] if len(seqs) == 1 else [starts[0]] + [starts[1]] * len(seqs), dtype=torch.int32))
        assert bool((attn(c, batch=b) == 77.0).all())
