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
