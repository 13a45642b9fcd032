"""Attention with shared prefixes on the CPU stand-in (tests/simt/) where one sequence has much more behind its prefix than the others: in no group, or behind a shorter prefix, so that
what lies there is divided by its own length.  Under the address sanitizer on buffers of exactly their size, against the definition in 64 bits."""
import pytest
import torch

from tests import page_util as pg
from tests import serving_util as sv
from tests.test_cpu_emulation_serving import BF16, F16, emulator, run  # noqa: F401  (the fixture)

# dtype, bits, group, page, H, gq, groups (shared tokens, sequences (new tokens, own tokens)), groups at the end that are none, causal, padding rows
LONGER = {
    "one_by_itself": (F16, 16, 128, 16, 1, 2, [(3000, [(1, 5), (1, 9)]), (0, [(1, 3100)])], 1, 1, 0),
    "a_short_prefix": (BF16, 8, 64, 32, 1, 4, [(3000, [(1, 5)] * 2), (70, [(1, 3050), (1, 20)])], 0, 1, 1),
    "two_column_tiles": (F16, 4, 32, 16, 1, 4, [(2600, [(5, 6)] * 2), (0, [(6, 2700), (5, 30)])], 1, 0, 0),
    "prefixes_of_many_columns": (F16, 16, 128, 64, 1, 4, [(1900, [(1, 5)] * 9), (0, [(1, 2000)])], 1, 1, 2),
    "many_behind": (F16, 16, 128, 16, 1, 4, [(64, [(9, 12), (33, 1700), (9, 9)]), (1500, [(1, 300), (2, 5)])], 0, 1, 1),
    "many_by_itself": (BF16, 4, 64, 16, 1, 2, [(1800, [(17, 30)] * 2), (0, [(80, 2000), (1, 1950)])], 1, 1, 0),
    "many_see_all": (F16, 8, 64, 64, 1, 4, [(1800, [(9, 30)] * 2), (0, [(33, 1900)])], 1, 0, 0),
    "no_page": (F16, 16, 128, 16, 1, 2, [(2500, [(1, 5), (1, 9)]), (0, [(1, 2600), (0, 40)])], 1, 1, 0),
}


@pytest.mark.parametrize("name", list(LONGER))
def test_what_lies_behind_a_prefix_may_be_long(emulator, tmp_path, name):  # noqa: F811
    dtype, bits, group, page, H, gq, groups, none, causal, pad = LONGER[name]
    gen = torch.Generator().manual_seed(len(name))
    n_pages = sum(-(-(s + o) // page) + 1 for s, seqs in groups for _, o in seqs) + 1
    q_start, kv, table, group_start, prefix, copies = sv.shared_table(page, groups, n_pages, gen)
    if none:
        group_start, prefix = group_start[:-none], prefix[:-none]
    x = torch.randn(2, n_pages, H, page, 128, generator=gen)
    x[..., 3] *= 6.0
    pool = torch.stack([pg.pack(t.to(dtype), bits, group, dtype) for t in x], 2)
    for a, b in copies:
        pool[b] = pool[a]
    if name == "no_page":
        table[2, 70], table[2, 120] = -1, n_pages + 3
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
