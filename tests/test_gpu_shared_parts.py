"""Attention with shared prefixes on the GPU where sequences have much more behind their prefix than the longest has behind the longest: in no group, or behind a shorter prefix."""
import pytest

from tests.test_gpu_serving import BF16, F16, FORMS, Batch, same_bits

pytestmark = pytest.mark.gpu

# page, H, gq, groups (shared tokens, sequences (new tokens, own tokens)), how many of them at the end are none, padding rows
LONGER = [
    (16, 2, 4, [(4000, [(1, 20)] * 6), (0, [(1, 4100), (1, 9)])], 1, 0),
    (32, 3, 2, [(5000, [(1, 30)] * 3), (100, [(1, 4900), (2, 700), (1, 5030)])], 0, 1),                  # a short prefix
    (64, 1, 4, [(6000, [(1, 100)] * 5), (0, [(1, 1500)]), (3000, [(1, 2900)] * 2), (0, [(1, 6050)])], 1, 0),   # between prefixes
    (16, 1, 8, [(3000, [(1, 9)] * 20), (0, [(1, 3000 - 700 * i) for i in range(4)])], 1, 2),                 # prefixes of many columns
    (16, 2, 4, [(2600, [(5, 20)] * 2), (0, [(5, 2600), (2, 10)])], 1, 0),                                    # two tiles of columns
    (128, 1, 2, [(2500, [(1, 1 + i % 7)] * 2) for i in range(30)] + [(0, [(1, 2500 - i) for i in range(9)])], 1, 0),   # more sequences than a wave has lanes
    (16, 2, 4, [(64, [(9, 12), (70, 3500), (9, 9)]), (2900, [(1, 300), (2, 5)])], 0, 1),                      # many columns, behind a short prefix
    (64, 1, 8, [(3000, [(5, 30)] * 9), (0, [(100, 3300), (1, 3200), (40, 60)])], 1, 0),                        # by themselves
    (16, 1, 2, [(2000, [(1, 1 + i % 7)] * 2) for i in range(30)] + [(0, [(70, 2100), (1, 1900), (33, 2222)])], 1, 0),
    (32, 2, 3, [(128, [(50, 5000), (43, 4100)])], 0, 3),                                                     # all of them long
    (256, 1, 1, [(70, [(1, 5)] * 2), (12000, [(0, 3), (1, 7)]), (0, [(1, 12000), (0, 5)])], 1, 0),
]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "%s-%d-%d" % (str(f[0])[6:], f[1], f[2]))
@pytest.mark.parametrize("shape", range(len(LONGER)))
def test_what_lies_behind_a_prefix_may_be_long(form, shape):
    dtype, bits, group = form
    page, H, gq, groups, none, pad = LONGER[shape]
    c = Batch(dtype, bits, group, page, H, gq, groups, pad, seed=shape)
    if none:
        c.group_start, c.prefix = c.group_start[:-none], c.prefix[:-none]
    first = None
    for causal in (True, False):
        out = c.run(causal=causal)
        c.check(out, causal=causal)
        first = out if first is None else first
    assert same_bits(c.run(), first)
    c.check(c.run(always=False))


def test_bounds_that_are_shorter_than_the_sequences():
    """max_kv and max_prefix are about the longest: with others the division is another, the results are the same."""
    c = Batch(F16, 16, 128, 16, 2, 4, [(3000, [(1, 20)] * 3), (100, [(1, 4000)] * 2)], seed=21)
    for max_kv in (1, 1000, 4100, 1 << 28):
        b, g = c.made()
        b.max_kv = max_kv
        c.check(c.run(made=(b, g)))
    c = Batch(BF16, 16, 128, 16, 2, 4, [(3000, [(1, 20)] * 3), (100, [(1, 4000)] * 2)], seed=22)
    for prefix in (64, 1500, 1 << 28):
        c.check(c.run(max_prefix=prefix))
