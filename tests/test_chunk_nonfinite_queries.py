"""A query row with a NaN or an infinity gives NaN in its own output row and in no other, in tiles of
every size."""
import math

import pytest
import torch

import paper_2605_17757_amd as ok
from paper_2605_17757_amd import build
from test_chunk_attn import Cache, _q

D, P = 128, 64
# rows (2 heads on one): tiles of 32, 128 and 256
NEW = [([1, 3], [300, 70]), ([100, 3], [300, 70]), ([600, 520], [600, 900])]


def test_nan_is_a_value_to_the_compiler():
    """Results with NaN are promised, so no unit may be compiled as if there were none."""
    for src, flags in build.SOURCES.items():
        for f in [*build.COMMON, *flags]:
            assert "nans" not in f and "fast" not in f and "finite" not in f, (src, f)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new,lens", NEW)
@pytest.mark.parametrize("splits", [0, 1, 4])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_rows_with_nan_or_infinity(fmt, new, lens, splits, window, sinks, value):
    c = Cache(fmt, lens, 1, seed=21)
    q = _q(new, 2)
    good = c.run(q, new, window, sinks, splits=splits)
    c.check(q, new, good, window, sinks)
    bad = q.clone()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for row, head, ch in ((0, 1, 7), (0, 0, 127), (q.shape[0] - 1, 1, 0), (q.shape[0] // 2, 0, 64)):
        bad[row, head, ch] = value
        hit[row, head] = True
    out = c.run(bad, new, window, sinks, splits=splits)
    assert torch.isnan(out[hit]).all()
    # The others: to the last bit where no row's reference moves at another time (NaN exceeds nothing).
    # The 32 rows of a wave move theirs together, each to its own maximum so far, whenever one exceeds its
    # own by 2^8, as infinite scores do; p / 2^m then rounds at another place: the definition's bounds hold.
    if math.isnan(value):
        assert torch.equal(out[~hit], good[~hit])
    out[hit] = good[hit]
    c.check(q, new, out, window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new,lens", NEW)
@pytest.mark.parametrize("splits", [0, 1, 4])
def test_scores_that_are_all_minus_infinity(fmt, new, lens, splits):
    """Keys positive in one channel, the query -infinity there: no score is left, and no softmax either."""
    c = Cache(fmt, lens, 1, seed=22, rot=False)
    g = torch.Generator(device="cuda").manual_seed(22)
    n = sum(lens)
    k, v = torch.randn(2, n, 1, D, generator=g, device="cuda").to(torch.bfloat16)
    k[:, :, 5] = 3.0
    slots = torch.cat([c.block_table[b].long()[torch.arange(m, device="cuda") // P] * P + torch.arange(m, device="cuda") % P
                       for b, m in enumerate(lens)])
    if fmt == "bf16":
        ok.bf16_kv_append(c.L, c.pool, k, v, slots)
    else:
        (ok.kv4_append if fmt == "kv4" else ok.kv_append)(c.L, c.pool, k, v, slots, None, None, 1.0, 1.0)
    q = _q(new, 2)
    good = c.run(q, new, splits=splits)
    bad = q.clone()
    bad[0, 1, 5] = bad[-1, 0, 5] = -math.inf
    out = c.run(bad, new, splits=splits)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(out[-1, 0]).all()
    out[0, 1], out[-1, 0] = good[0, 1], good[-1, 0]
    assert torch.equal(out, good)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new", [[3], [100], [600]])
def test_a_row_without_tokens_stays_zero(fmt, new):
    """seq_lens below the new tokens: the first rows see nothing, whatever they hold."""
    c = Cache(fmt, [new[0] - 1], 1, seed=23)
    q = _q(new, 2)
    q[0, 0, 3] = math.nan
    q[0, 1, 3] = math.inf
    c.check(q, new, c.run(q, new))
