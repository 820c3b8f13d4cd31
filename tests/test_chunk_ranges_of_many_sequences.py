"""Page ranges over more sequences than a wave looks at in one step: pieces of tiles of the 65th
sequence and on are found behind the sums of those before."""
import numpy as np
import pytest
import torch

from test_chunk_attn import Cache, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,Hkv", [("bf16", 1), ("kv4", 1), ("kv2", 2)])
@pytest.mark.parametrize("B,most", [(65, 1), (130, 3), (70, 60)])     # tiles of 32 and of 128 rows
@pytest.mark.parametrize("splits", [0, 9])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 70)])
def test_pieces(fmt, Hkv, B, most, splits, window, sinks):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 200, B)
    lens[rng.choice(B, 12, replace=False)] = rng.integers(1000, 1700, 12)
    lens[[3, B - 1]] = 1650, 1111
    new = [int(rng.integers(0, min(n, most) + 1)) for n in lens]
    new[3], new[40], new[B - 1] = min(most, 1), 0, most
    c = Cache(fmt, lens.tolist(), Hkv, seed=B)
    q = _q(new, 2 * Hkv, seed=B, more=2)
    out = torch.full_like(q, 7.0)
    c.run(q, new, window, sinks, splits=splits, out=out)
    c.check(q, new, out, window, sinks)
    assert bool((out[sum(new):] == 7.0).all())
    again = torch.full_like(q, 7.0)
    assert torch.equal(out, c.run(q, new, window, sinks, splits=splits, out=again))
