"""Rows of slots that come several times in one call of the 4-bit read-back, in tiles of 64
tokens: the four waves of a block each store a part of every row of a page, so that they
have to take a slot's tokens in the same order, and each token of a page that is left with
a few is stored by one wave alone."""
import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu

HKV, PAGES = 40, 12


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def tiles(kind, rng):
    """Slots of one tile after another."""
    out = []
    for i in range(9):
        p, q = rng.permutation(PAGES)[:2] * 64
        a = rng.permutation(64)
        out.append({
            "one slot": np.full(64, p + a[0]),                          # 64 tokens of it
            "threes": np.concatenate([np.repeat(p + a[:21], 3), [q]]),   # turns of 21, 21, 21
            "last few": np.concatenate([np.repeat(p + a[:8], 7), p + a[:8]])[:64],  # 8 slots in 8 turns
            "left over": np.concatenate([p + a[:50], p + a[:7], q + a[:7]]),  # 7 repeated ones, one by one
            "mixed": np.where(rng.random(64) < 0.1, -1, p + a[rng.integers(0, 1 + 7 * i, 64)]),
            "two pages": np.stack([p + a[rng.integers(0, 9, 32)], q + a[rng.integers(0, 20, 32)]], 1).reshape(-1),
        }[kind])
        if kind != "one slot":
            rng.shuffle(out[-1])
    return np.concatenate(out)


@pytest.mark.parametrize("kind", ("one slot", "threes", "last few", "left over", "mixed", "two pages"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("G,meta", ((32, 0), (128, 1)))
def test_repeated_slots_by_tiles(kind, dtype, G, meta):
    rng = np.random.default_rng(21)
    pool = R.random_pool(rng, PAGES, HKV, G, meta)
    slots = tiles(kind, rng)
    n = len(slots)
    assert n * HKV > 12288                                # by tiles
    lay = ok.Layout(HKV, PAGES, group_size=G, meta_dtype=meta)
    k, v = (torch.full((n, HKV, 128), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    ok.kv4_gather(lay, dev(pool), dev(slots.astype(np.int64)), k, v)
    blocks = pool.reshape(PAGES, HKV, -1)
    for out, is_v in ((k, 0), (v, 1)):
        vals = torch.from_numpy(R.block_values(blocks, G, meta, is_v))
        want = vals.permute(0, 2, 1, 3).reshape(PAGES * 64, HKV, 128)[np.maximum(slots, 0)].to(dtype)
        want[slots < 0] = 7.0
        assert torch.equal(out.cpu(), want)
