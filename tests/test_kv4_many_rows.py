"""The 4-bit cache's calls with more rows than one launch holds, and the merge's row counts."""
import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok
from test_kv4_attn import SM, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hq,Hkv,rot", ((9, 32, 8, "shared"), (20, 32, 8, "shared"), (40, 32, 8, "per_head"),
                                          (300, 16, 4, "identity_v")))   # 288, 640, 1280, 4800 rows
def test_rows_of_the_merge_with_weights(B, Hq, Hkv, rot):
    """2, 4, 8 and 16 rows per block of the merge that shares its launch with the weights."""
    rng = np.random.default_rng(B)
    c = Case(B, rng.integers(0, 150, B), Hq, Hkv, rot=rot)
    c.check((0,))
    w = torch.zeros(B, Hkv, c.mp * 64, device="cuda")
    assert torch.equal(c.run(0, torch.bfloat16, weights=w), c.run(0).bfloat16())


@pytest.mark.parametrize("splits", (1, 2))
def test_more_rows_than_a_launch(splits):
    """2^20 rows of queries and more: sequences dealt to several launches.  A sequence of one
    page has one partial state, whatever else is in the call."""
    B, Hq, Hkv, G = 17000, 64, 8, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    lay = ok.Layout(Hkv, B, group_size=G)
    pool = torch.randint(0, 256, (B, ok.kv4_page_bytes(lay)), dtype=torch.uint8, device="cuda", generator=g)
    meta = torch.from_numpy(R.random_pool(np.random.default_rng(1), 4, Hkv, G, 0).reshape(4, Hkv, -1)).cuda()
    pool.view(B, Hkv, -1)[..., 8192:] = meta[..., 8192:].repeat(B // 4, 1, 1)      # sane scales and zeros
    pool = pool.view(-1)
    table = torch.randperm(B, device="cuda", generator=g).to(torch.int32).view(B, 1)
    lens = torch.randint(0, 65, (B,), device="cuda", generator=g).to(torch.int32)
    q = torch.randn(B, Hq, 128, device="cuda", generator=g).bfloat16()
    rng = np.random.default_rng(2)
    Rk, Rv = (torch.from_numpy(R.rotation(rng)).cuda() for _ in range(2))
    k, v = (torch.randn(B, Hkv, 128, device="cuda", generator=g).bfloat16() for _ in range(2))
    slots = torch.where(lens > 0, table[:, 0].long() * 64 + lens.long() - 1, -1)

    def step(i):
        n = len(i)
        out = torch.full((n, Hq, 128), 7.0, device="cuda")
        w = torch.ones(n, Hkv, 64, device="cuda")
        ws = ok.kv4_alloc_workspace(lay, n, Hq, splits, 1, weights=True)
        p = pool.clone()
        ok.kv4_decode_step(lay, p, k[i], v[i], slots[i], 0.9, 0.9, q[i], table[i], lens[i], Rk, Rv, SM, splits, ws, out,
                           weights=w)
        plain = torch.full_like(out, 7.0)
        ok.kv4_decode_attn(lay, p, q[i], table[i], lens[i], Rk, Rv, SM, splits, ws, plain)
        assert torch.equal(out, plain)
        return out, w, p.view(B, -1)
    every = torch.arange(B, device="cuda")
    out, w, p = step(every)
    for first in (0, 16384 - 40, B - 80):
        i = every[first:first + 80]
        o1, w1, p1 = step(i)
        assert torch.equal(out[i], o1) and torch.equal(w[i], w1)
        at = table[i, 0].long()
        assert torch.equal(p[at], p1[at])
    assert (out[lens == 0] == 0).all() and (w[lens == 0] == 1).all()


def test_evictions_of_more_rows_than_a_launch():
    """More than 2^20 rows of (sequence, head): several launches of the select, and of the
    move (65535 rows)."""
    B, Hkv, G, budget = 16500, 64, 128, 30
    g = torch.Generator(device="cuda").manual_seed(3)
    lay = ok.Layout(Hkv, B, group_size=G)
    size = R.block_bytes(G)
    pool = torch.randint(0, 256, (B, Hkv, size), dtype=torch.uint8, device="cuda", generator=g)
    table = torch.randperm(B, device="cuda", generator=g).to(torch.int32).view(B, 1)
    lens = torch.randint(0, 65, (B,), device="cuda", generator=g).to(torch.int32)
    w = torch.rand(B, Hkv, 64, device="cuda", generator=g)
    pos = torch.full((B, Hkv, 64), -1, dtype=torch.int32, device="cuda")
    sample = torch.cat([torch.arange(12), torch.arange(16384 - 12, 16384 + 12), torch.arange(B - 12, B)]).cuda()
    small = pool[table[sample, 0].long()].cpu().numpy()
    n = len(sample)
    want = R.evict(small.reshape(-1), Hkv, G, np.arange(n, dtype=np.int32)[:, None], lens[sample].cpu().numpy(),
                   w[sample].cpu().numpy(), pos[sample].cpu().numpy(), lens[sample].cpu().numpy(), budget, 2, 5)
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    ok.kv4_evict(lay, pool.view(-1), table, lens, w, pos, lens, budget, 2, 5, new,
                 ok.kv4_alloc_evict_workspace(lay, B, 1))
    got = (pool[table[sample, 0].long()].reshape(-1), w[sample], pos[sample], new[sample])
    for a, b, name in zip(got, want, ("pages", "weights", "positions", "lengths")):
        assert np.array_equal(a.cpu().numpy(), b), name
    assert torch.equal(new, lens.clamp(max=budget))
