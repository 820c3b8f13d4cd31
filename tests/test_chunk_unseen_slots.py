"""Cached slots that no new token of a sequence sees, in pages that it reads: before the window
in the window's first page, after the first tokens in their last page.  They may hold anything."""
import pytest
import torch

import chunk_ref as R
import kv4_ref
from test_chunk_attn import Cache, _q

pytestmark = pytest.mark.gpu
D, P = 128, 64

CASES = [([1, 1], [700, 63], 100, 4), ([1], [300], 7, 0), ([3, 2], [449, 130], 64, 64), ([70, 3], [449, 65], 100, 70),
         ([300], [700], 130, 5), ([600], [900], 200, 1), ([600, 515], [777, 1000], 33, 100)]


def _spoil(c, b, slots, what):
    """K and V of cached tokens `slots` of sequence b: NaN, or the largest numbers."""
    pool = c.pool.cpu()
    at = [(int(c.table[b, t // P]), t % P) for t in slots]
    if c.fmt == "bf16":
        value = float("nan") if what == "nan" else 3e38
        view = pool.view(-1, c.Hkv, 2 * P * D)
        k, v = R.bf16_places()
        for page, t in at:
            view[page][:, k[t]] = value
            view[page][:, v[t]] = value if what == "nan" else -value
    else:
        ng = D // c.G
        size = pool.numel() // c.L.num_pages // c.Hkv
        view = pool.view(-1, c.Hkv, size).numpy()
        bits = 0xFFFF if what == "nan" else 0x7BFF if c.meta == 0 else 0x5B80    # 65504, 2^56
        for page, t in at:
            for is_v in (0, 1):
                for g in range(ng):
                    e = kv4_ref.sz_place(c.G, is_v, t, g) if c.fmt == "kv4" else \
                        2 * (P * D // 4) + is_v * ng * P * 4 + (g * P + t) * 4
                    view[page, :, e:e + 2] = (bits & 255, bits >> 8)
                    view[page, :, e + 2:e + 4] = (bits & 255, bits >> 8) if what == "nan" else 0
    c.pool = pool.cuda()


@pytest.mark.parametrize("fmt,meta", [("bf16", 0), ("kv4", 0), ("kv4", 1), ("kv2", 0), ("kv2", 1)])
@pytest.mark.parametrize("new,lens,window,sinks", CASES)
@pytest.mark.parametrize("splits", [0, 1, 4])
@pytest.mark.parametrize("what", ["nan", "large"])
def test_slots_that_no_new_token_sees(fmt, meta, new, lens, window, sinks, splits, what):
    c = Cache(fmt, lens, 1, seed=window + sinks, meta=meta)
    q = _q(new, 2)
    clean = c.run(q, new, window, sinks, splits=splits)
    spoiled = 0
    for b, (n, length) in enumerate(zip(new, lens)):
        seen = R.visible(n, length, window, sinks).any(0)
        shared = [t for t in range(length) if not seen[t] and seen[t // P * P:t // P * P + P].any()]
        _spoil(c, b, shared, what)
        spoiled += len(shared)
    assert spoiled
    out = c.run(q, new, window, sinks, splits=splits)
    c.check(q, new, out, window, sinks)
    assert torch.equal(out, c.run(q, new, window, sinks, splits=splits))
    if fmt == "bf16" or what == "large":
        c.check(q, new, clean, window, sinks)


@pytest.mark.parametrize("fmt,meta", [("kv4", 0), ("kv4", 1), ("kv2", 0), ("kv2", 1)])
@pytest.mark.parametrize("new,lens,window,sinks", CASES)
def test_their_scales_cost_no_bits(fmt, meta, new, lens, window, sinks):
    """Small values of the tokens that are seen, the largest scales in the others: the same bits come out."""
    c = Cache(fmt, lens, 1, seed=window, meta=meta, v_spread=1e-3)
    q = _q(new, 2)
    clean = c.run(q, new, window, sinks, splits=1)
    for b, (n, length) in enumerate(zip(new, lens)):
        seen = R.visible(n, length, window, sinks).any(0)
        _spoil(c, b, [t for t in range(length) if not seen[t] and seen[t // P * P:t // P * P + P].any()], "large")
    out = c.run(q, new, window, sinks, splits=1)
    c.check(q, new, out, window, sinks)
    # slots that some rows of a sequence see count among all of them, the others nowhere: only tiles'
    # powers of two may differ, which no normal number feels
    diff = (out.double() - clean.double()).abs()
    assert (diff <= 2.0 ** -8 * clean.double().abs() + 1e-8).all()
