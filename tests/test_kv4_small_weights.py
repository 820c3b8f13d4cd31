"""Small softmax weights beside a heavy token's in the 4-bit decode: the value sums take a
weight times its scale in two fp16 pieces, each rounded to nearest.

Per sequence the first four pages (one for each wave of a block) hold a heavy token; its
value is 0, so that the output comes from the other tokens alone.  These have the score 0
and the weight 2^-17 (head 0) down to 2^-25 (last head) of a heavy one, and the same value,
so that the errors of their pieces are the same and add up instead of averaging out.

Bound of the output's relative error, u = 2^-24:
  heavy score   16 u sum |q| sm s (15 + |z|) + 4 u |score|, as kv4_ref.attend derives it: it
                changes all small weights alike;
  pieces        x = w s 2^-ex, 2^10 <= s 2^-ex < 2^11.  A piece is off by half a step: the
                first by 2^-11 x at most, the second by 2^-11 of that remainder, 2^-22 x, or
                where the remainder is below 2^-14, by half of fp16's least value, 2^-25;
  within pages  sums of 64 terms, at most one last place each (128 u), and single operations
                (16 u);
  over pages    a wave adds one page after another to its sum of weights (the heavy token's 1
                and the small ones) and to its output.  Each addition is off by u times the
                sum so far, which is at most the final one: u per page in each, and all
                alike here, where every page adds the same.  A wave has a quarter of the
                sequence's pages at most.
"""
import math

import numpy as np
import pytest
import torch

import kv4_ref as R
from test_kv4_attn import SM, Case

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def entries(pool, c, is_v):
    """Scale and zero [pages, Hkv, slots, groups, 2] of the pool, a view."""
    blocks = pool.reshape(-1, c.Hkv, R.block_bytes(c.G))
    base = R.sz_place(c.G, is_v, 0, 0)
    return blocks[:, :, base:base + 64 * (128 // c.G) * 4].view(np.uint16).reshape(
        blocks.shape[0], c.Hkv, 64, 128 // c.G, 2)


def codes(pool, c, page, t, is_v, code):
    """Sets the codes [128] of slot t of a page, in all heads."""
    at, sh = R._PLACES[is_v]
    blocks = pool.reshape(-1, c.Hkv, R.block_bytes(c.G))[page]
    for half in (0, 4):
        m = sh[t] == half
        keep = 0xF0 if half == 0 else 0x0F
        blocks[:, at[t][m]] = (blocks[:, at[t][m]] & keep) | (code[m].astype(np.uint8) << half)


def small_weights(seed, n, g, G, meta, v_scale):
    c = Case(seed, (n, 700), g, 1, G, meta, rot="identity")
    c.pool[...] = 0x88                                   # every code 8
    size = R.block_bytes(G)
    region = c.pool.reshape(-1, size)[:, 64 * 64: 2 * 64 * 64]
    region[...] = 0xFF                                   # values: code 15
    put = lambda x: R.stored(np.float32(x), meta)  # noqa: E731
    for is_v in (0, 1):
        e = entries(c.pool, c, is_v)
        scales = v_scale * (1 + 0.11 * np.arange(128 // G)) if is_v else np.full(128 // G, 2.0 ** -10)
        e[..., 0], e[..., 1] = put(scales), put(8.0)     # s (8 - 8): small tokens' keys are 0
    rng = np.random.default_rng(seed)
    sign = rng.choice((-1.0, 1.0), 128)
    a = 1 + np.arange(g) * (8 / 17) / max(1, g - 1)      # gaps of 17 .. 25 in log2
    c.q = torch.from_numpy(np.broadcast_to((a[:, None] * sign).astype(np.float32), (2, g, 128)).copy()).bfloat16()
    s_heavy = 17 / (128 * 7.5 * SM * math.log2(math.e))
    for b in range(2):
        for i in range(4):
            page, t = int(c.table[b, i]), 5 * i + b
            codes(c.pool, c, page, t, 0, np.where(sign > 0, 15, 0))
            codes(c.pool, c, page, t, 1, np.full(128, 8))
            e = entries(c.pool, c, 0)
            e[page, :, t, :, 0], e[page, :, t, :, 1] = put(s_heavy), put(7.5)
    return c, a


@pytest.mark.parametrize("n,v_scale", ((5003, 0.113), (5003, 0.187), (60001, 0.149)))
@pytest.mark.parametrize("g,G,meta", ((1, 32, 0), (4, 32, 0), (3, 128, 1), (7, 64, 0), (12, 32, 1), (16, 128, 0)))
def test_small_weights_keep_their_bits(g, G, meta, n, v_scale):
    c, a = small_weights(50 + g, n, g, G, meta, v_scale)
    ref, w, tol, w_tol = R.attend(c.pool, 1, G, meta, c.q, c.table, c.lens, None, None, SM)
    K, V = R.sequence_values(c.pool, 1, G, meta, c.table[0], n)
    heavy = np.abs(K[:, 0]).sum(-1) > 0
    assert heavy.sum() == 4 and (V[heavy] == 0).all() and (V[~heavy] > 0).all()
    qn = c.q[0].double().numpy()
    score = (qn @ K[heavy, 0][0].astype(np.float64)) * SM           # natural units, per head
    p = np.exp(-score)                                              # a small token's weight beside a heavy one's
    assert p.max() < 2.0 ** -16.9 and p.min() > 2.0 ** -25.2
    s = float(np.abs(K[heavy, 0][0]).max()) / 7.5
    d_heavy = 16 * U * np.abs(qn).sum(-1) * SM * s * 22.5 + 4 * U * score
    s_v = V[~heavy, 0][0].astype(np.float64) / 7                    # per channel
    s_in = np.ldexp(np.frexp(s_v)[0], 11)                           # 2^10 .. 2^11
    pieces = np.maximum(2.0 ** -22, 2.0 ** -25 / (p[:, None] * s_in[None, :]))
    rel = d_heavy[:, None] * 1.01 + pieces + (144 + 2 * -(-n // 256)) * U
    assert (rel < 2.0 ** -9.5).all() and rel[0].max() < 2.0 ** -13  # one piece alone: up to 2^-12 off
    for splits in (1, 0, 3):
        got = c.run(splits).cpu().numpy().astype(np.float64)
        for b in range(2):
            err = np.abs(got[b] / ref[b] - 1)
            assert (err <= rel).all(), (splits, b, float((err / rel).max()), np.argwhere(err > rel)[:4])
    sums = torch.zeros(2, 1, c.mp * 64, device="cuda")
    c.run(0, weights=sums)
    got = sums.cpu().numpy().astype(np.float64)
    err = np.abs(got[0, 0, :n] / w[0, 0, :n] - 1)
    assert (err <= d_heavy.max() * 1.01 + (32 + -(-n // 256)) * U).all(), float(err.max())


@pytest.mark.parametrize("g,G,meta", ((4, 32, 0), (7, 64, 1), (16, 128, 0)))
def test_sum_of_many_small_weights(g, G, meta):
    """The softmax denominator beside heavy tokens, 60000 equal small weights to 4 of 1: here
    the heavy tokens have the value and the others none.  A wave adds a page's weights to its
    sum once (the page's four of a lane are added among themselves first), which is off by u
    times the sum; it has a quarter of the pages at most.  Beside that, as above: the heavy
    score, as far as the small weights' share of the sum goes, the pieces, and 144 u."""
    n = 60001
    c, a = small_weights(70 + g, n, g, G, meta, 0.149)
    blocks = c.pool.reshape(-1, 1, R.block_bytes(G))
    codes15 = np.full(128, 15)
    blocks[:, :, 64 * 64: 2 * 64 * 64] = 0x88                        # values: code 8, zero 8
    for b in range(2):
        for i in range(4):
            codes(c.pool, c, int(c.table[b, i]), 5 * i + b, 1, codes15)
    ref, w, tol, w_tol = R.attend(c.pool, 1, G, meta, c.q, c.table, c.lens, None, None, SM)
    K, V = R.sequence_values(c.pool, 1, G, meta, c.table[0], n)
    heavy = np.abs(K[:, 0]).sum(-1) > 0
    assert heavy.sum() == 4 and (V[heavy] > 0).all() and (V[~heavy] == 0).all()
    qn = c.q[0].double().numpy()
    score = (qn @ K[heavy, 0][0].astype(np.float64)) * SM
    small = (n - 4) * np.exp(-score)
    s = float(np.abs(K[heavy, 0][0]).max()) / 7.5
    d_heavy = 16 * U * np.abs(qn).sum(-1) * SM * s * 22.5 + 4 * U * score
    rel = (d_heavy * small / (4 + small) + 2.0 ** -22 + (144 + -(-n // 256)) * U)[:, None]
    got = c.run(1).cpu().numpy().astype(np.float64)
    err = np.abs(got[0] / ref[0] - 1)
    assert (err <= rel).all(), (float((err / rel).max()), float(err.max()))
