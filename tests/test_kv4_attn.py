"""Decode attention over the 4-bit cache against 64-bit attention on the pool's bytes.
The tolerance is the first-order bound of fp32 arithmetic that kv4_ref.attend derives
per output; bf16 outputs are the nearest-even rounding of the fp32 ones."""
import math

import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu

SM = 1.0 / math.sqrt(128)
FORMATS = [(32, 0), (64, 0), (128, 1), (32, 1), (64, 1), (128, 0)]


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Case:
    def __init__(self, seed, lens, Hq, Hkv, G=32, meta=0, spare=1, rot="shared", scale=0.1, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int32)
        self.B, self.Hq, self.Hkv, self.G, self.meta = len(lens), Hq, Hkv, G, meta
        self.mp = max(1, -(-int(self.lens.max()) // 64)) + spare
        used = [-(-int(n) // 64) for n in self.lens]
        num = sum(used) + 2
        perm = rng.permutation(num)
        self.table = np.full((self.B, self.mp), 2 ** 30, np.int32)   # entries past a sequence: never read
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        self.pool = R.random_pool(rng, num, Hkv, G, meta, scale)
        blocks = self.pool.reshape(num, Hkv, -1)
        for b, n in enumerate(self.lens):   # slots past a length: metadata of NaN and infinity
            if n % 64:
                blk = blocks[self.table[b, n // 64]]
                for is_v in (0, 1):
                    e = R.sz_place(G, is_v, int(n) % 64, 0)
                    end = R.sz_place(G, is_v, 63, 128 // G - 1) + 4
                    blk[:, e:end] = np.resize(np.array([0xFF, 0x7F, 0xC0, 0xFF, 0x00, 0x7C], np.uint8), end - e)
        self.q = torch.from_numpy(rng.standard_normal((self.B, Hq, 128)).astype(np.float32) * q_scale).bfloat16()
        rph = rot == "per_head"
        m = np.stack([R.rotation(rng) for _ in range(2 * Hkv)])
        self.Rk, self.Rv = {"shared": (m[0], m[1]), "identity": (None, None), "identity_v": (m[0], None),
                            "per_head": (m[:Hkv], m[Hkv:])}[rot]
        self.lay = ok.Layout(Hkv, num, group_size=G, meta_dtype=meta, rot_per_head=int(rph))
        self.rng = rng

    def run(self, splits, dtype=torch.float32, weights=None, weights_out=None, pool=None):
        out = torch.full((self.B, self.Hq, 128), float("nan"), dtype=dtype, device="cuda")
        s = splits or ok.default_num_splits(self.lay, self.B, self.Hq, self.mp * 64)
        ws = torch.full((ok.kv4_decode_workspace_bytes(self.lay, self.B, self.Hq, s, self.mp, weights is not None),),
                        255, dtype=torch.uint8, device="cuda")
        ok.kv4_decode_attn(self.lay, dev(self.pool) if pool is None else pool, self.q.cuda(), dev(self.table),
                           dev(self.lens), dev(self.Rk), dev(self.Rv), SM, splits, ws, out, weights=weights,
                           weights_out=weights_out)
        return out

    def check(self, splits=(0, 1, 3)):
        ref, w, tol, w_tol = R.attend(self.pool, self.Hkv, self.G, self.meta, self.q, self.table, self.lens,
                                      self.Rk, self.Rv, SM)
        for s in splits:
            out = self.run(s)
            got = out.cpu().numpy().astype(np.float64)
            assert np.isfinite(got).all()
            err = np.abs(got - ref)
            worst = float((err - tol).max())
            assert worst <= 0, (s, worst, float(err.max()), float(tol.max()))
            assert torch.equal(self.run(s, torch.bfloat16), out.bfloat16())
            assert (got[self.lens == 0] == 0).all()
        sums = torch.full((self.B, self.Hkv, self.mp * 64), 3.0, device="cuda")
        for b, n in enumerate(self.lens):
            sums[b, :, n:] = float("nan")
        for in_place in (False, True):
            w_in = sums.clone()
            w_out = w_in if in_place else torch.full_like(sums, 5.0)
            out_w = self.run(0, weights=w_in, weights_out=None if in_place else w_out)
            assert torch.equal(out_w, self.run(0))
            got = w_out.cpu().numpy().astype(np.float64)
            for b, n in enumerate(self.lens):
                err = np.abs(got[b, :, :n] - 3.0 - w[b, :, :n])
                assert (err <= w_tol[b, :, :n] + 2.0 ** -23 * (3 + w[b, :, :n])).all(), float(err.max())
                tail = got[b, :, n:]
                assert np.isnan(tail).all() if in_place else (tail == 5.0).all()


@pytest.mark.parametrize("g", range(1, 17))
def test_heads_per_kv_head(g):
    Case(g, (1, 130, 64, 0, 333), 2 * g, 2, *FORMATS[g % len(FORMATS)]).check()


@pytest.mark.parametrize("G,meta", FORMATS)
@pytest.mark.parametrize("g", (1, 4, 7, 12, 16))
def test_formats(G, meta, g):
    Case(40 + g, (65, 200), 3 * g, 3, G, meta).check((0,))


@pytest.mark.parametrize("n", (1, 2, 63, 64, 65, 127, 128, 129, 255, 257, 1000))
@pytest.mark.parametrize("g", (3, 10))
def test_lengths(n, g):
    Case(n, (n,), g, 1).check((0, 1, 2, 7))


@pytest.mark.parametrize("rot", ("identity", "identity_v", "per_head"))
def test_rotations(rot):
    Case(5, (70, 300, 1), 15, 3, rot=rot).check((0,))


@pytest.mark.parametrize("scale,q_scale,meta", [(2.0 ** -24, 1.0, 0), (300.0, 0.01, 0), (1e-20, 1.0, 1),
                                                (1e12, 1e-12, 1), (0.1, 12.0, 0)])
def test_magnitudes(scale, q_scale, meta):
    """Scales at the ends of their formats, and logits that leave one token all the weight."""
    c = Case(6, (90, 700), 8, 2, 32, meta, scale=scale, q_scale=q_scale)
    c.check((0, 1))


@pytest.mark.parametrize("g", (4, 9))
def test_smallest_bf16_scales(g):
    """Scales near the least normal bf16, whose reciprocals have no power of two in fp32."""
    Case(9, (90, 700), 2 * g, 2, 32, 1, rot="identity", scale=1e-37).check((0, 1))


def test_one_heavy_token_among_many():
    """A token with nearly all the weight, and 5000 others 2^-17 of it each: the small
    weights keep their bits."""
    c = Case(7, (5000,), 4, 1, 128, 0, rot="identity")
    blocks = c.pool.reshape(-1, 1, R.block_bytes(128))
    base = R.sz_place(128, 0, 0, 0)
    e = blocks[:, :, base:base + 256].view(np.uint16).reshape(-1, 1, 64, 2)
    e[..., 0] = np.float16(1e-4).view(np.uint16)       # small K scales: logits near 0
    first = int(c.table[0, 0])
    e[first, 0, 0, 0] = np.float16(0.12).view(np.uint16)
    c.check((0, 1))


@pytest.mark.parametrize("splits", (0, 1, 4))
def test_many_short_sequences(splits):
    """More sequences than a wave's lanes, most of them empty or a few tokens."""
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 4, 700) * rng.integers(0, 40, 700)
    Case(8, lens, 4, 2).check((splits,))


def test_many_pages_per_wave():
    """Ranges of more than 64 pages per wave (page ids are read 64 at a time)."""
    rng = np.random.default_rng(11)
    c = Case(11, (64 * 700 + 5,), 2, 1, 128, 1)
    c.check((1,))


def test_lengths_past_the_block_table_are_clamped():
    c = Case(12, (128, 100), 4, 1, spare=0)
    ref = c.run(0)
    c.lens = np.array([9999, 100], np.int32)
    assert torch.equal(c.run(0), ref)
    c.lens = np.array([-5, 100], np.int32)
    out = c.run(0)
    assert (out[0] == 0).all() and torch.equal(out[1], ref[1])


def test_pages_past_4_gib():
    c = Case(13, (200, 64), 8, 8)
    num = 54000
    lay = ok.Layout(8, num)
    pool = torch.zeros(ok.kv4_pool_bytes(lay), dtype=torch.uint8, device="cuda")
    size = R.block_bytes(32) * 8
    small = torch.from_numpy(c.pool).cuda().view(-1, size)
    far = num - small.shape[0]
    pool.view(num, size)[far:] = small
    ref = c.run(0)
    c.lay, c.table = lay, np.where(c.table < 2 ** 30, c.table + far, c.table).astype(np.int32)
    assert torch.equal(c.run(0, pool=pool), ref)


@pytest.mark.parametrize("g,Hkv", ((4, 2), (12, 1)))
@pytest.mark.parametrize("n_new", (0, 3))
def test_step_is_append_then_attention(g, Hkv, n_new):
    c = Case(14, (65, 1, 130), g * Hkv, Hkv)
    k, v = (torch.from_numpy(c.rng.standard_normal((n_new, Hkv, 128)).astype(np.float32)).bfloat16().cuda()
            for _ in range(2))
    slots = torch.tensor([int(c.table[b, (n - 1) // 64]) * 64 + (n - 1) % 64 for b, n in enumerate(c.lens)][:n_new],
                         dtype=torch.int64, device="cuda")
    pools = [dev(c.pool), dev(c.pool)]
    sums = torch.rand(c.B, Hkv, c.mp * 64, device="cuda")
    if n_new:
        ok.kv4_append(c.lay, pools[0], k, v, slots, dev(c.Rk), dev(c.Rv), 0.9, 0.95)
    w0 = torch.zeros_like(sums)
    ref = c.run(3, weights=sums, weights_out=w0, pool=pools[0])
    ws = ok.kv4_alloc_workspace(c.lay, c.B, c.Hq, 3, c.mp, weights=True)
    out, w1 = torch.empty_like(ref), torch.zeros_like(sums)
    ok.kv4_decode_step(c.lay, pools[1], k, v, slots, 0.9, 0.95, c.q.cuda(), dev(c.table), dev(c.lens), dev(c.Rk),
                       dev(c.Rv), SM, 3, ws, out, weights=sums, weights_out=w1)
    assert torch.equal(pools[0], pools[1]) and torch.equal(out, ref) and torch.equal(w0, w1)


def test_same_result_every_time_and_on_another_stream():
    c = Case(15, (3000, 77, 1500), 16, 2)
    ref = c.run(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [c.run(0) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    ws = ok.kv4_alloc_workspace(c.lay, c.B, c.Hq, 4, c.mp)
    args = (c.lay, dev(c.pool), c.q.cuda(), dev(c.table), dev(c.lens), dev(c.Rk), dev(c.Rv), SM, 4, ws)
    a, b = torch.zeros(c.B, c.Hq, 128, device="cuda"), torch.zeros(c.B, c.Hq, 128, device="cuda")
    ok.kv4_decode_attn(*args, a)
    torch.cuda.synchronize()
    ok.kv4_decode_attn(*args, b, stream=side)
    side.synchronize()
    assert torch.equal(a, b)


def test_python_refusals():
    c = Case(16, (65, 64), 4, 2)
    ws = ok.kv4_alloc_workspace(c.lay, 2, 4, 2, c.mp, weights=True)
    good = dict(pages=dev(c.pool), q=c.q.cuda(), block_table=dev(c.table), seq_lens=dev(c.lens), R_k=dev(c.Rk),
                R_v=dev(c.Rv), sm_scale=SM, num_splits=2, workspace=ws, out=torch.zeros(2, 4, 128, device="cuda"),
                weights=torch.zeros(2, 2, c.mp * 64, device="cuda"))
    ok.kv4_decode_attn(c.lay, **good)
    w = good["weights"]
    bad = [dict(q=good["q"].float()), dict(q=good["q"][:1]), dict(q=good["q"].cpu()), dict(out=good["out"].half()),
           dict(out=good["out"][:1]), dict(out=None), dict(weights=w[:, :1].contiguous()), dict(weights=w.double()),
           dict(weights=None, weights_out=w), dict(weights_out=w[..., :64].contiguous()),
           dict(block_table=good["block_table"].long()), dict(block_table=good["block_table"].t()),
           dict(seq_lens=good["seq_lens"][:1]), dict(pages=good["pages"][:-16]), dict(workspace=ws[:256]),
           dict(workspace=ws.cpu()), dict(num_splits=-1), dict(sm_scale=float("nan"))]
    for change in bad:
        with pytest.raises((TypeError, ValueError, ok.OscarError)):
            ok.kv4_decode_attn(c.lay, **{**good, **change})
