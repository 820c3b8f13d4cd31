"""Attention of chunks over the bf16, 4-bit and 2-bit caches against the definition in 64
bits, within bounds of the library's roundings derived per output."""
import math

import numpy as np
import pytest
import torch

import chunk_ref as R
import kv4_ref
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu
D, P = 128, 64
SM = 1 / math.sqrt(D)
FEW = 32   # (token, head) rows per sequence up to which softmax weights enter as two bf16 pieces


def _poison(n, dtype):
    """Bytes of NaN and infinities in every format that a page holds."""
    if dtype is torch.bfloat16:
        return torch.full((n // 2,), float("nan"), dtype=torch.bfloat16)
    return torch.full((n,), 0xFF, dtype=torch.uint8)


class Cache:
    """Sequences of `lens` tokens in a pool whose other slots and pages hold NaN."""

    def __init__(self, fmt, lens, Hkv, seed=0, G=32, meta=0, per_head=False, spread=1.0, v_spread=None, rot=True,
                 spare=1, pages=None):
        self.fmt, self.lens, self.Hkv, self.G, self.meta = fmt, lens, Hkv, G, meta
        rng = np.random.default_rng(seed)
        self.mp = max(max(lens), 1) // P + 1 + spare
        B = len(lens)
        num_pages = pages or B * self.mp + 1
        self.L = ok.Layout(Hkv, num_pages, group_size=G, meta_dtype=meta, rot_per_head=int(per_head))
        order = rng.permutation(num_pages - 1)[:B * self.mp] + 1        # page 0 stays poison
        self.table = order.reshape(B, self.mp).astype(np.int32)
        size = {"bf16": ok.bf16_pool_bytes, "kv4": ok.kv4_pool_bytes, "kv2": ok.pool_bytes}[fmt](self.L)
        pool = _poison(size, torch.bfloat16 if fmt == "bf16" else torch.uint8)
        self.k, self.v, self.koff, self.voff = [], [], [], []
        for b, n in enumerate(lens):
            at = np.arange(n)
            slots = self.table[b, at // P].astype(np.int64) * P + at % P
            if fmt == "bf16":
                k, v = (torch.from_numpy(rng.standard_normal((n, Hkv, D)) * s).to(torch.bfloat16)
                        for s in (spread, v_spread or spread))
                R.put_bf16(pool, Hkv, torch.from_numpy(slots), k, v)
                self.k.append(k.double().cuda())
                self.v.append(v.double().cuda())
                continue
            for x, (vals, offs) in enumerate(((self.k, self.koff), (self.v, self.voff))):
                code, s, z, val, off = R.random_codes(rng, n, Hkv, G, 16 if fmt == "kv4" else 4, meta,
                                                      (v_spread or spread) if x else spread)
                (kv4_ref.put_rows if fmt == "kv4" else R.put_int2)(pool.numpy(), Hkv, G, slots, x, code, s, z)
                vals.append(torch.from_numpy(val).cuda())
                offs.append(torch.from_numpy(off).cuda())
        self.pool = pool.cuda()
        self.Rk = self.Rv = None
        if fmt != "bf16" and rot:
            n = Hkv if per_head else 1
            q = np.linalg.qr(rng.standard_normal((2, n, D, D)))[0].astype(np.float32)
            q = torch.from_numpy(q).cuda()
            self.Rk, self.Rv = (q[0].contiguous(), q[1].contiguous()) if per_head else (q[0, 0].contiguous(), q[1, 0].contiguous())
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.block_table = torch.from_numpy(self.table).cuda()

    def run(self, q, new, window=0, sinks=0, splits=0, sm=SM, out=None, ws=None, stream=None):
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        out = torch.empty_like(q) if out is None else out
        if ws is None:
            ws = ok.chunk_alloc_workspace(self.L, q.shape[0], len(self.lens), q.shape[1], self.mp, splits,
                                          quantized=self.fmt != "bf16")
            ws.fill_(0xFF)
        args = (self.L, self.pool, q, start, self.block_table, self.seq_lens)
        more = (sm, window, sinks, splits, ws, out)
        if self.fmt == "bf16":
            ok.bf16_chunk_attn(*args, *more, stream=stream)
        else:
            (ok.kv4_chunk_attn if self.fmt == "kv4" else ok.chunk_attn)(*args, self.Rk, self.Rv, *more, stream=stream)
        return out

    def check(self, q, new, out, window=0, sinks=0, sm=SM):
        rows = q.shape[0] * (q.shape[1] // self.Hkv)
        pieces = 2 if rows <= FEW * len(new) else 1
        row = 0
        for b, (n, length) in enumerate(zip(new, self.lens)):
            if n == 0:
                continue
            live = min(n, length)
            dead, x = out[row:row + n - live], out[row + n - live:row + n]
            assert not dead.any(), "sequence %d: a row that sees nothing is not zero" % b
            okm = R.visible(live, length, window, sinks, "cuda")
            ref, tol = R.attend(q[row + n - live:row + n], self.k[b], self.v[b], okm, sm, self.Rk, self.Rv, pieces,
                                self.koff[b] if self.koff else None, self.voff[b] if self.voff else None)
            err = (x.double() - ref).abs()
            bad = ~(err <= tol)
            assert not bad.any(), "sequence %d: %d of %d off, worst %.3g of its bound, at %s" % (
                b, int(bad.sum()), bad.numel(), float((err / tol).nan_to_num(9e9).max()),
                torch.nonzero(bad)[0].tolist())
            row += n


def _q(new, Hq, seed=1, more=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(sum(new) + more, Hq, D, generator=g, device="cuda").to(torch.bfloat16)


CHUNKS = [
    ([1], [1]), ([1], [64]), ([1, 1, 1], [65, 1, 257]), ([2, 0, 5], [2, 30, 129]), ([31], [31]),
    ([64], [64]), ([130], [700]), ([5, 1, 200], [5, 640, 263]), ([0, 0, 1], [0, 70, 70]),
    ([4, 3, 2], [0, 2, 64]), ([257], [257]),
]


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new,lens", CHUNKS)
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (12, 4), (16, 1)])
def test_causal(fmt, new, lens, Hq, Hkv):
    c = Cache(fmt, lens, Hkv, seed=len(lens) + lens[0])
    q = _q(new, Hq)
    c.check(q, new, c.run(q, new))


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 64), (63, 65), (100, 4), (1000, 5), (300, 200),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("new,lens", [([1, 1], [700, 63]), ([70, 3], [449, 65]), ([300], [300])])
def test_window_and_first_tokens(fmt, window, sinks, new, lens):
    c = Cache(fmt, lens, 2, seed=window % 97 + sinks % 89)
    q = _q(new, 8)
    # entries of pages that no new token sees lead to a page of NaN
    for b, (n, length) in enumerate(zip(new, lens)):
        seen = R.visible(n, length, window, sinks).any(0)
        for i in range(c.mp):
            if not seen[i * P:(i + 1) * P].any():
                c.block_table[b, i] = 0
    c.check(q, new, c.run(q, new, window, sinks), window, sinks)


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new", [[1, 1], [90, 2]])
@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64])
def test_splits(fmt, new, splits):
    lens = [1500, 333]
    c = Cache(fmt, lens, 2, seed=3)
    q = _q(new, 8)
    c.check(q, new, c.run(q, new, splits=splits))
    c.check(q, new, c.run(q, new, 200, 70, splits=splits), 200, 70)


MANY = 512   # (token, head) rows per sequence past which 256 rows share a page, and codes are expanded first


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (90, 5), (300, 200)])
@pytest.mark.parametrize("new,lens,Hq,Hkv", [([600], [600], 1, 1), ([515, 0, 600], [900, 64, 610], 2, 1),
                                             ([200], [331], 16, 4), ([100, 170], [1000, 170], 16, 2)])
@pytest.mark.parametrize("splits", [0, 1, 6])
def test_many_rows(fmt, window, sinks, new, lens, Hq, Hkv, splits):
    assert sum(new) * Hq // Hkv > MANY * len(new)
    c = Cache(fmt, lens, Hkv, seed=window + sinks + Hq)
    q = _q(new, Hq)
    for b, (n, length) in enumerate(zip(new, lens)):
        seen = R.visible(n, length, window, sinks).any(0)
        for i in range(c.mp):
            if not seen[i * P:(i + 1) * P].any():
                c.block_table[b, i] = 0
    out = c.run(q, new, window, sinks, splits=splits)
    c.check(q, new, out, window, sinks)
    assert torch.equal(out, c.run(q, new, window, sinks, splits=splits))


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("meta,per_head,rot", [(0, False, True), (1, True, True), (1, False, False)])
@pytest.mark.parametrize("splits", [1, 3])
def test_many_rows_formats(fmt, G, meta, per_head, rot, splits):
    new, lens = [300, 260], [640, 261]
    c = Cache(fmt, lens, 3, seed=G, G=G, meta=meta, per_head=per_head, rot=rot)
    q = _q(new, 6)
    q[3] = 0
    q[5] *= 1e-20
    q[6] *= 40
    c.check(q, new, c.run(q, new, splits=splits))


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
@pytest.mark.parametrize("new", [[600], [80], [3]])
def test_tables_past_what_is_expanded(fmt, new):
    # more than 65536 (page, KV head) pairs in the table: codes are expanded by the blocks that read them
    c = Cache(fmt, [700], 1, seed=16)
    wide = torch.zeros(1, 66000, dtype=torch.int32, device="cuda")
    wide[:, :c.mp] = c.block_table
    c.block_table, c.mp = wide, 66000
    q = _q(new, 2)
    for splits in (0, 1):
        c.check(q, new, c.run(q, new, splits=splits))


@pytest.mark.parametrize("fmt,meta", [("kv4", 0), ("kv4", 1), ("kv2", 0), ("kv2", 1)])
@pytest.mark.parametrize("new", [[2], [90], [520]])
def test_rows_of_zeros_and_of_one_value(fmt, meta, new):
    """What the quantizer stores of rows without a range: scale 1, zero point -value, codes 0."""
    c = Cache(fmt, [600], 1, seed=17, meta=meta)
    Hkv, L = 1, c.L
    pool = ok.kv4_alloc_pool(L) if fmt == "kv4" else ok.alloc_pool(L)
    k = torch.zeros(600, Hkv, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[200:] = 0.75
    v[100:400] = -2.5
    v[400:] = 1e-3
    at = torch.arange(600, device="cuda")
    slots = c.block_table[0].long()[at // P] * P + at % P
    (ok.kv4_append if fmt == "kv4" else ok.kv_append)(L, pool, k, v, slots, None, None, 1.0, 1.0)
    c.pool, c.Rk, c.Rv = pool, None, None
    M = (lambda x: x.to(torch.bfloat16 if meta else torch.float16).double())
    c.k, c.v = [M(k.float())], [M(v.float())]
    c.koff, c.voff = [c.k[0].abs()], [c.v[0].abs()]
    q = _q(new, 2)
    c.check(q, new, c.run(q, new))


def test_one_workspace_for_smaller_chunks():
    for fmt in ("bf16", "kv4"):
        c = Cache(fmt, [3000], 2, seed=18)
        ws = ok.chunk_alloc_workspace(c.L, 1100, 1, 4, c.mp, 0, quantized=fmt != "bf16")
        for n in (1100, 600, 250, 30, 1):
            q = _q([n], 4)
            c.check(q, [n], c.run(q, [n], ws=ws))


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
def test_debug_checks(fmt, monkeypatch):
    monkeypatch.setenv("OSCAR_DEBUG", "1")
    new, lens = [2, 3], [200, 64]
    c = Cache(fmt, lens, 1, seed=19)
    q = _q(new, 2)
    out = torch.full_like(q, 3.0)
    c.run(q, new, out=out)
    c.check(q, new, out)
    table, lens_t = c.block_table.clone(), c.seq_lens.clone()
    out.fill_(3.0)

    def refused(**kw):
        with pytest.raises(ok.OscarError) as e:
            c.run(q, kw.pop("new", new), out=out, **kw)
        assert e.value.status == ok.ERR_INVALID_ARG and (out == 3.0).all()
    c.block_table[1, 0] = c.L.num_pages        # (never dereferenced)
    refused()
    c.block_table[1, 0] = -1
    refused()
    c.block_table.copy_(table)
    c.block_table[0, 0] = -1                    # outside the window: not looked at
    refused()
    c.run(q, new, window=70, out=out)
    c.block_table.copy_(table)
    out.fill_(3.0)
    c.seq_lens[0] = c.mp * P + 1
    refused()
    c.seq_lens.copy_(lens_t)
    refused(new=[4, 2])                          # 6 rows of 5
    refused(new=[3, -1])                         # descending


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("meta,per_head,rot", [(0, False, True), (1, True, True), (1, False, False)])
def test_formats(fmt, G, meta, per_head, rot):
    for new, lens in (([3, 1], [200, 65]), ([80, 60], [321, 60])):
        c = Cache(fmt, lens, 3, seed=G, G=G, meta=meta, per_head=per_head, rot=rot)
        q = _q(new, 6)
        c.check(q, new, c.run(q, new))


@pytest.mark.parametrize("fmt,meta,spread,v_spread", [
    ("bf16", 0, 1e-3, 1e-20), ("bf16", 0, 3.0, 1e30), ("kv4", 0, 1.0, 1e-3), ("kv4", 0, 4.0, 5e3), ("kv4", 1, 1e-6, 1e-12),
    ("kv4", 1, 4.0, 1e14), ("kv2", 0, 2.0, 8e3), ("kv2", 1, 1e-9, 1e12)])
@pytest.mark.parametrize("new", [[2], [150]])
def test_scales(fmt, meta, spread, v_spread, new):
    c = Cache(fmt, [400], 1, seed=4, meta=meta, spread=spread, v_spread=v_spread)
    q = _q(new, 4)
    c.check(q, new, c.run(q, new))


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
def test_scales_that_differ_between_pages(fmt):
    # the accumulators' exponent moves up and down again
    for new in ([1], [100]):
        c = Cache(fmt, [640], 1, seed=5, meta=1)
        grow = Cache(fmt, [640], 1, seed=5, meta=1)
        # the same codes; V's scales of the pages times 2^(0, 9, -7, 20, 3, ...)
        shift = [0, 9, -7, 20, 3, 18, -20, 1, 0, 2]
        half = P * D // (2 if fmt == "kv4" else 4)
        size = 2 * half + 2 * 4 * P * 4
        pool = grow.pool.view(-1, size)
        for i, e in enumerate(shift):
            page = int(grow.table[0, i])
            sz = pool[page, 2 * half + P * 16:].view(torch.bfloat16)
            sz[0::2] = (sz[0::2].float() * 2.0 ** e).to(torch.bfloat16)
            grow.v[0][i * P:(i + 1) * P] *= 2.0 ** e
            grow.voff[0][i * P:(i + 1) * P] *= 2.0 ** e
        q = _q(new, 4)
        grow.check(q, new, grow.run(q, new))
        assert not torch.equal(grow.run(q, new), c.run(q, new))


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("sm", [0.0, -0.07, 1.5])
def test_logit_scales(fmt, sm):
    for new in ([2], [77]):
        c = Cache(fmt, [150], 2, seed=6)
        q = _q(new, 4)
        c.check(q, new, c.run(q, new, sm=sm), sm=sm)


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
def test_queries_of_zero_and_of_any_size(fmt):
    c = Cache(fmt, [130, 90], 1, seed=7)
    for new in ([6, 6], [50, 60]):
        q = _q(new, 2)
        q[0] = 0
        q[1] *= 1e-20
        q[2] *= 30
        c.check(q, new, c.run(q, new))


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new", [[1, 3], [100, 3]])
@pytest.mark.parametrize("splits", [1, 4])
def test_a_row_with_nan_spoils_itself_only(fmt, new, splits):
    c = Cache(fmt, [600, 100], 2, seed=8)
    q = _q(new, 4)
    good = c.run(q, new, splits=splits)
    bad = q.clone()
    bad[0, 1, 7] = float("nan")
    bad[-1, 3, 100] = float("nan")
    out = c.run(bad, new, splits=splits)
    hit = torch.zeros(q.shape[0], 4, dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[-1, 3] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], good[~hit])


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("splits", [1, 5])
def test_rows_behind_the_last_sequence_stay(fmt, splits):
    for new in ([2, 1], [70, 1]):
        c = Cache(fmt, [300, 64], 2, seed=9)
        q = _q(new, 4, more=37)
        out = torch.full_like(q, 7.0)
        c.run(q, new, splits=splits, out=out)
        c.check(q, new, out)
        assert (out[sum(new):] == 7.0).all()


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
def test_many_sequences(fmt):
    # more than a wave looks at in one step, and more than 64 of those
    rng = np.random.default_rng(10)
    lens = rng.integers(0, 70, 300).tolist()
    new = [int(rng.integers(0, min(n, 5) + 1)) for n in lens]
    new[17], lens[17] = 40, 40
    c = Cache(fmt, lens, 1, seed=10, spare=0)
    q = _q(new, 2)
    c.check(q, new, c.run(q, new))


@pytest.mark.parametrize("fmt,Hkv", [("bf16", 8), ("bf16", 1), ("kv4", 8), ("kv2", 1)])
@pytest.mark.parametrize("B,most", [(33, 4), (64, 90), (65, 8), (129, 9), (256, 2), (257, 40)])
def test_tiles_of_many_sequences(fmt, Hkv, B, most):
    # each block finds its tile among the sequences'; none, one or more of a sequence, some without new tokens
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 150, B).tolist()
    new = [int(rng.integers(0, min(n, most) + 1)) for n in lens]
    new[0], new[B // 2], new[B - 1] = 0, min(lens[B // 2], most), 0
    c = Cache(fmt, lens, Hkv, seed=B, spare=0)
    q = _q(new, 4 * Hkv, seed=B, more=3)
    out = torch.full_like(q, 7.0)
    c.run(q, new, splits=1, out=out)
    c.check(q, new, out)
    assert bool((out[sum(new):] == 7.0).all())


def test_thousands_of_sequences():
    B = 5000
    c = Cache("bf16", [3], 1, seed=11)
    rng = np.random.default_rng(11)
    new = rng.integers(0, 3, B)
    q = _q(new.tolist(), 2)
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    table = c.block_table[:1].expand(B, -1).contiguous()
    lens = torch.full((B,), 3, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = ok.chunk_alloc_workspace(c.L, q.shape[0], B, 2, c.mp, quantized=False)
    ok.bf16_chunk_attn(c.L, c.pool, q, start, table, lens, SM, 0, 0, 0, ws, out)
    one, two = np.flatnonzero(new == 1), np.flatnonzero(new == 2)
    s = np.concatenate([[0], np.cumsum(new)])
    for rows, n in ((s[one], 1), (s[two], 2)):
        at = torch.from_numpy(rows).cuda()
        at = torch.stack([at + i for i in range(n)], 1).flatten()
        for j in range(n):
            okm = R.visible(n, 3, 0, 0, "cuda")[j:j + 1]
            x = q[at[j::n]]
            ref, tol = R.attend(x, c.k[0], c.v[0], okm.expand(x.shape[0], -1), SM, pieces=2)
            assert ((out[at[j::n]].double() - ref).abs() <= tol).all()


def test_pool_past_4_gib():
    pages = (5 << 30) // (2 * P * D * 2)
    c = Cache("bf16", [100], 1, seed=12)
    L = ok.Layout(1, pages)
    pool = torch.empty(ok.bf16_pool_bytes(L) // 2, dtype=torch.bfloat16, device="cuda")
    moved = torch.arange(pages - c.mp, pages, dtype=torch.int32, device="cuda")[None]
    pool.view(-1, 2 * P * D)[moved[0].long()] = c.pool.view(-1, 2 * P * D)[c.block_table[0].long()]
    for new in ([3], [60]):
        q = _q(new, 4)
        ref = c.run(q, new)
        out = torch.empty_like(q)
        start = torch.tensor([0, new[0]], dtype=torch.int32, device="cuda")
        ws = ok.chunk_alloc_workspace(L, new[0], 1, 4, c.mp, quantized=False)
        ok.bf16_chunk_attn(L, pool, q, start, moved, c.seq_lens, SM, 0, 0, 0, ws, out)
        assert torch.equal(out, ref)


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
def test_one_token_agrees_with_decode(fmt):
    lens = [1000, 77, 64]
    c = Cache(fmt, lens, 2, seed=13)
    q = _q([1, 1, 1], 8)
    out = c.run(q, [1, 1, 1])
    dec = torch.empty(3, 8, D, device="cuda")
    if fmt == "bf16":
        ws = ok.alloc_workspace(c.L, 3, 8, 4)
        ok.bf16_decode_attn(c.L, c.pool, q, c.block_table, c.seq_lens, SM, 4, ws, dec)
    elif fmt == "kv4":
        ws = ok.kv4_alloc_workspace(c.L, 3, 8, 4, c.mp)
        ok.kv4_decode_attn(c.L, c.pool, q, c.block_table, c.seq_lens, c.Rk, c.Rv, SM, 4, ws, dec)
    else:
        ws = ok.alloc_workspace(c.L, 3, 8, 4)
        ok.decode_attn(c.L, c.pool, q, c.block_table, c.seq_lens, c.Rk, c.Rv, SM, 4, ws, dec)
    row = 0
    for b, n in enumerate(lens):
        okm = R.visible(1, n, 0, 0, "cuda")
        _, tol = R.attend(q[b:b + 1], c.k[b], c.v[b], okm, SM, c.Rk, c.Rv, 2, c.koff[b] if c.koff else None,
                          c.voff[b] if c.voff else None)
        # (decode's own distance from the definition: 2e-3, as its tests ask)
        assert ((out[b:b + 1].double() - dec[b:b + 1].double()).abs() <= tol + 2e-3).all()


@pytest.mark.parametrize("fmt", ["bf16", "kv4", "kv2"])
@pytest.mark.parametrize("new", [[1, 4], [90, 33]])
def test_captured_and_replayed_and_on_two_streams(fmt, new):
    lens = [800, 300]
    c = Cache(fmt, lens, 2, seed=14)
    q = _q(new, 8)
    want = c.run(q, new, splits=3)
    start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    wss = [ok.chunk_alloc_workspace(c.L, sum(new), 2, 8, c.mp, 3, quantized=fmt != "bf16") for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]

    def call(i, x, stream=None):
        args = (c.L, c.pool, x, start, c.block_table, c.seq_lens)
        more = (SM, 0, 0, 3, wss[i], outs[i])
        if fmt == "bf16":
            ok.bf16_chunk_attn(*args, *more, stream=stream)
        else:
            (ok.kv4_chunk_attn if fmt == "kv4" else ok.chunk_attn)(*args, c.Rk, c.Rv, *more, stream=stream)
    call(0, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    x = q.clone()
    with torch.cuda.graph(graph):
        call(0, x)
    for k in range(3):
        x.copy_(q * (k + 1))
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = c.run(x, new, splits=3)
        assert torch.equal(outs[0], eager)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            call(i, q, s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_path_from_the_projection():
    """A prompt in chunks, then drafted tokens, through norm and rotation, both caches and their attention."""
    Hq, Hkv, T = 8, 2, 150
    g = torch.Generator(device="cuda").manual_seed(15)
    x = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = (y.unflatten(1, (-1, D)) for y in x.split((Hq * D, Hkv * D, Hkv * D), 1))
    w = (1 + 0.1 * torch.randn(2, D, generator=g, device="cuda")).to(torch.bfloat16)
    rope = ok.Rope(64, ok.rope_freqs(64, 1e4, ok.ROPE_BY_INDEX, 4.0, 64.0), interleaved=True, attn_scale=1.1)
    pos = torch.arange(T, device="cuda")
    L = ok.Layout(Hkv, 5)
    table = torch.tensor([[3, 0, 4]], dtype=torch.int32, device="cuda")
    slots = table[0].long()[pos // P] * P + pos % P
    R0 = torch.linalg.qr(torch.randn(2, D, D, generator=g, device="cuda", dtype=torch.float64))[0].float()
    Rk, Rv = R0[0].contiguous(), R0[1].contiguous()
    bf = torch.zeros(ok.bf16_pool_bytes(L) // 2, dtype=torch.bfloat16, device="cuda")
    k4, k2 = ok.kv4_alloc_pool(L), ok.alloc_pool(L)
    outs = {n: torch.zeros(T, Hq, D, dtype=torch.bfloat16, device="cuda") for n in ("bf16", "kv4", "kv2")}
    qs, ks = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, Hkv, D, dtype=torch.bfloat16, device="cuda")
    ws = ok.chunk_alloc_workspace(L, T, 1, Hq, 3, 4)
    for a, b in ((0, 70), (70, 71), (71, 140), (140, 145), (145, 150)):
        e = slice(a, b)
        ok.bf16_kv_append_rope(L, bf, rope, k[e], v[e], slots[e], pos[e], q=q[e], q_out=qs[e], q_weight=w[0], k_weight=w[1])
        q2 = torch.empty_like(qs[e])
        ok.qk_norm_rope(L, rope, q[e], k[e], pos[e], q2, ks[e], q_weight=w[0], k_weight=w[1])
        assert torch.equal(q2, qs[e])
        ok.kv4_append(L, k4, ks[e], v[e].contiguous(), slots[e], Rk, Rv, 1.0, 1.0)
        ok.kv_append(L, k2, ks[e], v[e].contiguous(), slots[e], Rk, Rv, 1.0, 1.0)
        start = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        n = torch.tensor([b], dtype=torch.int32, device="cuda")
        ok.bf16_chunk_attn(L, bf, qs[e], start, table, n, SM, 100, 4, 0, ws, outs["bf16"][e])
        ok.kv4_chunk_attn(L, k4, qs[e], start, table, n, Rk, Rv, SM, 100, 4, 0, ws, outs["kv4"][e])
        ok.chunk_attn(L, k2, qs[e], start, table, n, Rk, Rv, SM, 100, 4, 0, ws, outs["kv2"][e])
    okm = R.visible(T, T, 100, 4, "cuda")
    ref, tol = R.attend(qs, ks.double(), v.double(), okm, SM)
    assert ((outs["bf16"].double() - ref).abs() <= tol).all()
    # 4 bits: against the values that the cache reads back (fp32 products and differences)
    kk, vv = (torch.empty(T, Hkv, D, device="cuda") for _ in range(2))
    ok.kv4_gather(L, k4, slots, kk, vv)
    top = [y.abs().amax().expand_as(y).double() for y in (kk, vv)]   # |s z| is below twice a row's largest value
    ref4, tol4 = R.attend(qs, kk.double(), vv.double(), okm, SM, Rk, Rv, 1, 2 * top[0], 2 * top[1])
    assert ((outs["kv4"].double() - ref4).abs() <= tol4).all()
    # 2 bits lose a lot, but not the direction
    cos = torch.nn.functional.cosine_similarity(outs["kv2"].double().flatten(1), ref.flatten(1))
    assert cos.min() > 0.5
