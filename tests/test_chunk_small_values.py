"""Attention of chunks over the 4-bit and 2-bit caches where small values lie beside large
scales: rows without a range (stored with scale 1 whatever their value) and outliers.  Bounds
per page and per token, from the roundings that include/oscar.h names."""
import math

import numpy as np
import pytest
import torch

import chunk_ref as R
import kv4_ref
import paper_2605_17757_amd as ok
from test_chunk_attn import SM, Cache

pytestmark = pytest.mark.gpu
D, P = 128, 64
U32, U16, UB = R.U32, R.U16, R.UB
ROWS = [2, 90, 600]                      # tiles of 32, 128 and 256 rows (one head)
FORMATS = [("kv4", 0, 32), ("kv4", 1, 128), ("kv2", 0, 128), ("kv2", 1, 32), ("kv2", 0, 64)]


def quantized(x, G, levels, meta):
    """The library's quantizer without clipping: rows [n, H, D] -> codes, scale and zero bits."""
    n, H, _ = x.shape
    y = np.asarray(x, np.float32).reshape(n, H, D // G, G)
    lo, hi = y.min(-1), y.max(-1)
    s = kv4_ref.stored((hi - lo) / np.float32(levels - 1), meta).reshape(lo.shape)
    deg = (s & 0x7FFF) == 0
    s = np.where(deg, 0x3F80 if meta else 0x3C00, s).astype(np.uint16)
    sf = kv4_ref.f32_of(s, meta).reshape(lo.shape)
    z = kv4_ref.stored(np.where(deg, -lo, -lo / sf), meta).reshape(lo.shape)
    zf = kv4_ref.f32_of(z, meta).reshape(lo.shape)
    code = np.clip(np.rint(y / sf[..., None] + zf[..., None]), 0, levels - 1)
    return np.where(deg[..., None], 0, code).astype(np.uint8).reshape(n, H, D), s, z


class Rows(Cache):
    """One sequence whose rows are the quantizer's of k and v [n, D] (identity rotations)."""

    def __init__(self, fmt, meta, G, k, v):
        super().__init__(fmt, [len(k)], 1, seed=1, G=G, meta=meta, rot=False)
        levels = 16 if fmt == "kv4" else 4
        pool = self.pool.cpu()
        at = np.arange(len(k))
        slots = self.table[0, at // P].astype(np.int64) * P + at % P
        self.err = []
        for is_v, x in enumerate((k, v)):
            code, s, z = quantized(x[:, None], G, levels, meta)
            (kv4_ref.put_rows if fmt == "kv4" else R.put_int2)(pool.numpy(), 1, G, slots, is_v, code, s, z)
            sf, zf = (kv4_ref.f32_of(y, meta).reshape(len(k), D // G).astype(np.float64) for y in (s, z))
            val = (sf[..., None] * (code.reshape(len(k), D // G, G) - zf[..., None])).reshape(len(k), D)
            # x to fp16, -s z before it, and every entry against its page's largest
            top = np.maximum(abs(sf) * (levels - 1), abs(sf * zf)).max(-1)
            page = np.array([top[i // P * P:i // P * P + P].max() for i in range(len(k))])
            err = U16 * (abs(val) + np.repeat(abs(sf * zf), G, 1)) * 1.001 + page[:, None] * 2.0 ** -31
            (self.v if is_v else self.k)[0] = torch.from_numpy(val).cuda()[:, None]
            self.err.append(torch.from_numpy(err).cuda())
        self.pool = pool.cuda()

    def check_closely(self, q, out, sm=SM):
        n, length = q.shape[0], self.lens[0]
        K, V, (dk, dv) = self.k[0][:, 0], self.v[0][:, 0], self.err
        okm = R.visible(n, length, 0, 0, "cuda")
        x = q[:, 0].double()
        mag = abs(sm) * (x.abs() @ K.abs().T)
        s = (sm * (x @ K.T)).masked_fill(~okm, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - m)
        den = p.sum(-1, keepdim=True)
        p = p / den
        o = p @ V
        # a score: q to fp16 (before and after a rotation by the identity), K's errors, 128 products
        # summed in fp32, its factor and exponent
        ds = abs(sm) * (x.abs() @ dk.T) + 3 * U16 * mag + 150 * U32 * (mag + m.abs() + s.abs()) + 2.0 ** -20
        ds = torch.where(okm, ds, torch.zeros_like(ds)).clamp(max=80)
        # a weight that is off moves the output by that times the value's distance from the output, for any
        # constant c at most |v - c| + |o - c|; its rounding to fp16 is the numerator's alone
        w, c = p * torch.expm1(2 * ds), V.mean(0)
        t = w @ (V - c).abs() + (o - c).abs() * w.sum(-1, keepdim=True) + p @ dv
        w = p * (U16 + 2 * (length + 128) * U32) + okm * (p.amax(-1, keepdim=True) * 2.0 ** -30)
        t = t + w @ V.abs() + o.abs() * 2 * (length + 128) * U32
        t = t + o.abs() * (2 * U16 + 150 * U32)        # o to fp16, rotated by the identity, 1 / sum
        t = t + UB * (o.abs() + t) + 1e-38
        err = (out[:, 0].double() - o).abs()
        bad = ~(err <= t)
        assert not bad.any(), "%d of %d off, worst %.3g of its bound, %.3g of its value, at %s" % (
            int(bad.sum()), bad.numel(), float((err / t).nan_to_num(9e9).max()),
            float((err / o.abs()).nan_to_num(0.0).max()), torch.nonzero(bad)[0].tolist())
        return o, t


def _q(n, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(3)
    return (scale * torch.randn(n, 1, D, generator=g, device="cuda")).to(torch.bfloat16)


@pytest.mark.parametrize("fmt,meta,G", FORMATS)
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("value", [1e-3, 1e-4, -7e-5])
def test_values_without_a_range(fmt, meta, G, n, value):
    rng = np.random.default_rng(1)
    v = np.full((max(n, 300), D), value)
    c = Rows(fmt, meta, G, rng.standard_normal(v.shape), v)
    q = _q(n)
    o, t = c.check_closely(q, c.run(q, [n]))
    assert (t <= 2.0 ** -6 * o.abs()).all()       # the bound itself is no larger than some roundings


@pytest.mark.parametrize("fmt,meta,G", FORMATS)
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("size", [1e-3, 1e-4])
def test_a_row_of_zeros_among_small_values(fmt, meta, G, n, size):
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, max(n, 300), D))
    v *= size
    v[5] = 0.0
    c = Rows(fmt, meta, G, k, v)
    q = _q(n)
    c.check_closely(q, c.run(q, [n]))


@pytest.mark.parametrize("fmt,meta,G", FORMATS)
@pytest.mark.parametrize("n", ROWS)
def test_keys_beside_a_row_of_zeros(fmt, meta, G, n):
    rng = np.random.default_rng(4)
    k, v = rng.standard_normal((2, max(n, 300), D))
    k *= 1e-3
    k[::64] = 0.0
    k[1::64] = 1e-3
    c = Rows(fmt, meta, G, k, v)
    q = _q(n)
    c.check_closely(q, c.run(q, [n], sm=100.0), sm=100.0)


@pytest.mark.parametrize("fmt,meta,G", FORMATS)
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("page", [0, 2])
@pytest.mark.parametrize("shift", [14, 17])
def test_an_outlier_that_no_query_looks_at(fmt, meta, G, n, page, shift):
    """A token of 2^shift times the others' values, before or after them, with a weight of about e^-100."""
    rng = np.random.default_rng(5)
    k, v = 0.3 * rng.standard_normal((2, max(n, 300), D))
    if meta == 0:
        v *= 2.0 ** -6                             # its zero point and scale stay fp16 numbers
    at = 64 * page + 7
    g = torch.Generator().manual_seed(6)
    u = torch.randn(D, generator=g)
    k[at] = -9.0 * u.numpy()
    v[at] *= 2.0 ** shift
    q = (u + 0.2 * torch.randn(n, 1, D, generator=g)).to(torch.bfloat16).cuda()
    c = Rows(fmt, meta, G, k, v)
    c.check_closely(q, c.run(q, [n]))


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("shifts", [(40, 0, 0, -20, 0), (0, -30, 30, 0, 0), (0, 20, -20, 20, -20), (55, 0, 55, 0, 0)])
def test_pages_of_other_sizes_that_no_query_looks_at(fmt, n, shifts):
    """Pages of 2^shift times the values of others, with small weights, around those that count (shift 0)."""
    rng = np.random.default_rng(7)
    k, v = 0.3 * rng.standard_normal((2, max(n, 320), D))
    g = torch.Generator().manual_seed(8)
    u = torch.randn(D, generator=g)
    for i, e in enumerate(shifts):
        if e:
            k[64 * i:64 * i + 64] = -12.0 * u.numpy()
            v[64 * i:64 * i + 64] *= 2.0 ** e
    q = (u + 0.2 * torch.randn(n, 1, D, generator=g)).to(torch.bfloat16).cuda()
    c = Rows(fmt, 1, 32, k, v)
    if n > 64:                                     # rows that see none of the pages that count
        c.check_closely(q[-40:], c.run(q, [n])[-40:])
    else:
        c.check_closely(q, c.run(q, [n]))
