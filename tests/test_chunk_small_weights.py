"""Softmax weights far below their row's largest, over many cached tokens of the 4-bit and
2-bit caches: together they count."""
import math

import numpy as np
import pytest
import torch

import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu
D, P = 128, 64


@pytest.mark.parametrize("fmt", ["kv4", "kv2"])
@pytest.mark.parametrize("n", [1, 90, 600])      # tiles of 32, 128 and 256 rows
@pytest.mark.parametrize("tokens,bits", [(131072, 23.3), (131072, 25.2), (1 << 20, 26.0)])
def test_many_equal_small_weights_beside_a_heavy_one(fmt, n, tokens, bits):
    """Token 0 has a score of `bits` (log2) and the value 0, all others the score 0 and the value 1:
    the output is N 2^-bits / (1 + N 2^-bits) for the row's N other tokens."""
    L = ok.Layout(1, 2)
    pool = ok.kv4_alloc_pool(L) if fmt == "kv4" else ok.alloc_pool(L)
    k = torch.zeros(2 * P, 1, D, dtype=torch.bfloat16, device="cuda")
    v = torch.ones_like(k)
    k[0], v[0] = 1.0, 0.0
    slots = torch.arange(2 * P, device="cuda")
    (ok.kv4_append if fmt == "kv4" else ok.kv_append)(L, pool, k, v, slots, None, None, 1.0, 1.0)
    mp = tokens // P + n // P + 2
    table = torch.ones(1, mp, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    q = torch.ones(n, 1, D, dtype=torch.bfloat16, device="cuda")
    sm = np.float32(bits * math.log(2.0) / D)
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    length = tokens + n
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = ok.chunk_alloc_workspace(L, n, 1, 1, mp, 1)
    (ok.kv4_chunk_attn if fmt == "kv4" else ok.chunk_attn)(L, pool, q, start, table, lens, None, None, float(sm), 0, 0,
                                                          1, ws, out)
    N = (length - n + torch.arange(n, dtype=torch.float64)).cuda()[:, None, None]
    share = torch.exp(torch.tensor(-float(sm) * D, dtype=torch.float64)).item()
    den = 1.0 + N * share
    ref = N * share / den
    # A weight as one fp16 value: off by 2^-11 of itself, or by 2^-30 of the largest; the exponent of
    # 2 (25 and its reference in fp32, 2^-19 each at most), the denominator's sum of 2^20 weights in
    # fp32 (a lane's partial sums: 2^14 additions of 2^-24 each at most), the output in bf16.
    tol = ref * (2.0 ** -11 + 2.0 ** -18 + 2.0 ** -10) + N * 2.0 ** -30 / den
    tol = tol + 2.0 ** -8 * (ref + tol)
    err = (out.double() - ref).abs()
    assert (err <= tol).all(), "off by %.3g of its value, %.3g of the bound" % (
        float((err / ref).max()), float((err / tol).max()))
