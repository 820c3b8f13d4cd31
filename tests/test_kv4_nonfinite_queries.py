"""A query with a NaN or an infinity: softmax over scores that are NaN (or infinite) is NaN,
so its head's output is NaN, and so are the weights of the KV head, which sum over its
heads.  Other heads, other KV heads and other sequences keep their results."""
import numpy as np
import pytest
import torch

import kv4_ref as R
from test_kv4_attn import FORMATS, SM, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g", (1, 3, 4, 7, 12, 16))
@pytest.mark.parametrize("rot", ("identity", "shared"))
@pytest.mark.parametrize("value", (float("nan"), float("inf"), -float("inf")))
def test_query_that_is_not_finite(g, rot, value):
    Hkv = 2
    c = Case(30 + g, (700, 1, 0, 130), Hkv * g, Hkv, *FORMATS[g % len(FORMATS)], rot=rot)
    ref, w, tol, w_tol = R.attend(c.pool, Hkv, c.G, c.meta, c.q, c.table, c.lens, c.Rk, c.Rv, SM)
    bad = np.zeros((c.B, c.Hq), bool)
    for b, head in ((0, g - 1), (1, g), (2, 0), (3, 2 * g - 1)):    # one head of one KV head per sequence
        c.q[b, head, 17 * b + 5] = value
        bad[b, head] = c.lens[b] > 0                                # no tokens: no scores, the output is 0
    for splits in (0, 1, 3):
        out = c.run(splits)
        got = out.cpu().numpy().astype(np.float64)
        assert np.isnan(got[bad]).all()
        ok_rows = ~bad
        assert (np.abs(got[ok_rows] - ref[ok_rows]) <= tol[ok_rows]).all()
        half = c.run(splits, torch.bfloat16).float().cpu().numpy()
        assert np.isnan(half[bad]).all() and np.isfinite(half[ok_rows]).all()
    sums = torch.full((c.B, Hkv, c.mp * 64), 3.0, device="cuda")
    c.run(0, weights=sums)
    got = sums.cpu().numpy().astype(np.float64)
    for b, n in enumerate(c.lens):
        for h in range(Hkv):
            if bad[b, h * g:(h + 1) * g].any():
                assert np.isnan(got[b, h, :n]).all()
            else:
                err = np.abs(got[b, h, :n] - 3.0 - w[b, h, :n])
                assert (err <= w_tol[b, h, :n] + 2.0 ** -23 * (3 + w[b, h, :n])).all()
            assert (got[b, h, n:] == 3.0).all()
