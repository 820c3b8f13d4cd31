"""Norm and rotation of rows whose squares leave fp32's range: bf16 reaches from 1e-38 to 3e38, and eps may be 0."""
import pytest
import torch

import chunk_ref as R
import paper_2605_17757_amd as ok
from test_rope import _close, _weights

pytestmark = pytest.mark.gpu
D, P = 128, 64


@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-6, 1e30])
@pytest.mark.parametrize("pages", [False, True])
@pytest.mark.parametrize("n", [9, 700])
def test_rows_of_any_magnitude(eps, pages, n):
    """Rows from 2^-120 to 2^124, next to each other and to ordinary ones."""
    Hq, Hkv = 8, 2
    g = torch.Generator(device="cuda").manual_seed(n)
    e = torch.randint(-120, 125, (n, Hq + Hkv, 1), generator=g, device="cuda").double()
    e[::3] = 0.0
    e[1, 0], e[1, 1], e[1, Hq], e[2, Hq] = 124, -120, 124, -120
    # (|x| >= 1/4: no element is a subnormal number)
    x = torch.randn(n, Hq + Hkv, D, generator=g, device="cuda").double()
    x = torch.where(x < 0, -1.0, 1.0) * x.abs().clamp(0.25, 3.5) * 2.0 ** e
    x = x.to(torch.bfloat16)
    q, k = x[:, :Hq], x[:, Hq:]
    w = _weights(5)
    pos = torch.arange(n, device="cuda") * 77
    f = ok.rope_freqs(64, 1e4)
    rope = ok.Rope(64, f)
    qo = torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda")
    ko = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    if pages:
        L = ok.Layout(Hkv, n // P + 1)
        pool = torch.zeros(ok.bf16_pool_bytes(L) // 2, dtype=torch.bfloat16, device="cuda")
        ok.bf16_kv_append_rope(L, pool, rope, k, k, pos // 77, pos, q=q, q_out=qo, q_weight=w[0], k_weight=w[1], eps=eps)
        at = R.bf16_places()[0].cuda()
        ko = pool.view(-1, Hkv, 2 * P * D)[:, :, at].transpose(1, 2).reshape(-1, Hkv, D)[:n]
    else:
        ok.qk_norm_rope(ok.Layout(Hkv, 1), rope, q, k, pos, qo, ko, q_weight=w[0], k_weight=w[1], eps=eps)
    # eps is an fp32 number in the call
    eps = float(torch.tensor(eps, dtype=torch.float32))
    for got, y, wt, what in ((qo, q, w[0], "q"), (ko, k, w[1], "k")):
        ref, tol = R.rope(y, wt, eps, pos, f, 64, False, 1.0)
        assert bool(torch.isfinite(ref).all())
        assert bool(torch.isfinite(got).all()), what
        _close(got, ref, tol, what)


def test_rows_of_zeros_and_of_nan():
    """0 / sqrt(eps) is 0, 0 / 0 NaN; a NaN or an infinity spoils its own row only."""
    x = torch.randn(4, 8, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    x[1, 2] = 0.0
    x[2, 3, 5] = float("nan")
    x[2, 4, 6] = float("inf")
    w = _weights(6)
    pos = torch.arange(4, device="cuda")
    rope = ok.Rope(128, ok.rope_freqs(128, 1e4))
    for eps in (1e-6, 0.0):
        out = [torch.empty_like(x) for _ in range(2)]
        ok.qk_norm_rope(ok.Layout(8, 1), rope, x, x, pos, *out, q_weight=w[0], k_weight=w[0], eps=eps)
        for o in out:
            nan = torch.isnan(o).any(-1)
            want = torch.zeros_like(nan)
            want[2, 3] = want[2, 4] = True
            want[1, 2] = eps == 0.0
            assert torch.equal(nan, want)
            assert eps == 0.0 or not o[1, 2].any()


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40])
def test_rows_of_subnormal_numbers(eps):
    """Elements of 2^-133 to 2^-126: normalised to numbers near 1 unless eps outweighs them."""
    g = torch.Generator(device="cuda").manual_seed(7)
    n, H = 600, 8
    x = torch.randint(1, 128, (n, H, D), generator=g, device="cuda").to(torch.int16)      # bf16 bits
    x[::2] //= 16
    x[1::4, :, ::3] = 0
    x[..., 0] = 3                                       # (no row of zeros: 0 / 0)
    x = x.view(torch.bfloat16)
    w = _weights(8)[0]
    pos = torch.arange(n, device="cuda")
    out = [torch.empty_like(x) for _ in range(2)]
    ok.qk_norm_rope(ok.Layout(H, 1), ok.Rope(0, None), x, x, pos, *out, q_weight=w, k_weight=w, eps=eps)
    ref, tol = R.rope(x, w, float(torch.tensor(eps, dtype=torch.float32)), pos, None, 0, False, 1.0)
    assert bool(torch.isfinite(ref).all())
    for o in out:
        _close(o, ref, tol, "row")
