"""Norm and rotation of new tokens' queries and keys, and the bf16 cache update with them,
against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import chunk_ref as R
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu
D, P = 128, 64


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _fused(n, Hq, Hkv, seed, pad=0):
    """A projection's rows and views of its q, k, v."""
    x = torch.randn(n, (Hq + 2 * Hkv) * D + pad, generator=_gen(seed), device="cuda")
    x[:, 5::37] *= 8
    x = x.to(torch.bfloat16)
    q, k, v = (y.unflatten(1, (-1, D)) for y in x[:, :(Hq + 2 * Hkv) * D].split((Hq * D, Hkv * D, Hkv * D), 1))
    return q, k, v


def _weights(seed):
    return (1 + 0.3 * torch.randn(2, D, generator=_gen(seed), device="cuda")).to(torch.bfloat16)


def _close(got, ref, tol, what):
    bad = (got.double() - ref).abs() > tol
    assert not bad.any(), "%s: %d of %d off, worst %.3g over its bound" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - ref).abs() / tol).max()))


@pytest.mark.parametrize("rotary,inter", [(128, False), (128, True), (64, False), (64, True), (96, False),
                                          (16, True), (16, False), (0, False)])
@pytest.mark.parametrize("n,Hq,Hkv,norm", [(1, 32, 8, True), (7, 3, 1, True), (65, 20, 5, False), (300, 16, 2, True)])
def test_qk_norm_rope(rotary, inter, n, Hq, Hkv, norm):
    q, k, _ = _fused(n, Hq, Hkv, 1)
    w = _weights(2) if norm else (None, None)
    pos = torch.randint(0, 1 << 20, (n,), generator=_gen(3), device="cuda")
    pos[0] = 0
    pos[-1] = 131071
    f = ok.rope_freqs(max(rotary, 2), 1e6)
    rope = ok.Rope(rotary, f, interleaved=inter, attn_scale=1.25)
    L = ok.Layout(Hkv, 1)
    qo = torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda")
    ko = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    ok.qk_norm_rope(L, rope, q, k, pos, qo, ko, q_weight=w[0], k_weight=w[1], eps=1e-5)
    for got, x, wt, what in ((qo, q, w[0], "q"), (ko, k, w[1], "k")):
        _close(got, *R.rope(x, wt, 1e-5, pos, f, rotary, inter, 1.25), what)
    if not norm and not rotary:
        assert torch.equal(qo, q) and torch.equal(ko, k)


def test_angles_of_far_positions():
    # cosines and sines themselves: x = (1, 0) in every pair
    n = 64
    pos = torch.cat([torch.arange(32), (1 << 24) + torch.arange(16) * 977, 2 ** 31 + torch.arange(16) * 65537]).cuda()
    f = ok.rope_freqs(128, 10000.0)
    x = torch.zeros(n, 1, D, dtype=torch.bfloat16, device="cuda")
    x[..., :64] = 1.0
    out = [torch.empty_like(x) for _ in range(2)]
    ok.qk_norm_rope(ok.Layout(1, 1), ok.Rope(128, f), x, x, pos, *out)
    t = pos.double()[:, None] * f.double()
    ref = torch.cat([t.cos(), t.sin()], 1)[:, None]
    _close(out[0], ref, R.UB * ref.abs() + 2.0 ** -20 + 2.0 ** -23, "cos, sin")
    assert torch.equal(out[0], out[1])


def test_in_place_and_other_stream():
    n, Hq, Hkv = 37, 8, 2
    q, k, _ = (x.contiguous() for x in _fused(n, Hq, Hkv, 11))
    w = _weights(12)
    pos = torch.arange(n, device="cuda") + 100
    rope = ok.Rope(64, ok.rope_freqs(64, 1e4), interleaved=True)
    L = ok.Layout(Hkv, 1)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ok.qk_norm_rope(L, rope, q, k, pos, qo, ko, q_weight=w[0], k_weight=w[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ok.qk_norm_rope(L, rope, q, k, pos, q, k, q_weight=w[0], k_weight=w[1], stream=s)
    s.synchronize()
    assert torch.equal(q, qo) and torch.equal(k, ko)


def _slots(kind, n, pages):
    if kind == "run":        # a prompt from the middle of a page on, pages in any order
        order = np.random.default_rng(5).permutation(pages)
        at = np.arange(n) + 13
        return order[at // P] * P + at % P
    if kind == "aligned":
        return np.arange(n) + P
    if kind == "scattered":
        return np.random.default_rng(6).permutation(pages * P)[:n]
    if kind == "reversed":
        return np.arange(n)[::-1] + 3
    s = np.arange(n) + 5     # "holes": some tokens skipped
    s[::3] = -1
    return s


@pytest.mark.parametrize("kind", ["run", "aligned", "scattered", "reversed", "holes"])
@pytest.mark.parametrize("n,Hkv,with_q", [(1, 8, True), (9, 1, False), (130, 3, True), (4100, 8, True)])
def test_bf16_append(kind, n, Hkv, with_q):
    Hq = 4 * Hkv
    pages = n // P + 4
    q, k, v = _fused(n, Hq, Hkv, 21, pad=24)
    w = _weights(22)
    pos = torch.randint(0, 200000, (n,), generator=_gen(23), device="cuda")
    slots = torch.from_numpy(np.ascontiguousarray(_slots(kind, n, pages)).astype(np.int64)).cuda()
    f = ok.rope_freqs(128, 5e5, ok.ROPE_BY_TURNS, 8.0, 8192, 1.0, 4.0)
    rope = ok.Rope(128, f)
    L = ok.Layout(Hkv, pages)
    fill = torch.randint(0, 1 << 15, (ok.bf16_pool_bytes(L) // 2,), generator=_gen(24), device="cuda",
                         dtype=torch.int16).view(torch.bfloat16)
    pool = fill.clone()
    qo = torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda") if with_q else None
    ok.bf16_kv_append_rope(L, pool, rope, k, v, slots, pos, q=q if with_q else None, q_out=qo,
                           q_weight=w[0], k_weight=w[1])
    # the keys and queries are those of the call without a cache, to the bit
    q2 = torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda")
    k2 = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    ok.qk_norm_rope(L, rope, q, k, pos, q2, k2, q_weight=w[0], k_weight=w[1])
    _close(k2, *R.rope(k, w[1], 1e-6, pos, f, 128, False, 1.0), "k")
    if with_q:
        assert torch.equal(qo, q2)
    # the pool: plain update of those rows; every other byte as it was
    ref = fill.cpu()
    R.put_bf16(ref, Hkv, slots.cpu(), k2.cpu(), v.cpu())
    assert torch.equal(pool.cpu().view(torch.int16), ref.view(torch.int16))
    if kind != "holes":
        plain = fill.clone()
        ok.bf16_kv_append(L, plain, k2, v.contiguous(), slots)
        assert torch.equal(pool.view(torch.int16), plain.view(torch.int16))


def test_append_past_4_gib():
    Hkv, n = 8, 70
    pages = (5 << 30) // (Hkv * 2 * P * D * 2)
    L = ok.Layout(Hkv, pages)
    pool = torch.empty(ok.bf16_pool_bytes(L) // 2, dtype=torch.bfloat16, device="cuda")
    _, k, v = _fused(n, Hkv, Hkv, 31)
    slots = torch.arange(n, device="cuda") + (pages - 2) * P
    rope = ok.Rope(128, ok.rope_freqs(128, 1e6))
    pos = torch.arange(n, device="cuda")
    ok.bf16_kv_append_rope(L, pool, rope, k, v, slots, pos)
    small = ok.Layout(Hkv, 2)
    part = torch.zeros(ok.bf16_pool_bytes(small) // 2, dtype=torch.bfloat16, device="cuda")
    ok.bf16_kv_append_rope(small, part, rope, k, v, slots - (pages - 2) * P, pos)
    block = part.view(2, Hkv, 2 * P * D)
    got = pool[-part.numel():].view(2, Hkv, 2 * P * D)
    kp, vp = R.bf16_places()
    for t in range(n):
        for a in (kp, vp):
            i = a[t % P].cuda()
            assert torch.equal(got[t // P][:, i], block[t // P][:, i]), t


def test_captured_and_replayed():
    n, Hq, Hkv = 19, 8, 4
    q, k, v = (x.contiguous() for x in _fused(n, Hq, Hkv, 41))
    pos = torch.arange(n, device="cuda")
    slots = torch.arange(n, device="cuda") + 7
    rope = ok.Rope(128, ok.rope_freqs(128, 1e6))
    L = ok.Layout(Hkv, 3)
    pool = torch.zeros(ok.bf16_pool_bytes(L) // 2, dtype=torch.bfloat16, device="cuda")
    qo = torch.empty_like(q)
    call = lambda p, o: ok.bf16_kv_append_rope(L, p, rope, k, v, slots, pos, q=q, q_out=o)
    call(pool, qo)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(pool, qo)
    for i in range(4):
        q.mul_(-0.5)
        k.add_(0.25)
        pos.add_(31)
        graph.replay()
        torch.cuda.synchronize()
        p2, o2 = torch.zeros_like(pool), torch.empty_like(qo)
        call(p2, o2)
        assert torch.equal(p2, pool) and torch.equal(o2, qo), i


def test_frequencies_on_the_gpu_side():
    f = ok.rope_freqs(128, 1e6)
    i = torch.arange(64, dtype=torch.float64)
    assert torch.equal(f.cpu(), (1e6 ** (-2 * i / 128)).float())
    assert f.is_cuda and math.isclose(float(f[0]), 1.0)
