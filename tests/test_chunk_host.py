"""Host side of norm and rotation and of the attention of chunks: frequencies, sizes,
refusals (no GPU: validation fails before anything is launched)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2605_17757_amd as ok

A = lambda i: ctypes.c_void_p(i << 32)   # addresses 4 GiB apart, never dereferenced


def _freqs(*a):
    return ok.rope_freqs(*a, device="cpu").numpy()


def test_frequencies():
    i = np.arange(32.0)
    f = 1e4 ** (-2 * i / 64)
    assert np.array_equal(_freqs(64, 1e4), f.astype(np.float32))
    assert np.array_equal(_freqs(64, 1e4, ok.ROPE_LINEAR, 8.0), (f / 8).astype(np.float32))
    turns = 8192 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / (4 - 1), 0, 1)
    want = f * keep + f / 8 * (1 - keep)
    assert np.allclose(_freqs(64, 1e4, ok.ROPE_BY_TURNS, 8.0, 8192, 1.0, 4.0), want, rtol=2e-7, atol=0)
    # by index: 32 turns and 1 turn over 4096 positions
    at = lambda r: 64 * math.log(4096 / (r * 2 * math.pi)) / (2 * math.log(1e4))
    lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), 63)
    keep = 1 - np.clip((i - lo) / (hi - lo), 0, 1)
    want = f * keep + f / 16 * (1 - keep)
    assert np.allclose(_freqs(64, 1e4, ok.ROPE_BY_INDEX, 16.0, 4096, 1.0, 32.0), want, rtol=2e-7, atol=0)
    assert want[0] == f[0] and np.isclose(want[-1], f[-1] / 16)


@pytest.mark.parametrize("args", [(0, 1e4), (63, 1e4), (64, 1.0), (64, math.nan), (64, 1e4, 4), (64, 1e4, 1, 0.0),
                                  (64, 1e4, 1, math.inf), (64, 1e4, 2, 8.0, 0.0), (64, 1e4, 2, 8.0, 4096, 4.0, 1.0),
                                  (64, 1e4, 3, 8.0, 4096, 0.0, 1.0)])
def test_frequency_refusals(args):
    with pytest.raises(ok.OscarError) as e:
        _freqs(*args)
    assert e.value.status == ok.ERR_INVALID_ARG


def _rope(**kw):
    d = dict(rotary_dim=128, interleaved=0, attn_scale=1.0, inv_freq=0x700000000000)
    d.update(kw)
    return ok._RopeArg(d["rotary_dim"], d["interleaved"], d["attn_scale"], d["inv_freq"])


def _norm_rope(lay=None, rope=None, **kw):
    d = dict(q=A(1), qs=32 * 128, qo=A(2), Hq=32, k=A(3), ks=8 * 128, ko=A(4), pos=A(5), n=10, qw=A(6), kw=A(7), eps=1e-6)
    d.update(kw)
    lay = lay or ok.Layout(8, 10)
    rope = rope or _rope()
    return ok.lib().oscar_qk_norm_rope(ctypes.byref(lay), ctypes.byref(rope), d["q"], d["qs"], d["qo"], d["Hq"], d["k"],
                                       d["ks"], d["ko"], d["pos"], d["n"], d["qw"], d["kw"], d["eps"], None)


def _append(lay=None, rope=None, **kw):
    d = dict(pages=A(9), q=A(1), qs=32 * 128, qo=A(2), Hq=32, k=A(3), ks=8 * 128, v=A(4), vs=8 * 128, slots=A(5), pos=A(6),
             n=10, qw=A(7), kw=A(8), eps=1e-6)
    d.update(kw)
    lay = lay or ok.Layout(8, 10)
    rope = rope or _rope()
    return ok.lib().oscar_bf16_kv_append_rope(ctypes.byref(lay), d["pages"], ctypes.byref(rope), d["q"], d["qs"], d["qo"],
                                              d["Hq"], d["k"], d["ks"], d["v"], d["vs"], d["slots"], d["pos"], d["n"],
                                              d["qw"], d["kw"], d["eps"], None)


@pytest.mark.parametrize("call", [_norm_rope, _append])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(eps=-1.0), 1), (dict(eps=math.nan), 1), (dict(k=None), 1), (dict(pos=None), 1), (dict(q=None), 1),
    (dict(qo=None), 1), (dict(qs=32 * 128 - 8), 1), (dict(ks=8), 1), (dict(qs=32 * 128 + 4), 2), (dict(q=ctypes.c_void_p(8)), 1),
    (dict(k=ctypes.c_void_p(24)), 1), (dict(qw=ctypes.c_void_p(8)), 1), (dict(Hq=-1), 1), (dict(Hq=65536, qs=65536 * 128), 2),
    # written arrays that share bytes with others
    (dict(qo=A(3)), 1), (dict(qo=ctypes.c_void_p((1 << 32) + 256)), 1), (dict(q=A(1), qo=A(1), qs=40 * 128), 1), (dict(qo=A(5)), 1)])
def test_row_refusals(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("call", [_norm_rope, _append])
@pytest.mark.parametrize("kw,status", [(dict(rotary_dim=-16), 1), (dict(rotary_dim=144), 1), (dict(rotary_dim=24), 2),
                                       (dict(interleaved=2), 1), (dict(attn_scale=math.inf), 1), (dict(inv_freq=0), 1),
                                       (dict(inv_freq=0x700000000008), 1)])
def test_rope_refusals(call, kw, status):
    assert call(rope=_rope(**kw)) == status


def test_append_refusals():
    assert _append(pages=None) == 1 and _append(slots=None) == 1 and _append(v=None) == 1 and _append(vs=64) == 1
    assert _append(v=ctypes.c_void_p((9 << 32) + 64)) == 1            # values inside the pages
    assert _append(lay=ok.Layout(8, 10, head_dim=64)) == 2 and _append(lay=ok.Layout(0, 10)) == 1
    assert _append(n=0, pages=None, k=None, v=None, slots=None, pos=None) == 0
    assert _norm_rope(n=0, q=None, k=None, pos=None) == 0 and _norm_rope(Hq=0) == 1


CALLS = {"oscar_bf16_chunk_attn": False, "oscar_kv4_chunk_attn": True, "oscar_chunk_attn": True}


def _chunk(name, lay=None, **kw):
    d = dict(pages=A(1), q=A(2), n_q=50, B=4, Hq=32, start=A(3), table=A(4), mp=100, lens=A(5), Rk=A(6), Rv=A(7), sm=0.1,
             window=0, sinks=0, splits=2, ws=A(8), ws_bytes=1 << 40, out=A(9))
    d.update(kw)
    lay = lay or ok.Layout(8, 1000)
    rot = (d["Rk"], d["Rv"]) if CALLS[name] else ()
    return getattr(ok.lib(), name)(ctypes.byref(lay), d["pages"], d["q"], d["n_q"], d["B"], d["Hq"], d["start"], d["table"],
                                   d["mp"], d["lens"], *rot, d["sm"], d["window"], d["sinks"], d["splits"], d["ws"],
                                   d["ws_bytes"], d["out"], None)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(n_q=-1), 1), (dict(B=0), 1), (dict(B=65536), 2), (dict(Hq=0), 1), (dict(Hq=12), 1), (dict(Hq=8 * 17), 2),
    (dict(mp=0), 1), (dict(mp=(1 << 24) + 1), 2), (dict(window=-1), 1), (dict(sinks=-1), 1), (dict(sm=math.nan), 1),
    (dict(splits=-1), 1), (dict(splits=1025), 2), (dict(n_q=1 << 26, Hq=32), 2), (dict(n_q=1 << 25, Hq=32, splits=1024), 2),
    (dict(pages=None), 1), (dict(q=None), 1), (dict(start=None), 1), (dict(table=None), 1), (dict(lens=None), 1),
    (dict(ws=None), 1), (dict(out=None), 1), (dict(q=ctypes.c_void_p(8)), 1), (dict(out=ctypes.c_void_p(8)), 1),
    (dict(ws=ctypes.c_void_p(128)), 1), (dict(ws_bytes=1000), 3), (dict(out=A(2)), 1), (dict(out=A(1)), 1),
    (dict(out=ctypes.c_void_p((8 << 32) + 4096)), 1), (dict(ws=ctypes.c_void_p((1 << 32) + 256)), 1), (dict(out=A(5)), 1)])
def test_chunk_refusals(name, kw, status):
    assert _chunk(name, **kw) == status


@pytest.mark.parametrize("name", CALLS)
def test_chunk_of_nothing(name):
    assert _chunk(name, n_q=0, q=None, out=None, ws=None, start=None) == 0
    assert _chunk(name, lay=ok.Layout(8, 10, page_size=32)) == 2


def test_chunk_rotations_stay_apart_from_what_is_written():
    for name in ("oscar_kv4_chunk_attn", "oscar_chunk_attn"):
        assert _chunk(name, out=A(6)) == 1 and _chunk(name, Rv=A(9)) == 1 and _chunk(name, Rk=ctypes.c_void_p(8)) == 1


def test_workspace_and_splits():
    lay = ok.Layout(8, 1000)
    size = lambda *a: ok.chunk_workspace_bytes(lay, *a)
    assert size(100, 4, 32, 100, 1, False) == 256
    assert 100 * 32 * 520 * 3 <= size(100, 4, 32, 100, 3, False) <= 100 * 32 * 520 * 3 + 512
    # codes: 32 rows of a KV head to a sequence are rotated apart, more by the blocks that take them
    assert 32 * 32 * (512 + 520) <= size(32, 4, 32, 100, 1, True) <= 32 * 32 * (512 + 520) + 768
    assert size(32, 4, 32, 100, 1, True) <= size(100, 4, 32, 100, 1, True) <= size(1000, 4, 32, 100, 1, True)
    assert size(0, 4, 32, 100, 1, True) == 256 and size(100, 4, 12, 100, 1, True) == 0
    s = ok.chunk_default_splits
    assert s(lay, 1, 1, 32, 8) == 1                    # a short table: one piece
    assert s(lay, 1, 1, 32, 2048) > 8                  # one user, a long one: many
    assert s(lay, 8192, 1, 32, 128) == 1               # a long chunk fills the GPU
    assert size(100, 4, 32, 1000, 0, True) == size(100, 4, 32, 1000, s(lay, 100, 4, 32, 1000), True)


def test_python_refuses_host_tensors():
    lay = ok.Layout(2, 4)
    t = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(Exception):
        ok.bf16_chunk_attn(lay, torch.zeros(4), t, torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32),
                           torch.zeros(1, dtype=torch.int32), 0.1, 0, 0, 1, torch.zeros(256, dtype=torch.uint8), t)
