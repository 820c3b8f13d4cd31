"""The 4-bit cache's C and Python entry points without a GPU: sizes, refusals (none of
these calls reaches a launch), and the test definitions' own consistency."""
import ctypes

import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: validation fails first
INV, UNS, SMALL = ok.ERR_INVALID_ARG, ok.ERR_UNSUPPORTED, ok.ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def L():
    return ok.lib()


@pytest.mark.parametrize("G", (32, 64, 128))
def test_page_layout_is_a_partition(G):
    """Every nibble and metadata byte of a block belongs to one (tensor, slot, channel)."""
    seen = np.zeros(R.block_bytes(G), int)
    for place in (R.k_place, R.v_place):
        for t in range(64):
            for c in range(128):
                b, sh = place(t, c)
                seen[b] += 1 if sh == 0 else 16
    for is_v in (0, 1):
        for t in range(64):
            for g in range(128 // G):
                e = R.sz_place(G, is_v, t, g)
                seen[e:e + 4] += 17
    assert (seen == 17).all()
    # no byte holds two slots
    for place in (R.k_place, R.v_place):
        owner = {}
        for t in range(64):
            for c in range(128):
                assert owner.setdefault(place(t, c)[0], t) == t


def test_sizes(L):
    for G in (32, 64, 128):
        lay = ok.Layout(3, 7, group_size=G)
        assert ok.kv4_page_bytes(lay) == 3 * R.block_bytes(G)
        assert ok.kv4_pool_bytes(lay) == 21 * R.block_bytes(G)
    assert ok.kv4_page_bytes(ok.Layout(0, 7)) == 0 and ok.kv4_pool_bytes(ok.Layout(3, 7, head_dim=64)) == 0
    assert L.oscar_kv4_page_bytes(None) == 0 and L.oscar_kv4_pool_bytes(None) == 0
    lay = ok.Layout(8, 10)
    plain = ok.kv4_decode_workspace_bytes(lay, 4, 32, 3, 20)
    assert plain == ok.decode_workspace_bytes(lay, 4, 32, 3)
    with_w = ok.kv4_decode_workspace_bytes(lay, 4, 32, 3, 20, weights=True)
    assert with_w - plain >= 4 * 32 * 20 * 64 * 4 and with_w % 256 == 0
    assert ok.kv4_decode_workspace_bytes(lay, 0, 32, 3, 20) == 0
    assert ok.kv4_decode_workspace_bytes(lay, 4, 30, 3, 20) == 0
    assert ok.kv4_decode_workspace_bytes(lay, 4, 32, 3, 0) == 0
    assert ok.kv4_decode_workspace_bytes(lay, 4, 32, 3, 1 << 25) == 0   # slots pass 32 bits
    assert ok.kv4_evict_workspace_bytes(lay, 4, 20) >= 4 * 8 * 20 * 64 * 4
    for args in ((0, 20), (65536, 20), (4, 0), (4, 1 << 25)):
        assert ok.kv4_evict_workspace_bytes(lay, *args) == 0


def test_append_refusals(L):
    def call(lay=ok.Layout(8, 10), pages=FAKE, k=FAKE, v=FAKE, slots=FAKE, n=4, Rk=FAKE, Rv=FAKE, ck=0.9, cv=0.9):
        return L.oscar_kv4_append(ctypes.byref(lay), pages, k, v, slots, n, Rk, Rv, ck, cv, None)
    assert call(n=-1) == INV and call(ck=0.0) == INV and call(cv=1.5) == INV and call(ck=float("nan")) == INV
    assert call(pages=None) == INV and call(k=None) == INV and call(v=None) == INV and call(slots=None) == INV
    assert call(pages=ctypes.c_void_p(0x10008)) == INV and call(k=ctypes.c_void_p(0x10002)) == INV
    assert call(Rk=ctypes.c_void_p(0x10004)) == INV and call(slots=ctypes.c_void_p(0x10004)) == INV
    assert call(lay=ok.Layout(8, 10, head_dim=256)) == UNS
    assert call(lay=ok.Layout(60000, 10), n=1 << 20) == UNS            # rows pass 32 bits
    assert call(n=0, pages=None) == ok.OK
    assert L.oscar_kv4_append(None, FAKE, FAKE, FAKE, FAKE, 4, None, None, 0.9, 0.9, None) == INV


def test_gather_refusals(L):
    def call(lay=ok.Layout(8, 10), pages=FAKE, slots=FAKE, n=4, k=FAKE, v=FAKE, dt=1):
        return L.oscar_kv4_gather(ctypes.byref(lay), pages, slots, n, k, v, dt, None)
    assert call(n=-1) == INV and call(dt=2) == INV and call(pages=None) == INV and call(slots=None) == INV
    assert call(k=None) == INV and call(v=None) == INV and call(k=ctypes.c_void_p(0x10008)) == INV
    assert call(lay=ok.Layout(8, 10, page_size=32)) == UNS
    assert call(n=0, k=None) == ok.OK


def _attn(L, step, lay=ok.Layout(8, 10), pages=FAKE, q=FAKE, B=2, Hq=32, bt=FAKE, mp=4, lens=FAKE, Rk=FAKE,
          Rv=FAKE, sm=0.088, S=2, w=None, wo=None, ws=FAKE, size=1 << 40, out=FAKE, dt=0, n_new=0, k=None, ck=0.9):
    tail = (q, B, Hq, bt, mp, lens, Rk, Rv, sm, S, w, wo, ws, size, out, dt, None)
    if step:
        return L.oscar_kv4_decode_step(ctypes.byref(lay), pages, k, k, k, n_new, ck, 0.9, *tail)
    return L.oscar_kv4_decode_attn(ctypes.byref(lay), pages, *tail)


@pytest.mark.parametrize("step", (False, True))
def test_decode_refusals(L, step):
    def call(**kw):
        return _attn(L, step, **kw)
    assert call(Hq=30) == INV and call(Hq=8 * 17) == UNS and call(B=0) == INV and call(S=-1) == INV
    assert call(B=65536) == UNS and call(mp=0) == INV and call(mp=1 << 25) == UNS
    assert call(dt=7) == INV and call(sm=float("inf")) == INV
    for name in ("pages", "q", "bt", "lens", "ws", "out"):
        assert call(**{name: None}) == INV, name
    assert call(ws=ctypes.c_void_p(0x10010)) == INV and call(Rv=ctypes.c_void_p(0x10004)) == INV
    assert call(w=FAKE) == INV and call(wo=FAKE) == INV                      # one without the other
    assert call(w=ctypes.c_void_p(0x10004), wo=FAKE) == INV
    n = 2 * 8 * 4 * 64 * 4                                                   # weights: [2][8][4 * 64] fp32
    for d in (16, n - 16, 16 - n):                                           # partly the same bytes
        assert call(w=FAKE, wo=ctypes.c_void_p(FAKE.value + d)) == INV
    lay = ok.Layout(8, 10)
    assert call(size=ok.kv4_decode_workspace_bytes(lay, 2, 32, 2, 4) - 1) == SMALL
    assert call(w=FAKE, wo=FAKE, size=ok.kv4_decode_workspace_bytes(lay, 2, 32, 2, 4, True) - 1) == SMALL
    if step:
        assert call(n_new=-1) == INV and call(n_new=2) == INV and call(ck=0.0) == INV
        assert call(n_new=2, k=ctypes.c_void_p(0x10002)) == INV


def test_evict_refusals(L):
    def call(lay=ok.Layout(8, 10), pages=FAKE, B=2, bt=FAKE, mp=4, lens=FAKE, w=FAKE, wo=FAKE, p=FAKE, po=FAKE,
             seen=FAKE, budget=64, sink=4, recent=16, new=ctypes.c_void_p(0x20000), ws=FAKE, size=1 << 40):
        return L.oscar_kv4_evict(ctypes.byref(lay), pages, B, bt, mp, lens, w, wo, p, po, seen, budget, sink,
                                 recent, new, ws, size, None)
    assert call(budget=0) == INV and call(sink=-1) == INV and call(recent=-1) == INV and call(B=0) == INV
    assert call(B=65536) == UNS and call(mp=0) == INV and call(mp=1 << 25) == UNS
    for name in ("pages", "bt", "lens", "w", "wo", "p", "po", "seen", "new", "ws"):
        assert call(**{name: None}) == INV, name
    assert call(new=FAKE) == INV                                             # seq_lens itself
    assert call(new=ctypes.c_void_p(FAKE.value + 4)) == INV                  # part of it
    n = 2 * 8 * 4 * 64 * 4
    for d in (16, n - 16, 16 - n):
        assert call(wo=ctypes.c_void_p(FAKE.value + d)) == INV and call(po=ctypes.c_void_p(FAKE.value + d)) == INV
    for name in ("pages", "w", "wo", "p", "po"):
        assert call(**{name: ctypes.c_void_p(0x10008)}) == INV, name
    assert call(size=ok.kv4_evict_workspace_bytes(ok.Layout(8, 10), 2, 4) - 1) == SMALL
    assert call(lay=ok.Layout(8, 10, group_size=16)) == UNS


def test_python_refusals_of_host_tensors():
    if torch.cuda.is_available():
        dev = torch.cuda.current_device()
    else:
        dev = 0
    with pytest.raises(ValueError):
        ok._arg(torch.zeros(4), torch.float32, "x", 4, dev)          # not a GPU tensor
    with pytest.raises(TypeError):
        ok._arg([1.0], torch.float32, "x", None, dev)
    with pytest.raises(TypeError):
        ok._out_code(torch.zeros(4, dtype=torch.float16), "out")
    with pytest.raises(TypeError):
        ok._out_code(None, "out")
    with pytest.raises(ok.OscarError):
        ok.kv4_alloc_pool(ok.Layout(8, 10, head_dim=64), device="cpu")
    with pytest.raises(ok.OscarError):
        ok.kv4_alloc_workspace(ok.Layout(8, 10), 0, 32, 1, 4, device="cpu")
    with pytest.raises(ok.OscarError):
        ok.kv4_alloc_evict_workspace(ok.Layout(8, 10), 0, 4, device="cpu")


def test_reference_round_trip():
    """The test definitions against each other: rows put into a pool and read back."""
    rng = np.random.default_rng(0)
    for G, meta, mode in ((32, 0, 0), (64, 1, 1), (128, 1, 0)):
        x = torch.randn(5, 2, 128).bfloat16()
        pool = np.zeros(2 * 2 * R.block_bytes(G), np.uint8)
        slots = [3, 70, 127, -1, 0]
        Rk = R.rotation(rng)
        R.append(pool, 2, G, meta, mode, x, x, slots, Rk, None, 1.0, 0.9)
        xt = R.rotated(x.float().numpy(), Rk)
        vals = R.block_values(pool.reshape(2, 2, -1), G, meta, 0)
        for i, s in enumerate(slots):
            if s < 0:
                continue
            step = (xt[i].reshape(2, -1, G).max(-1) - xt[i].reshape(2, -1, G).min(-1)) / 15
            err = np.abs(vals[s // 64, :, s % 64] - xt[i]).reshape(2, -1, G).max(-1)
            if mode == 0:
                assert (err <= step * (0.5 + 2.0 ** -7 * 16)).all()  # half a step, and the rounding of s and z
