"""Eviction from the 4-bit cache against the definition in Python: pages, weights,
positions and lengths are equal.  Attention before and after, a serving loop, a graph."""
import math

import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu

SM = 1.0 / math.sqrt(128)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def setup(seed, lens, Hkv, G=32, meta=0, spare=1, mp=None):
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    B = len(lens)
    mp = mp or max(1, -(-int(lens.max()) // 64)) + spare
    used = [-(-int(n) // 64) for n in lens]
    num = sum(used) + 1
    perm = rng.permutation(num)
    table = np.full((B, mp), 2 ** 30, np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    pool = R.random_pool(rng, num, Hkv, G, meta)
    weights = np.exp(2 * rng.standard_normal((B, Hkv, mp * 64))).astype(np.float32)
    pos = np.full(weights.shape, -1, np.int32)
    return rng, lens, table, pool, weights, pos, ok.Layout(Hkv, num, group_size=G, meta_dtype=meta)


def check(lay, lens, table, pool, weights, pos, seen, budget, sink, recent, G=32, in_place=(False, True)):
    seen = np.asarray(seen, np.int32)
    want = R.evict(pool, lay.num_kv_heads, G, table, lens, weights, pos, seen, budget, sink, recent)
    for inp in in_place:
        p, w, ps = dev(pool), dev(weights), dev(pos)
        w_out = None if inp else torch.full_like(w, 9.0)
        p_out = None if inp else torch.full_like(ps, 9)
        new = torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
        ws = torch.full((ok.kv4_evict_workspace_bytes(lay, len(lens), table.shape[1]),), 255, dtype=torch.uint8,
                        device="cuda")
        ok.kv4_evict(lay, p, dev(table), dev(lens), w, ps, dev(seen), budget, sink, recent, new, ws,
                     weights_out=w_out, pos_out=p_out)
        got = (p.cpu().numpy(), (w if inp else w_out).cpu().numpy(), (ps if inp else p_out).cpu().numpy(),
               new.cpu().numpy())
        for name, a, b in zip(("pages", "weights", "pos", "lens"), got, want):
            assert np.array_equal(a, b, equal_nan=name == "weights"), (name, inp, np.argwhere(a != b)[:4])
    return want


@pytest.mark.parametrize("G,meta", ((32, 0), (64, 1), (128, 0)))
@pytest.mark.parametrize("budget,sink,recent", ((1, 0, 0), (64, 4, 16), (100, 0, 0), (130, 64, 64), (200, 300, 10),
                                                (128, 0, 500), (1000, 4, 64)))
def test_budgets(G, meta, budget, sink, recent):
    rng, lens, table, pool, weights, pos, lay = setup(budget, (333, 1, 0, 64, 200, 129), 3, G, meta)
    check(lay, lens, table, pool, weights, pos, lens, budget, sink, recent, G)


def test_few_and_many_moves_per_page():
    """Weights that make one page receive all its rows, another a few, a third none."""
    rng, lens, table, pool, weights, pos, lay = setup(1, (640, 640), 2)
    weights[...] = 1.0
    weights[:, :, :64] = 0.5           # every slot of page 0 goes
    weights[:, :, 64:69] = 0.25        # five of page 1
    weights[:, :, 400:475] = 2.0       # and these come in their places
    check(lay, lens, table, pool, weights, pos, lens, 192, 0, 0)


@pytest.mark.parametrize("kind", ("equal", "zeros", "nan", "negative", "infinite"))
def test_ties_and_odd_weights(kind):
    rng, lens, table, pool, weights, pos, lay = setup(2, (300, 170), 2)
    if kind == "equal":
        weights[...] = 1.5
        weights[0, 0, 250:] = 2.0
    elif kind == "zeros":
        weights[...] = np.where(rng.random(weights.shape) < 0.5, 0.0, -0.0)
        weights[:, :, ::7] = 1e-40
    elif kind == "nan":
        weights[:, :, ::3] = np.nan
    elif kind == "negative":
        weights *= np.where(rng.random(weights.shape) < 0.5, -1, 1).astype(np.float32)
    else:
        weights[:, :, ::4] = np.inf
        weights[:, :, 1::4] = -np.inf
    check(lay, lens, table, pool, weights, pos, lens, 99, 2, 5)


def test_evicted_before():
    """Kept positions of an earlier eviction, out of order, and tokens since then."""
    rng, lens, table, pool, weights, pos, lay = setup(3, (260, 190), 3)
    seen = np.array([1000, 191], np.int32)
    for b, n in enumerate(lens):
        old = int(n) - 60
        for h in range(3):
            pos[b, h, :old] = rng.permutation(int(seen[b]) - 60)[:old]
    check(lay, lens, table, pool, weights, pos, seen, 128, 8, 100)


@pytest.mark.parametrize("mp", (70, 200, 500, 600))
def test_slots_per_thread(mp):
    """Every way of keeping the keys: 4, 12 or 32 of a thread in registers, or none."""
    n = mp * 64 - 29
    rng, lens, table, pool, weights, pos, lay = setup(mp, (n, n // 2), 1, 128, mp=mp)
    weights[:, :, : n // 3] = np.float32(0.7)   # ties over many waves
    check(lay, lens, table, pool, weights, pos, lens, n // 3, 4, 64, 128, in_place=(mp % 200 == 0,))


def test_many_rows():
    rng, lens, table, pool, weights, pos, lay = setup(5, [70 + i % 61 for i in range(90)], 2, 128)
    check(lay, lens, table, pool, weights, pos, lens, 66, 1, 8, 128, in_place=(False,))


def test_nothing_to_evict_keeps_pages():
    rng, lens, table, pool, weights, pos, lay = setup(6, (64, 10), 2)
    want = check(lay, lens, table, pool, weights, pos, lens, 64, 0, 0)
    assert np.array_equal(want[0], pool)


def attend(lay, pool, q, table, lens, weights=None):
    B, Hq = q.shape[0], q.shape[1]
    mp = table.shape[1]
    s = ok.default_num_splits(lay, B, Hq, mp * 64)
    out = torch.empty(B, Hq, 128, device="cuda")
    ws = ok.kv4_alloc_workspace(lay, B, Hq, s, mp, weights=weights is not None)
    ok.kv4_decode_attn(lay, pool, q, table, lens, None, None, SM, s, ws, out, weights=weights)
    return out


def test_attention_is_that_over_the_kept_tokens():
    """After an eviction the attention over the shorter cache is the softmax over the kept
    tokens, wherever their rows lie now."""
    rng, lens, table, pool, weights, pos, lay = setup(7, (500, 300), 2)
    want_pool, _, _, want_lens = R.evict(pool, 2, 32, table, lens, weights, pos, lens, 150, 4, 32)
    q = torch.from_numpy(rng.standard_normal((2, 8, 128)).astype(np.float32)).bfloat16()
    p, w, ps, new = dev(pool), dev(weights), dev(pos), torch.zeros(2, dtype=torch.int32, device="cuda")
    ok.kv4_evict(lay, p, dev(table), dev(lens), w, ps, dev(lens), 150, 4, 32, new,
                 ok.kv4_alloc_evict_workspace(lay, 2, table.shape[1]))
    got = attend(lay, p, q.cuda(), dev(table), new).cpu().numpy()
    for b in range(2):
        K, V = R.sequence_values(pool, 2, 32, 0, table[b], int(lens[b]))
        for h in range(2):
            src, _ = R.evict_row(weights[b, h], pos[b, h], int(lens[b]), int(lens[b]), 150, 4, 32)
            x = (R.bf16_bits(q[b, 4 * h:4 * h + 4]).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
            s = x @ K[src, h].astype(np.float64).T * SM
            e = np.exp(s - s.max(-1, keepdims=True))
            ref = (e / e.sum(-1, keepdims=True)) @ V[src, h]
            tol = R.attend(want_pool, 2, 32, 0, q, table, want_lens, None, None, SM)[2][b, 4 * h:4 * h + 4]
            assert (np.abs(got[b, 4 * h:4 * h + 4] - ref) <= tol).all()


def test_serving_loop():
    """Prompt, steps with weights, and an eviction whenever the cache reaches its limit;
    every step against 64-bit attention over the tokens that the definition keeps."""
    rng = np.random.default_rng(8)
    Hkv, Hq, mp, limit, budget, sink, recent = 2, 6, 4, 200, 128, 4, 32
    lay = ok.Layout(Hkv, 2 * mp)
    pool = ok.kv4_alloc_pool(lay)
    table = dev(np.arange(2 * mp, dtype=np.int32).reshape(2, mp)[::-1].copy())
    tab = table.cpu().numpy()
    Rk, Rv = R.rotation(rng), R.rotation(rng)
    n = np.array([150, 97], np.int32)
    seen = n.copy()
    weights = torch.zeros(2, Hkv, mp * 64, device="cuda")
    pos = torch.full((2, Hkv, mp * 64), -1, dtype=torch.int32, device="cuda")
    slot_of = lambda b, t: int(tab[b, t // 64]) * 64 + t % 64  # noqa: E731

    def new_rows(m):
        return [torch.from_numpy(rng.standard_normal((m, Hkv, 128)).astype(np.float32)).bfloat16() for _ in range(2)]
    for b in range(2):
        k, v = new_rows(int(n[b]))
        ok.kv4_append(lay, pool, k.cuda(), v.cuda(), dev(np.array([slot_of(b, t) for t in range(n[b])])), dev(Rk),
                      dev(Rv), 0.96, 0.96)
    splits = ok.default_num_splits(lay, 2, Hq, mp * 64)
    ws = ok.kv4_alloc_workspace(lay, 2, Hq, splits, mp, weights=True)
    ews = ok.kv4_alloc_evict_workspace(lay, 2, mp)
    out = torch.empty(2, Hq, 128, device="cuda")
    evictions = 0
    for step in range(130):
        k, v = new_rows(2)
        q = torch.from_numpy(rng.standard_normal((2, Hq, 128)).astype(np.float32)).bfloat16()
        n += 1
        seen += 1
        slots = dev(np.array([slot_of(b, int(n[b]) - 1) for b in range(2)]))
        before = weights.clone()
        ok.kv4_decode_step(lay, pool, k.cuda(), v.cuda(), slots, 0.96, 0.96, q.cuda(), table, dev(n), dev(Rk), dev(Rv),
                           SM, splits, ws, out, weights=weights)
        if step % 13 == 0 or (n >= limit).any():
            host = pool.cpu().numpy()
            ref, w, tol, w_tol = R.attend(host, Hkv, 32, 0, q, tab, n, Rk, Rv, SM)
            assert (np.abs(out.cpu().numpy() - ref) <= tol).all()
            grown = (weights - before).cpu().numpy()
            slack = 2.0 ** -23 * weights.cpu().numpy()
            assert (np.abs(grown - w) <= w_tol + slack).all()
        if (n >= limit).any():
            host, w0, p0 = pool.cpu().numpy(), weights.cpu().numpy(), pos.cpu().numpy()
            want = R.evict(host, Hkv, 32, tab, n, w0, p0, seen, budget, sink, recent)
            new = torch.empty(2, dtype=torch.int32, device="cuda")
            ok.kv4_evict(lay, pool, table, dev(n), weights, pos, dev(seen), budget, sink, recent, new, ews)
            n = new.cpu().numpy()
            for a, b in zip((pool.cpu().numpy(), weights.cpu().numpy(), pos.cpu().numpy(), n), want):
                assert np.array_equal(a, b)
            for b in range(2):      # the newest tokens are all there, each once
                for h in range(Hkv):
                    kept = set(want[2][b, h, :n[b]].tolist())
                    assert set(range(int(seen[b]) - recent, int(seen[b]))) <= kept and len(kept) == n[b]
            evictions += 1
    assert evictions >= 1


def test_captured_and_replayed():
    """A step with weights and an eviction in one captured graph: every replay gives what
    the eager calls give on the inputs of that replay."""
    rng, lens, table, pool, weights, pos, lay = setup(9, (300, 190), 2)
    B, Hq, mp = 2, 8, table.shape[1]
    s = ok.default_num_splits(lay, B, Hq, mp * 64)
    t, ln = dev(table), dev(lens)
    p, w, ps = dev(pool), dev(weights), dev(pos)
    q = torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(B, 2, 128, dtype=torch.bfloat16, device="cuda")
    slots = dev(np.array([int(table[b, (n - 1) // 64]) * 64 + (n - 1) % 64 for b, n in enumerate(lens)], np.int64))
    ws, ews = ok.kv4_alloc_workspace(lay, B, Hq, s, mp, weights=True), ok.kv4_alloc_evict_workspace(lay, B, mp)
    out, w1, w2 = torch.zeros(B, Hq, 128, device="cuda"), torch.zeros_like(w), torch.zeros_like(w)
    p2, new = torch.zeros_like(ps), torch.zeros(B, dtype=torch.int32, device="cuda")

    def calls():
        ok.kv4_decode_step(lay, p, k, k, slots, 1.0, 1.0, q, t, ln, None, None, SM, s, ws, out, weights=w, weights_out=w1)
        ok.kv4_evict(lay, p, t, ln, w1, ps, ln, 100, 4, 16, new, ews, weights_out=w2, pos_out=p2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        q.copy_(torch.from_numpy(rng.standard_normal((B, Hq, 128)).astype(np.float32)))
        k.copy_(torch.from_numpy(rng.standard_normal((B, 2, 128)).astype(np.float32)))
        p.copy_(dev(pool))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (p, out, w1, w2, p2, new)]
        for x in (out, w1, w2, p2, new):
            x.zero_()
        p.copy_(dev(pool))
        calls()
        torch.cuda.synchronize()
        for a, b in zip(got, (p, out, w1, w2, p2, new)):
            assert torch.equal(a, b), i


def test_python_refusals():
    rng, lens, table, pool, weights, pos, lay = setup(10, (100, 80), 2)
    good = dict(pages=dev(pool), block_table=dev(table), seq_lens=dev(lens), weights=dev(weights), pos=dev(pos),
                num_seen=dev(lens), budget=64, sink=0, recent=0, new_lens=torch.zeros(2, dtype=torch.int32, device="cuda"),
                workspace=ok.kv4_alloc_evict_workspace(lay, 2, table.shape[1]))
    ok.kv4_evict(lay, **good)
    bad = [dict(weights=good["weights"].double()), dict(weights=good["weights"][:1]), dict(pos=good["pos"].long()),
           dict(pos=good["pos"].cpu()), dict(num_seen=good["num_seen"][:1]), dict(budget=0), dict(sink=-1),
           dict(recent=-1), dict(new_lens=good["seq_lens"]), dict(workspace=good["workspace"][:512]),
           dict(block_table=good["block_table"][0]), dict(weights_out=good["weights"][:1]), dict(pages=good["pages"][:-1])]
    for change in bad:
        with pytest.raises((TypeError, ValueError, ok.OscarError)):
            ok.kv4_evict(lay, **{**good, **change})


def test_debug_checks(monkeypatch):
    """OSCAR_DEBUG: lengths and page ids out of range are refused before any launch."""
    monkeypatch.setenv("OSCAR_DEBUG", "1")
    rng, lens, table, pool, weights, pos, lay = setup(11, (100, 80), 2)
    ws = ok.kv4_alloc_evict_workspace(lay, 2, table.shape[1])
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    bad_table = table.copy()
    bad_table[1, 1] = 2 ** 30
    for t, n in ((bad_table, lens), (table, np.array([100, 64 * table.shape[1] + 1], np.int32))):
        with pytest.raises(ok.OscarError) as e:
            ok.kv4_evict(lay, dev(pool), dev(t), dev(n), dev(weights), dev(pos), dev(lens), 64, 0, 0, new, ws)
        assert e.value.status == ok.ERR_INVALID_ARG
        with pytest.raises(ok.OscarError) as e:
            attend(lay, dev(pool), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), dev(t), dev(n))
        assert e.value.status == ok.ERR_INVALID_ARG


@pytest.mark.parametrize("budget,sink,recent", ((1, 0, 0), (700, 4, 16), (9000, 0, 1), (19999, 30000, 5), (33000, 1, 1)))
@pytest.mark.parametrize("kind", ("plain", "equal", "nan"))
def test_select_in_parts(budget, sink, recent, kind):
    """Tables of more slots than one block takes, with rows of any length in them."""
    rng, lens, table, pool, weights, pos, lay = setup(budget, (33270, 0, 700, 20000, 1), 2, 128, mp=520)
    if kind == "equal":
        weights[:, :, : 15000] = np.float32(0.7)
        weights[:, 1] = 3.0
    elif kind == "nan":
        weights[:, :, ::3] = np.nan
        weights[:, :, 1::5] = -np.inf
    pos[3, :, :9000] = rng.permutation(19000)[:9000]   # evicted before
    seen = lens + np.int32(12000) * (np.arange(5) == 3).astype(np.int32)
    check(lay, lens, table, pool, weights, pos, seen, budget, sink, recent, 128, in_place=(kind == "plain",))


def test_many_rows_in_parts():
    """So many rows that a row's select is of two parts only."""
    rng, lens, table, pool, weights, pos, lay = setup(11, [66 + i % 70 for i in range(300)], 2, 128, mp=520)
    check(lay, lens, table, pool, weights, pos, lens, 66, 1, 8, 128, in_place=(True,))


def test_parts_captured_and_two_at_once():
    """The select in parts from a captured graph, replayed, and in two calls on two streams."""
    rng, lens, table, pool, weights, pos, lay = setup(15, (20000, 700, 33000), 2, 128, mp=520)
    t, ln, ps = dev(table), dev(lens), dev(pos)

    def buffers():
        return dict(p=dev(pool), w=dev(weights), w2=torch.zeros_like(ps, dtype=torch.float32), p2=torch.zeros_like(ps),
                    new=torch.zeros(3, dtype=torch.int32, device="cuda"), ws=ok.kv4_alloc_evict_workspace(lay, 3, 520))

    def call(b):
        ok.kv4_evict(lay, b["p"], t, ln, b["w"], ps, ln, 3000, 4, 100, b["new"], b["ws"], weights_out=b["w2"],
                     pos_out=b["p2"])
    x, y = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(x)
    for i in range(4):
        w = np.exp(2 * rng.standard_normal(weights.shape)).astype(np.float32)
        for b in (x, y):
            b["w"].copy_(dev(w))
            b["p"].copy_(dev(pool))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            call(y)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        want = R.evict(pool, 2, 128, table, lens, w, pos, lens, 3000, 4, 100) if i == 0 else None
        for name, j in (("p", 0), ("w2", 1), ("p2", 2), ("new", 3)):
            assert torch.equal(x[name], y[name]), (i, name)
            assert want is None or np.array_equal(x[name].cpu().numpy(), want[j]), name
