"""4-bit cache update and read-back against the numpy definitions: page bytes and values
are equal, bit for bit."""
import numpy as np
import pytest
import torch

import kv4_ref as R
import paper_2605_17757_amd as ok

pytestmark = pytest.mark.gpu

FORMATS = {"G32 f16 absmax": (32, 0, 0), "G128 bf16 quantile": (128, 1, 1), "G64 f16 quantile": (64, 0, 1),
           "G32 bf16 absmax": (32, 1, 0)}


def layout(Hkv, pages, fmt, rph=0):
    G, meta, mode = fmt
    return ok.Layout(Hkv, pages, group_size=G, meta_dtype=meta, clip_mode=mode, rot_per_head=rph)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rows(rng, n, Hkv, scale=1.0):
    x = rng.standard_normal((n, Hkv, 128)).astype(np.float32) * scale
    x[..., rng.choice(128, 3, replace=False)] *= 15
    return torch.from_numpy(x).bfloat16()


def check_append(fmt, Hkv, k, v, slots, pages, Rk, Rv, ck, cv, rph=0):
    rng = np.random.default_rng(9)
    lay = layout(Hkv, pages, fmt, rph)
    want = rng.integers(0, 256, ok.kv4_pool_bytes(lay), dtype=np.uint8)  # untouched bytes keep their values
    pool = dev(want)
    ok.kv4_append(lay, pool, k.cuda(), v.cuda(), dev(np.asarray(slots, np.int64)), dev(Rk), dev(Rv), ck, cv)
    R.append(want, Hkv, fmt[0], fmt[1], fmt[2], k, v, slots, Rk, Rv, ck, cv)
    got = pool.cpu().numpy()
    bad = np.nonzero(got != want)[0]
    assert bad.size == 0, (bad.size, bad[:8])


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("n,Hkv", [(1, 1), (15, 3), (17, 2), (64, 1), (700, 8)])  # the last: the bulk kernel
def test_append_bytes(name, n, Hkv):
    rng = np.random.default_rng(n + Hkv)
    pages = -(-n // 64) + 3
    slots = rng.permutation(pages * 64)[:n]
    check_append(FORMATS[name], Hkv, rows(rng, n, Hkv), rows(rng, n, Hkv, 3.0), slots, pages, R.rotation(rng),
                 R.rotation(rng), 0.96, 0.9)


@pytest.mark.parametrize("n", (5, 700))
@pytest.mark.parametrize("rot", ("none", "identity_v", "per_head"))
def test_append_rotations_and_skipped_slots(n, rot):
    rng = np.random.default_rng(n)
    Hkv, pages = 7, -(-n // 64) + 2
    slots = rng.permutation(pages * 64)[:n]
    slots[::5] = -1
    per = np.stack([R.rotation(rng) for _ in range(Hkv)])
    Rk, Rv = {"none": (None, None), "identity_v": (per[0], None), "per_head": (per, per[::-1].copy())}[rot]
    check_append(FORMATS["G32 f16 absmax"], Hkv, rows(rng, n, Hkv), rows(rng, n, Hkv), slots, pages, Rk, Rv, 1.0,
                 0.5, int(rot == "per_head"))


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("n", (9, 700))
def test_append_extreme_rows(name, n):
    """Rows of zeros, constants, one outlier, subnormal and huge values (scales that
    underflow, saturate, and pass the fast division's bounds)."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((n, 2, 128)).astype(np.float32)
    x[0] = 0.0
    x[1] = -3.25
    x[2] = 0.0
    x[2, :, 5] = 1000.0
    x[3] *= 1e-30
    x[4] *= 1e-6
    x[5] *= 1e6
    x[6] *= 1e30
    x[7] = np.where(np.arange(128) % 2, 1.0, -1.0)
    x[8, :, :64] = 0.0
    k = torch.from_numpy(x).bfloat16()
    pages = -(-n // 64) + 1
    check_append(FORMATS[name], 2, k, k.flip(0), np.arange(n) + 3, pages, R.rotation(rng), None, 0.96, 1.0)


def gathered(lay, pool, slots, dtype, fill=7.0):
    n = len(slots)
    k, v = (torch.full((n, lay.num_kv_heads, 128), fill, dtype=dtype, device="cuda") for _ in range(2))
    ok.kv4_gather(lay, pool, dev(np.asarray(slots, np.int64)), k, v)
    return k, v


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("kind", ("one", "scattered", "pages", "short runs", "twice", "long"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_gather_values(name, kind, dtype):
    fmt = FORMATS[name]
    rng = np.random.default_rng(3)
    Hkv, pages = 3, 40
    lay = layout(Hkv, pages, fmt)
    pool = R.random_pool(rng, pages, Hkv, fmt[0], fmt[1])
    every = np.arange(pages * 64)
    slots = {"one": [130], "scattered": rng.permutation(every)[:191],
             "pages": np.concatenate([p * 64 + np.arange(64) for p in (5, 3, 39, 0)]),
             "short runs": np.concatenate([p * 64 + 11 + np.arange(7 + p % 3) for p in range(30)]),
             "twice": np.concatenate([np.arange(64, 100), np.arange(80, 120), [64] * 12]),
             "long": np.concatenate([np.arange(7, 1403), [-1] * 5, np.arange(64, 64 + 700)])}[kind]
    slots = np.asarray(slots)
    k, v = gathered(lay, dev(pool), slots, dtype)
    blocks = pool.reshape(pages, Hkv, -1)
    for out, is_v in ((k, 0), (v, 1)):
        vals = torch.from_numpy(R.block_values(blocks, fmt[0], fmt[1], is_v))  # [pages, Hkv, 64, 128]
        want = vals.permute(0, 2, 1, 3).reshape(pages * 64, Hkv, 128)[np.maximum(slots, 0)].to(dtype)
        want[slots < 0] = 7.0
        assert torch.equal(out.cpu(), want)


def test_append_then_gather_past_4_gib():
    """Blocks past 2^32 bytes of the pool."""
    rng = np.random.default_rng(4)
    Hkv = 8
    lay = ok.Layout(Hkv, 54000)          # 4.4e9 bytes
    pool = torch.empty(ok.kv4_pool_bytes(lay), dtype=torch.uint8, device="cuda")
    slots = np.array([53999 * 64 + 63, 53999 * 64, 30000 * 64 + 5, 53000 * 64 + 17], np.int64)
    k, v = rows(rng, 4, Hkv), rows(rng, 4, Hkv)
    ok.kv4_append(lay, pool, k.cuda(), v.cuda(), dev(slots), None, None, 1.0, 1.0)
    small = np.zeros(4 * Hkv * R.block_bytes(32), np.uint8)
    at = [0 * 64 + 63, 1 * 64, 2 * 64 + 5, 3 * 64 + 17]
    R.append(small, Hkv, 32, 0, 0, k, v, at, None, None, 1.0, 1.0)
    for many in (slots, np.concatenate([slots] * 20)):   # both gather kernels
        got = gathered(lay, pool, many, torch.float32)
        for out, is_v in zip(got, (0, 1)):
            vals = R.block_values(small.reshape(4, Hkv, -1), 32, 0, is_v)
            want = np.stack([vals[i, :, a % 64] for i, a in enumerate(at)])
            assert np.array_equal(out.cpu().numpy(), np.concatenate([want] * (len(many) // 4)))


def test_python_refusals():
    lay = ok.Layout(2, 4)
    pool = ok.kv4_alloc_pool(lay)
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(3, device="cuda")
    out = torch.zeros(3, 2, 128, device="cuda")
    ok.kv4_append(lay, pool, k, k, slots, None, None, 1.0, 1.0)
    for bad in (dict(pool=pool[:-1]), dict(k=k.float()), dict(k=k[:2]), dict(k=k.transpose(0, 1)),
                dict(slots=slots.int()), dict(slots=slots.cpu()), dict(clip=0.0), dict(clip=2.0),
                dict(R=torch.zeros(64, 64, device="cuda"))):
        with pytest.raises((TypeError, ValueError, ok.OscarError)):
            ok.kv4_append(lay, bad.get("pool", pool), bad.get("k", k), k, bad.get("slots", slots), bad.get("R"),
                          None, bad.get("clip", 1.0), 1.0)
    for a, b in ((out, out.bfloat16()), (out.half(), out.half()), (out[:2], out), (out, out.cpu())):
        with pytest.raises((TypeError, ValueError)):
            ok.kv4_gather(lay, pool, slots, a, b)


def test_debug_checks(monkeypatch):
    """OSCAR_DEBUG: slots past the pool are refused on the host, before any launch."""
    monkeypatch.setenv("OSCAR_DEBUG", "1")
    lay = ok.Layout(1, 2)
    pool = ok.kv4_alloc_pool(lay)
    k = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(1, 1, 128, device="cuda")
    bad = torch.tensor([128], device="cuda")
    for call in (lambda: ok.kv4_append(lay, pool, k, k, bad, None, None, 1.0, 1.0),
                 lambda: ok.kv4_gather(lay, pool, bad, out, out.clone())):
        with pytest.raises(ok.OscarError) as e:
            call()
        assert e.value.status == ok.ERR_INVALID_ARG


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("kind", ("pages", "scattered", "short runs", "twice"))
def test_gather_by_tiles(name, kind):
    """Calls of more than 12288 rows, which read whole pages where a tile of tokens has
    several of one."""
    fmt = FORMATS[name]
    rng = np.random.default_rng(13)
    Hkv, pages = 40, 60
    lay = layout(Hkv, pages, fmt)
    pool = R.random_pool(rng, pages, Hkv, fmt[0], fmt[1])
    every = np.arange(pages * 64)
    slots = {"pages": np.concatenate([p * 64 + np.arange(64) for p in rng.permutation(pages)])[: 64 * 13 + 5],
             "scattered": rng.permutation(every)[:777],
             "short runs": np.concatenate([p * 64 + 11 + np.arange(3 + p % 11) for p in range(pages)] * 2),
             "twice": np.concatenate([np.arange(64, 100), np.arange(80, 120), [64] * 12, [-1] * 3, every[::5]])}[kind]
    assert len(slots) * Hkv > 12288
    for dtype in (torch.float32, torch.bfloat16):
        k, v = gathered(lay, dev(pool), slots, dtype)
        blocks = pool.reshape(pages, Hkv, -1)
        for out, is_v in ((k, 0), (v, 1)):
            vals = torch.from_numpy(R.block_values(blocks, fmt[0], fmt[1], is_v))
            want = vals.permute(0, 2, 1, 3).reshape(pages * 64, Hkv, 128)[np.maximum(slots, 0)].to(dtype)
            want[slots < 0] = 7.0
            assert torch.equal(out.cpu(), want)


def test_gather_by_tiles_past_4_gib():
    rng = np.random.default_rng(14)
    Hkv = 8
    lay = ok.Layout(Hkv, 54000)
    pool = torch.empty(ok.kv4_pool_bytes(lay), dtype=torch.uint8, device="cuda")
    ends = R.random_pool(rng, 2, Hkv, 32, 0)
    for i, p in enumerate((30000, 53999)):
        pool[p * ok.kv4_page_bytes(lay):(p + 1) * ok.kv4_page_bytes(lay)] = dev(ends[i * ok.kv4_page_bytes(lay):(i + 1) * ok.kv4_page_bytes(lay)])
    runs = np.concatenate([53999 * 64 + np.arange(64), 30000 * 64 + np.arange(3), [53999 * 64 + 5], 30000 * 64 + np.arange(60)])
    slots = np.concatenate([runs] * 32)
    got = gathered(lay, pool, slots, torch.float32)
    page = np.where(slots // 64 == 53999, 1, 0)
    for out, is_v in zip(got, (0, 1)):
        vals = R.block_values(ends.reshape(2, Hkv, -1), 32, 0, is_v)
        assert np.array_equal(out.cpu().numpy(), vals[page, :, slots % 64])


@pytest.mark.parametrize("n,Hkv", ((530, 8), (1700, 3)))   # just past the small kernel's calls, and several items a wave
@pytest.mark.parametrize("rot", ("identity_k", "per_head_k", "per_head_v"))
def test_append_one_rotated_tensor(n, Hkv, rot):
    """Longer calls of which one tensor is rotated: the blocks are shared out unevenly."""
    rng = np.random.default_rng(n)
    pages = -(-n // 64) + 2
    slots = rng.permutation(pages * 64)[:n]
    slots[::11] = -1
    per = np.stack([R.rotation(rng) for _ in range(Hkv)])
    Rk, Rv = {"identity_k": (None, per[0]), "per_head_k": (per, None), "per_head_v": (None, per)}[rot]
    for name in FORMATS:
        check_append(FORMATS[name], Hkv, rows(rng, n, Hkv), rows(rng, n, Hkv), slots, pages, Rk, Rv, 0.97, 0.97,
                     int(rot != "identity_k"))
