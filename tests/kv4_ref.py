"""The 4-bit cache's definitions in numpy, for the tests: page layout, quantizer, decode
attention in 64 bits, eviction.  Written from include/oscar.h, without the library."""
from __future__ import annotations

import numpy as np
import torch

D, P = 128, 64


def block_bytes(G):
    return 2 * (P * D // 2) + 2 * (D // G) * P * 4


def k_place(t, c):
    """(byte, shift) of K channel c of slot t in a page-head block."""
    u, lo = t % 4, t // 4
    kc, hi, e = c // 32, c // 8 % 4, c % 8
    nibble = e // 2 + 4 * (e % 2)
    return ((64 * u + 16 * hi + lo) * 4 + kc) * 4 + nibble // 2, 4 * (nibble % 2)


def v_place(t, c):
    kt, hi, f, x = t // 32, t // 8 % 4, t // 4 % 2, t % 4
    j, n, lo = c // 32, c // 16 % 2, c % 16
    return P * D // 2 + (64 * j + 16 * hi + lo) * 16 + 8 * kt + 4 * f + x // 2 + 2 * (x % 2), 4 * n


def sz_place(G, is_v, t, g):
    """Byte of the (scale, zero) entry of slot t, group g."""
    ng = D // G
    return P * D + is_v * ng * P * 4 + (t * ng + g) * 4


_T, _C = np.meshgrid(np.arange(P), np.arange(D), indexing="ij")
_PLACES = [tuple(np.vectorize(f)(_T, _C)) for f in (k_place, v_place)]


def bf16_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16)


def f32_of(bits16: np.ndarray, meta: int) -> np.ndarray:
    b = np.ascontiguousarray(bits16).astype(np.uint16)
    return (b.astype(np.uint32) << 16).view(np.float32) if meta else b.view(np.float16).astype(np.float32)


def stored(x: np.ndarray, meta: int) -> np.ndarray:
    """fp32 -> 16 bits of the metadata format: nearest even, saturating."""
    x = np.asarray(x, np.float32)
    if not meta:
        return np.clip(x, -65504, 65504).astype(np.float16).view(np.uint16)
    u = x.view(np.uint32).astype(np.uint64)
    h = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where((h & 0x7FFF) == 0x7F80, (h & 0x8000) | 0x7F7F, h).astype(np.uint16)


def rotated(x: np.ndarray, R) -> np.ndarray:
    """fp32 rows x~ of fp32-valued rows x [n, Hkv, D]: products summed in fp64 in channel
    order, rounded once."""
    if R is None:
        return x.astype(np.float32)
    R = np.broadcast_to(np.asarray(R, np.float64), (x.shape[1], D, D))
    acc = np.zeros(x.shape, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        for c in range(D):
            acc += x[:, :, c, None].astype(np.float64) * R[None, :, c, :]
        return acc.astype(np.float32)


def quantize(xt: np.ndarray, G, meta, clip_mode, clip):
    """x~ [n, H, D] fp32 -> codes [n, H, D], scale and zero bits [n, H, D / G]; fp32 steps."""
    n, H, _ = xt.shape
    f = np.float32
    y = xt.reshape(n, H, D // G, G)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if clip_mode == 0:
            tau = f(clip) * np.abs(y).max(-1, keepdims=True)
        else:
            a = np.sort(np.abs(xt), -1)
            pos = f(f(clip) * f(D - 1))
            k = int(np.floor(pos))
            fr = f(pos - f(k))
            lo, hi = a[..., k], a[..., min(k + 1, D - 1)]
            tau = (lo + fr * (hi - lo))[:, :, None, None]
        y = np.minimum(np.maximum(y, -tau), tau)
        lo, hi = y.min(-1), y.max(-1)
        s = stored((hi - lo) / f(15), meta)
        deg = (s & 0x7FFF) == 0
        s = np.where(deg, 0x3F80 if meta else 0x3C00, s).astype(np.uint16)
        sf = f32_of(s, meta).reshape(lo.shape)
        z = stored(np.where(deg, -lo, -lo / sf), meta).reshape(lo.shape)
        z = np.where((z & 0x7FFF) == 0, 0, z).astype(np.uint16)
        zf = f32_of(z, meta).reshape(lo.shape)
        code = np.clip(np.rint(y / sf[..., None] + zf[..., None]), 0, 15)
    code = np.where(deg[..., None], 0, code).astype(np.uint8).reshape(n, H, D)
    return code, s.reshape(lo.shape), z.reshape(lo.shape)


def put_rows(pool: np.ndarray, Hkv, G, slots, is_v, code, s, z):
    """Writes rows (as from quantize) to their slots (negative: none) of the pool's bytes."""
    size = block_bytes(G)
    at, sh = _PLACES[is_v]
    view = pool.reshape(-1, Hkv, size)
    for i, slot in enumerate(slots):
        if slot < 0:
            continue
        page, t = divmod(int(slot), P)
        for h in range(Hkv):
            blk = view[page, h]
            for half in (0, 4):
                m = sh[t] == half
                b = at[t][m]
                blk[b] = (blk[b] & (0xF0 if half == 0 else 0x0F)) | (code[i, h, m] << half)
            for g in range(D // G):
                e = sz_place(G, is_v, t, g)
                blk[e:e + 4] = np.array([s[i, h, g], z[i, h, g]], np.uint16).view(np.uint8)


def append(pool, Hkv, G, meta, clip_mode, k, v, slots, Rk, Rv, clip_k, clip_v):
    for is_v, (x, R, clip) in enumerate(((k, Rk, clip_k), (v, Rv, clip_v))):
        x = (bf16_bits(x).astype(np.uint32) << 16).view(np.float32).reshape(x.shape)
        put_rows(pool, Hkv, G, slots, is_v, *quantize(rotated(x, R), G, meta, clip_mode, clip))


def block_values(blocks: np.ndarray, G, meta, is_v) -> np.ndarray:
    """fp32 values [..., P, D] of page-head blocks [..., bytes]: s * (n - z), fp32 steps."""
    at, sh = _PLACES[is_v]
    code = ((blocks[..., at] >> sh) & 15).astype(np.float32)
    ng = D // G
    base = sz_place(G, is_v, 0, 0)
    e = np.ascontiguousarray(blocks[..., base:base + P * ng * 4]).view(np.uint16)
    e = e.reshape(*blocks.shape[:-1], P, ng, 2)
    with np.errstate(over="ignore", invalid="ignore"):
        s, z = f32_of(e[..., 0], meta), f32_of(e[..., 1], meta)
        return (s[..., None] * (code.reshape(*code.shape[:-1], ng, G) - z[..., None])).reshape(code.shape)


def sequence_values(pool, Hkv, G, meta, table_row, n):
    """K, V values [n, Hkv, D] of a sequence's tokens."""
    pages = table_row[: -(-n // P)].astype(np.int64)
    blocks = pool.reshape(-1, Hkv, block_bytes(G))[pages]
    out = []
    for is_v in (0, 1):
        x = block_values(blocks, G, meta, is_v)              # [pages, Hkv, P, D]
        out.append(x.transpose(0, 2, 1, 3).reshape(-1, Hkv, D)[:n])
    return out


def attend(pool, Hkv, G, meta, q, table, lens, Rk, Rv, sm_scale):
    """64-bit decode attention: (out [B, Hq, D], weights [B, Hkv, slots], error scale
    [B, Hq, D] for the tolerance, see attn_tolerance)."""
    B, Hq, _ = q.shape
    g = Hq // Hkv
    qf = (bf16_bits(q).astype(np.uint32) << 16).view(np.float32).reshape(q.shape).astype(np.float64)
    out = np.zeros((B, Hq, D))
    tol = np.zeros((B, Hq, D))
    w = np.zeros((B, Hkv, table.shape[1] * P))
    w_tol = np.zeros_like(w)
    I = np.eye(D)
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        K, V = (x.astype(np.float64) for x in sequence_values(pool, Hkv, G, meta, table[b], n))
        for h in range(Hkv):
            rk = I if Rk is None else np.asarray(Rk if Rk.ndim == 2 else Rk[h], np.float64)
            rv = I if Rv is None else np.asarray(Rv if Rv.ndim == 2 else Rv[h], np.float64)
            x = qf[b, h * g:(h + 1) * g]
            qt = x @ rk
            s = qt @ K[:, h].T * sm_scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            ot = p @ V[:, h]
            out[b, h * g:(h + 1) * g] = ot @ rv.T
            w[b, h, :n] = p.sum(0)
            # First-order error of fp32 arithmetic, half a last place (2^-24) per operation:
            # q~ is a chain of 128 multiply-adds; a score sums 128 products of q~ and codes
            # below 16 with scales (the zero points' part is of the same size), whose low
            # bits the matrix cores may drop 7 bits early (a code is a subnormal operand).
            u = 2.0 ** -24
            kmax = np.abs(K[:, h]).max(0) if n else 0
            code_part = _code_part(pool, Hkv, G, meta, table[b], n, h)
            dq = 128 * u * (np.abs(x) @ np.abs(rk)) * sm_scale
            ds = dq @ kmax[:, None] + 16 * u * (np.abs(qt) * sm_scale) @ code_part[:, None] + \
                4 * u * np.abs(s).max(-1, keepdims=True)
            rel = 2 * ds + 8 * u                                  # of every weight
            spread = p @ np.abs(V[:, h])
            vcode = _code_part(pool, Hkv, G, meta, table[b], n, h, 1)
            do = rel * spread + 16 * u * vcode[None, :]
            tol[b, h * g:(h + 1) * g] = do @ np.abs(rv).T + 128 * u * np.abs(ot) @ np.abs(rv).T
            w_tol[b, h, :n] = (rel * p).sum(0) + 1e-30
    return out, w, tol, w_tol


def _code_part(pool, Hkv, G, meta, table_row, n, h, is_v=0):
    """Per channel, the largest scale * (15 + |zero|) of a head's tokens."""
    ng = D // G
    pages = table_row[: -(-n // P)].astype(np.int64)
    blocks = pool.reshape(-1, Hkv, block_bytes(G))[pages, h]
    base = sz_place(G, is_v, 0, 0)
    e = np.ascontiguousarray(blocks[:, base:base + P * ng * 4]).view(np.uint16).reshape(-1, ng, 2)[:n]
    s, z = f32_of(e[..., 0], meta).astype(np.float64), f32_of(e[..., 1], meta).astype(np.float64)
    return np.repeat((s * (15 + np.abs(z))).max(0), G)


def evict_row(w, pos, n, seen, budget, sink, recent):
    """One (sequence, head): (source slot of each of the m kept places, positions)."""
    m = min(n, budget)
    at = [int(p) if p >= 0 else seen - (n - t) for t, p in enumerate(pos[:n])]

    def key(t):
        x = float(w[t])
        safe = at[t] < sink or at[t] >= seen - recent
        return (0,) if safe else (2, 0.0) if x != x else (1, -x)

    kept = sorted(sorted(range(n), key=key)[:m])     # (sorted is stable: ties to the lowest slot)
    source = list(range(m))
    holes = sorted(set(source) - set(kept))
    for hole, t in zip(holes, [t for t in kept if t >= m]):
        source[hole] = t
    return source, at


def evict(pool, Hkv, G, table, lens, weights, pos, seen, budget, sink, recent):
    """(pool, weights, pos, lens) after an eviction."""
    size = block_bytes(G)
    src_pool = pool.reshape(-1, Hkv, size)
    pool = src_pool.copy()
    w_out, p_out = np.zeros_like(weights), np.full_like(pos, -1)
    for b in range(len(lens)):
        n = int(lens[b])
        for h in range(Hkv):
            source, at = evict_row(weights[b, h], pos[b, h], n, int(seen[b]), budget, sink, recent)
            for dst, src in enumerate(source):
                w_out[b, h, dst], p_out[b, h, dst] = weights[b, h, src], at[src]
                if dst == src:
                    continue
                a, c = src_pool[table[b, src // P], h], pool[table[b, dst // P], h]
                for is_v in (0, 1):
                    c[_PLACES[is_v][0][dst % P]] = a[_PLACES[is_v][0][src % P]]
                    for g in range(D // G):
                        i, o = sz_place(G, is_v, src % P, g), sz_place(G, is_v, dst % P, g)
                        c[o:o + 4] = a[i:i + 4]
    return pool.reshape(-1), w_out, p_out, np.minimum(lens, budget).astype(np.int32)


def random_pool(rng, num_pages, Hkv, G, meta, scale=0.1):
    """A pool of random codes with sane metadata: scales around `scale`, zeros around 7.5."""
    size = block_bytes(G)
    pool = rng.integers(0, 256, (num_pages, Hkv, size), dtype=np.uint8)
    ng = D // G
    for is_v in (0, 1):
        base = sz_place(G, is_v, 0, 0)
        s = stored((scale * np.exp(0.5 * rng.standard_normal((num_pages, Hkv, P, ng)))).astype(np.float32), meta)
        z = stored((7.5 + 2 * rng.standard_normal((num_pages, Hkv, P, ng))).astype(np.float32), meta)
        e = np.stack([s.reshape(num_pages, Hkv, P, ng), z.reshape(num_pages, Hkv, P, ng)], -1)
        pool[:, :, base:base + P * ng * 4] = np.ascontiguousarray(e).view(np.uint8).reshape(num_pages, Hkv, -1)
    return pool.reshape(-1)


def rotation(rng):
    return np.linalg.qr(rng.standard_normal((D, D)))[0].astype(np.float32)
