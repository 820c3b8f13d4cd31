"""Definitions in 64 bits of the norm and rotation of new tokens and of the attention of
chunks over paged caches, with bounds of the library's roundings, for the tests.  Written
from include/oscar.h, without the library."""
from __future__ import annotations

import math

import numpy as np
import torch

import kv4_ref

D, P = 128, 64
U32, U16, UB = 2.0 ** -24, 2.0 ** -11, 2.0 ** -8   # half steps of fp32, fp16, bf16


# ---- page layouts: rows [n, Hkv, D] at their slots -------------------------------------

def bf16_places():
    """Element of (slot, channel) in a page-head block: K and V, [P, D] each."""
    t, c = np.meshgrid(np.arange(P), np.arange(D), indexing="ij")
    k = ((t % 4 * 4 + c // 8 % 4) * 64 + t // 4 + 16 * (c // 32)) * 8 + c % 8
    v = P * D + ((c // 16 * 2 + t // 8 % 2) * 64 + c % 16 + 16 * (t // 16)) * 8 + t % 8
    return torch.from_numpy(k), torch.from_numpy(v)


def put_bf16(pool, Hkv, slots, k, v):
    """bf16 rows into the pool's elements (all on the CPU; negative slots skipped)."""
    at = bf16_places()
    view = pool.view(-1, Hkv, 2 * P * D)
    for i, slot in enumerate(slots.tolist()):
        if slot < 0:
            continue
        for x, a in ((k, at[0]), (v, at[1])):
            view[slot // P][:, a[slot % P]] = x[i]


def put_int2(pool, Hkv, G, slots, is_v, code, s, z):
    """Codes [n, Hkv, D] (0 .. 3) and scale, zero bits [n, Hkv, D / G] into 2-bit pages."""
    ng = D // G
    size = 2 * (P * D // 4) + 2 * ng * P * 4
    view = pool.reshape(-1, Hkv, size)
    byte = code.reshape(*code.shape[:2], D // 4, 4)
    byte = (byte[..., 0] | byte[..., 1] << 2 | byte[..., 2] << 4 | byte[..., 3] << 6).astype(np.uint8)
    for i, slot in enumerate(slots):
        page, t = divmod(int(slot), P)
        for h in range(Hkv):
            blk = view[page, h]
            if is_v:
                blk[P * D // 4 + np.arange(D // 4) * P + t] = byte[i, h]
            else:
                blk[t * (D // 4):(t + 1) * (D // 4)] = byte[i, h]
            for g in range(ng):
                e = 2 * (P * D // 4) + is_v * ng * P * 4 + (g * P + t) * 4
                blk[e:e + 4] = np.array([s[i, h, g], z[i, h, g]], np.uint16).view(np.uint8)


def random_codes(rng, n, Hkv, G, levels, meta, spread=1.0):
    """Codes, scale and zero bits, and the values they stand for (fp64), of rows of about `spread`."""
    x = rng.standard_normal((n, Hkv, D // G, G)) * spread
    lo, hi = x.min(-1), x.max(-1)
    s = kv4_ref.stored(((hi - lo) / (levels - 1)).astype(np.float32), meta)
    sf = kv4_ref.f32_of(s, meta).reshape(lo.shape).astype(np.float64)
    z = kv4_ref.stored((-lo / np.where(sf == 0, 1.0, sf)).astype(np.float32), meta)
    zf = kv4_ref.f32_of(z, meta).reshape(lo.shape).astype(np.float64)
    code = np.clip(np.rint(x / np.where(sf == 0, 1.0, sf)[..., None] + zf[..., None]), 0, levels - 1)
    val = sf[..., None] * (code - zf[..., None])
    off = np.abs(sf * zf)[..., None] + 0.0 * val     # |s z|, which the kernels round
    shape = (n, Hkv, D)
    return code.astype(np.uint8).reshape(shape), s.reshape(lo.shape), z.reshape(lo.shape), val.reshape(shape), off.reshape(shape)


# ---- norm and rotation ------------------------------------------------------------------

def rope(x, weight, eps, pos, freq, rotary, interleaved, factor):
    """bf16 [n, H, D] -> (fp64 values, bound of the errors of a bf16 result)."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y, mag = x.clone(), x.abs()
    if rotary:
        i = torch.arange(rotary // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        t = pos.double()[:, None, None] * freq.double()
        c, s = t.cos() * factor, t.sin() * factor
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        mag[..., a] = mag[..., b] = abs(factor) * (x[..., a].abs() + x[..., b].abs())
    # fp32: the norm's sum of 128 squares (11 additions deep), root, quotient and two products; the
    # rotation's products and sum; the angle's fraction of a turn to 2^-26 of one (2^-23 in radians)
    # and sine and cosine to 2^-20
    return y, UB * y.abs() + mag * (40 * U32 + 2.0 ** -20) + 1e-38


# ---- attention --------------------------------------------------------------------------

def visible(n, length, window, sinks, device="cpu"):
    """bool [n, length]: which cached tokens the new ones see."""
    p = torch.arange(length - n, length, device=device)[:, None]
    t = torch.arange(length, device=device)[None, :]
    ok = t <= p
    if window:
        ok &= (t > p - window) | (t < sinks)
    return ok


def attend(q, k, v, ok, sm_scale, Rk=None, Rv=None, pieces=1, k_off=None, v_off=None):
    """One sequence: q bf16 [n, Hq, D]; k, v fp64 [len, Hkv, D]; ok [n, len] -> (fp64 [n, Hq, D], bound).
    pieces: bf16 pieces of a softmax weight; k_off, v_off (|s z| of quantized rows): fp16 operands."""
    n, Hq, _ = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    out = torch.zeros(n, Hq, D, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    quant = k_off is not None
    L = k.shape[0]
    if L == 0:
        return out, tol
    for h in range(Hq):
        kv = h // g
        rot = (lambda R: None if R is None else (R[kv] if R.dim() == 3 else R).double())
        x = q[:, h].double()
        rk, rv = rot(Rk), rot(Rv)
        x = x if rk is None else x @ rk
        K, V = k[:, kv], v[:, kv]
        s = (x @ K.T) * sm_scale
        m = s.masked_fill(~ok, -math.inf).amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        p = torch.exp(s - m).masked_fill(~ok, 0.0)
        den = p.sum(-1, keepdim=True)
        p = p / torch.where(den == 0, torch.ones_like(den), den)
        o, A = p @ V, p @ V.abs()
        # a score: 128 products summed in fp32, its factor, the exponent's rounding, exp2
        mag = abs(sm_scale) * (x.abs() @ K.abs().T)
        top = (mag + m.abs() + s.abs()).masked_fill(~ok, 0.0)
        ds = 150 * U32 * top + 2.0 ** -20
        pv = (2.0 ** -16 if pieces == 2 else UB)
        extra = 0.0
        if quant:
            # q~ to fp16 (and fp32 before), K to fp16 after a product and with -s z rounded; the
            # same for V; small ones against the page's (row's) largest
            koff = k_off[:, kv]
            ds = ds + abs(sm_scale) * (x.abs() @ (3 * K.abs() + koff).T) * U16
            ds = ds + abs(sm_scale) * 2.0 ** -18 * x.abs().amax(-1, keepdim=True) * K.abs().amax() * D
            voff = v_off[:, kv]
            extra = p @ (2 * V.abs() + voff) * U16 + 2.0 ** -18 * V.abs().amax() * (den > 0)
            pv = 2 * U16
        ds = torch.where(ok, ds, torch.zeros_like(ds)).amax(-1, keepdim=True)
        # off by the weights' roundings, the scores' (numerator and denominator), fp32 sums over the tokens
        t = A * (pv + 2 * torch.expm1(ds) + 2 * (L + 128) * U32) + extra
        if rv is not None:
            o, t = o @ rv.T, t @ rv.abs().T + (A @ rv.abs().T) * 140 * U32
        out[:, h], tol[:, h] = o, t + UB * (o.abs() + t) + 1e-38
    return out, tol
