"""Timed workloads of the 4-bit cache's operators and their plain forms.

Each case is one layer's work in a program that serves a model with a KV cache held in
4 bits:

  write    rows of new tokens into the cache, and the same rows read back as values
           (``kv4_append``, ``kv4_gather``): what a prompt's chunk does before the next
           chunk attends to it;
  attend   one decode step's attention over the cache (``kv4_decode_attn``), with
           ``weigh`` also adding every token's attention weight to its running sum;
  step     the newest token of every sequence into the cache, and the attention over it
           (``kv4_decode_step``); the new rows are read back;
  evict    keeping the tokens with the largest running sums (``kv4_evict``); the kept
           rows are read back;
  cycle    eviction, then a decode step's attention over what was kept, weights and all.

With ``own`` set, ``run`` makes the package's calls; otherwise it computes the same in
elementary torch operations, from the same page bytes.  ``exact`` evaluates the
definitions in 64 bits from the rows the pages were made of.

Page layout (pages of 64 token slots; the block of page p, head h starts at byte
(p Hkv + h) (8192 + 512 ng), ng = 128 / G groups):
  K codes, 4096 bytes: slot t = 4 lo + u, channel 32 kc + 8 hi + e: dword
      (64 u + 16 hi + lo) 4 + kc, nibble e / 2 + 4 (e % 2)
  V codes, 4096 bytes: slot t = 32 kt + 8 hi + 4 f + x, channel 32 j + 16 n + lo: byte
      (64 j + 16 hi + lo) 16 + 8 kt + 4 f + (x / 2 + 2 (x % 2)), nibble n
  K scale and zero, 2 x 16 bits: entry t ng + g; then V's.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D, P = 128, 64
DEV = "cuda"
SM_SCALE = 1.0 / math.sqrt(D)
MAX_TOKENS = 131072  # the longest sequence
CHUNK = 16384        # tokens that a plain form unpacks at a time

# Quantizer formats: the library's default, the paper's (larger groups, bfloat16 scale
# and zero, the token's quantile as the clip bound), and two between them.
DEFAULT = {"G": 32, "meta": "f16", "clip_mode": "absmax", "clip": 0.96}
PAPER = {"G": 128, "meta": "bf16", "clip_mode": "quantile", "clip": 0.96}
HALF = {"G": 64, "meta": "f16", "clip_mode": "quantile", "clip": 0.98}
WIDE = {"G": 32, "meta": "bf16", "clip_mode": "absmax", "clip": 1.0}


def _write(name, n, Hkv, prompts=1, rot="shared", fmt=DEFAULT):
    return {"name": name, "kind": "write", "n": n, "prompts": prompts, "Hkv": Hkv, "rot": rot,
            "outliers": 4, **fmt}


def _attend(name, kind, B, Hq, Hkv, len_min, len_max, out="bf16", weigh=False, idle=0, rot="shared",
            fmt=DEFAULT, outliers=4):
    return {"name": name, "kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "len_min": len_min,
            "len_max": len_max, "out": out, "weigh": weigh, "idle": idle, "rot": rot,
            "outliers": outliers, **fmt}


def _evict(name, kind, B, Hq, Hkv, len_min, len_max, budget, sink, recent, again=False, out="bf16",
           rot="shared", fmt=DEFAULT):
    return {"name": name, "kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "len_min": len_min,
            "len_max": len_max, "budget": budget, "sink": sink, "recent": recent, "again": again,
            "out": out, "weigh": True, "idle": 0, "rot": rot, "outliers": 4, **fmt}


def listed():
    return [
        # One new token of a small layer: nothing but the latency of two launches.
        _write("write_1_h8", 1, 8),
        # The prompts of a few short chats written together, in the paper's format.
        _write("write_3x701_h8", 2103, 8, prompts=3, fmt=PAPER),
        # One long document: the largest write.
        _write("write_128k_h8", MAX_TOKENS, 8),
        # One user at the start of a chat, a Qwen3-4B-shaped layer: latency again.
        _attend("attend_b1_h32x8_ctx257", "attend", 1, 32, 8, 257, 257, out="f32"),
        # The benchmark's Qwen3-8B-shaped layer, reasoning traces of 16k to 32k tokens.
        _attend("attend_b64_h32x8_ctx32k", "attend", 64, 32, 8, 16384, 32768),
        # Long documents, 12 query heads per KV head, heavy-tailed keys: the largest decode.
        _attend("attend_b16_h96x8_ctx128k", "attend", 16, 96, 8, MAX_TOKENS, MAX_TOKENS, outliers=0),
        # A server's step with two idle places in its batch, uneven lengths, 8 query heads
        # per KV head, the paper's format.
        _attend("step_b16_h64x8_ctx4k", "step", 16, 64, 8, 301, 4099, idle=2, fmt=PAPER),
        # Steps that also weigh the tokens: a small batch on a long context, and the
        # benchmark's batch on a cache that is kept at 8k tokens.
        _attend("weigh_b2_h32x8_ctx31k", "attend", 2, 32, 8, 31001, 31001, weigh=True, fmt=HALF),
        _attend("weigh_b64_h32x8_ctx8k", "attend", 64, 32, 8, 7937, 8192, weigh=True),
        # One conversation that passes its budget of 2048 tokens by a page.
        _evict("evict_b1_h8_2k", "evict", 1, 32, 8, 2112, 2112, 2048, 4, 256, again=True),
        # Prompts of 8k to 16k tokens cut to 1024 before decoding.
        _evict("evict_b32_h8_16k", "evict", 32, 32, 8, 8192, 16384, 1024, 64, 256),
        # Eviction and the step after it, as a server runs them.
        _evict("cycle_b8_h16x4_4k", "cycle", 8, 16, 4, 1900, 4133, 2048, 4, 512, fmt=WIDE),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "attend", "attend", "weigh", "step", "evict", "evict", "cycle"))
    fmt = rng.choice((DEFAULT, PAPER, HALF, WIDE))
    rot = rng.choice(("shared", "shared", "identity_v", "per_head"))
    Hkv = rng.choice((1, 2, 4, 8))
    if kind == "write":
        prompts = rng.choice((1, 1, 2, 3, 8))
        c = _write("", max(prompts, _log_int(rng, 1, MAX_TOKENS)), Hkv, prompts, rot, fmt)
    else:
        g = rng.choice((1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 10, 12, 16))
        B = _log_int(rng, 1, 128)
        lo = 66 if kind in ("evict", "cycle") else 1
        # no more tokens x KV heads than 64 sequences of 24576 tokens and 8 heads, nor, with
        # kept rows read back, than a quarter of that
        most = 64 * 24576 * 8 // (4 if kind in ("evict", "cycle") else 1)
        hi = max(lo, min(_log_int(rng, lo, MAX_TOKENS), most // (B * Hkv), MAX_TOKENS))
        low = max(1, hi // rng.choice((1, 2, 4, 16)))
        out = rng.choice(("f32", "bf16"))
        if kind in ("evict", "cycle"):
            budget = min(_log_int(rng, 16, hi), max(16, 2 ** 18 // (B * Hkv)))
            sink = rng.choice((0, 4, 64))
            c = _evict("", kind, B, Hkv * g, Hkv, low, hi, budget, min(sink, budget // 4),
                       budget // rng.choice((2, 4, 8)), rng.random() < 0.5, out, rot, fmt)
        else:
            c = _attend("", "step" if kind == "step" else "attend", B, Hkv * g, Hkv, low, hi, out,
                        kind == "weigh" or rng.random() < 0.2, rng.choice((0, 0, 1)) if B > 1 else 0, rot,
                        fmt, rng.choice((4, 4, 0)))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed, stream, device=None):
    return torch.Generator(device=device or DEV).manual_seed((seed * 1_000_003 + stream) & 0x7FFFFFFFFFFF)


def _lens(case):
    """Tokens of each sequence: spread evenly from len_min to len_max, in the same
    shuffled order for every seed; the last `idle` places of that order hold none."""
    B, lo, hi = case["B"], case["len_min"], case["len_max"]
    n = [hi if B == 1 else lo + (hi - lo) * i // (B - 1) for i in range(B)]
    for i in range(case["idle"]):
        n[i] = 0
    order = torch.randperm(B, generator=torch.Generator().manual_seed(5)).tolist()
    return [n[i] for i in order]


def _rows(case, seed, stream, n, which):
    """bf16 rows [n, Hkv, D]: Gaussian with a few channels an order of magnitude larger
    (as activations of served models have), or Student-t(3) keys without."""
    g = _gen(seed, stream)
    x = torch.randn(n, case["Hkv"], D, generator=g, device=DEV, dtype=torch.bfloat16)
    if case["outliers"]:
        ch = torch.randperm(D, generator=_gen(seed, which, "cpu"))[: case["outliers"]]
        x[..., ch.to(DEV)] *= 15.0
    elif which == 1:
        c = torch.zeros(n, case["Hkv"], D, device=DEV)
        for _ in range(3):
            c += torch.randn(n, case["Hkv"], D, generator=g, device=DEV).square_()
        x = (x / c.div_(3.0).sqrt_()).to(torch.bfloat16)
    return x


def _kv(case, seed, b, n):
    """The n tokens of sequence b: K and V rows."""
    return _rows(case, seed, 2 * b + 101, n, 1), _rows(case, seed, 2 * b + 102, n, 2)


def _rotations(case, seed):
    """fp32 orthogonal matrices R_k, R_v ([Hkv, D, D] per head; None: identity)."""
    n = case["Hkv"] if case["rot"] == "per_head" else 1
    R = torch.linalg.qr(torch.randn(2, n, D, D, generator=_gen(seed, 3, "cpu"), dtype=torch.float64))[0]
    R = R.float().to(DEV)
    Rk, Rv = (R[0], R[1]) if case["rot"] == "per_head" else (R[0, 0], R[1, 0])
    return Rk.contiguous(), None if case["rot"] == "identity_v" else Rv.contiguous()


def _queries(case, seed):
    return torch.randn(case["B"], case["Hq"], D, generator=_gen(seed, 6), device=DEV).to(torch.bfloat16)


def _history(case, seed, b, n, S):
    """What a server has of sequence b before an eviction, per KV head: the running sums
    of n cached tokens (a few heavy ones, some that underflowed to 0), their positions
    (-1: not set; all of them, or those since the last eviction), and the tokens seen."""
    g, Hkv = _gen(seed, 50_000 + b), case["Hkv"]
    w = torch.exp(2.0 * torch.randn(Hkv, n, generator=g, device=DEV) - 3.0)
    w[torch.rand(Hkv, n, generator=g, device=DEV) < 0.05] = 0.0
    weights = torch.zeros(Hkv, S, device=DEV)
    weights[:, :n] = w
    pos = torch.full((Hkv, S), -1, dtype=torch.int32, device=DEV)
    seen = n
    if case["again"]:  # kept tokens of an earlier eviction, and a page of new ones
        old = n - min(P, n - 1)
        seen = 2 * n
        for h in range(Hkv):
            pos[h, :old] = torch.randperm(seen - (n - old), generator=g, device=DEV)[:old].to(torch.int32)
    return weights, pos, seen


# ---------------------------------------------------------------------------
# the page layout
# ---------------------------------------------------------------------------

def _block_bytes(case):
    return 8192 + 512 * (D // case["G"])


def _code_map():
    """For slot t and byte i of a row: the byte's place in the K and in the V region, and
    the channels of its low and high nibble (the same for every slot)."""
    t, i = torch.arange(P)[:, None], torch.arange(64)[None, :]
    kc, hi, s, f = i // 16, i // 4 % 4, i // 2 % 2, i % 2   # K byte: channels 32 kc + 8 hi + 4 f + s, + 2
    k_at = ((64 * (t % 4) + 16 * hi + t // 4) * 4 + kc) * 4 + 2 * s + f
    k_low = (32 * kc + 8 * hi + 4 * f + s)[0]
    j, lo = i // 16, i % 16                                 # V byte: channels 32 j + lo, + 16
    x = t % 4
    v_at = 4096 + (64 * j + 16 * (t // 8 % 4) + lo) * 16 + 8 * (t // 32) + 4 * (t // 4 % 2) + x // 2 + 2 * (x % 2)
    v_low = (32 * j + lo)[0]
    return k_at.to(DEV), k_low.to(DEV), v_at.to(DEV), v_low.to(DEV)


def _sz_map(case):
    """For slot t: the 16-bit places of its K and V scales (the zeros follow them)."""
    ng = D // case["G"]
    k = (8192 + 4 * (torch.arange(P)[:, None] * ng + torch.arange(ng)[None, :])) // 2
    return k.to(DEV), (k + 128 * ng).to(DEV)


def _quantize(x, R, case):
    """bf16 rows [n, Hkv, D] -> codes uint8 [n, Hkv, D] and the stored scale and zero
    (16-bit patterns, [n, Hkv, groups]).  The rotation is summed in 64 bits and rounded
    once; every later step is one fp32 operation, as the format is defined."""
    if R is None:
        xt = x.float()
    elif R.dim() == 2:
        xt = (x.reshape(-1, D).double() @ R.double()).float().reshape(x.shape)
    else:
        xt = torch.stack([(x[:, h].double() @ R[h].double()).float() for h in range(x.shape[1])], 1)
    G = case["G"]
    y = xt.unflatten(-1, (D // G, G))
    clip = torch.tensor(case["clip"], dtype=torch.float32, device=x.device)
    if case["clip_mode"] == "absmax":
        tau = clip * y.abs().amax(-1, keepdim=True)
    else:
        at = clip * 127.0
        k = at.floor()
        i = int(k)
        a = xt.abs().sort(-1).values
        tau = (a[..., i] + (at - k) * (a[..., min(i + 1, D - 1)] - a[..., i]))[..., None, None]
    y = torch.minimum(torch.maximum(y, -tau), tau)
    dt, top = (torch.bfloat16, 3.3895313892515355e38) if case["meta"] == "bf16" else (torch.float16, 65504.0)
    a, b = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = ((b - a) / torch.full_like(a, 15.0)).clamp(-top, top).to(dt)
    flat = s == 0
    sf = torch.where(flat, torch.ones_like(s), s).float()
    z = torch.where(flat, -a, -a / sf).clamp(-top, top).to(dt)
    z = torch.where(z == 0, torch.zeros_like(z), z)
    code = (y / sf + z.float()).round().clamp(0.0, 15.0)
    code = torch.where(flat, torch.zeros_like(code), code).to(torch.uint8).flatten(-2)
    return code, sf.to(dt).squeeze(-1).view(torch.int16), z.squeeze(-1).view(torch.int16)


def _plain_append(case, pages, k, v, slots, Rk, Rv, maps):
    k_at, k_low, v_at, v_low = maps["code"]
    Hkv, size = case["Hkv"], _block_bytes(case)
    words = pages.view(torch.int16)
    for i in range(0, slots.numel(), CHUNK):
        sl = slots[i:i + CHUNK]
        t = sl % P
        block = ((sl // P)[:, None] * Hkv + torch.arange(Hkv, device=DEV)) * size
        for x, R, at, low, step, sz_at in ((k, Rk, k_at, k_low, 2, maps["sz"][0]),
                                           (v, Rv, v_at, v_low, 16, maps["sz"][1])):
            code, s, z = _quantize(x[i:i + CHUNK], R, case)
            pages[block[..., None] + at[t][:, None]] = code[..., low] | (code[..., low + step] << 4)
            w = (block // 2)[..., None] + sz_at[t][:, None]
            words[w] = s
            words[w + 1] = z


def _values(case, blocks, maps):
    """Page blocks uint8 [..., size] -> fp32 K and V values [..., P, D]."""
    k_at, k_low, v_at, v_low = maps["code"]
    ng = D // case["G"]
    dt = torch.bfloat16 if case["meta"] == "bf16" else torch.float16
    out = []
    for at, low, step, sz_at in ((k_at, k_low, 2, maps["sz"][0]), (v_at, v_low, 16, maps["sz"][1])):
        byte = blocks[..., at]                                     # [..., P, 64]
        code = torch.empty(*byte.shape[:-1], D, device=DEV)
        code[..., low] = (byte & 15).float()
        code[..., low + step] = (byte >> 4).float()
        sz = blocks.view(torch.int16)
        s, z = sz[..., sz_at].view(dt).float(), sz[..., sz_at + 1].view(dt).float()  # [..., P, ng]
        code = code.unflatten(-1, (ng, case["G"]))
        out.append((s[..., None] * (code - z[..., None])).flatten(-2))
    return out


def _plain_gather(case, pages, slots, maps):
    """fp32 K and V values [n, Hkv, D] of the slots."""
    k_at, k_low, v_at, v_low = maps["code"]
    Hkv, size, ng = case["Hkv"], _block_bytes(case), D // case["G"]
    dt = torch.bfloat16 if case["meta"] == "bf16" else torch.float16
    words = pages.view(torch.int16)
    out = [torch.empty(slots.numel(), Hkv, D, device=DEV) for _ in range(2)]
    for i in range(0, slots.numel(), CHUNK):
        sl = slots[i:i + CHUNK]
        t = sl % P
        block = ((sl // P)[:, None] * Hkv + torch.arange(Hkv, device=DEV)) * size
        for o, at, low, step, sz_at in ((out[0], k_at, k_low, 2, maps["sz"][0]),
                                        (out[1], v_at, v_low, 16, maps["sz"][1])):
            byte = pages[block[..., None] + at[t][:, None]]
            code = torch.empty(*byte.shape[:-1], D, device=DEV)
            code[..., low] = (byte & 15).float()
            code[..., low + step] = (byte >> 4).float()
            w = (block // 2)[..., None] + sz_at[t][:, None]
            s, z = words[w].view(dt).float(), words[w + 1].view(dt).float()
            o[i:i + CHUNK] = (s[..., None] * (code.unflatten(-1, (ng, case["G"])) - z[..., None])).flatten(-2)
    return out


def _plain_attend(case, pages, q, table, lens, Rk, Rv, weights, maps):
    """(out [B, Hq, D], weights + every token's attention weight, or None)."""
    Hkv, Hq = case["Hkv"], case["Hq"]
    g = Hq // Hkv
    out = torch.zeros(len(lens), Hq, D, device=DEV)
    total = torch.zeros_like(weights) if weights is not None else None
    blocks = pages.view(-1, Hkv, _block_bytes(case))
    for b, n in enumerate(lens):
        if n == 0:
            continue
        qb = q[b].float().view(Hkv, g, D)
        qb = qb @ Rk if Rk is not None else qb                 # one matrix, or one per head
        V, S = [], []
        n_pages = -(-n // P)
        for i in range(0, n_pages, CHUNK // P):
            kk, vv = _values(case, blocks[table[b, i:min(i + CHUNK // P, n_pages)].long()], maps)
            kk = kk.transpose(0, 1).reshape(Hkv, -1, D)        # [Hkv, tokens, D]
            V.append(vv.transpose(0, 1).reshape(Hkv, -1, D))
            S.append(qb @ kk.transpose(1, 2).contiguous())
        s = torch.cat(S, 2)[..., :n] * SM_SCALE
        e = torch.exp(s - s.amax(-1, keepdim=True))
        p = e / e.sum(-1, keepdim=True)
        o = p @ torch.cat(V, 1)[:, :n].contiguous()
        out[b] = (o @ Rv.transpose(-1, -2).contiguous() if Rv is not None else o).reshape(Hq, D)
        if weights is not None:
            total[b, :, :n] = weights[b, :, :n] + p.sum(1)
    return out.to(torch.float32 if case["out"] == "f32" else torch.bfloat16), total


def _plain_evict(case, s):
    """Keeps the heaviest tokens; rows of pages move in place."""
    Hkv, size = case["Hkv"], _block_bytes(case)
    k_at, _, v_at, _ = s["maps"]["code"]
    ng = D // case["G"]
    weights, pos = torch.zeros_like(s["weights"]), torch.full_like(s["pos"], -1)
    new = torch.minimum(s["lens"], torch.full_like(s["lens"], case["budget"]))
    sz = s["maps"]["sz"][0][:, :1] * 2 + torch.arange(4 * ng, device=DEV)         # bytes of a slot's entries
    place = torch.cat([k_at, v_at, sz, sz + 256 * ng], 1)                          # [P, bytes of a row]
    heads = torch.arange(Hkv, device=DEV)[:, None]
    for b, n in enumerate(s["n"]):
        m, seen = min(n, case["budget"]), int(s["n_seen"][b])
        at = torch.arange(n, device=DEV)
        p = s["pos"][b, :, :n]
        p = torch.where(p >= 0, p, (seen - n + at).to(torch.int32))
        w = s["weights"][b, :, :n]
        rank = torch.where((p < case["sink"]) | (p >= seen - case["recent"]), math.inf, w)
        order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :m]
        keep = torch.zeros(Hkv, n, dtype=torch.bool, device=DEV).scatter_(1, order, True)
        weights[b, :, :m], pos[b, :, :m] = w[:, :m], p[:, :m]
        h_dst, dst = torch.nonzero(~keep[:, :m], as_tuple=True)     # by head, ascending
        h_src, src = torch.nonzero(keep[:, m:], as_tuple=True)      # as many in every head
        src = src + m
        weights[b, h_dst, dst], pos[b, h_dst, dst] = w[h_src, src], p[h_src, src]
        page = s["table"][b].long()
        for i in range(0, dst.numel(), 1 << 17):
            e = slice(i, i + (1 << 17))
            to = ((page[dst[e] // P] * Hkv + h_dst[e]) * size)[:, None] + place[dst[e] % P]
            fr = ((page[src[e] // P] * Hkv + h_src[e]) * size)[:, None] + place[src[e] % P]
            s["pages"][to] = s["pages"][fr]
    return new, weights, pos


# ---------------------------------------------------------------------------
# the program around a call
# ---------------------------------------------------------------------------

def _paging(case, seed):
    """int32 [B, pages a sequence]: a pool dealt out shuffled, with room for 64 more
    tokens in every sequence."""
    mp = -(-(case["len_max"] + P) // P)
    perm = torch.randperm(case["B"] * mp, generator=_gen(seed, 4, "cpu")).to(torch.int32)
    return perm.reshape(case["B"], mp).to(DEV)


def _slots(table_row, at):
    return table_row.long()[at // P] * P + at % P


def _write_slots(case, seed):
    """Slots of the prompts' tokens (the prompts as long as can be alike), each prompt in
    pages of its own from a shuffled pool; a lone token comes at the end of a page's first half."""
    n, m = case["n"], case["prompts"]
    each = [n // m + (i < n % m) for i in range(m)]
    need = [-(-e // P) for e in each]
    perm = torch.randperm(sum(need) + 3, generator=_gen(seed, 4, "cpu")).to(DEV)
    slots, used = [], 0
    for e, c in zip(each, need):
        slots.append(_slots(perm[used:used + c], torch.arange(e, device=DEV)))
        used += c
    slots = torch.cat(slots)
    return (slots + 31 if n == 1 else slots), sum(need) + 3


def prepare(case, seed):
    Rk, Rv = _rotations(case, seed)
    maps = {"code": _code_map(), "sz": _sz_map(case)}
    s = {"case": case, "Rk": Rk, "Rv": Rv, "maps": maps}
    Hkv = case["Hkv"]
    if case["kind"] == "write":
        s["slots"], num_pages = _write_slots(case, seed)
        s["k"], s["v"] = _kv(case, seed, 0, case["n"])
    else:
        B, Hq, lens = case["B"], case["Hq"], _lens(case)
        s["table"] = _paging(case, seed)
        mp = s["table"].shape[1]
        num_pages = B * mp
        s["n"], s["lens"] = lens, torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["q"] = _queries(case, seed)
        s["out"] = torch.empty(B, Hq, D, device=DEV,
                               dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16)
        s["weights"] = None
        if case["weigh"]:
            s["weights"] = torch.zeros(B, Hkv, mp * P, device=DEV)
            s["weights_out"] = torch.zeros_like(s["weights"])
    s["pages"] = torch.zeros(num_pages * Hkv * _block_bytes(case), dtype=torch.uint8, device=DEV)
    if case["kind"] in ("evict", "cycle"):
        s["pos"] = torch.empty(B, Hkv, mp * P, dtype=torch.int32, device=DEV)
        s["pos_out"], s["weights_kept"] = torch.empty_like(s["pos"]), torch.empty_like(s["weights"])
        s["n_seen"] = []
        s["new"] = torch.empty_like(s["lens"])
        for b, n in enumerate(lens):
            s["weights"][b], s["pos"][b], seen = _history(case, seed, b, n, mp * P)
            s["n_seen"].append(seen)
        s["seen"] = torch.tensor(s["n_seen"], dtype=torch.int32, device=DEV)
        kept = [_slots(s["table"][b], torch.arange(min(n, case["budget"]), device=DEV))
                for b, n in enumerate(lens)]
        s["slots"] = torch.cat(kept)
    elif case["kind"] != "write" and case["weigh"]:
        for b, n in enumerate(lens):  # sums of the steps so far
            g = _gen(seed, 50_000 + b)
            s["weights"][b, :, :n] = torch.exp(2.0 * torch.randn(Hkv, n, generator=g, device=DEV) - 3.0)
    if case["kind"] != "write":
        step = case["kind"] == "step"
        new = []
        for b, n in enumerate(lens):
            if n == 0:
                continue
            k, v = _kv(case, seed, b, n)
            old = n - 1 if step else n
            _plain_append(case, s["pages"], k[:old], v[:old],
                          _slots(s["table"][b], torch.arange(old, device=DEV)), Rk, Rv, maps)
            new.append((k[-1], v[-1], _slots(s["table"][b], torch.tensor([n - 1], device=DEV))))
        if step:
            s["k"], s["v"] = (torch.stack([x[i] for x in new]) for i in (0, 1))
            s["slots"] = torch.cat([x[2] for x in new])
    if case["kind"] in ("write", "step", "evict"):
        s["values"] = [torch.empty(s["slots"].numel(), Hkv, D, device=DEV) for _ in range(2)]
    if own:
        import paper_2605_17757_amd as oscar
        s["L"] = L = oscar.Layout(
            Hkv, num_pages, group_size=case["G"],
            clip_mode=oscar.CLIP_TOKEN_QUANTILE if case["clip_mode"] == "quantile" else oscar.CLIP_GROUP_ABSMAX,
            meta_dtype=oscar.META_BF16 if case["meta"] == "bf16" else oscar.META_F16,
            rot_per_head=int(case["rot"] == "per_head"))
        if case["kind"] in ("attend", "step", "cycle"):
            s["splits"] = oscar.default_num_splits(L, B, Hq, case["len_max"])
            s["ws"] = oscar.kv4_alloc_workspace(L, B, Hq, s["splits"], mp, weights=case["weigh"])
        if case["kind"] in ("evict", "cycle"):
            s["evict_ws"] = oscar.kv4_alloc_evict_workspace(L, B, mp)
    return s


def _run_own(s):
    import paper_2605_17757_amd as oscar
    case = s["case"]
    kind, clip = case["kind"], case["clip"]
    if kind == "write":
        oscar.kv4_append(s["L"], s["pages"], s["k"], s["v"], s["slots"], s["Rk"], s["Rv"], clip, clip)
        oscar.kv4_gather(s["L"], s["pages"], s["slots"], *s["values"])
        return {"k": s["values"][0], "v": s["values"][1]}
    res, lens, weights = {}, s["lens"], s["weights"]
    if kind in ("evict", "cycle"):
        oscar.kv4_evict(s["L"], s["pages"], s["table"], s["lens"], s["weights"], s["pos"], s["seen"],
                        case["budget"], case["sink"], case["recent"], s["new"], s["evict_ws"],
                        weights_out=s["weights_kept"], pos_out=s["pos_out"])
        res = {"lens": s["new"], "kept": s["weights_kept"], "pos": s["pos_out"]}
        lens, weights = s["new"], s["weights_kept"]
    if kind == "step":
        oscar.kv4_decode_step(s["L"], s["pages"], s["k"], s["v"], s["slots"], clip, clip, s["q"], s["table"],
                              lens, s["Rk"], s["Rv"], SM_SCALE, s["splits"], s["ws"], s["out"],
                              weights=weights, weights_out=s.get("weights_out"))
    elif kind != "evict":
        oscar.kv4_decode_attn(s["L"], s["pages"], s["q"], s["table"], lens, s["Rk"], s["Rv"], SM_SCALE,
                              s["splits"], s["ws"], s["out"], weights=weights,
                              weights_out=s.get("weights_out"))
    if kind in ("step", "evict"):
        oscar.kv4_gather(s["L"], s["pages"], s["slots"], *s["values"])
        res["k"], res["v"] = s["values"]
    if kind != "evict":
        res["out"] = s["out"]
        if weights is not None:
            res["weights"] = s["weights_out"]
    return res


def run(s):
    if own:
        return _run_own(s)
    case, maps = s["case"], s["maps"]
    kind = case["kind"]
    if kind in ("write", "step"):
        _plain_append(case, s["pages"], s["k"], s["v"], s["slots"], s["Rk"], s["Rv"], maps)
    if kind == "write":
        k, v = _plain_gather(case, s["pages"], s["slots"], maps)
        return {"k": k, "v": v}
    res, n, weights = {}, s["n"], s["weights"]
    if kind in ("evict", "cycle"):
        new, weights, pos = _plain_evict(case, s)
        res = {"lens": new, "kept": weights, "pos": pos}
        n = [min(x, case["budget"]) for x in n]
    if kind in ("step", "evict"):
        res["k"], res["v"] = _plain_gather(case, s["pages"], s["slots"], maps)
    if kind != "evict":
        res["out"], total = _plain_attend(case, s["pages"], s["q"], s["table"], n, s["Rk"], s["Rv"], weights,
                                          maps)
        if weights is not None:
            res["weights"] = total
    return res


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    Hkv, ng = case["Hkv"], D // case["G"]
    row = D + 8 * ng  # bytes of a token's K and V of one head, codes and metadata
    rots = 1 if case["rot"] == "identity_v" else 2
    if case["kind"] == "write":
        n = case["n"]
        return {"bytes": n * Hkv * (4 * D + row + 8 * D) + 8 * n, "flops": rots * 2 * D * D * n * Hkv}
    lens, Hq = _lens(case), case["Hq"]
    nbytes = flops = 0
    if case["kind"] in ("evict", "cycle"):
        S = -(-(case["len_max"] + P) // P) * P
        for n in lens:
            m = min(n, case["budget"])
            beyond = min(n - m, case["recent"])  # moved: the recent ones behind m, and the heavy ones' share
            free = max(0, m - case["sink"] - case["recent"])
            moved = beyond + free * max(0, n - m - case["recent"]) / max(1, n - case["sink"] - case["recent"])
            nbytes += Hkv * (8 * n + 8 * S + 2 * row * moved)
        lens = [min(n, case["budget"]) for n in lens]
        if case["kind"] == "evict":
            m = sum(lens)
            return {"bytes": int(nbytes + Hkv * m * (row + 8 * D)), "flops": 2 * D * Hkv * m}
    for n in lens:
        if n == 0:
            continue
        nbytes += Hkv * n * (row + (8 if case["weigh"] else 0))
        flops += Hq * n * 4 * D + rots * 2 * D * D * Hq
        if case["kind"] == "step":
            nbytes += Hkv * (4 * D + 8 * D + row)
            flops += rots * 2 * D * D * Hkv
    nbytes += len(lens) * Hq * D * (2 + (4 if case["out"] == "f32" else 2))
    return {"bytes": int(nbytes), "flops": int(flops)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits, from the rows
# ---------------------------------------------------------------------------

def _held(x, R, case):
    """fp64 values that the cache holds of bf16 rows [n, Hkv, D] in the rotated basis."""
    n, H, _ = x.shape
    if R is None:
        r = x.double()
    else:
        r = torch.einsum("nhc,hcd->nhd", x.double(), R.double().expand(H, D, D)) if R.dim() == 3 else \
            torch.matmul(x.double().view(n * H, D), R.double()).view(n, H, D)
    r = r.to(torch.float32)
    G, ng = case["G"], D // case["G"]
    mag = r.abs()
    ratio = torch.full((), case["clip"], dtype=torch.float32, device=DEV)
    if case["clip_mode"] == "quantile":
        srt = torch.sort(mag, dim=-1)[0]
        where = (ratio * torch.full((), D - 1.0, device=DEV)).item()
        k0 = math.floor(where)
        bound = srt[:, :, k0]
        if k0 + 1 < D:
            bound = bound + torch.tensor(where - k0, dtype=torch.float32, device=DEV) * (srt[:, :, k0 + 1] - bound)
        bound = bound[:, :, None].expand(n, H, ng)
    else:
        bound = ratio * mag.view(n, H, ng, G).max(-1)[0]
    y = r.view(n, H, ng, G)
    y = torch.where(y > bound[..., None], bound[..., None], y)
    y = torch.where(y < -bound[..., None], -bound[..., None], y)
    lo, hi = y.min(-1)[0], y.max(-1)[0]

    def stored(v):
        kind = torch.float16 if case["meta"] == "f16" else torch.bfloat16
        top = torch.finfo(kind).max
        return torch.clamp(v, -top, top).to(kind).float()

    scale = stored(torch.div(hi - lo, torch.tensor(15.0, device=DEV)))
    none = scale == 0
    zero = stored(torch.where(none, -lo, torch.div(-lo, torch.where(none, torch.ones_like(scale), scale))))
    scale = torch.where(none, torch.ones_like(scale), scale)
    c = torch.clamp(torch.round(torch.div(y, scale[..., None]) + zero[..., None]), 0, 15)
    c = torch.where(none[..., None], torch.zeros_like(c), c)
    return ((c.double() - zero.double()[..., None]) * scale.double()[..., None]).view(n, H, D)


def _held_rows(x, R, case):
    return torch.cat([_held(x[i:i + 8192], R, case) for i in range(0, x.shape[0], 8192)]) if x.shape[0] else x.double()


def _exact_order(case, w, pos, n, seen):
    """Slots of one head after an eviction: the source slot of each kept place."""
    m = min(n, case["budget"])
    w, pos, t = w[:n].astype(np.float64), pos[:n].astype(np.int64), np.arange(n)
    at = np.where(pos >= 0, pos, seen - (n - t))
    safe = np.logical_or(at < case["sink"], at >= seen - case["recent"])
    kept = np.sort(np.lexsort((t, np.where(safe, 0.0, -w), np.where(safe, 0, 1)))[:m])  # last key first
    source = np.arange(m)
    source[np.setdiff1d(source, kept)] = kept[kept >= m]
    return source, at


def exact(case, seed):
    Rk, Rv = _rotations(case, seed)
    Hkv = case["Hkv"]
    if case["kind"] == "write":
        k, v = _kv(case, seed, 0, case["n"])
        return {"k": _held_rows(k, Rk, case), "v": _held_rows(v, Rv, case)}
    B, Hq, lens = case["B"], case["Hq"], _lens(case)
    g = Hq // Hkv
    S = -(-(case["len_max"] + P) // P) * P
    evicting, cycle, step = case["kind"] in ("evict", "cycle"), case["kind"] == "cycle", case["kind"] == "step"
    q = _queries(case, seed).double()
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=DEV)
    total = torch.zeros(B, Hkv, S, dtype=torch.float64, device=DEV) if case["weigh"] else None
    if evicting:
        kept = torch.zeros(B, Hkv, S, dtype=torch.float64, device=DEV)
        places = torch.full((B, Hkv, S), -1, dtype=torch.int32, device=DEV)
    ks, vs = [], []
    for b, n in enumerate(lens):
        if n == 0:
            continue
        k, v = _kv(case, seed, b, n)
        if step:
            ks.append(_held(k[-1:], Rk, case))
            vs.append(_held(v[-1:], Rv, case))
        K, V = _held_rows(k, Rk, case), _held_rows(v, Rv, case)
        if evicting:
            w, pos, seen = _history(case, seed, b, n, S)
            w, pos = w.cpu().numpy(), pos.cpu().numpy()
            KK, VV = [], []
            for h in range(Hkv):
                source, at = _exact_order(case, w[h], pos[h], n, seen)
                kept[b, h, :len(source)] = torch.from_numpy(w[h][source].astype(np.float64)).to(DEV)
                places[b, h, :len(source)] = torch.from_numpy(at[source].astype(np.int32)).to(DEV)
                source = torch.from_numpy(source).to(DEV)
                KK.append(K[source, h])
                VV.append(V[source, h])
            K, V = torch.stack(KK, 1), torch.stack(VV, 1)
            n = K.shape[0]
            if not cycle:
                ks.append(K)
                vs.append(V)
                continue
        for h in range(Hkv):
            rk = None if Rk is None else (Rk if Rk.dim() == 2 else Rk[h]).double()
            rv = None if Rv is None else (Rv if Rv.dim() == 2 else Rv[h]).double()
            x = q[b, h * g:(h + 1) * g]
            x = x if rk is None else x @ rk
            p = torch.softmax((x @ K[:, h].T) / math.sqrt(D), -1)
            o = p @ V[:, h]
            out[b, h * g:(h + 1) * g] = o if rv is None else o @ rv.T
            if total is not None:
                total[b, h, :n] = p.sum(0)
        if total is not None:
            if cycle:
                total[b, :, :n] += kept[b, :, :n]
            else:
                gen = _gen(seed, 50_000 + b)
                total[b, :, :n] += torch.exp(2.0 * torch.randn(Hkv, n, generator=gen, device=DEV) - 3.0).double()
    res = {}
    if evicting:
        res = {"lens": torch.tensor([min(n, case["budget"]) for n in lens], dtype=torch.int32, device=DEV),
               "kept": kept, "pos": places}
    if step or case["kind"] == "evict":
        res["k"], res["v"] = torch.cat(ks), torch.cat(vs)
    if case["kind"] != "evict":
        res["out"] = out
        if total is not None:
            res["weights"] = total
    return res
