"""Eviction refuses arrays that it writes while other arguments of the call are read from
the same bytes (CPU: no call reaches a launch)."""
import ctypes

import pytest
import torch

import paper_2605_17757_amd as ok

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: for machines without a GPU")

B, Hkv, MP = 2, 8, 4
LAY = ok.Layout(Hkv, 10)
SLOTS = B * Hkv * MP * 64 * 4      # bytes of weights and of pos
SIZES = {"pages": ok.kv4_pool_bytes(LAY), "table": B * MP * 4, "lens": B * 4, "w": SLOTS, "wo": SLOTS, "p": SLOTS,
         "po": SLOTS, "seen": B * 4, "new": B * 4, "ws": ok.kv4_evict_workspace_bytes(LAY, B, MP)}
AT = {name: (i + 1) << 24 for i, name in enumerate(SIZES)}     # addresses far apart, never dereferenced
WRITTEN = ("pages", "wo", "po", "new", "ws")
IN_PLACE = {("wo", "w"), ("po", "p")}


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    """A call that passes all checks of its arrays ends at the checks of indices, whose copy
    of the made-up addresses the runtime refuses."""
    monkeypatch.setenv("OSCAR_DEBUG", "1")


def call(**at):
    a = {**AT, **at}
    p = {k: ctypes.c_void_p(v) for k, v in a.items()}
    return ok.lib().oscar_kv4_evict(ctypes.byref(LAY), p["pages"], B, p["table"], MP, p["lens"], p["w"], p["wo"],
                                    p["p"], p["po"], p["seen"], 64, 4, 16, p["new"], p["ws"], SIZES["ws"], None)


PAIRS = [(a, b) for a in WRITTEN for b in SIZES if a != b and not (b in WRITTEN and b < a)]


@pytest.mark.parametrize("a,b", PAIRS, ids=["%s-%s" % x for x in PAIRS])
def test_shared_bytes_are_refused(a, b):
    """The written array `a` begins with b's first bytes, holds its last ones, or ends with its first."""
    align = 256 if "ws" in (a, b) else 16
    last = (SIZES[b] - 1) // align * align       # aligned, inside b
    for d in {0, last, -((SIZES[a] - 1) // align * align)}:
        if d == 0 and (a, b) in IN_PLACE:
            continue
        assert call(**{a: AT[b] + d}) == ok.ERR_INVALID_ARG, (a, b, d)


def test_lengths_over_the_tokens_so_far():
    """new_lens in num_seen's place: written by one block while others read num_seen."""
    assert call(new=AT["seen"]) == ok.ERR_INVALID_ARG
    assert call(new=AT["seen"] + 4) == ok.ERR_INVALID_ARG
    assert call(new=AT["seen"] - 4) == ok.ERR_INVALID_ARG
