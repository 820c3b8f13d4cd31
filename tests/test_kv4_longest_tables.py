"""The longest block tables that eviction takes (CPU: no call reaches a launch)."""
import ctypes

import pytest
import torch

import paper_2605_17757_amd as ok

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: for machines without a GPU")

LAY = ok.Layout(1, 10, group_size=128)


def call(mp, budget):
    at = [ctypes.c_void_p((i + 1) << 40) for i in range(10)]     # far apart, never dereferenced
    return ok.lib().oscar_kv4_evict(ctypes.byref(LAY), at[0], 1, at[1], mp, at[2], at[3], at[3], at[4], at[4], at[5],
                                    budget, 4, 16, at[6], at[7], 1 << 39, None)


@pytest.mark.parametrize("budget", (64, 2 ** 30 - 64, 2 ** 30 - 63, 2 ** 30 - 1))
def test_a_launch_holds_every_page_that_receives_rows(budget, monkeypatch):
    """2^24 pages of 256 threads are 2^32 in one launch, of which none would run: rows,
    weights and positions would disagree.  One page less is the longest table."""
    monkeypatch.setenv("OSCAR_DEBUG", "1")                       # the indices' copy fails before any launch
    assert call(1 << 24, budget) == ok.ERR_UNSUPPORTED
    assert ok.kv4_evict_workspace_bytes(LAY, 1, 1 << 24) == 0
    assert call((1 << 24) - 1, budget) == ok.ERR_HIP
    assert ok.kv4_evict_workspace_bytes(LAY, 1, (1 << 24) - 1) >= 2 ** 30
    # attention has no such launch
    assert ok.kv4_decode_workspace_bytes(LAY, 1, 1, 2, 1 << 24, True) >= 2 ** 32
