"""Every form of eviction's select at its own sizes and at their borders: keys of up to 4, 12
or 32 slots a thread in the registers of one block of 1024 threads (tables of up to 64, 192
and 512 pages), several blocks a row beyond."""
import numpy as np
import pytest

from test_kv4_evict import check, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mp", (17, 20, 40, 64,             # 4 slots a thread, 2 to 4 of them used
                                65, 97, 120, 192,           # 12: the first batch of six loads, and the second
                                193, 300, 512,              # 32
                                513))                       # several blocks
@pytest.mark.parametrize("kind", ("distinct", "ties", "evicted before"))
def test_slots_per_thread(mp, kind):
    n = mp * 64
    rng, lens, table, pool, weights, pos, lay = setup(mp, (n, n - 29, n // 2 + 1), 1, 128, mp=mp)
    seen = lens.copy()
    if kind == "ties":
        weights[:, :, : n // 3] = np.float32(0.7)            # over many waves
        weights[1] = np.where(rng.random(weights[1].shape) < 0.5, np.float32(2), np.float32(1))
    elif kind == "evicted before":
        seen += 777
        for b in range(3):
            old = int(lens[b]) - 50
            pos[b, 0, :old] = rng.permutation(int(seen[b]) - 50)[:old]
    budget = {"distinct": n // 3, "ties": n - 64, "evicted before": min(2048, n // 2)}[kind]
    check(lay, lens, table, pool, weights, pos, seen, budget, 4, 64, 128, in_place=(mp % 2 == 0,))


@pytest.mark.parametrize("mp", (40, 120, 300))
def test_budgets_of_one_and_all_but_one(mp):
    n = mp * 64
    for budget in (1, n - 1):
        rng, lens, table, pool, weights, pos, lay = setup(mp + 1, (n, n - 1), 2, 128, mp=mp)
        check(lay, lens, table, pool, weights, pos, lens, budget, 0, 0, 128, in_place=(True,))
