"""CPU tests of the rules that lay out the linear layers' work (mtn_linear.h)."""
import random

import pytest

from tests._linear_rules import Rules

SEG_UNITS, MAX_SEG, TILE = 3, 1024, 64  # kLinSegUnits, kLinMaxSeg, kLinTile


@pytest.fixture(scope="module")
def rules():
    r = Rules()
    yield r
    r.close()


@pytest.mark.parametrize("n_cu", [1, 7, 64, 256, 304, 2048])
def test_segments_fit_their_workspace_and_items(rules, n_cu):
    rnd, plans = random.Random(n_cu), []
    for _ in range(400):
        hkv = rnd.choice([1, 2, 3, 4, 8, 32, 64, 255, 256])
        hq = hkv * rnd.choice([1, 2, 4, 8])
        n_seq = rnd.randint(1, max(1, min(300, n_cu // hkv + 1)))
        top = rnd.choice([1, 2, 65, 130, 1000, 9000, 100000])
        plans.append((n_cu, 1, hq, hkv, 128, [rnd.randint(1, top) for _ in range(n_seq)]))
    cut = 0
    for (_, _, hq, hkv, _, n), (length, items, _) in zip(plans, rules.ask(plans)):
        assert (length == 0) == (len(n) * hkv >= n_cu)
        if length:
            assert length % TILE == 0 and length >= 2 * TILE
            assert items * hkv < SEG_UNITS * n_cu and items <= len(n) + MAX_SEG
            cut += items > len(n)
    assert cut > 20 or n_cu < 64
