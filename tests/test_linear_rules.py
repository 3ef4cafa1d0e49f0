"""CPU tests of the rules that lay out the linear layers' work (mtn_linear.h)."""
import random

import pytest

from tests._linear_rules import CHUNKS, N_CU, SINGLES, Rules

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
    for (_, _, hq, hkv, _, n), (length, items, *_) in zip(plans, rules.ask(plans)):
        assert (length == 0) == (len(n) * hkv >= n_cu)
        if length:
            assert length % TILE == 0 and length >= 2 * TILE
            assert items * hkv < SEG_UNITS * n_cu and items <= len(n) + MAX_SEG
            cut += items > len(n)
    assert cut > 20 or n_cu < 64


def test_the_layouts_that_the_device_tests_are_made_for(rules):
    dt = {"f32": 0, "bf16": 1}
    got = rules.ask([(N_CU, dt[t], hq, hkv, d, n) for t, hq, hkv, d, n, *_ in CHUNKS])
    for case, (length, items, tile, heads, _) in zip(CHUNKS, got):
        assert (tile, heads, items > len(case[4])) == case[5:], case
    # every form with several heads, whole and cut, is among them
    assert {(c[0], c[3], c[5], c[6]) for c in CHUNKS} >= {(t, d, b, h) for t, b in (("bf16", 64), ("bf16", 32), ("f32", 32))
                                                          for d in (64, 128) for h in (2, 4, 8)}
    assert {(c[0], c[3]) for c in CHUNKS if c[7]} == {(t, d) for t in dt for d in (64, 128)}
    got = rules.ask([(N_CU, dt[t], hq, hkv, d, [1] * n) for t, hq, hkv, d, n, _ in SINGLES])
    for case, (*_, slices) in zip(SINGLES, got):
        assert slices == case[5], case
    assert {(c[3], c[5]) for c in SINGLES} == {(64, 1), (64, 2), (128, 1), (128, 2), (128, 4)}
