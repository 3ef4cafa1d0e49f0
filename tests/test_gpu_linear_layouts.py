"""GPU parity of the linear layers in the layouts that full batches and long prompts take:
chunk workgroups that walk several query heads, single-token workgroups that hold
half a state or a whole one (test_linear_rules.py holds which plans take which)."""
import numpy as np
import pytest
import torch

from tests._gpu_util import say
from tests._linear_rules import CHUNKS, N_CU, SINGLES
from tests._linear_util import Linear, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    n = torch.cuda.get_device_properties(0).multi_processor_count
    assert n == N_CU, f"the layouts are pinned for {N_CU} compute units, this device has {n}"


def _step(x, n_tok, some):
    """One plan of every session; the oracles of the sessions `some` follow."""
    rows = x.rows(sum(n_tok))
    x.plan(x.sids, n_tok)
    out = x.attend(*rows)
    x.pool.plan_commit()
    torch.cuda.synchronize()
    assert bool((out[:, -1] == 7.0).all()), "a row behind the last token was written"
    at = np.cumsum([0] + list(n_tok))
    for i in some:
        s, cut = x.sids[i], slice(at[i], at[i + 1])
        ref, mag = x.orc[s][0].step(*(f64(r[0, cut]) for r in rows))
        x.compare(out[0, cut], ref, mag, x.orc[s][0].length, f"session {s}")
        x.check_state(s)


def _name(case):
    return "-".join(str(c if not isinstance(c, list) else f"{len(c)}x{max(c)}") for c in case)


@pytest.mark.parametrize("case", CHUNKS, ids=_name)
def test_chunks_of_several_heads(case):
    """Fresh, then over a state, some sessions of each length range."""
    dtype, hq, hkv, d, n_tok, *_ = case
    n = len(n_tok)
    say(f"layout {_name(case)}")
    x = Linear(dtype, hq, hkv, d, n=n, cmax=max(n_tok), seed=hq + d)
    some = sorted({0, n // 2, n - 1} | ({int(np.argmin(n_tok)), int(np.argmax(n_tok))} if n > 3 else set(range(n))))
    _step(x, n_tok, some)
    if sum(n_tok) < 8000:
        _step(x, n_tok[::-1], some)
    say(f"  worst {x.worst:.3f} of the bound")


@pytest.mark.parametrize("dtype,hq,hkv,d,n,slices", SINGLES)
def test_single_tokens_of_full_batches(dtype, hq, hkv, d, n, slices):
    say(f"single tokens {dtype} {hq}/{hkv} D={d}, {n} sequences, {slices} slices")
    x = Linear(dtype, hq, hkv, d, n=n, seed=n + hq)
    for _ in range(3):
        _step(x, [1] * n, [0, 1, n // 2, n - 1])
    say(f"  worst {x.worst:.3f} of the bound")


@pytest.mark.parametrize("case", [c for c in CHUNKS if c[6] in (4, 8) and c[3] == 128 and len(c[4]) > 1], ids=_name)
def test_a_value_that_is_not_finite_stays_with_later_tokens_of_every_head(case):
    dtype, hq, hkv, d, n_tok, *_ = case
    g, n = hq // hkv, len(n_tok)
    s = int(np.argmax(n_tok))
    at = sum(n_tok[:s])
    outs, states, end = [], [], at + n_tok[s]
    bad = at + n_tok[s] // 2
    for value in (None, float("inf"), float("nan")):
        x = Linear(dtype, hq, hkv, d, n=n, cmax=max(n_tok), seed=3)
        q, k, v = x.rows(sum(n_tok))
        if value is not None:
            v[0, bad, 1, 70] = value
        x.plan(x.sids, n_tok)
        outs.append(x.attend(q, k, v)[0, :-1])
        x.pool.plan_commit()
        states.append(torch.stack([x.pool.session_state(i)[0] for i in x.sids]))
    keep = torch.ones_like(outs[0], dtype=torch.bool)
    keep[bad:end, g:2 * g, 70] = False
    same = torch.ones_like(states[0], dtype=torch.bool)
    same[s, 1, 70] = False
    assert torch.isfinite(outs[0]).all()
    for o, st in zip(outs[1:], states[1:]):
        assert torch.equal(o[keep], outs[0][keep]) and not torch.isfinite(o[~keep]).any()
        assert torch.equal(st[same], states[0][same]) and not torch.isfinite(st[~same]).any()
