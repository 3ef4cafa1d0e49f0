"""States of the linear layers over many plans, in every form that carries one on:
single tokens beside a chunk, short chunks, whole tiles, segments and their scan.

A decay that is rounded is off the same way plan after plan; roundings of the state
are not, for long: a piece of a plan (tile or segment) that takes the part
delta = 1 - lambda^m of an element of mantissa X, 2^23 <= X < 2^24, moves what is
rounded of it by X delta units, and that by X delta^2 from one plan to the next, so
the roundings come round once in 1 / (2^23 delta^2) =: L plans or sooner and are alike
for no longer.  r roundings by at most 2^-24 of an element, in runs of L alike (L at
least 1 and at most r), over M elements on their own: the mean relative error has a
standard deviation of 2^-24 sqrt(r L / (3 M)) at most (six are allowed).  A piece may
round an element twice.  Decays in two fp32 terms are off by 2^-48 a piece, the scan's
by its exponent's rounding in 64 bits, too: 2^-52 of 1.45 |a| a token."""
import numpy as np
import pytest
import torch

from tests._gpu_util import say
from tests._linear_util import TDT, Linear, f64

pytestmark = pytest.mark.gpu

# tokens of the checked session and of the one beside it (0: alone), plans, pieces of
# a plan at most, tokens of the shortest
PLANS = [(1, 2, 600, 1, 1), (2, 0, 400, 1, 2), (3, 1, 400, 1, 3), (4, 4, 400, 1, 4), (40, 5, 200, 2, 8),
         (64, 0, 200, 2, 32), (300, 0, 100, 8, 12)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("a", [-2.0 ** -14, -3e-5, -1.1e-6])
@pytest.mark.parametrize("n_tok,beside,plans,pieces,shortest", PLANS)
def test_states_decay_without_drift(dtype, a, n_tok, beside, plans, pieces, shortest):
    d = 64
    x = Linear(dtype, 1, 1, d, n=2, cmax=max(n_tok, 8), log_decay=[[a]])
    s, other = x.sids
    state = x.pool.session_state
    x.step([1], [s], check=False)
    state(s).copy_(torch.rand_like(state(s)) + 0.5)
    before = f64(state(s))[0, 0]
    sids, cuts = ([s, other], [n_tok, beside]) if beside else ([s], [n_tok])
    zero = [torch.zeros((1, sum(cuts), 1, d), dtype=TDT[dtype]) for _ in range(3)]
    for _ in range(plans):
        x.plan(sids, cuts)
        x.attend(*zero)
        x.pool.plan_commit()
    got = f64(state(s))[0, 0]
    n, r = plans * n_tok, 2 * plans * pieces
    rel = got / (before * np.exp(n * float(np.float32(a)))) - 1.0
    alike = np.clip(1 / (2 ** 23 * np.expm1(shortest * a) ** 2), 1, r)
    tol = 6 * 2.0 ** -24 * np.sqrt(r * alike / (3 * d * d)) + 2.0 ** -48 * plans * pieces + 2.0 ** -51 * n * abs(a)
    say(f"{dtype} a {a} {n_tok} tokens x {plans}: mean relative error {rel.mean():.2e}, {tol:.2e} allowed")
    assert abs(rel.mean()) <= tol
    assert np.abs(rel).max() <= r * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_tok,plans", [(2, 4000), (4, 2000)])
def test_a_steady_input_comes_to_its_state(dtype, n_tok, plans):
    """The same positive rows over and over: the state nears its end and moves by the part
    rho delta of itself a plan, rho = e^(-8000 2^-12) at the last.  What is rounded of it
    moves by X rho delta^2 units from one plan to the next (see above), runs of roundings
    alike are 1 / (2^23 rho delta^2) plans at most (one at least), and the relative
    error's rms is 2^-24 sqrt(plans L / 3) at most, were none of it decayed, plus 4 2^-24
    of rows, weights and products.  Elements share their rows, 64 of each: twice
    that is allowed."""
    a, d = -2.0 ** -12, 64
    x = Linear(dtype, 1, 1, d, log_decay=[[a]])
    k, v = ((torch.rand((1, 1, d)) + 0.5).to(TDT[dtype]) for _ in range(2))
    q, kk, vv = (t.expand(n_tok, 1, d).contiguous().cuda() for t in (torch.ones_like(k), k, v))
    out = torch.empty_like(q)
    for _ in range(plans):
        x.plan(x.sids, [n_tok])
        x.pool.attend_linear(0, q, kk, vv, out)
        x.pool.plan_commit()
    n = n_tok * plans
    ref = np.expm1(n * a) / np.expm1(a) * np.outer(f64(v).ravel(), f64(k).ravel())
    rel = f64(x.pool.session_state(x.sids[0]))[0, 0] / ref - 1.0
    alike = max(1.0, 1 / (2 ** 23 * np.exp(n * a) * np.expm1(n_tok * a) ** 2))
    tol = 2 * 2.0 ** -24 * (np.sqrt(plans * alike / 3) + 4)
    rms = np.sqrt(np.mean(rel ** 2))
    say(f"{dtype} {n_tok} tokens x {plans}: rms {rms * 2 ** 24:.1f} 2^-24, {tol * 2 ** 24:.1f} allowed")
    assert rms <= tol
