"""CPU tests of the norms of queries and keys (mtn_pool_set_qk_norm): the oracle's
norm against closed forms, and the calls that are refused."""
import math

import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from oracle import windowed_attention as wa


def _pool(layers=2, d=64):
    return mtn.Pool(n_layers=layers, n_q_heads=4, n_kv_heads=2, head_dim=d, n_sink=4, window=32, max_chunk=8,
                    max_sessions=2, n_blocks=8, dtype="bf16", host_only=True)


def _code(fn, *a, **kw):
    try:
        fn(*a, **kw)
        return mtn.MTN_OK
    except mtn.MtnError as e:
        return e.code


def test_oracle_norm_closed_forms():
    d, w = 64, np.linspace(0.5, 2.0, 64)
    # a row of equal magnitudes c: sign(x) w c / sqrt(c^2 + eps)
    x = np.where(np.arange(d) % 3 == 0, -2.0, 2.0)
    assert np.allclose(wa.rms_norm(x, w, 1e-6), np.sign(x) * w * 2.0 / math.sqrt(4.0 + 1e-6), rtol=1e-15)
    # one element: sqrt(D) w there, 0 elsewhere; zero rows stay zero
    y = wa.rms_norm(np.eye(d)[5] * 7.0, w, 1e-30)
    assert abs(y[5] - w[5] * math.sqrt(d)) < 1e-13 and not np.delete(y, 5).any()
    assert not wa.rms_norm(np.zeros(d), w, 1e-6).any()
    # independent of the row's scale where eps is small against it
    r = np.random.default_rng(0).standard_normal(d)
    assert np.allclose(wa.rms_norm(r, w, 1e-300), wa.rms_norm(1e9 * r, w, 1e-300), rtol=1e-14)


def test_oracle_session_norms_before_it_rotates():
    """One key, one query, no window effects: the score is that of normed, rotated rows."""
    rng, d = np.random.default_rng(1), 16
    s = wa.OracleSession(1, 1, d, 0, 8, n_layers=1)
    wq, wk = rng.uniform(0.5, 1.5, (1, d)), rng.uniform(0.5, 1.5, (1, d))
    s.qk_norm = (wq, wk, 1e-6)
    q, k, v = (rng.standard_normal((3, 1, d)) for _ in range(3))
    _, lse = s.step(q, k, v)
    norm = lambda x, w: x / math.sqrt((x * x).sum() / d + 1e-6) * w
    want = [wa.rope_rotate(norm(q[2, 0], wq[0]), 2, 1e4) @ wa.rope_rotate(norm(k[j, 0], wk[0]), j, 1e4)
            for j in range(3)]
    assert abs(lse[2, 0] - np.logaddexp.reduce(np.array(want) / math.sqrt(d))) < 1e-12


@pytest.mark.parametrize("eps", [0.0, -1e-6, float("nan"), float("inf"), 1.5, 1e-39])
def test_eps_outside_its_range_is_refused(eps):
    assert _code(_pool().set_qk_norm, eps=eps) == mtn.MTN_ERR_INVALID_ARG


@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-6, 1.0])
def test_eps_of_its_range_is_taken(eps):
    assert _code(_pool().set_qk_norm, eps=eps) == mtn.MTN_OK


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_weights_that_are_not_finite_are_refused(bad):
    w = torch.ones(2, 64)
    w[1, 63] = bad
    for kw in (dict(q_weight=w), dict(k_weight=w)):
        assert _code(_pool().set_qk_norm, **kw) == mtn.MTN_ERR_INVALID_ARG


def test_weights_of_another_size_are_refused():
    for w in (torch.ones(64), torch.ones(3, 64), [[1.0] * 64], np.ones((2, 63))):
        assert _code(_pool().set_qk_norm, q_weight=w) == mtn.MTN_ERR_INVALID_ARG
    assert _code(_pool().set_qk_norm, q_weight=[[1.0] * 64] * 2, k_weight=np.ones((2, 64))) == mtn.MTN_OK


def test_only_without_open_plans_and_tokens():
    pool = _pool()
    sid = pool.session_open()
    assert _code(pool.set_qk_norm) == mtn.MTN_OK       # a session without tokens is none
    pool.plan_begin([sid], [3])
    for fn in (pool.set_qk_norm, pool.clear_qk_norm):
        assert _code(fn) == mtn.MTN_ERR_BAD_STATE
    pool.plan_commit()
    for fn in (pool.set_qk_norm, pool.clear_qk_norm):
        assert _code(fn) == mtn.MTN_ERR_BAD_STATE
    pool.session_close(sid)
    for fn in (pool.clear_qk_norm, pool.set_qk_norm, pool.set_rope):
        assert _code(fn) == mtn.MTN_OK
