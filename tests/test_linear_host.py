"""CPU tests of the linear layers: the oracle's recurrence against other forms of the
same sums, and the calls that are refused."""
import math

import numpy as np
import pytest

import paper_2607_02640_amd as mtn
from oracle.linear_attention import LinearState, all_pairs


def _pool(max_sessions=2):
    return mtn.Pool(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, n_sink=4, window=32, max_chunk=8,
                    max_sessions=max_sessions, n_blocks=16, dtype="bf16", host_only=True)


GOOD = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, log_decay=[[-0.1, 0.0]] * 2)


def _code(fn, *a, **kw):
    try:
        fn(*a, **kw)
        return mtn.MTN_OK
    except mtn.MtnError as e:
        return e.code


def test_oracle_recurrence_is_the_sum_over_all_pairs():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((11, 4, 8)), rng.standard_normal((11, 2, 8)), rng.standard_normal((11, 2, 8))
    a = np.array([-0.3, 0.0])
    s = LinearState(4, 2, 8, a)
    parts = [s.step(q[i:j], k[i:j], v[i:j])[0] for i, j in ((0, 4), (4, 5), (5, 11))]
    assert np.allclose(np.concatenate(parts), all_pairs(q, k, v, a, 1 / math.sqrt(8)), atol=1e-13)


def test_oracle_closed_forms():
    # orthonormal keys without decay: o_t = scale (q . k_j) v_j picks value j
    d = 8
    s = LinearState(1, 1, d, [0.0], scale=1.0)
    v = np.arange(d * d, dtype=np.float64).reshape(d, 1, d)
    s.step(np.zeros((d, 1, d)), np.eye(d)[:, None], v)
    assert np.array_equal(s.S[0], v[:, 0].T)
    # one key over and over: a geometric series
    s, lam = LinearState(1, 1, d, [math.log(0.5)], scale=1.0), 0.5
    one = np.zeros((5, 1, d))
    one[..., 0] = 1.0
    out, mag = s.step(one, one, one)
    assert np.allclose(out[:, 0, 0], [sum(lam ** j for j in range(i + 1)) for i in range(5)])
    assert np.array_equal(out, mag)


@pytest.mark.parametrize("change,code", [
    (dict(n_layers=0, log_decay=[]), mtn.MTN_ERR_INVALID_ARG),
    (dict(n_layers=-1, log_decay=[]), mtn.MTN_ERR_INVALID_ARG),
    (dict(n_kv_heads=0, log_decay=[]), mtn.MTN_ERR_INVALID_ARG),
    (dict(n_q_heads=7), mtn.MTN_ERR_INVALID_ARG),
    (dict(n_q_heads=6), mtn.MTN_ERR_UNSUPPORTED),      # groups of three
    (dict(n_q_heads=32), mtn.MTN_ERR_UNSUPPORTED),     # groups of sixteen
    (dict(head_dim=96), mtn.MTN_ERR_UNSUPPORTED),
    (dict(dtype="fp8"), mtn.MTN_ERR_UNSUPPORTED),
    (dict(scale=-1.0), mtn.MTN_ERR_INVALID_ARG),
    (dict(scale=float("nan")), mtn.MTN_ERR_INVALID_ARG),
    (dict(scale=float("inf")), mtn.MTN_ERR_INVALID_ARG),
    (dict(log_decay=[[0.1, 0.0]] * 2), mtn.MTN_ERR_INVALID_ARG),
    (dict(log_decay=[[float("nan"), 0.0]] * 2), mtn.MTN_ERR_INVALID_ARG),
    (dict(log_decay=[[0.0, -float("inf")]] * 2), mtn.MTN_ERR_INVALID_ARG),
    (dict(log_decay=[[0.0, 0.0]]), mtn.MTN_ERR_INVALID_ARG),
    (dict(n_layers=5000, log_decay=np.zeros((5000, 2))), mtn.MTN_ERR_UNSUPPORTED),
])
def test_refused_configurations(change, code):
    pool = _pool()
    assert _code(pool.set_linear, **{**GOOD, **change}) == code
    assert _code(pool.state_slot, pool.session_open()) == mtn.MTN_ERR_BAD_STATE  # nothing was set


def test_required_bytes():
    pool, n = _pool(3), mtn._lib.C.c_size_t()
    cfg = mtn._lib.LinearConfig(2, 8, 2, 64, 1, 0.0, None)
    assert pool.lib.mtn_linear_required_bytes(pool.h, mtn._lib.C.byref(cfg), mtn._lib.C.byref(n)) == 0
    assert n.value == 3 * 2 * 2 * 2 * 64 * 64 * 4


def test_only_without_open_plans_and_tokens():
    pool = _pool()
    sid = pool.session_open()
    assert _code(pool.set_linear, **GOOD) == mtn.MTN_OK
    pool.plan_begin([sid], [3])
    assert _code(pool.set_linear, **GOOD) == _code(pool.clear_linear) == mtn.MTN_ERR_BAD_STATE
    pool.plan_commit()
    assert _code(pool.set_linear, **GOOD) == _code(pool.clear_linear) == mtn.MTN_ERR_BAD_STATE
    pool.session_close(sid)
    assert _code(pool.clear_linear) == mtn.MTN_OK


def test_slots_turn_with_commits_alone():
    pool = _pool()
    pool.set_linear(**GOOD)
    a, b = pool.session_open(), pool.session_open()
    assert pool.state_slot(a) == pool.state_slot(b) == 0
    pool.plan_begin([a], [3])
    assert pool.state_slot(a) == 0
    pool.plan_abort()
    assert pool.state_slot(a) == 0
    pool.plan_begin([a], [3])
    pool.plan_commit()
    assert (pool.state_slot(a), pool.state_slot(b)) == (1, 0)
    pool.plan_begin([b, a], [1, 1])
    pool.plan_commit()
    assert (pool.state_slot(a), pool.state_slot(b)) == (0, 1)
    pool.session_close(a)
    c = pool.session_fork(b)[0]
    assert c == a and pool.state_slot(c) == pool.state_slot(b) == 1
    pool.session_close(b)
    assert _code(pool.state_slot, b) == mtn.MTN_ERR_BAD_SESSION
    assert pool.session_open() == b and pool.state_slot(b) == 0


def test_frame_step_is_refused():
    pool = _pool()
    pool.set_linear(**GOOD)
    sid = pool.session_open()
    assert _code(pool.frame_step, [sid], [2], [1], None, None, None, None) == mtn.MTN_ERR_BAD_STATE
    assert pool.session_info(sid)[0] == 0
    pool.clear_linear()
    assert _code(pool.frame_step, [sid], [2], [1], None, None, None, None) == mtn.MTN_OK


def test_attend_on_a_host_only_pool_is_refused():
    pool = _pool()
    pool.set_linear(**GOOD)
    sid = pool.session_open()
    pool.plan_begin([sid], [1])
    assert pool.lib.mtn_attend_linear(pool.h, 0, None, None, None, None, None) == mtn.MTN_ERR_BAD_STATE


def test_a_failed_fork_launch_takes_the_copies_back():
    pool = _pool(3)
    pool.set_linear(**GOOD)
    sid = pool.session_open()
    pool.plan_begin([sid], [3])
    pool.plan_commit()
    before = pool.stats()
    for launch in range(3):  # before the first work, the pages' launch, the states'
        pool.inject_failure(launch)
        assert _code(pool.session_fork, sid, 2) == mtn.MTN_ERR_DEVICE
        assert pool.stats() == before
    assert pool.session_fork(sid, 2) == [1, 2]
