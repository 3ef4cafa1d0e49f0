"""CPU tests of the page operations' bookkeeping (host-only pools): fork and
resize against the independent index model among random plans, their refusals,
and that an error changes nothing."""
import random

import pytest

import paper_2607_02640_amd as mtn
from oracle import index_model as im


def _pair(n_blocks, S, W, cmax, max_sessions, max_len=None, dtype="f32"):
    pool = mtn.Pool(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, n_sink=S, window=W,
                    max_chunk=cmax, max_sessions=max_sessions, n_blocks=n_blocks, dtype=dtype,
                    max_len=max_len or 0, host_only=True)
    return pool, im.IndexModel(n_blocks, 16, S, W, cmax, max_sessions, max_len=max_len)


def _code(fn, *a):
    try:
        return 0, fn(*a)
    except (mtn.MtnError, im.IndexError_) as e:
        return e.code, None


def _compare(pool, model):
    st = pool.stats()
    assert st["capacity"] == model.n_blocks
    assert st["assigned"] == model.assigned()
    assert st["reserved"] == model.reserved_blocks()
    assert st["open_sessions"] == len(model.sessions)
    for sid, s in model.sessions.items():
        assert pool.block_table(sid) == model.block_table(sid)
        assert pool.session_info(sid) == (s.length, sum(b >= 0 for b in s.row))


@pytest.mark.parametrize("policy", ["windowed", "unbounded"])
@pytest.mark.parametrize("seed", range(8))
def test_fork_and_resize_match_the_index_model(policy, seed):
    rnd = random.Random(100 * seed + len(policy))
    S = rnd.choice([0, 1, 4, 16, 20, 33])
    W = None if policy == "unbounded" else rnd.choice([1, 5, 16, 33, 64])
    cmax = rnd.choice([1, 3, 25, 40])
    pool, model = _pair(rnd.choice([30, 60, 90]), S, W, cmax, 6, rnd.choice([40, 100]) if W is None else None)
    for _ in range(200):
        op, sids = rnd.random(), list(model.sessions)
        if op < 0.15:
            got, want = _code(pool.session_open), _code(model.open)
        elif op < 0.25 and sids:
            sid = rnd.choice(sids)
            got, want = _code(pool.session_close, sid), _code(model.close, sid)
        elif op < 0.45:
            sid, n = rnd.choice(sids + [5]), rnd.choice([1, 1, 2, 3, 0])
            got, want = _code(pool.session_fork, sid, n), _code(model.fork, sid, n)
        elif op < 0.55:
            n = rnd.choice([0, 12, 25, 40, 60, 90])
            got, want = (_code(f, n)[0] for f in (pool.resize, model.resize))
        elif sids:
            pick = rnd.sample(sids, rnd.randint(1, len(sids)))
            nt = [rnd.randint(1, cmax) for _ in pick]
            got, want = _code(pool.plan_begin, pick, nt), _code(model.plan_begin, pick, nt)
            if not got[0]:
                end = rnd.choice(["plan_commit", "plan_commit", "plan_abort"])
                getattr(pool, end)()
                getattr(model, end)()
        else:
            continue
        assert got == want
        _compare(pool, model)


def test_refusals_change_nothing():
    pool, model = _pair(12, 4, 32, 8, 4)  # rows of 4 blocks: three sessions fit
    lib = mtn.load()
    a = pool.session_open()
    model.open()
    pool.plan_begin([a], [8])
    for call in (lambda: pool.session_fork(a), lambda: pool.resize(20)):
        with pytest.raises(mtn.MtnError) as e:
            call()
        assert e.value.code == mtn.MTN_ERR_BAD_STATE
    pool.plan_commit()
    model.plan_begin([a], [8])
    model.plan_commit()
    for call, code in [(lambda: pool.session_fork(a, 0), mtn.MTN_ERR_INVALID_ARG),
                       (lambda: pool.session_fork(a, -1), mtn.MTN_ERR_INVALID_ARG),
                       (lambda: pool.session_fork(3), mtn.MTN_ERR_BAD_SESSION),
                       (lambda: pool.session_fork(-1), mtn.MTN_ERR_BAD_SESSION),
                       (lambda: pool.session_fork(9), mtn.MTN_ERR_BAD_SESSION),
                       (lambda: pool.session_fork(a, 4), mtn.MTN_ERR_NO_SESSION_SLOT),
                       (lambda: pool.session_fork(a, 3), mtn.MTN_ERR_POOL_EXHAUSTED),
                       (lambda: pool.resize(0), mtn.MTN_ERR_INVALID_ARG),
                       (lambda: pool.resize(-5), mtn.MTN_ERR_INVALID_ARG),
                       (lambda: pool.resize(1 << 31), mtn.MTN_ERR_INVALID_ARG),
                       (lambda: pool.resize(3), mtn.MTN_ERR_POOL_EXHAUSTED)]:
        with pytest.raises(mtn.MtnError) as e:
            call()
        assert e.value.code == code
        _compare(pool, model)
    assert lib.mtn_session_fork(pool.h, a, 1, None, None) == mtn.MTN_ERR_INVALID_ARG
    assert lib.mtn_session_fork(None, a, 1, None, None) == mtn.MTN_ERR_INVALID_ARG
    assert lib.mtn_pool_resize(None, 1, None, 0, None) == mtn.MTN_ERR_INVALID_ARG
    _compare(pool, model)


def test_a_failed_launch_changes_nothing():
    pool, model = _pair(40, 4, 32, 8, 4)
    sid = pool.session_open()
    model.open()
    for _ in range(6):
        for p in (pool, model):
            p.plan_begin([sid], [8])
            p.plan_commit()
    for call in (lambda: pool.session_fork(sid, 2), lambda: pool.resize(20)):
        pool.inject_failure(0)
        with pytest.raises(mtn.MtnError) as e:
            call()
        assert e.value.code == mtn.MTN_ERR_DEVICE
        _compare(pool, model)
    assert pool.session_fork(sid, 2) == model.fork(sid, 2)
    pool.resize(20)
    model.resize(20)
    _compare(pool, model)


def test_an_empty_session_forks_into_empty_ones():
    pool, model = _pair(40, 4, 32, 8, 4)
    assert pool.session_open() == model.open()
    assert pool.session_fork(0, 2) == model.fork(0, 2) == [1, 2]
    _compare(pool, model)
