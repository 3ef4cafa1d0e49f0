"""CPU tests (host-only pools) of forks and resizes that fail at any of their
launches: tables, counters and free blocks are as before, and later calls go on
as the independent index model does."""
import random

import pytest

import paper_2607_02640_amd as mtn
from tests.test_pages_host import _compare, _pair


def _refused(call):
    with pytest.raises(mtn.MtnError) as e:
        call()
    assert e.value.code == mtn.MTN_ERR_DEVICE


def _plan(pool, model, sids, n_tok):
    for p in (pool, model):
        p.plan_begin(sids, n_tok)
        p.plan_commit()


# launch points: one before any work; a fork's pages, then an int8 pool's tails; a
# resize's pages, tails, tables (pages and tables per 240 sessions, tails per 480)
@pytest.mark.parametrize("dtype,fork_points,resize_points", [("f32", 2, 3), ("int8", 3, 4)])
@pytest.mark.parametrize("W,max_len", [(32, None), (None, 90)])
def test_every_launch_point(dtype, fork_points, resize_points, W, max_len):
    pool, model = _pair(70, 4, W, 8, 7, max_len=max_len, dtype=dtype)
    sids = [pool.session_open() for _ in range(3)]
    assert sids == [model.open() for _ in range(3)]
    for _ in range(7):
        _plan(pool, model, sids, [8, 5, 3])  # open blocks in all of them at the end
    pool.session_close(1)
    model.close(1)
    for name, points, args in (("fork", fork_points, (2, 3)), ("resize", resize_points, (50,))):
        call = {"fork": pool.session_fork, "resize": pool.resize}[name]
        for at in range(points):
            pool.inject_failure(at)
            _refused(lambda: call(*args))
            _compare(pool, model)
            _plan(pool, model, [0, 2], [1, 1])
            _compare(pool, model)
        pool.inject_failure(points)  # one past the last: not met
        got, want = call(*args), getattr(model, name)(*args)
        assert name == "resize" or got == want
        pool.inject_failure(-1)
        _compare(pool, model)
        _plan(pool, model, [0, 1, 2, 3], [3, 8, 1, 2])
        _compare(pool, model)


@pytest.mark.parametrize("dtype,points", [("f32", 5), ("int8", 6)])
def test_launches_of_many_sessions(dtype, points):
    pool, model = _pair(2000, 3, 40, 20, 300, dtype=dtype)
    sids = [pool.session_open() for _ in range(300)]
    assert sids == [model.open() for _ in range(300)]
    for turn in range(3):
        _plan(pool, model, sids, [1 + (7 * s + turn) % 20 for s in sids])
    for s in sids[::11]:
        pool.session_close(s)
        model.close(s)
    for at in range(points):
        pool.inject_failure(at)
        _refused(lambda: pool.resize(1900))
        _compare(pool, model)
    pool.inject_failure(points)
    pool.resize(1900)
    model.resize(1900)
    _compare(pool, model)


@pytest.mark.parametrize("seed", range(4))
def test_int8_pools_match_the_index_model(seed):
    """Random opens, closes, forks, resizes and plans of an int8 pool, one in
    three of the page operations failing at a launch."""
    rnd = random.Random(seed)
    S, W, cmax = rnd.choice([0, 4, 20]), rnd.choice([5, 33]), rnd.choice([3, 25])
    pool, model = _pair(60, S, W, cmax, 6, dtype="int8")
    for _ in range(150):
        op, sids = rnd.random(), list(model.sessions)
        room = (len(sids) + 1) * (-(-S // 16) + -(-(W + cmax - 1) // 16)) <= model.n_blocks
        if op < 0.2 and len(sids) < 6 and room:
            assert pool.session_open() == model.open()
        elif op < 0.3 and sids:
            sid = rnd.choice(sids)
            pool.session_close(sid)
            model.close(sid)
        elif op < 0.5 and sids and len(sids) < 6 and room:
            sid = rnd.choice(sids)
            if rnd.random() < 0.33:
                pool.inject_failure(0)
                _refused(lambda: pool.session_fork(sid))
            else:
                assert pool.session_fork(sid) == model.fork(sid, 1)
        elif op < 0.6 and sids:
            if rnd.random() < 0.33:
                pool.inject_failure(0)
                _refused(lambda: pool.resize(70))
            else:
                n = rnd.choice([60, 75])
                pool.resize(n)
                model.resize(n)
        elif sids:
            _plan(pool, model, sids, [rnd.randint(1, cmax) for _ in sids])
        _compare(pool, model)
