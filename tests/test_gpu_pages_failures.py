"""GPU tests of forks and resizes that fail between their launches (the failure is
forced on the host, before a launch): the sessions answer from the old pages as
before, whatever the launches before the failure wrote."""
import pytest
import torch

import paper_2607_02640_amd as mtn
from tests._gpu_util import make_pool
from tests.test_gpu_pages import _code

pytestmark = pytest.mark.gpu


def _many(dtype, n=260, d=64):
    """Sessions of many lengths (more than one launch of a move takes), and what
    they answer to one query each."""
    pool = make_pool(n_layers=2, hq=2, hkv=1, d=d, S=3, W=40, cmax=20, max_sessions=n + 3, n_blocks=5 * (n + 3),
                     dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(9)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    sids = [pool.session_open() for _ in range(n)]
    for turn in range(4):
        nt = [1 + (7 * s + turn) % 20 for s in sids]
        pool.plan_begin(sids, nt)
        k, v = draw(sum(nt), 1, d), draw(sum(nt), 1, d)
        for l in range(2):
            pool.frame_append_kv(l, k, v)
        pool.plan_commit()
    k, v, q = draw(n, 1, d), draw(n, 1, d), draw(n, 2, d)

    def answers(who=None):
        rows = list(range(n)) if who is None else [s for s, _ in who]
        ids = sids if who is None else [c for _, c in who]
        out = torch.empty_like(q[rows])
        pool.plan_begin(ids, [1] * len(ids))
        pool.attend_decode_append(1, k[rows].contiguous(), v[rows].contiguous(), q[rows].contiguous(), out)
        pool.plan_abort()
        return out
    return pool, answers


@pytest.mark.parametrize("dtype,points", [("bf16", 5), ("int8", 6)])
def test_a_move_that_fails_at_a_launch(dtype, points):
    pool, answers = _many(dtype)
    want = answers()
    for at in range(points):
        kv = torch.empty_like(pool.kv)
        pool.inject_failure(at)
        assert _code(lambda: pool.resize(pool.cfg.n_blocks, kv)) == mtn.MTN_ERR_DEVICE
        kv.fill_(0xFF)
        assert torch.equal(answers(), want), at
    pool.inject_failure(points)
    old, kv = pool.kv, torch.empty_like(pool.kv)
    pool.resize(pool.cfg.n_blocks, kv)
    pool.inject_failure(-1)
    old.fill_(0xFF)
    assert torch.equal(answers(), want)


@pytest.mark.parametrize("dtype,points", [("bf16", 2), ("int8", 3)])
def test_a_fork_that_fails_at_a_launch(dtype, points):
    pool, answers = _many(dtype)
    want, src = answers(), 7
    for at in range(points):
        pool.inject_failure(at)
        assert _code(lambda: pool.session_fork(src, 3)) == mtn.MTN_ERR_DEVICE
        assert torch.equal(answers(), want), at
    other = pool.session_open()  # takes blocks that the failed forks wrote
    copies = pool.session_fork(src, 2)
    assert torch.equal(answers(), want)
    for c in copies:
        assert torch.equal(answers([(src, c)]), want[[src]])
    pool.session_close(other)
