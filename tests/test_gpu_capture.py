"""GPU tests of calls that change a pool while a graph is being captured: refused
where the graph's stream is theirs or the previous plan's, and harmless to a
capture on any other stream."""
import ctypes as C
import random

import pytest
import torch

import paper_2607_02640_amd as mtn
from paper_2607_02640_amd import _lib
from tests._gpu_util import Harness
from tests.test_gpu_pages import _code, _frames, _harness

pytestmark = pytest.mark.gpu


def _captured(stream, inside):
    """What `inside` returns while `stream` captures x += 1, and whether three
    replays, with other work between them, then give 3."""
    x, g = torch.zeros(100, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=stream):
        x += 1
        got = inside()
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        torch.randn(1000, device="cuda").sum()
    return got, bool((x == 3).all())


def _set_rope(pool, layout):
    """mtn_pool_set_rope itself, without the wrapper's look at the current stream."""
    cfg = _lib.RopeConfig(layout, 0, 0, 0, 0.0, 0.0, 0.0, 0.0)
    return pool.lib.mtn_pool_set_rope(pool.h, C.byref(cfg))


def _sessions(pool, rope):
    """Two new sessions of a pool of `_harness` that holds no other."""
    h = Harness(pool, n_sessions=2, n_layers=2, hq=8, hkv=1, d=128, S=4, W=40, dtype="bf16", seed=7)
    for o in h.orc:
        o.rope = rope
    return h


@pytest.mark.parametrize("used", [False, True])
def test_set_rope_while_another_stream_is_captured(used):
    """A pool that never used the captured stream takes the form at once, and the
    capture goes on; the wrapper, whose stream is the captured one, refuses."""
    h, rnd = _harness("bf16", 8, 1, 128, n=0), random.Random(1)
    h.pool.set_rope()
    if used:  # the previous plan ran on the default stream
        sid = h.pool.session_open()
        h.pool.plan_begin([sid], [1])
        h.pool.plan_abort()
        h.pool.session_close(sid)
    got, whole = _captured(torch.cuda.Stream(), lambda: (
        _code(lambda: h.pool.set_rope(layout="interleaved")), _set_rope(h.pool, 1)))
    assert got == (mtn.MTN_ERR_BAD_STATE, mtn.MTN_OK) and whole
    _frames(_sessions(h.pool, dict(layout="interleaved")), rnd, 3)


def test_refused_while_the_previous_plans_stream_is_captured():
    h, rnd, side, other = _harness("bf16", 8, 1, 128), random.Random(2), torch.cuda.Stream(), torch.cuda.Stream()
    kv = torch.empty_like(h.pool.kv)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _frames(h, rnd, 2)
    before = h.pool.stats()

    def inside():
        with torch.cuda.stream(other):
            return (_code(lambda: h.pool.session_fork(h.sids[0])),
                    _code(lambda: h.pool.resize(h.pool.cfg.n_blocks, kv)))
    got, whole = _captured(side, inside)
    assert got == (mtn.MTN_ERR_BAD_STATE,) * 2 and whole and h.pool.stats() == before
    for sid in h.sids:
        h.pool.session_close(sid)
    got, whole = _captured(side, lambda: _set_rope(h.pool, 1))
    assert got == mtn.MTN_ERR_BAD_STATE and whole
    _frames(_sessions(h.pool, None), rnd, 3)  # the form is the one before
