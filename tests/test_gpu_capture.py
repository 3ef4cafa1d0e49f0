"""GPU tests of calls that change a pool while a graph is being captured: refused
where the graph's stream is the previous plan's."""
import random

import pytest
import torch

import paper_2607_02640_amd as mtn
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
    _frames(h, rnd, 2)
