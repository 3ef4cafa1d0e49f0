"""GPU tests of fork and resize: copies and moved sessions go on exactly as the
float64 oracle's copies do, with every slot that no query may read poisoned,
and pages are copied bit for bit."""
import copy
import random

import pytest
import torch

import paper_2607_02640_amd as mtn
from tests._gpu_util import Harness, make_pool, say

pytestmark = pytest.mark.gpu

SHAPES = [("f32", 4, 2, 64), ("bf16", 8, 1, 128), ("bf16", 3, 3, 64), ("fp8", 8, 2, 128)]


def _harness(dtype, hq, hkv, d, W=40, S=4, n=2, room=6, layers=2, cmax=9, spare=3):
    ring = 64 if W is None else -(-(W + cmax - 1) // 16) + -(-S // 16)
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, cmax=cmax, max_sessions=room,
                     n_blocks=room * ring + spare, dtype=dtype, max_len=200 if W is None else 0)
    return Harness(pool, n_sessions=n, n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, dtype=dtype, seed=3)


def _code(call):
    """The error code of a refused call.  (Kept exceptions would keep the pool, in
    a cycle that a later test's collection frees, device synchronisation and all.)"""
    try:
        call()
    except mtn.MtnError as e:
        return e.code
    return mtn.MTN_OK


def _fork(h, i, copies, **kw):
    """Fork session i of the harness, oracle and generators with it; the copies'
    generators then draw other tokens."""
    for sid in h.pool.session_fork(h.sids[i], copies, **kw):
        h.sids.append(sid)
        h.orc.append(copy.deepcopy(h.orc[i]))
        h.rng.append(copy.deepcopy(h.rng[i]))
        h.rng[-1].standard_normal(7 * len(h.rng))


def _frames(h, rnd, n):
    for f in range(n):
        h.frame([rnd.randint(1, 9) for _ in h.sids], [rnd.randint(0, 2) for _ in h.sids],
                use_frame_step=f % 2 == 0, fused=True)


@pytest.mark.parametrize("W", [40, None])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_forked_sessions_go_on_apart(dtype, hq, hkv, d, W):
    h, rnd = _harness(dtype, hq, hkv, d, W=W), random.Random(1)
    _fork(h, 1, 1)  # empty
    _frames(h, rnd, 3)
    _fork(h, 0, 2)  # mid-window, copies of one source
    h.pool.poison_dead()
    _frames(h, rnd, 4)
    _fork(h, 3, 1)  # a copy of a copy, windows wrapped
    h.pool.poison_dead()
    _frames(h, rnd, 3)
    say(f"{dtype} W={W}: max err {h.max_err:.2e}")


@pytest.mark.parametrize("W", [40, None])
@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_resized_pools_go_on(dtype, hq, hkv, d, W):
    h, rnd = _harness(dtype, hq, hkv, d, W=W, n=3), random.Random(2)
    _frames(h, rnd, 3)
    h.pool.session_close(h.sids.pop(1))  # holes
    del h.orc[1], h.rng[1]
    _frames(h, rnd, 1)
    for blocks in (max(h.pool.stats()["reserved"] + (8 if W is None else 0), 1), 64, 30):
        kw = {k: getattr(h.pool.cfg, k) for k in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim",
                                                  "n_sink", "max_chunk", "max_sessions", "max_len")}
        need = mtn.Pool.required(**kw, window=W, n_blocks=blocks, dtype=dtype)
        old, kv = h.pool.kv, torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        h.pool.resize(blocks, kv)
        old.fill_(0xFF)  # NaN in every type
        assert h.pool.kv is kv and h.pool.stats()["capacity"] == blocks and h.pool.required_bytes == need
        h.pool.poison_dead()
        _frames(h, rnd, 2)
    say(f"{dtype} W={W}: max err {h.max_err:.2e}")


@pytest.mark.parametrize("hkv,d,layers,tokens", [(1, 64, 1, 1), (2, 64, 3, 250), (3, 128, 2, 700), (8, 128, 1, 90)])
def test_pages_are_copied_whole(hkv, d, layers, tokens):
    """Blocks of 4, 8, 24 and 64 KiB, from one to many: every byte of every page
    arrives, every other byte of the pool stays."""
    copies, per = 33, -(-tokens // 16)
    pool = make_pool(n_layers=layers, hq=hkv, hkv=hkv, d=d, S=0, W=None, cmax=64, max_sessions=copies + 1,
                     n_blocks=per * (copies + 1) + 2, dtype="bf16", max_len=tokens)
    sid, done = pool.session_open(), 0
    rows = torch.zeros((64, hkv, d), dtype=torch.bfloat16, device="cuda")
    while done < tokens:
        n = min(64, tokens - done)
        pool.plan_begin([sid], [n])
        for l in range(layers):
            pool.frame_append_kv(l, rows, rows)
        pool.plan_commit()
        done += n
    pool.kv.copy_(torch.randint(0, 256, pool.kv.shape, dtype=torch.uint8, device="cuda"))
    want = pool.kv.clone()
    sids = pool.session_fork(sid, copies)
    pages = want.view(layers, pool.cfg.n_blocks, -1)
    src = [b for b in pool.block_table(sid) if b >= 0]
    for s in sids:
        dst = [b for b in pool.block_table(s) if b >= 0]
        assert len(dst) == len(src) == per
        pages[:, dst] = pages[:, src]
    assert torch.equal(pool.kv, want)
    kv = torch.randint(0, 256, (pool.required_bytes + 4 * pool.required_bytes // pool.cfg.n_blocks,),
                       dtype=torch.uint8, device="cuda")
    after, n_blocks = kv.clone(), pool.cfg.n_blocks + 4
    pool.session_close(sids[5])
    order = [b for s in [sid] + sids if s != sids[5] for b in pool.block_table(s) if b >= 0]
    pool.resize(n_blocks, kv)
    after.view(layers, n_blocks, -1)[:, :len(order)] = pages[:, order]
    assert torch.equal(kv, after)


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
def test_many_sessions_move(dtype):
    """More sessions than one launch's arguments hold, of different lengths, with
    holes between them: each returns after the move what it does before."""
    n, d = 300, 64
    kw = dict(n_layers=1, hq=2, hkv=1, d=d, S=3, W=40, cmax=20, max_sessions=n, dtype=dtype)
    pool = make_pool(**kw, n_blocks=5 * n)
    gen = torch.Generator(device="cuda").manual_seed(8)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    sids = [pool.session_open() for _ in range(n)]
    for turn in range(5):
        who = [s for s in sids if s % 5 <= turn]
        nt = [1 + (7 * s + turn) % 20 for s in who]
        pool.plan_begin(who, nt)
        pool.frame_append_kv(0, draw(sum(nt), 1, d), draw(sum(nt), 1, d))
        pool.plan_commit()
        if turn == 3:
            for s in sids[::11]:
                pool.session_close(s)
            sids = [s for s in sids if s % 11]
    k, v, q = draw(len(sids), 1, d), draw(len(sids), 1, d), draw(len(sids), 2, d)

    def answers():
        out = torch.empty_like(q)
        pool.plan_begin(sids, [1] * len(sids))
        pool.attend_decode_append(0, k, v, q, out)
        pool.plan_abort()  # asked again below
        return out
    want = answers()
    old, kv = pool.kv, torch.empty_like(pool.kv)
    pool.resize(pool.cfg.n_blocks, kv)
    old.fill_(0xFF)
    assert torch.equal(answers(), want)


def test_plans_and_page_operations_on_different_streams():
    """Each call waits for the work of the one before it, whatever its stream."""
    h, rnd = _harness("bf16", 8, 1, 128), random.Random(4)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        _frames(h, rnd, 3)
        torch.cuda._sleep(20_000_000)
        q = torch.randn((5, 8, 128), device="cuda").bfloat16()
        k, v = torch.randn((2, 5, 1, 128), device="cuda").bfloat16()
        h.pool.plan_begin([h.sids[0]], [5])
        for l in range(2):
            h.pool.frame_append_kv(l, k, v)
        h.pool.plan_commit()
    sid = h.pool.session_fork(h.sids[0], stream=two.cuda_stream)[0]  # while stream one sleeps
    outs = []
    for s in (h.sids[0], sid):  # on the default stream
        out = torch.empty_like(q)
        h.pool.plan_begin([s], [5])
        for l in range(2):
            h.pool.frame_append_kv(l, k, v)
        h.pool.attend_chunk_prefill(1, q, out)
        h.pool.plan_commit()
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0].float()).all())


def test_refused_while_a_graph_is_captured():
    h, rnd = _harness("bf16", 8, 1, 128), random.Random(5)
    _frames(h, rnd, 2)
    kv = torch.empty_like(h.pool.kv)
    torch.cuda.synchronize()
    before, g = h.pool.stats(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        codes = [_code(lambda: h.pool.session_fork(h.sids[0])),
                 _code(lambda: h.pool.resize(h.pool.cfg.n_blocks, kv))]
    assert codes == [mtn.MTN_ERR_BAD_STATE] * 2
    assert h.pool.stats() == before
    _frames(h, rnd, 2)


def test_bad_buffers_are_refused():
    h = _harness("f32", 4, 2, 64)
    n = h.pool.required_bytes
    for kv, blocks in [(None, h.pool.cfg.n_blocks), (h.pool.kv, h.pool.cfg.n_blocks),
                       (torch.empty(n - 256, dtype=torch.uint8, device="cuda"), h.pool.cfg.n_blocks),
                       (torch.empty(n, dtype=torch.uint8), h.pool.cfg.n_blocks),
                       (torch.empty(1, dtype=torch.uint8, device="cuda").expand(n), h.pool.cfg.n_blocks),
                       (torch.empty(n + 16, dtype=torch.uint8, device="cuda")[16:], h.pool.cfg.n_blocks)]:
        assert _code(lambda: h.pool.resize(blocks, kv)) == mtn.MTN_ERR_INVALID_ARG
    _frames(h, random.Random(6), 2)
