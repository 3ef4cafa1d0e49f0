"""The int8 cache, a scaled rotary form, forks and moves together, as a server
uses them; and offsets past 32 bits."""
import copy
import random

import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from tests._gpu_util import Harness, make_pool, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d", [("int8", 16, 2, 128), ("int8", 4, 4, 64), ("bf16", 16, 2, 128),
                                            ("fp8", 8, 2, 128), ("f32", 4, 2, 64)])
def test_a_serving_run(dtype, hq, hkv, d):
    """Calls come and go; one is forked to try two replies, the better of them
    goes on; the pool shrinks for the night and grows again."""
    rope = dict(layout="interleaved", rotary_dim=48, scaling="yarn", factor=4.0, original_len=64)
    S, W, cmax, room, layers = 4, 70, 24, 6, 2
    row = -(-(W + cmax - 1) // 16) + 1
    kw = dict(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_sink=S, window=W, max_chunk=cmax,
              max_sessions=room, dtype=dtype, rope_theta=1e4)
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, cmax=cmax, max_sessions=room,
                     n_blocks=room * row, dtype=dtype)
    pool.set_rope(**rope)
    h = Harness(pool, n_sessions=3, n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, dtype=dtype, seed=11)
    for o in h.orc:
        o.rope = rope
    rnd = random.Random(d + hq)

    def frames(n):
        for f in range(n):
            pool.poison_dead()
            h.frame([rnd.randint(1, cmax) for _ in h.sids], [rnd.randint(0, 4) for _ in h.sids],
                    use_frame_step=f % 2 == 0, fused=True)

    def hang_up(i):
        pool.session_close(h.sids.pop(i))
        del h.orc[i], h.rng[i]

    def move(blocks):
        old = pool.kv
        pool.resize(blocks, torch.empty(mtn.Pool.required(**kw, n_blocks=blocks), dtype=torch.uint8, device="cuda"))
        old.fill_(0xFF)

    frames(3)
    for sid in pool.session_fork(h.sids[2], 2):
        h.sids.append(sid)
        h.orc.append(copy.deepcopy(h.orc[2]))
        h.rng.append(np.random.default_rng(sid))
    frames(2)
    hang_up(2)
    hang_up(3)
    move(3 * row)
    with pytest.raises(mtn.MtnError):
        pool.session_open()
    frames(3)
    move(room * row + 5)
    frames(1)
    k, v = torch.randn((2, 2 * cmax, hkv, d), device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    pool.plan_begin(h.sids[:2], [cmax, cmax])  # a frame that is abandoned half way
    pool.frame_append_kv(0, k, v)
    pool.plan_abort()
    frames(3)
    say(f"{dtype}: max err {h.max_err:.2e}, rms {h.rms_err():.2e}")


@pytest.mark.parametrize("dtype", ["int8", "bf16"])
def test_layers_past_four_gigabytes(dtype):
    """The last layer's blocks (and an int8 pool's tails behind them) lie past 2^32
    bytes; given the first layer's rows it holds and returns the same."""
    layers, blocks, hkv, d = 40, 8000 if dtype == "int8" else 4000, 4, 128
    kw = dict(n_layers=layers, hq=16, hkv=hkv, d=d, S=4, W=100, cmax=40, max_sessions=3, n_blocks=blocks, dtype=dtype)
    pool = make_pool(**kw)
    assert pool.required_bytes // layers * (layers - 1) > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(6)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    sids = [pool.session_open()]
    for turn in range(6):
        if turn == 4:
            sids += pool.session_fork(sids[0])
        if turn == 5:
            n = blocks + 100
            size = pool.required_bytes + 101 * (pool.required_bytes // blocks)
            old = pool.kv
            pool.resize(n, torch.empty(size, dtype=torch.uint8, device="cuda"))
            old.fill_(0xFF)
        nt = [40 - turn] * len(sids) if turn % 2 == 0 else [1] * len(sids)
        k, v, q = draw(sum(nt), hkv, d), draw(sum(nt), hkv, d), draw(sum(nt), 16, d)
        pool.plan_begin(sids, nt)
        outs = []
        for l in range(layers):
            pool.frame_append_kv(l, k, v)
            if l in (0, layers - 1):
                outs.append(torch.empty_like(q))
                pool.attend_chunk_prefill(l, q, outs[-1])
        pool.plan_commit()
        assert torch.equal(*outs) and bool(torch.isfinite(outs[0].float()).all())
