"""Infinite and NaN elements under norms of queries and keys: they reach the outputs
as they do without norms, whatever kernel a call takes."""
import math

import pytest
import torch

from tests._gpu_util import TDT, make_pool, say

pytestmark = pytest.mark.gpu

BAD = {3: float("nan"), 17: float("inf"), 40: float("-inf"), 61: float("inf")}  # dim: value
INF = float("inf")


def _decode(pool, dtype, hq, hkv, d, rows, have, kind, fused, n_split):
    """The last of have + 1 tokens as a single token of a fresh session."""
    pool.set_decode_kernel(0 if kind == 2 and d == 64 else kind)  # (head dim 64: taken by shape)
    q, k, v = rows
    sid = pool.session_open()
    pool.plan_begin([sid], [have])
    pool.frame_append_kv(0, k[:have], v[:have])
    pool.plan_commit()
    pool.plan_begin([sid], [1])
    out = torch.empty((1, hq, d), dtype=TDT[dtype], device="cuda")
    lse = torch.empty((1, hq), device="cuda")
    if fused:
        pool.attend_decode_append(0, k[have:], v[have:], q, out, lse, n_split=n_split)
    else:
        pool.frame_append_kv(0, k[have:], v[have:])
        pool.attend_decode(0, q, out, lse, n_split=n_split)
    pool.plan_commit()
    torch.cuda.synchronize()
    pool.session_close(sid)
    return out, lse


@pytest.mark.parametrize("n_split", [1, 3])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dtype,g,d,kind", [
    *[("bf16", g, d, kind) for g, d in ((1, 64), (2, 128), (4, 64), (4, 128), (8, 128)) for kind in (1, 2)],
    ("f32", 4, 128, 1), ("f32", 1, 64, 1)])
def test_an_infinite_value_stays_infinite(dtype, g, d, kind, fused, n_split):
    """Every weight is above 0 (scores of normed rows lie within sqrt(d) of 0)."""
    say(f"{dtype} G={g} D={d} kernel {kind} fused {fused} split {n_split}")
    hkv, have = 2, 90
    pool = make_pool(n_layers=1, hq=hkv * g, hkv=hkv, d=d, S=4, W=100, cmax=have, max_sessions=1, n_blocks=13,
                     dtype=dtype)
    pool.set_qk_norm()
    gen = torch.Generator(device="cuda").manual_seed(g + d)
    q, k, v = (torch.randn(s, generator=gen, device="cuda").to(TDT[dtype])
               for s in ((1, hkv * g, d), (have + 1, hkv, d), (have + 1, hkv, d)))
    args = (pool, dtype, hkv * g, hkv, d)
    clean, lse = _decode(*args, (q, k, v), have, kind, fused, n_split)
    assert torch.isfinite(clean).all()
    ok = torch.ones(d, dtype=torch.bool, device="cuda")
    ok[list(BAD)] = False
    for at in (1, 50, have):  # a sink, one in the window, the newest
        bad = v.clone()
        for dim, x in BAD.items():
            bad[at, 1, dim] = x
        out, l2 = _decode(*args, (q, k, bad), have, kind, fused, n_split)
        assert torch.equal(l2, lse) and torch.equal(out[:, :g], clean[:, :g])
        assert torch.equal(out[:, g:, ok], clean[:, g:, ok])
        for dim, x in BAD.items():
            got = out[:, g:, dim]
            assert bool((torch.isnan(got) if x != x else got == x).all()), f"value {x} at {at}: {got}"


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_score_of_minus_infinity_has_weight_zero(d, fused, kind):
    """A weight takes two dims of one key past the largest float (pair 0, rotated by the
    key's position in radians); the query's pair has the opposite signs."""
    hq, have, p = 4, 40, 22
    pool = make_pool(n_layers=1, hq=hq, hkv=1, d=d, S=4, W=100, cmax=have, max_sessions=1, n_blocks=12, dtype="bf16")
    w = torch.ones((1, d))
    w[0, 0] = 3e38
    pool.set_qk_norm(None, w)
    gen = torch.Generator(device="cuda").manual_seed(d)
    q, k, v = (torch.randn(s, generator=gen, device="cuda") for s in ((1, hq, d), (have + 1, 1, d), (have + 1, 1, d)))
    k[:, 0, 0] = 0.0
    k[p, 0, 0] = 6.0  # normed to 6 / sqrt((36 + d) / d) at most, times 3e38: above 2^128
    a, b = -math.copysign(1.5, math.cos(p)), -math.copysign(1.5, math.sin(p))
    c, s = math.cos(-have), math.sin(-have)  # turned back, so that position `have` turns it to (a, b)
    q[0, :, 0], q[0, :, d // 2] = a * c - b * s, a * s + b * c
    outs = []
    for x in (0.0, 1000.0):
        v[p] = x
        outs.append(_decode(pool, "bf16", hq, 1, d, tuple(t.bfloat16() for t in (q, k, v)), have, kind, fused, 1))
    assert all(torch.isfinite(t).all() for o in outs for t in o), outs
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("g,split", [(8, False), (4, True), (1, False)])
def test_an_fp8_value_past_bf16_stays_infinite(g, split, norm):
    """The largest bf16 value rounds to 2^128 as an E4M3 code under its row's scale,
    which is infinite as the chunk prefill's bf16 operand."""
    hkv, d, n = 2, 128, 30
    W = 700 if split else 60
    pool = make_pool(n_layers=1, hq=hkv * g, hkv=hkv, d=d, S=4, W=W, cmax=n, max_sessions=1,
                     n_blocks=2 + -(-(W + n) // 16), dtype="fp8")
    if norm:
        pool.set_qk_norm()
    gen = torch.Generator(device="cuda").manual_seed(g)
    outs = []
    for bad in (False, True):
        sid, at = pool.session_open(), 0
        gen.manual_seed(g)
        have = n * (24 if split else 1)
        while at <= have:
            q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").bfloat16() for h in (hkv * g, hkv, hkv))
            v[:, :, 5] = 0.0  # (a code of its own beside the large ones)
            if bad and at == have:
                v[7, 1, :] = 0.0
                v[7, 1, 9] = torch.finfo(torch.bfloat16).max
                v[7, 1, 70] = -torch.finfo(torch.bfloat16).max
            out = torch.empty_like(q)
            pool.plan_begin([sid], [n])
            pool.frame_append_kv(0, k, v)
            pool.attend_chunk_prefill(0, q, out)
            pool.plan_commit()
            at += n
        torch.cuda.synchronize()
        pool.session_close(sid)
        outs.append(out)
    clean, out = outs
    assert torch.equal(out[:7], clean[:7]) and torch.equal(out[:, :g], clean[:, :g])
    assert bool((out[7:, g:, 9] == INF).all()) and bool((out[7:, g:, 70] == -INF).all()), (out[7:, g:, 9], out[7:, g:, 70])
    assert torch.isfinite(out[7:, g:, 5]).all()
