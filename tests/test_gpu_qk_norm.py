"""GPU parity of normed queries and keys (mtn_pool_set_qk_norm) on every cache type
and every kernel that rotates.  Tolerances are those of rows that are only
rotated: a normed row of weights near 1 has elements of the same size, its factor
r adds a relative error of a few 2^-24 to a product that is rounded to bf16
(2^-9) or used in fp32 (2^-24 per product of a score, of which the f32 bound of
1e-5 leaves room for a hundred)."""
import random

import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from oracle import windowed_attention as wa
from tests._gpu_util import TDT, Harness, f64, make_pool, say

pytestmark = pytest.mark.gpu

FORMS = [None, dict(layout="interleaved", rotary_dim=48), dict(layout="half", rotary_dim=32),
         dict(layout="interleaved")]


def _weights(layers, d, seed=0):
    rng = np.random.default_rng(seed)
    return [rng.uniform(0.6, 1.4, (layers, d)).astype(np.float32) for _ in range(2)]


def _harness(dtype, hq, hkv, d, form=None, S=4, W=40, n=3, layers=2, cmax=9, seed=0, eps=1e-6, norm_first=False):
    ring = -(-(W + cmax - 1) // 16) + -(-S // 16)
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, cmax=cmax, max_sessions=n,
                     n_blocks=n * ring, dtype=dtype)
    wq, wk = _weights(layers, d, seed)
    if norm_first:
        pool.set_qk_norm(wq, wk, eps)
    if form:
        pool.set_rope(**form)
    if not norm_first:
        pool.set_qk_norm(torch.from_numpy(wq).cuda(), wk, eps)
    h = Harness(pool, n_sessions=n, n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, dtype=dtype, seed=seed)
    for o in h.orc:
        o.qk_norm = (wq, wk, eps)
        o.rope = form
    return h


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,hq,hkv,d", [("f32", 8, 2, 64), ("f32", 8, 1, 128), ("bf16", 8, 2, 64),
                                            ("bf16", 16, 2, 128), ("bf16", 2, 2, 128), ("fp8", 8, 2, 128),
                                            ("int8", 8, 2, 64), ("int8", 16, 2, 128)])
def test_frames(dtype, hq, hkv, d, form):
    say(f"normed frames {dtype} {hq}/{hkv} D={d} form {form}")
    h = _harness(dtype, hq, hkv, d, FORMS[form], seed=form, norm_first=form % 2 == 0)
    rnd = random.Random(form)
    for f in range(6):
        h.frame([rnd.randint(1, 9) for _ in h.sids], [rnd.randint(0, 3) for _ in h.sids],
                use_frame_step=f % 3 != 2, fused=f % 2 == 0)
    say(f"  max err {h.max_err:.2e}, lse {h.max_lse_err:.2e}")


@pytest.mark.parametrize("kind", [1, 2])
def test_both_decode_kernels(kind):
    h = _harness("bf16", 4, 1, 128, seed=kind)
    h.pool.set_decode_kernel(kind)
    for f in range(4):
        h.frame([1] * 3, [2] * 3, use_frame_step=f % 2 == 0, fused=f > 2)


@pytest.mark.parametrize("split", [2, 5])
def test_split_decode(split):
    h = _harness("bf16", 8, 1, 128, W=200, n=1)
    for f in range(3):
        h.frame([9], [3], n_split=split)


def _pool_bytes(dtype, d, fused, seed):
    """The pool after frames of chunks and decodes from rows whose magnitudes lie up
    to 2^6 apart, appended by kernels of their own or by those that attend."""
    n, hq, hkv, layers, cmax = 2, 8, 2, 1, 7
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=4, W=40, cmax=cmax, max_sessions=n,
                     n_blocks=n * 4, dtype=dtype)
    pool.kv.zero_()
    pool.set_qk_norm(*_weights(layers, d), 1e-6)
    sids = [pool.session_open() for _ in range(n)]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rows(t, h):
        x = torch.randn((1, t, h, d), generator=gen, device="cuda")
        return (x * torch.exp2(torch.randint(-3, 4, x.shape, generator=gen, device="cuda"))).to(TDT[dtype])
    for f in range(8):
        c = [1, 1] if f % 3 == 2 else [cmax, 3 + f % 4]
        q, k, v = rows(sum(c), hq), rows(sum(c), hkv), rows(sum(c), hkv)
        o = torch.empty_like(q)
        if fused:
            pool.frame_step(sids, c, [0] * n, q, k, v, o)
        else:
            pool.plan_begin(sids, c)
            pool.frame_append_kv(0, k[0], v[0])
            pool.attend_chunk_prefill(0, q[0], o[0])
            pool.plan_commit()
    torch.cuda.synchronize()
    return pool.kv.clone()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("fp8", 128), ("int8", 128)])
def test_fused_and_separate_calls_store_identical_pools(dtype, d):
    for seed in range(3):
        assert torch.equal(_pool_bytes(dtype, d, True, seed), _pool_bytes(dtype, d, False, seed))


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128), ("int8", 128)])
@pytest.mark.parametrize("scale", [1e38, 1e19, 1e-19, 1e-38, 0.0])
def test_largest_and_smallest_rows(dtype, d, scale):
    """Rows whose squares overflow or vanish in fp32: a large row's outputs are those
    of any row of its direction, a small one's eps decides."""
    h = _harness(dtype, 4, 2, d, n=1, layers=1, eps=2.0 ** -126 if scale == 1e-19 else 1e-6)
    draw = h._draw
    h._draw = lambda i, n: tuple(x if j == 2 else (x.double().clamp(-3, 3) * scale).to(x.dtype)
                                 for j, x in enumerate(draw(i, n)))
    for f in range(3):
        h.frame([5], [2], use_frame_step=f != 1, fused=f == 1)
    say(f"{dtype} D={d} scale {scale}: max err {h.max_err:.2e}")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8", "int8"])
def test_a_bad_key_stays_with_its_head(dtype):
    """A NaN in one key makes the outputs of its head's queries NaN and no other's
    (int8: every key of its block, here the sinks that the plan completes, is NaN
    from the append on, also for the queries before it)."""
    d, hq, hkv, n = 128, 4, 2, 6
    outs = []
    for bad in (False, True):
        pool = make_pool(n_layers=1, hq=hq, hkv=hkv, d=d, S=4, W=40, cmax=n, max_sessions=1, n_blocks=4, dtype=dtype)
        pool.set_qk_norm(*_weights(1, d))
        gen = torch.Generator(device="cuda").manual_seed(3)
        q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").to(TDT[dtype]) for h in (hq, hkv, hkv))
        if bad:
            k[2, 1, 7] = float("nan")
        out, sid = torch.empty_like(q), pool.session_open()
        pool.plan_begin([sid], [n])
        pool.frame_append_kv(0, k, v)
        pool.attend_chunk_prefill(0, q, out)
        pool.plan_commit()
        outs.append(out)
    first = 0 if dtype == "int8" else 2
    assert torch.equal(outs[0][:, :2], outs[1][:, :2]) and torch.equal(outs[0][:first], outs[1][:first])
    assert torch.isnan(outs[1][first:, 2:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8", "int8"])
def test_cleared_norms_give_the_created_pools_results(dtype):
    def frames(pool):
        gen = torch.Generator(device="cuda").manual_seed(5)
        sid, outs = pool.session_open(), []
        for n in (5, 1, 9, 1):
            q, k, v = (torch.randn((n, h, 128), generator=gen, device="cuda").to(TDT[dtype]) for h in (8, 2, 2))
            out = torch.empty_like(q)
            pool.plan_begin([sid], [n])
            pool.frame_append_kv(0, k, v)
            pool.attend_chunk_prefill(0, q, out)
            pool.plan_commit()
            outs.append(out)
        pool.session_close(sid)
        return outs
    kw = dict(n_layers=1, hq=8, hkv=2, d=128, S=4, W=40, cmax=9, max_sessions=1, n_blocks=5, dtype=dtype)
    a, b = make_pool(**kw), make_pool(**kw)
    want = frames(a)
    b.set_qk_norm(*_weights(1, 128))
    other = frames(b)
    b.clear_qk_norm()
    for x, y, z in zip(want, frames(b), other):
        assert torch.equal(x, y)
        assert x.shape[0] == 1 or not torch.equal(x, z)


def test_refused_while_the_current_stream_is_captured():
    pool = _harness("bf16", 4, 1, 128, n=1).pool
    x, g, codes = torch.zeros(8, device="cuda"), torch.cuda.CUDAGraph(), []
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        x += 1
        for fn in (pool.set_qk_norm, pool.clear_qk_norm):
            try:
                fn()
                codes.append(0)
            except mtn.MtnError as e:
                codes.append(e.code)
    assert codes == [mtn.MTN_ERR_BAD_STATE] * 2
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
    assert bool((x == 3).all())


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (8, 2), (4, 4)])
def test_fp8_decode_is_off_by_its_outputs_rounding(hq, hkv, fused):
    """The stored rows are exact operands, queries and probabilities have two bf16
    terms (2^-16 and less of theirs): what is left is the output's rounding, of
    which half a step is 2^-8 of values of [1, 2) and less, evenly spread: 2^-8 / sqrt(3)
    in rms, were all of them at the lower end, and 2^-13 for everything else (queries
    in one term would add as much again as the outputs' rounding, 0.0024 together with it
    the least, probabilities in one the same)."""
    d, n, layers = 128, 150, 1
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=4, W=200, cmax=n, max_sessions=1, n_blocks=23, dtype="fp8")
    w = _weights(layers, d)
    pool.set_qk_norm(*w)
    o = wa.OracleSession(hq, hkv, d, 4, 200, n_layers=layers, kv_quant="fp8_e4m3")
    o.qk_norm = (*w, 1e-6)
    gen, sid, err, size = torch.Generator(device="cuda").manual_seed(hq), pool.session_open(), [], []
    for t in [n] + [1] * 12:
        q, k, v = (torch.randn((t, h, d), generator=gen, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
        out = torch.empty_like(q)
        pool.plan_begin([sid], [t])
        if t == 1 and fused:
            pool.attend_decode_append(0, k, v, q, out)
        else:
            pool.frame_append_kv(0, k, v)
            (pool.attend_decode if t == 1 else pool.attend_chunk_prefill)(0, q, out)
        pool.plan_commit()
        o.begin(t)
        ref = o.layer_step(0, *(f64(x) for x in (q, k, v)))[0]
        o.commit()
        if t == 1:
            err.append(f64(out) - ref)
            size.append(ref)
    rms = np.sqrt(np.mean(np.square(err)) / np.mean(np.square(size)))
    say(f"fp8 {hq}/{hkv} fused {fused}: {rms:.5f}")
    assert rms <= 2.0 ** -8 / np.sqrt(3) + 2.0 ** -13
