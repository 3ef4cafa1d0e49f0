"""GPU parity of the rotary forms (mtn_pool_set_rope) on every cache type and
every kernel that rotates: fused and separate appends, chunk prefill, vector
and matrix-core decode.  Tolerances are those of the whole-row form (the
rotation of an element is two products in fp32 either way; a magnitude m
multiplies scores, and the roundings in them, by m^2 <= 1.3 here)."""
import random

import pytest
import torch

import paper_2607_02640_amd as mtn
from oracle import windowed_attention as wa
from tests._gpu_util import Harness, make_pool, say

pytestmark = pytest.mark.gpu

FORMS = [
    dict(layout="interleaved"),
    dict(layout="half", rotary_dim=16),
    dict(layout="interleaved", rotary_dim=48, scaling="linear", factor=8.0),
    dict(layout="half", rotary_dim=48, scaling="base", factor=4.0),
    dict(layout="half", scaling="yarn", factor=4.0, original_len=64),
    dict(layout="interleaved", rotary_dim=32, scaling="yarn", factor=2.0, original_len=40, beta_fast=8.0,
         beta_slow=0.5, magnitude=1.1),
]


def _harness(dtype, hq, hkv, d, form, S=4, W=40, n=3, layers=2, cmax=9, seed=0):
    ring = -(-(W + cmax - 1) // 16) + -(-S // 16)
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, cmax=cmax, max_sessions=n,
                     n_blocks=n * ring, dtype=dtype)
    pool.set_rope(**form)
    h = Harness(pool, n_sessions=n, n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, dtype=dtype, seed=seed)
    for o in h.orc:
        o.rope = {k: v for k, v in form.items()}
    return h


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,hq,hkv,d", [("f32", 8, 2, 64), ("f32", 8, 1, 128), ("bf16", 8, 2, 64),
                                            ("bf16", 16, 2, 128), ("bf16", 2, 2, 128), ("fp8", 8, 2, 128)])
def test_frames(dtype, hq, hkv, d, form):
    h = _harness(dtype, hq, hkv, d, FORMS[form], seed=form)
    rnd = random.Random(form)
    for f in range(6):
        h.frame([rnd.randint(1, 9) for _ in h.sids], [rnd.randint(0, 3) for _ in h.sids],
                use_frame_step=f % 3 != 2, fused=f % 2 == 0)
    say(f"{dtype} {hq}/{hkv} D={d} form {form}: max err {h.max_err:.2e}, lse {h.max_lse_err:.2e}")


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_both_decode_kernels(kind, layout):
    h = _harness("bf16", 4, 1, 128, dict(layout=layout, rotary_dim=96), seed=kind)
    h.pool.set_decode_kernel(kind)
    for f in range(4):
        h.frame([1] * 3, [2] * 3, use_frame_step=f % 2 == 0, fused=f > 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_set_back_to_the_created_form(dtype):
    """An all-default set_rope after another form gives the created form's results bit for bit."""
    def frames(pool):
        gen = torch.Generator(device="cuda").manual_seed(5)
        sid, outs = pool.session_open(), []
        io = torch.float32 if dtype == "f32" else torch.bfloat16
        for n in (5, 1, 9, 1):
            q, k, v = (torch.randn((n, h, 128), generator=gen, device="cuda").to(io) for h in (8, 2, 2))
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
    b.set_rope(layout="interleaved", rotary_dim=64, scaling="linear", factor=3.0)
    other = frames(b)
    b.set_rope()
    for x, y, z in zip(want, frames(b), other):
        assert torch.equal(x, y)
        assert x.shape[0] == 1 or not torch.equal(x, z)
