"""GPU parity of the int8 cache against the float64 oracle: appends fused and
apart, decode, chunk prefill with and without key segments, open and complete
blocks, wrapped rings, abandoned plans and dead slots poisoned.

Tolerances.  Values are N(0, 1), at most 4.5 of them large enough to matter.  A
bf16 rounding is off by at most 2^-8 relative: the output by 0.018 (at 4.5), the
probabilities' share of it by as much, and a score by at most about 4 standard
deviations of the query's 128 roundings, 4 * 2^-8 / sqrt(3) / sqrt(128) * sqrt(128) =
0.009 before the products' mean size 0.72: 0.0065, which moves two keys' shares by
a quarter of twice that, times values 7 apart: 0.023.  Together 0.058; the
harness holds every element to 0.06.  (Most are far closer: windows of many keys
average.)  The root mean square over a test is held to 4e-3: the output's
rounding contributes 2^-8 / sqrt(3) * 0.7 = 1.6e-3 at unit size, the probabilities'
as much at most, the scores' 0.0016 * 0.25 * 2 * 1.4 = 1.1e-3; together 2.5e-3.

The oracle quantizes from the same bf16 rows as the kernels, but for keys whose
rotation lies within fp32 rounding of a bf16 border, a few elements in 10^4; the
code of such an element may differ by one step of its block, max|k| / 127 = 0.035,
which moves one score by at most 0.035 * 4.5 / sqrt(128) = 0.014 and leaves the root
mean square where it is."""
import random

import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from tests._gpu_util import Harness, make_pool, say

pytestmark = pytest.mark.gpu


def _harness(hq, hkv, d, S=4, W=40, n=3, layers=2, cmax=9, seed=0, rope=None, max_len=300):
    ring = -(-max_len // 16) if W is None else -(-(W + cmax - 1) // 16) + -(-S // 16)
    pool = make_pool(n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, cmax=cmax, max_sessions=n + 2,
                     n_blocks=(n + 2) * ring, dtype="int8", max_len=0 if W else max_len)
    if rope:
        pool.set_rope(**rope)
    h = Harness(pool, n_sessions=n, n_layers=layers, hq=hq, hkv=hkv, d=d, S=S, W=W, dtype="int8", seed=seed)
    for o in h.orc:
        o.rope = rope
    return h


def _settled(h):
    assert h.rms_err() <= 4e-3
    say(f"max err {h.max_err:.2e}, rms {h.rms_err():.2e}, lse {h.max_lse_err:.2e}")


def _frames(h, rnd, n, cmax=9, poison=True):
    for f in range(n):
        if poison:
            h.pool.poison_dead()
        h.frame([rnd.randint(1, cmax) for _ in h.sids], [rnd.randint(0, 3) for _ in h.sids],
                use_frame_step=f % 3 != 2, fused=f % 2 == 0)
    _settled(h)


@pytest.mark.parametrize("W", [3, 40, 57, None])
@pytest.mark.parametrize("S", [0, 1, 4, 16, 20])
@pytest.mark.parametrize("hq,hkv,d", [(8, 1, 128), (3, 3, 64)])
def test_frames(hq, hkv, d, S, W):
    h = _harness(hq, hkv, d, S=S, W=W, seed=S)
    _frames(h, random.Random(S), 8)


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 128), (4, 2, 128), (8, 2, 128), (16, 2, 128), (5, 5, 128),
                                      (2, 1, 64), (4, 1, 64), (8, 1, 64)])
def test_head_layouts(hq, hkv, d):
    h = _harness(hq, hkv, d, seed=hq)
    _frames(h, random.Random(hq), 5)


@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_through_every_slot(d):
    """One-token plans from an empty session on, over the sinks' and the ring's
    block edges and a ring's turn, with the append fused and apart."""
    h = _harness(4, 2, d, S=5, W=20, n=2, layers=1, cmax=1)
    for t in range(70):
        if t % 7 == 0:
            h.pool.poison_dead()
        h.frame([1, 1], [0, 0], use_frame_step=t % 3 == 0, fused=t % 2 == 0)
    _settled(h)


@pytest.mark.parametrize("n_split", [1, 2, 5, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_split(n_split, d):
    h = _harness(8, 2, d, W=300, n=2, layers=1, cmax=64, seed=n_split)
    for c in (64, 64, 50, 64, 64, 33):
        h.frame([c, c - 7], [0, 0])
    for f in range(20):
        h.frame([1, 1], [0, 0], n_split=n_split, use_frame_step=False, fused=f % 2 == 0)
    assert h.pool.last_split() == n_split
    _settled(h)


@pytest.mark.parametrize("rows", [0, 128, 256])
@pytest.mark.parametrize("hq,hkv,d,W", [(8, 1, 128, 500), (2, 2, 128, None), (4, 1, 64, 700), (8, 1, 64, None)])
def test_long_chunks(hq, hkv, d, W, rows):
    """Chunks over several passes and key segments, longer than a block, over
    blocks of every kind; then decodes of what they left."""
    h = _harness(hq, hkv, d, S=17, W=W, n=2, layers=1, cmax=180, seed=rows, max_len=700)
    h.pool.set_prefill_pass_rows(rows)
    for c in ((180, 33), (150, 180), (9, 16), (180, 175)):
        h.pool.poison_dead()
        h.frame(list(c), [2, 1])
    _settled(h)


@pytest.mark.parametrize("rope", [dict(layout="interleaved"), dict(rotary_dim=32, scaling="linear", factor=4.0),
                                  dict(layout="interleaved", rotary_dim=48, scaling="yarn", factor=4.0, original_len=64)])
@pytest.mark.parametrize("d", [64, 128])
def test_rotary_forms(d, rope):
    h = _harness(8, 2, d, rope=rope)
    _frames(h, random.Random(d), 6)


def test_an_abandoned_plan_leaves_the_rows_whole():
    """Plans of every length over the open block, appended in every layer and
    then abandoned, before each frame."""
    h, rnd = _harness(8, 2, 128, cmax=50, W=60), random.Random(9)
    for f in range(8):
        n = [1, 3, 15, 16, 17, 32, 40, 50][f]
        k, v = torch.randn((2, n * len(h.sids), 2, 128), device="cuda").bfloat16() * 50
        h.pool.plan_begin(h.sids, [n] * len(h.sids))
        for l in range(2):
            h.pool.frame_append_kv(l, k, v)
        h.pool.plan_abort()
        h.frame([rnd.randint(1, 20) for _ in h.sids], [1] * len(h.sids), use_frame_step=f % 2 == 0, fused=True)
    _settled(h)


def test_forks_and_moves_take_the_open_rows_along():
    import copy
    h, rnd = _harness(8, 2, 64, n=2), random.Random(4)
    _frames(h, rnd, 3)
    for sid in h.pool.session_fork(h.sids[1], 2):
        h.sids.append(sid)
        h.orc.append(copy.deepcopy(h.orc[1]))
        h.rng.append(np.random.default_rng(sid))
    _frames(h, rnd, 2)
    old, blocks = h.pool.kv, h.pool.stats()["reserved"] + 7
    kw = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, n_sink=4, window=40, max_chunk=9,
              max_sessions=4, n_blocks=blocks, dtype="int8")
    h.pool.resize(blocks, torch.full((mtn.Pool.required(**kw),), 0xFF, dtype=torch.uint8, device="cuda"))
    old.fill_(0xFF)
    _frames(h, rnd, 4)


def _attend(pool, sid, q, k, v):
    n = q.shape[0]
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    pool.plan_begin([sid], [n])
    pool.frame_append_kv(0, k, v)
    pool.attend_chunk_prefill(0, q, out, lse)
    pool.plan_commit()
    return out, lse


def _plain_pool(d, W=None, hkv=2, g=4, S=0, n=2):
    ring = 20 if W is None else -(-(W + 63) // 16) + -(-S // 16)
    return make_pool(n_layers=1, hq=hkv * g, hkv=hkv, d=d, S=S, W=W, cmax=64, max_sessions=n, n_blocks=n * ring,
                     dtype="int8", max_len=320 if W is None else 0)


@pytest.mark.parametrize("d", [64, 128])
def test_plans_do_not_change_what_a_block_reads(d):
    """The same 96 tokens in other chunks, by every append: the pools hold the
    same bytes and a query sees the same."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    k, v, q = draw(96, 2, d), draw(96, 2, d), draw(1, 8, d)
    kept = []
    for cuts in ([64, 32], [1] * 96, [7] * 13 + [5], [16] * 6):
        pool = _plain_pool(d)
        pool.kv.zero_()
        sid, at = pool.session_open(), 0
        for c in cuts:
            ks, vs, qs = k[at:at + c], v[at:at + c], draw(c, 8, d)
            if c == 1:
                pool.plan_begin([sid], [1])
                pool.attend_decode_append(0, ks, vs, qs, torch.empty_like(qs))
                pool.plan_commit()
            else:
                _attend(pool, sid, qs, ks, vs)
            at += c
        blocks = pool.kv[:pool.cfg.n_blocks * (2 * 32 * d + 128)].clone()
        kept.append((blocks, _attend(pool, sid, q, k[:1], v[:1])))
    for blocks, (out, lse) in kept[1:]:
        assert torch.equal(blocks, kept[0][0])
        assert torch.equal(out, kept[0][1][0]) and torch.equal(lse, kept[0][1][1])


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-10, 1e10, 2.0 ** 100])
def test_magnitudes(scale):
    """Values of any size, a block of huge ones beside a block of small ones: the
    outputs stay within a step of the block that carries the weight."""
    pool = _plain_pool(128)
    gen = torch.Generator(device="cuda").manual_seed(2)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda")
    sid = pool.session_open()
    k, v, q = draw(48, 2, 128).bfloat16(), (draw(48, 2, 128) * scale).bfloat16(), draw(48, 8, 128).bfloat16()
    k[:16] = 0
    out, _ = _attend(pool, sid, q, k, v)
    kf, vf, qf = k.double(), v.double(), q.double()
    pos = torch.arange(48, device="cuda").double()
    inv = 1e4 ** (-torch.arange(64, device="cuda").double() / 64)
    c, s = (pos[:, None] * inv).cos()[:, None], (pos[:, None] * inv).sin()[:, None]
    rot = lambda x: torch.cat([x[..., :64] * c - x[..., 64:] * s, x[..., 64:] * c + x[..., :64] * s], -1)
    sc = torch.einsum("thd,khd->htk", rot(qf), rot(kf).repeat_interleave(4, 1)) / 128 ** 0.5
    sc = sc.masked_fill(pos[None, None, :] > pos[None, :, None], -torch.inf)
    want = torch.einsum("htk,khd->thd", sc.softmax(-1), vf.repeat_interleave(4, 1))
    # Half a step of the values (max 4.5, so 0.018), what half a step of the keys
    # moves the probabilities by (a score by 0.0095 on average, at most about 4
    # times that; two keys' shares by a quarter of it, values 7 apart: 0.066),
    # roundings of probabilities and output to bf16 (2^-9 of 4.5 each: 0.018)
    assert torch.isfinite(out).all()
    assert (out.double() - want).abs().max() <= 0.102 * scale


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("what", ["k", "v"])
def test_a_bad_element_stays_with_the_rows_that_see_its_block(what, bad, d):
    """A non-finite element makes its block, head and tensor NaN: rows that see
    no key of the block, and the other heads, are bitwise what they were."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    k, v, q = draw(60, 2, d), draw(60, 2, d), draw(60, 8, d)
    for at in (5, 20, 58):  # a complete block before the others, between, the open one
        outs = []
        for x in (None, bad):
            pool = _plain_pool(d)
            sid = pool.session_open()
            ks, vs = k.clone(), v.clone()
            if x is not None:
                (ks if what == "k" else vs)[at, 1, 3] = x
            outs.append(_attend(pool, sid, q, ks, vs)[0])
        first = at if at >= 48 else at // 16 * 16  # an open block keeps its rows apart
        clean, dirty = outs
        assert torch.equal(clean[:, :4], dirty[:, :4])
        assert torch.equal(clean[:first, 4:], dirty[:first, 4:])
        rest = dirty[first:, 4:].float()
        if what == "k" and at >= 48 and bad == float("inf"):
            continue  # an open key of score -inf is a key of probability 0
        hit = rest if what == "k" or at < 48 else rest[..., 3]
        assert not torch.isfinite(hit).any()
        if what == "v" and at >= 48:
            keep = [i for i in range(d) if i != 3]
            assert torch.equal(clean[:, :, keep], dirty[:, :, keep])


def test_noalloc_decode_and_graph_replay():
    """The allocation-free decode, captured once and replayed over the same open
    plan: every replay gives the eager result."""
    pool = _plain_pool(128, W=200, S=4, n=2)
    gen = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    sids = [pool.session_open() for _ in range(2)]
    for _ in range(4):
        pool.plan_begin(sids, [60, 41])
        pool.frame_append_kv(0, draw(101, 2, 128), draw(101, 2, 128))
        pool.plan_commit()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        pool.plan_begin(sids, [1, 1])
        pool.frame_append_kv(0, draw(2, 2, 128), draw(2, 2, 128))
        q = draw(2, 8, 128)
        want, out = torch.empty_like(q), torch.empty_like(q)
        pool.attend_decode(0, q, want, n_split=3)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            pool.attend_decode_noalloc(0, q, out, n_split=3)
        for _ in range(4):
            out.zero_()
            g.replay()
            side.synchronize()
            assert torch.equal(out, want)
            torch.matmul(torch.randn(256, 256, device="cuda"), torch.randn(256, 256, device="cuda"))
        pool.plan_commit()
    torch.cuda.synchronize()
