"""GPU tests of the int8 cache with blocks of very different scales: a row's sum
and log-sum-exp depend on its scores alone, whatever the values' size, and
scores on the product of a query's and a block's size.

A power of two on the rows of a block moves its scale by that power and leaves
its codes, so most of what follows is exact.  Where fp32 or bf16 operands
become subnormal it is not: a probability times a V scale may then be off by up
to 2^-126 (if it is taken for zero), times a code of at most 127, for each of
at most 300 keys and before the division by a sum of at least 1.
"""
import pytest
import torch

import paper_2607_02640_amd as mtn
from tests.test_gpu_int8 import _attend, _plain_pool

pytestmark = pytest.mark.gpu

SUBNORMAL = 300 * 127 * 2.0 ** -126
LENGTHS = [60, 60, 60, 60, 57]  # the last block, of 9 rows, stays open


def _draw(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()


def _rows(d, seed=0):
    draw, n = _draw(seed), sum(LENGTHS)
    return draw(n, 8, d), draw(n, 2, d), draw(n, 2, d)


def _within(out, want, tol):
    bad = ~((out - want).abs() <= tol)
    assert not bad.any(), [(i, out[i].item(), want[i].item()) for i in map(tuple, bad.nonzero()[:4].tolist())]


def _run(pool, q, k, v):
    """Every chunk's rows and their sums, then those of a decode that sees all."""
    n, d = sum(LENGTHS), pool.cfg.head_dim
    assert (q.shape, k.shape, v.shape) == ((n, 8, d), (n, 2, d), (n, 2, d))
    sid, at, outs, lses = pool.session_open(), 0, [], []
    for n in LENGTHS:
        out, lse = _attend(pool, sid, *(x[at:at + n].contiguous() for x in (q, k, v)))
        outs.append(out)
        lses.append(lse)
        at += n
    pool.plan_begin([sid], [1])
    out, lse = torch.empty_like(q[:1]), torch.empty((1, 8), device="cuda")
    pool.attend_decode_append(0, k[-1:].contiguous(), v[-1:].contiguous(), q[:1].contiguous(), out, lse)
    pool.plan_commit()
    pool.session_close(sid)
    return torch.cat(outs + [out]).double(), torch.cat(lses + [lse])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-133, -130, -127, -125, -122, -119, -116, -110, -100, -60, 60, 100])
def test_the_size_of_a_block_of_values_leaves_the_sums(power, d):
    q, k, v = _rows(d)
    pool = _plain_pool(d)
    out1, lse1 = _run(pool, q, k, v)
    for b in (0, 7, 18):  # the first block, one between, the open one
        rows = slice(16 * b, 16 * b + 16)
        vs, v0, vb = v.clone(), v.clone(), torch.zeros_like(v)
        vs[rows] = (vs[rows].float() * 2.0 ** power).bfloat16()
        v0[rows] = 0
        vb[rows] = v[rows]
        out, lse = _run(pool, q, k, vs)
        assert torch.equal(lse, lse1)
        rest, alone = _run(pool, q, k, v0)[0], _run(pool, q, k, vb)[0]
        # to a bf16 step: what the other blocks give and what this one adds (the
        # larger of the two may cancel, which leaves its own rounding)
        want = rest + alone * 2.0 ** power
        tol = 2.0 ** -7 * (rest.abs() + alone.abs() * 2.0 ** power) + SUBNORMAL
        # An fp32 sum of terms of both sizes (at most 300, whose weights add up to 1)
        # is off by 2^-24 of a partial sum at each: where the larger terms cancel, the
        # smaller ones are lost.
        mixed = rest.abs().amax(-1, keepdim=True) > 0
        tol = tol + mixed * 300 * 2.0 ** -24 * 4.5 * max(1.0, 2.0 ** power)
        if power < -110:  # bf16 rows, their scale and codes then have few bits
            tol = tol + 4.5 * 2.0 ** power
        _within(out, want, tol)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-133, -127, -120, -100, 100])
def test_all_values_of_one_size(power, d):
    q, k, v = _rows(d, 1)
    pool = _plain_pool(d)
    out1, lse1 = _run(pool, q, k, v)
    out, lse = _run(pool, q, k, (v.float() * 2.0 ** power).bfloat16())
    assert torch.equal(lse, lse1)
    tol = 2.0 ** -7 * out1.abs() * 2.0 ** power + SUBNORMAL
    if power < -110:
        tol = tol + 4.5 * 2.0 ** power
    _within(out, out1 * 2.0 ** power, tol)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_value_leaves_the_sums(bad, d):
    """Rows with a non-finite sum of values are computed once more, under other
    references: their log-sum-exp is off by what fp32 exponents (of at most 32:
    2^-20 in log2) and the sums of 300 terms in two orders (300 * 2^-24) are."""
    q, k, v = _rows(d, 2)
    pool = _plain_pool(d)
    lse1 = _run(pool, q, k, v)[1]
    for at in (5, 130, 290):
        vs = v.clone()
        vs[at, 1, 3] = bad
        out, lse = _run(pool, q, k, vs)
        assert (lse - lse1).abs().max() <= 2.5e-5
        assert not torch.isfinite(out[290:, 4:, 3]).any() and torch.isfinite(out[:, :4]).all()


def _scaled_pool(d, softmax_scale):
    kw = dict(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=d, n_sink=0, window=None, max_chunk=64,
              max_sessions=2, n_blocks=40, dtype="int8", max_len=320)
    kv = torch.empty(mtn.Pool.required(**kw), dtype=torch.uint8, device="cuda")
    return mtn.Pool(**kw, softmax_scale=softmax_scale, kv=kv)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 1.0])
@pytest.mark.parametrize("power", [-120, -110, -60, 60, 100, 125])
def test_small_queries_over_large_keys_and_the_reverse(power, scale, d):
    """Queries times 2^power over keys times 2^-power: the same scores.  (Where a
    rotated element is subnormal in fp32 it may round to another bf16 value, which
    moves a key by a step of its block, 0.035 of the largest, and a score by
    0.035 * 4.5 * the softmax scale.)"""
    q, k, v = _rows(d, 3)
    if scale:
        q = (q.float() / 8).bfloat16()
    out1 = lse1 = None
    for p in (0, power):
        ks = (k.float() * 2.0 ** -p).bfloat16()
        out, lse = _run(_scaled_pool(d, scale), (q.float() * 2.0 ** p).bfloat16(), ks, v)
        if out1 is None:
            out1, lse1 = out, lse
    step = 0.035 * 4.5 * (scale / 8 if scale else d ** -0.5)
    assert (lse - lse1).abs().max() <= step
    assert (out - out1).abs().max() <= 2 * step * 2 * 4.5 / 4 + 2.0 ** -7 * 4.5


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pq,pk", [(-84, -84), (-130, -20), (-20, -130), (-133, -133)])
def test_scores_too_small_to_matter(pq, pk, d):
    """Every key that a row sees has the same weight, and masked keys none: the
    log-sum-exp is ln n, the output the mean (to half a step of a code, 0.018, and
    three bf16 roundings of at most 4.5)."""
    q, k, v = _rows(d, 4)
    q, k = (q.float() * 2.0 ** pq).bfloat16(), (k.float() * 2.0 ** pk).bfloat16()
    out, lse = _run(_plain_pool(d), q, k, v)
    n = torch.arange(1, 299, device="cuda").double()
    vf = torch.cat([v, v[-1:]]).double().repeat_interleave(4, 1)
    assert (lse - n.log()[:, None]).abs().max() <= 2.5e-5
    assert (out - vf.cumsum(0) / n[:, None, None]).abs().max() <= 0.018 + 3 * 2.0 ** -8 * 4.5


@pytest.mark.parametrize("d", [64, 128])
def test_queries_near_the_largest_float_over_zero_keys(d):
    """Scaled and rotated elements of up to 1.5 * 2^126 * log2(e) * sqrt(2) = 1.53 *
    2^127: finite, so that their scores over zero keys are 0 and every key has the
    same weight (tolerances as above)."""
    _, k, v = _rows(d, 5)
    q = torch.zeros((len(k), 8, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, [3, 3 + d // 2]] = 1.5 * 2.0 ** 126
    out, lse = _run(_scaled_pool(d, 1.0), q, torch.zeros_like(k), v)
    n = torch.arange(1, 299, device="cuda").double()
    vf = torch.cat([v, v[-1:]]).double().repeat_interleave(4, 1)
    assert (lse - n.log()[:, None]).abs().max() <= 2.5e-5
    assert (out - vf.cumsum(0) / n[:, None, None]).abs().max() <= 0.018 + 3 * 2.0 ** -8 * 4.5
