"""GPU parity of the linear layers (mtn_attend_linear) with the float64 recurrence:
chunk and single-token forms, segmented prompts, state slots, forks, graphs."""
import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from tests._gpu_util import say
from tests._linear_util import TDT, Linear, f64

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 2, 2, 128), ("bf16", 4, 2, 64), ("bf16", 8, 1, 128), ("bf16", 4, 1, 128), ("bf16", 16, 2, 64),
          ("f32", 2, 2, 64), ("f32", 2, 1, 128), ("f32", 8, 1, 64), ("f32", 4, 1, 128), ("f32", 1, 1, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_single_tokens(dtype, hq, hkv, d):
    say(f"single tokens {dtype} {hq}/{hkv} D={d}")
    x = Linear(dtype, hq, hkv, d, n=3, layers=2)
    for _ in range(5):
        x.step([1, 1, 1])
    x.step([1], x.sids[1:2])  # one of them alone, then all again, in another order
    x.step([1, 1, 1], x.sids[::-1])
    say(f"  worst {x.worst:.3f} of the bound")


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("first", [2, 16, 17, 31, 32, 33])
def test_short_chunks(dtype, hq, hkv, d, first):
    """Chunks around the 16- and 32-token tiles, fresh and over a state."""
    say(f"short chunks {dtype} {hq}/{hkv} D={d} first {first}")
    x = Linear(dtype, hq, hkv, d, n=2, seed=first)
    for n_tok in ([first, 1], [1, 1], [3, first], [32, 25]):
        x.step(n_tok)
    say(f"  worst {x.worst:.3f} of the bound")


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_long_chunks_and_segments(dtype, hq, hkv, d):
    """Chunks around the 64-token tiles, and prompts that the plan cuts into segments
    (few sequences and heads), beside short ones, fresh and over a state."""
    say(f"long chunks {dtype} {hq}/{hkv} D={d}")
    x = Linear(dtype, hq, hkv, d, n=3, cmax=700, seed=d + hq)
    for n_tok in ([63, 64, 65], [1, 128, 129], [700, 2, 300], [1, 1, 1], [300, 640, 5]):
        x.step(n_tok)
    say(f"  worst {x.worst:.3f} of the bound")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_unsegmented(dtype):
    """As many sequences as compute units: one workgroup walks each sequence's tiles."""
    n = torch.cuda.get_device_properties(0).multi_processor_count + 1
    x = Linear(dtype, 1, 1, 64, n=n, cmax=200)
    some = [0, 1, n // 2, n - 1]
    keep = {s: x.orc[s] for s in (x.sids[i] for i in some)}
    n_tok = [65 + (i * 37) % 136 for i in range(n)]
    rows = x.rows(sum(n_tok))
    x.plan(x.sids, n_tok)
    out = x.attend(*rows)
    x.pool.plan_commit()
    at = np.cumsum([0] + n_tok)
    for i in some:
        s = x.sids[i]
        ref, mag = keep[s][0].step(*(f64(r[0, at[i]:at[i + 1]]) for r in rows))
        x.compare(out[0, at[i]:at[i + 1]], ref, mag, n_tok[i], f"session {s}")
        x.check_state(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("a", [0.0, -1e-6, -0.7, -50.0, -1e30, -3.4e38])
def test_decays(dtype, a):
    """From none to one that forgets everything at once; a second head decays mildly."""
    x = Linear(dtype, 2, 2, 64, n=2, cmax=200, log_decay=[[a, -0.1]])
    for n_tok in ([40, 150], [1, 1], [33, 1]):
        x.step(n_tok)


def test_scale():
    x = Linear("f32", 2, 1, 64, scale=3.25)
    x.step([20])
    x.step([1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_tok", [1, 25, 300])
def test_abandoned_plans_leave_the_state(dtype, n_tok):
    x = Linear(dtype, 4, 2, 128, n=2, cmax=300)
    x.step([30, 7])
    before = [x.pool.session_state(s).clone() for s in x.sids]
    x.plan(x.sids, [n_tok, 1])
    x.attend(*x.rows(n_tok + 1))
    x.pool.plan_abort()
    for s, b in zip(x.sids, before):
        assert torch.equal(x.pool.session_state(s), b)
    x.step([n_tok, 1])


def test_a_reopened_session_starts_from_nothing():
    x = Linear("bf16", 2, 2, 64, n=2)
    x.step([5, 40])
    x.step([1, 1])
    x.pool.session_close(x.sids[0])
    assert x.pool.session_open() == x.sids[0]
    x.orc[x.sids[0]] = x.fresh()
    x.step([1, 3])
    x.step([4, 1])


@pytest.mark.parametrize("n_tok", [1, 40])
def test_poisoned_dead_slots_are_never_read(n_tok):
    x = Linear("bf16", 2, 2, 128, n=2, cmax=200)
    for s in ([3, 9], [1, 1], [n_tok, 2]):
        x.pool.poison_dead()
        x.step(s)
    x.pool.session_close(x.sids[0])
    x.pool.poison_dead()
    x.pool.session_open()
    x.orc[x.sids[0]] = x.fresh()
    x.step([n_tok, n_tok])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forks_go_on_independently(dtype):
    x = Linear(dtype, 2, 2, 64, n=2, layers=3, spare=3)
    x.step([9, 20])
    x.step([1], x.sids[:1])
    new = x.pool.session_fork(x.sids[0], 3)
    for s in new:
        x.orc[s] = [o.copy() for o in x.orc[x.sids[0]]]
        x.check_state(s)
    x.sids += new
    x.step([5, 1, 2, 70 - 20, 1])
    x.step([1] * 5)
    x.pool.session_close(new[1])
    x.sids.remove(new[1])
    x.step([1, 2, 3, 4])


def test_a_fork_of_a_session_without_tokens():
    x = Linear("f32", 1, 1, 64, n=1, spare=1)
    s = x.pool.session_fork(x.sids[0])[0]
    x.orc[s] = x.fresh()
    x.sids.append(s)
    x.step([2, 3])


def test_a_state_changed_by_the_caller():
    """Saved, overwritten and put back between plans: a session goes on from it."""
    x = Linear("f32", 2, 1, 64)
    x.step([10])
    saved, orc = x.pool.session_state(x.sids[0]).clone(), [o.copy() for o in x.orc[x.sids[0]]]
    first = x.rows(4)
    a = x.step([4], rows=first)
    x.pool.session_state(x.sids[0]).copy_(saved)
    x.orc[x.sids[0]] = orc
    assert torch.equal(x.step([4], rows=first), a)


def test_plans_alternating_between_streams():
    x = Linear("bf16", 4, 2, 128, n=2, cmax=400)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for j, n_tok in enumerate(([400, 3], [1, 1], [30, 30], [1, 1], [300, 1])):
        with torch.cuda.stream(streams[j % 2]):
            x.step(n_tok)


@pytest.mark.parametrize("n_tok", [[1, 1], [25, 3], [300, 40]])
def test_a_captured_layer_replays(n_tok):
    """Replays while the plan is open, with other work between them, all give the
    eager call's outputs and state."""
    x = Linear("bf16", 4, 2, 128, n=2, cmax=300)
    x.step([12, 5])
    rows = x.rows(sum(n_tok))
    q, k, v = (r[0].cuda() for r in rows)
    side, out, g = torch.cuda.Stream(), torch.zeros_like(q), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.plan(x.sids, n_tok)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            x.pool.attend_linear(0, q, k, v, out)
        got = []
        for _ in range(4):
            out.zero_()
            torch.randn(4096, device="cuda").sort()
            g.replay()
            torch.cuda.synchronize()
            got.append(out.clone())
        x.pool.plan_commit()
    at = 0
    for s, n in zip(x.sids, n_tok):
        ref, mag = x.orc[s][0].step(*(f64(r[0, at:at + n]) for r in rows))
        for o in got:
            x.compare(o[at:at + n], ref, mag, x.orc[s][0].length, f"session {s}")
        x.check_state(s)
        at += n


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,at", [(30, 0), (30, 13), (64, 16), (64, 63), (150, 70), (400, 150), (400, 399), (1, 0)])
def test_values_that_are_not_finite_stay_with_later_tokens(dtype, d, n, at):
    """In one token's value, key or query: earlier tokens, other heads and other
    sessions are bitwise what they are without; the value's other dims too."""
    for kind in ("v", "k", "q"):
        outs, states = [], []
        for bad in (None, float("inf"), float("nan")):
            x = Linear(dtype, 4, 2, d, n=2, cmax=400, seed=n)
            x.step([6, 6])
            q, k, v = x.rows(n + 4)
            if bad is not None:
                {"q": q, "k": k, "v": v}[kind][0, at, 1, 5] = bad
            x.plan(x.sids, [n, 4])
            outs.append(x.attend(q, k, v)[0, :n + 4])
            x.pool.plan_commit()
            states.append([x.pool.session_state(s)[0].clone() for s in x.sids])
        hit = [2, 3] if kind != "q" else [1]  # query heads that see the bad row
        for o, st in zip(outs[1:], states[1:]):
            keep = torch.ones_like(outs[0], dtype=torch.bool)
            for h in hit:
                if kind == "q":
                    keep[at, h] = False
                elif kind == "k":
                    keep[at:n, h] = False
                else:
                    keep[at:n, h, 5] = False
            assert torch.equal(o[keep], outs[0][keep]), f"{kind} at {at}"
            assert not torch.isfinite(o[~keep]).any(), f"{kind} at {at}"
            assert torch.equal(st[1], states[0][1]) and torch.equal(st[0][0], states[0][0][0])
            if kind == "q":
                assert torch.equal(st[0], states[0][0])
            else:  # the key dim's column, the value dim's row of its head's state
                dim = (slice(None), 5) if kind == "k" else (5, slice(None))
                assert not torch.isfinite(st[0][1][dim]).any()
                same = torch.ones((d, d), dtype=torch.bool, device="cuda")
                same[dim] = False
                assert torch.equal(st[0][1][same], states[0][0][1][same])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_small_rows(dtype):
    """Products near both ends of fp32's range."""
    for s in (1e15, 1e-15):
        x = Linear(dtype, 2, 2, 64, n=1)
        for n in (20, 1, 40):
            x.step([n], rows=(x.draw(n, 2), x.draw(n, 2, s), x.draw(n, 2, s)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_whatever_the_cuts(dtype):
    """A prompt brought at once, in chunks and token by token ends in the same state
    within the bound of fp32 sums."""
    n = 97
    xs = [Linear(dtype, 2, 1, 128, n=1, cmax=128, seed=4) for _ in range(3)]
    rows = xs[0].rows(n)
    for x, cuts in zip(xs, ([n], [40, 1, 33, 23], [1] * n)):
        at = 0
        for c in cuts:
            x.step([c], rows=[r[:, at:at + c] for r in rows], check=c > 1)
            at += c
        x.check_state(x.sids[0])


def test_times_and_stats():
    x = Linear("bf16", 2, 2, 64, n=1, layers=2)
    x.pool.set_timing(True)
    x.step([30])
    x.step([1])
    t = x.pool.kernel_times()
    assert t["linear"][0] == 4 and t["linear"][1] > 0.0 and t["append"][0] == 2
    assert x.pool.kernel_times()["linear"] == (0, 0.0)


def test_taken_away_and_given_again():
    x = Linear("f32", 2, 2, 64, n=1)
    x.step([5])
    x.pool.session_close(x.sids[0])
    x.pool.clear_linear()
    sid = x.pool.session_open()
    z = torch.zeros((3, 1, 64), device="cuda")
    x.pool.plan_begin([sid], [3])
    x.pool.frame_append_kv(0, z, z)
    x.pool.plan_commit()  # no linear layer to bring
    x.pool.session_close(sid)
    y = Linear("bf16", 4, 1, 128, n=0, spare=1)
    y.sids, y.orc = [y.pool.session_open()], {0: y.fresh()}
    y.step([9])
    y.step([1])


@pytest.mark.parametrize("a", [-2.0 ** -14, -3e-5, -0.0123, -0.7])
def test_single_tokens_decay_without_drift(a):
    """A state that nothing is added to is e^(n a) of what it was.  Each of n steps
    rounds each of M elements on its own, by at most 2^-24 of it and at most twice (a
    standard deviation of 2^-24 sqrt(2 / 3) at most): the mean of the M relative errors
    is off by 2^-24 sqrt(2 n / (3 M)) (one deviation; six are allowed) and by what the
    decay is off, n times over: 2^-48 for two terms of 24 bits."""
    n, d = 600, 64
    x = Linear("f32", 1, 1, d, log_decay=[[a]])
    q, k, v = x.rows(1)
    x.step([1], rows=(q, torch.randn_like(k), v))
    state = x.pool.session_state(x.sids[0])
    state.copy_(torch.rand_like(state) + 0.5)
    before = f64(state)
    zero = [torch.zeros_like(r) for r in (q, k, v)]
    for _ in range(n):
        x.plan(x.sids, [1])
        x.attend(*zero)
        x.pool.plan_commit()
    got, ref = f64(x.pool.session_state(x.sids[0])), before * np.exp(n * float(np.float32(a)))
    if ref.max() < 2.0 ** -126:
        # relative errors end where fp32's normal numbers do (e^-420 is no fp32 number
        # at all); what falls below them only falls further
        assert got.min() >= 0.0 and got.max() < 2.0 ** -126
        return
    rel = got / ref - 1.0
    say(f"a {a}: mean relative error {rel.mean():.2e}")
    assert abs(rel.mean()) <= 6 * 2.0 ** -24 * np.sqrt(2 * n / (3 * d * d)) + n * 2.0 ** -48
    assert np.abs(rel).max() <= 2 * n * 2.0 ** -24


def test_refused_calls_change_nothing():
    x = Linear("bf16", 4, 2, 64, n=2, layers=2, cmax=40)
    x.step([5, 9])
    bad, n = [], 40
    rows = x.rows(n)
    q, k, v = (r[0].cuda() for r in rows)
    out = torch.full_like(q, 7.0)
    pool, sides = x.pool, torch.cuda.Stream()

    def code(fn, *args, **kw):
        try:
            fn(*args, **kw)
            return 0
        except mtn.MtnError as e:
            return e.code
    bad.append(code(pool.attend_linear, 0, q, k, v, out) == mtn.MTN_ERR_BAD_STATE)  # no plan
    x.plan(x.sids, [39, 1])
    bad.append(code(pool.plan_commit) == mtn.MTN_ERR_BAD_STATE)  # no linear layer yet
    strided = torch.cat([q, q], 2)[..., :64]
    shifted = torch.empty(q.numel() + 8, dtype=q.dtype, device="cuda")[1:1 + q.numel()].view_as(q)
    for args in ((2, q, k, v, out), (-1, q, k, v, out), (0, None, k, v, out), (0, q, None, v, out),
                 (0, q, k, None, out), (0, q, k, v, None), (0, q.float(), k, v, out), (0, strided, k, v, out),
                 (0, q, k.cpu(), v, out), (0, q, k, v, shifted)):
        bad.append(code(pool.attend_linear, *args) == mtn.MTN_ERR_INVALID_ARG)
    bad.append(code(pool.attend_linear, 0, q, k, v, out, stream=sides.cuda_stream) == mtn.MTN_ERR_INVALID_ARG)
    assert all(bad), bad
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    pool.attend_linear(0, q, k, v, out)
    assert code(pool.attend_linear, 0, q, k, v, out) == mtn.MTN_ERR_BAD_STATE  # again
    assert code(pool.plan_commit) == mtn.MTN_ERR_BAD_STATE  # the other layer
    pool.plan_abort()
    for s in x.sids:
        x.check_state(s)
    x.step([39, 1], rows=rows)


def test_states_that_set_linear_refuses():
    x = Linear("bf16", 2, 2, 64, n=1)
    shape = tuple(x.states.shape)
    for states in (None, torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape),
                   torch.zeros(shape[:-1] + (shape[-1] * 2,), device="cuda")[..., ::2],
                   torch.zeros((2,) + shape[1:], device="cuda")):
        with pytest.raises(mtn.MtnError) as e:
            x.pool.set_linear(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype="bf16",
                              log_decay=x.log_decay, states=states)
        assert e.value.code == mtn.MTN_ERR_INVALID_ARG
    x.step([9])
    x.step([1])


def test_states_past_2_to_the_31_elements():
    """1100 sessions of 2 x 2 x 32 states; the last ones lie past 2^31 elements."""
    n = 1100
    x = Linear("bf16", 32, 32, 128, n=n, layers=2, cmax=16)
    assert x.states.numel() > 2 ** 31
    last = x.sids[-2:]
    assert last == [n - 2, n - 1]
    for n_tok in ([16, 3], [1, 1], [7, 1]):
        x.step(n_tok, last)
    x.step([2], x.sids[:1])


def test_a_resized_pool_keeps_the_states():
    x = Linear("bf16", 2, 2, 64, n=2, cmax=32)
    x.step([20, 5])
    kw = dict(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, n_sink=0, window=32, max_chunk=32,
              max_sessions=2, n_blocks=16, dtype="bf16")
    x.pool.resize(16, torch.empty(mtn.Pool.required(**kw), dtype=torch.uint8, device="cuda"))
    for s in x.sids:
        x.check_state(s)
    x.step([1, 1])
    x.step([9, 32])
