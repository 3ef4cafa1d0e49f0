"""A hybrid model's layers together, as a serving loop runs them: windowed layers
with normed queries and keys and linear layers of other heads in turn under one
plan, chunks and single tokens, forks, abandoned plans, sessions that come and go,
a captured frame; all against the float64 oracles of both kinds."""
import copy

import numpy as np
import pytest
import torch

import paper_2607_02640_amd as mtn
from oracle import windowed_attention as wa
from tests._gpu_util import TDT, TOL, make_pool, say
from tests._linear_util import Linear, f64

pytestmark = pytest.mark.gpu

ORDER = [("w", 0), ("l", 0), ("l", 1), ("w", 1), ("l", 2)]
EPS = 1e-6


class Hybrid(Linear):
    """Two windowed layers (4 query, 2 KV heads of 128) and three linear ones."""

    W = dict(hq=4, hkv=2, d=128, S=4, W=40)

    def __init__(self, dtype, hq, hkv, d, n=2, spare=2, cmax=100, form=None, seed=0):
        io = "f32" if dtype == "f32" else "bf16"
        self.dtype, self.kv, self.hq, self.hkv, self.d, self.layers, self.scale = io, dtype, hq, hkv, d, 3, 0.0
        w, self.form = self.W, form
        ring = -(-(w["W"] + cmax - 1) // 16) + 1
        self.pool = make_pool(n_layers=2, cmax=cmax, max_sessions=n + spare, n_blocks=(n + spare) * ring,
                              dtype=dtype, **w)
        self.rng = np.random.default_rng(seed)
        self.weights = [self.rng.uniform(0.6, 1.4, (2, w["d"])).astype(np.float32) for _ in range(2)]
        if form:
            self.pool.set_rope(**form)
        self.pool.set_qk_norm(*self.weights, EPS)
        self.log_decay = -self.rng.uniform(0.01, 0.9, (3, hkv)).astype(np.float32)
        self.states = torch.full(mtn.Pool.linear_shape(n + spare, 3, hkv, d), float("nan"), device="cuda")
        self.pool.set_linear(n_layers=3, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=io,
                             log_decay=self.log_decay, states=self.states)
        self.sids = [self.pool.session_open() for _ in range(n)]
        self.orc = {s: self.fresh() for s in self.sids}
        self.win = {s: self.fresh_windowed() for s in self.sids}
        self.worst = 0.0

    def fresh_windowed(self):
        w = self.W
        o = wa.OracleSession(w["hq"], w["hkv"], w["d"], w["S"], w["W"], n_layers=2,
                             kv_quant={"fp8": "fp8_e4m3", "int8": "int8_block"}.get(self.kv), rope=self.form)
        o.qk_norm = (*self.weights, EPS)
        return o

    def wrows(self, n):
        w = self.W
        return [torch.from_numpy(self.rng.standard_normal((2, n, h, w["d"])).astype(np.float32)).to(TDT[self.kv])
                for h in (w["hq"], w["hkv"], w["hkv"])]

    def run(self, n_tok, wrows, rows, wout, out, fused=False):
        """Every layer of the open plan, in the model's order."""
        for kind, l in ORDER:
            if kind == "l":
                self.pool.attend_linear(l, *(x[l] for x in rows), out[l])
            elif max(n_tok) == 1 and fused:
                self.pool.attend_decode_append(l, wrows[1][l], wrows[2][l], wrows[0][l], wout[l])
            else:
                self.pool.frame_append_kv(l, wrows[1][l], wrows[2][l])
                if max(n_tok) == 1:
                    self.pool.attend_decode(l, wrows[0][l], wout[l])
                else:
                    self.pool.attend_chunk_prefill(l, wrows[0][l], wout[l])

    def verify(self, sids, n_tok, wrows, rows, wout, out):
        at = 0
        for s, n in zip(sids, n_tok):
            o = self.win[s]
            o.begin(n)
            for l in range(2):
                ref = o.layer_step(l, *(f64(x[l, at:at + n]) for x in wrows))[0]
                got = f64(wout[l, at:at + n])
                assert np.isfinite(got).all()
                err = np.abs(got - ref).max()
                assert err <= TOL[self.kv], f"windowed layer {l} of session {s}: {err:.3e}"
            o.commit()
            for l in range(3):
                ref, mag = self.orc[s][l].step(*(f64(x[l, at:at + n]) for x in rows))
                self.compare(out[l, at:at + n], ref, mag, self.orc[s][l].length, f"linear layer {l} of session {s}")
            self.check_state(s)
            at += n

    def draw_frame(self, n):
        wrows, rows = self.wrows(n), self.rows(n)
        return [x.cuda() for x in wrows], [x.cuda() for x in rows]

    def frame(self, n_tok, sids=None, fused=False, abandon=False):
        sids = self.sids if sids is None else sids
        wrows, rows = self.draw_frame(sum(n_tok))
        wout, out = torch.empty_like(wrows[0]), torch.empty_like(rows[0])
        self.pool.plan_begin(sids, n_tok)
        self.run(n_tok, wrows, rows, wout, out, fused)
        if abandon:
            self.pool.plan_abort()
            return
        self.pool.plan_commit()
        torch.cuda.synchronize()
        self.verify(sids, n_tok, wrows, rows, wout, out)


CASES = [("bf16", 4, 4, 64, None), ("bf16", 8, 2, 128, dict(layout="interleaved", rotary_dim=32)),
         ("fp8", 4, 1, 128, None), ("int8", 2, 2, 64, dict(layout="half", rotary_dim=32)),
         ("f32", 4, 2, 64, dict(layout="interleaved"))]


@pytest.mark.parametrize("dtype,hq,hkv,d,form", CASES)
def test_frames(dtype, hq, hkv, d, form):
    say(f"hybrid frames {dtype} linear {hq}/{hkv} D={d} form {form}")
    x = Hybrid(dtype, hq, hkv, d, form=form)
    x.frame([90, 7])
    for fused in (False, True):
        x.frame([1, 1], fused=fused)
    x.frame([20, 33])
    x.frame([40, 1], abandon=True)
    x.frame([1], x.sids[1:], fused=True)
    x.frame([1, 1], abandon=True)
    x.frame([3, 64])
    say(f"  worst linear output {x.worst:.3f} of the bound")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sessions_that_fork_close_and_open(dtype):
    x = Hybrid(dtype, 4, 2, 64, n=1, spare=2)
    x.frame([50])
    x.frame([1])
    new = x.pool.session_fork(x.sids[0], 2)
    for s in new:
        x.win[s] = copy.deepcopy(x.win[x.sids[0]])
        x.orc[s] = [o.copy() for o in x.orc[x.sids[0]]]
    x.sids += new
    x.frame([1, 9, 70])
    x.frame([1, 1, 1], fused=True)
    x.pool.session_close(new[0])
    x.pool.poison_dead()
    assert x.pool.session_open() == new[0]
    x.win[new[0]], x.orc[new[0]] = x.fresh_windowed(), x.fresh()
    x.frame([2, 30, 1])
    x.frame([1, 1, 1], x.sids[::-1])


@pytest.mark.parametrize("n_tok", [[1, 1], [33, 5]])
def test_a_captured_frame_replays(n_tok):
    """All layers of an open plan in one graph, replayed with eager work of another
    pool of the same shapes between; every replay gives the frame's outputs."""
    x, y = Hybrid("bf16", 4, 2, 128), Hybrid("bf16", 4, 2, 128, seed=1)
    x.frame([30, 12])
    y.frame([9, 9])
    wrows, rows = x.draw_frame(sum(n_tok))
    wout, out = torch.zeros_like(wrows[0]), torch.zeros_like(rows[0])
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    got = []
    with torch.cuda.stream(side):
        x.pool.plan_begin(x.sids, n_tok)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            x.run(n_tok, wrows, rows, wout, out)
        for _ in range(3):
            wout.zero_()
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            got.append((wout.clone(), out.clone()))
            y.frame([n_tok[0], 2])
        x.pool.plan_commit()
    for a, b in got[1:]:
        assert torch.equal(a, got[0][0]) and torch.equal(b, got[0][1])
    x.verify(x.sids, n_tok, wrows, rows, *got[0])
    x.frame([4, 1])
