"""Helpers for the tests of the linear layers: sessions driven through the C ABI
and, in lockstep, through the float64 recurrence.

Bounds, relative to the sum of magnitudes of the products that make an element
(the same recurrence over |k|, |v|, |q|): fp32 arithmetic rounds a term at most once
per addition, 2^-24 each, on its way through a dot product of D terms, a tile's and
the tiles' sums (fewer than 2 n additions for n tokens) and a second dot product of
D; a decay e^-x computed as 2^y has |x| 2^-24 from y's rounding, twice, and is below
fp32's smallest number past x = 104: together (2 D + 2 n + 210) 2^-24.  With bf16
rows, scores and states enter an output's products in two terms: the first 8
significant bits cut off, which leaves less than 2^-7, and that rounded to 8 bits,
half a step of which is 2^-8 of it: 2^-15 each.  The output's own rounding is half a
step of 2^-7, 2^-8 of itself (spacing of 8 significant bits in [1, 2): 2^-7)."""
import numpy as np
import torch

import paper_2607_02640_amd as mtn
from oracle.linear_attention import LinearState

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


class Linear:
    """A pool with one small windowed layer and linear layers, and N sessions of it."""

    def __init__(self, dtype, hq, hkv, d, n=1, layers=1, cmax=64, log_decay=None, scale=0.0, seed=0, spare=0):
        self.dtype, self.hq, self.hkv, self.d, self.layers = dtype, hq, hkv, d, layers
        ring = -(-(32 + cmax - 1) // 16)
        kw = dict(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, n_sink=0, window=32, max_chunk=cmax,
                  max_sessions=n + spare, n_blocks=(n + spare) * ring, dtype=dtype)
        self.pool = mtn.Pool(**kw, kv=torch.empty(mtn.Pool.required(**kw), dtype=torch.uint8, device="cuda"))
        rng = np.random.default_rng(seed)
        if log_decay is None:
            log_decay = -np.exp2(-8.0 * (np.arange(hkv) + 1) / hkv) * np.linspace(1.0, 0.2, layers)[:, None]
        self.log_decay = np.broadcast_to(np.asarray(log_decay, np.float32), (layers, hkv))
        # garbage where no plan has written yet
        self.states = torch.full(mtn.Pool.linear_shape(n + spare, layers, hkv, d), float("nan"), device="cuda")
        self.scale = scale
        self.pool.set_linear(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, scale=scale,
                             log_decay=self.log_decay, states=self.states)
        self.sids = [self.pool.session_open() for _ in range(n)]
        self.orc = {s: self.fresh() for s in self.sids}
        self.rng = rng
        self.worst = 0.0  # largest error over its bound

    def fresh(self):
        return [LinearState(self.hq, self.hkv, self.d, self.log_decay[l], self.scale) for l in range(self.layers)]

    def draw(self, n, h, scale=1.0):
        x = torch.from_numpy((self.rng.standard_normal((self.layers, n, h, self.d)) * scale).astype(np.float32))
        return x.to(TDT[self.dtype])

    def rows(self, n):
        return self.draw(n, self.hq), self.draw(n, self.hkv), self.draw(n, self.hkv)

    def plan(self, sids, n_tok):
        """Open a plan with its windowed layer appended."""
        self.pool.plan_begin(sids, n_tok)
        z = torch.zeros((sum(n_tok), 1, 64), dtype=TDT[self.dtype], device="cuda")
        self.pool.frame_append_kv(0, z, z)

    def attend(self, q, k, v):
        """Every layer of the open plan: outputs with one guard row behind them."""
        n = q.shape[1]
        out = torch.full((self.layers, n + 1, self.hq, self.d), 7.0, dtype=TDT[self.dtype], device="cuda")
        for l in range(self.layers):
            self.pool.attend_linear(l, *(x[l].contiguous().cuda() for x in (q, k, v)), out[l])
        return out

    def step(self, n_tok, sids=None, rows=None, check=True):
        sids = self.sids if sids is None else sids
        q, k, v = rows if rows is not None else self.rows(sum(n_tok))
        self.plan(sids, n_tok)
        out = self.attend(q, k, v)
        self.pool.plan_commit()
        torch.cuda.synchronize()
        assert bool((out[:, -1] == 7.0).all()), "a row behind the last token was written"
        at = 0
        for s, n in zip(sids, n_tok):
            for l in range(self.layers):
                ref, mag = self.orc[s][l].step(*(f64(x[l, at:at + n]) for x in (q, k, v)))
                if check:
                    self.compare(out[l, at:at + n], ref, mag, self.orc[s][l].length, f"session {s} layer {l}")
            at += n
            if check:
                self.check_state(s)
        return out[:, :-1]

    def bound(self, n):
        return (2 * self.d + 2 * n + 210) * 2.0 ** -24

    def compare(self, got, ref, mag, n, what):
        tol = self.bound(n) * mag + 1e-37
        if self.dtype == "bf16":
            tol = tol + 2 * 2.0 ** -15 * mag
            tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
        self._within(f64(got), ref, tol, what)

    def check_state(self, s):
        got = f64(self.pool.session_state(s))
        for l in range(self.layers):
            o = self.orc[s][l]
            self._within(got[l], o.S, self.bound(o.length) * o.A + 1e-37, f"state of session {s} layer {l}")

    def _within(self, got, ref, tol, what):
        assert np.isfinite(got).all(), f"{what}: not finite"
        off = np.abs(got - ref) / tol
        self.worst = max(self.worst, float(off.max()))
        assert off.max() <= 1.0, f"{what}: {off.max():.2f} of the bound, at {np.unravel_index(off.argmax(), off.shape)}"
