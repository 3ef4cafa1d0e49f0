"""Float64 oracle of the linear-attention layers: the recurrence itself, token by
token, and the sums of magnitudes that rounding bounds are taken of.  Test
infrastructure only.

    S_t = exp(a) S_(t-1) + v_t k_t^T,    o_t = scale S_t q_t,    S = 0 before token 0
"""
from __future__ import annotations

import math

import numpy as np


class LinearState:
    """One session's state in one layer."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, log_decay, scale: float = 0.0):
        self.g = n_q_heads // n_kv_heads
        self.decay = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
        self.scale = scale or 1.0 / math.sqrt(head_dim)
        self.S = np.zeros((n_kv_heads, head_dim, head_dim))  # [head][value dim][key dim]
        self.A = np.zeros_like(self.S)                       # the same of magnitudes
        self.length = 0

    def copy(self) -> "LinearState":
        c = object.__new__(LinearState)
        c.__dict__.update(self.__dict__)
        c.S, c.A = self.S.copy(), self.A.copy()
        return c

    def step(self, q: np.ndarray, k: np.ndarray, v: np.ndarray):
        """q [n, Hq, D], k and v [n, Hkv, D]: (outputs [n, Hq, D], the outputs' sums
        of magnitudes)."""
        out, mag = np.zeros(q.shape), np.zeros(q.shape)
        for t in range(q.shape[0]):
            self.S = self.decay * self.S + v[t][:, :, None] * k[t][:, None, :]
            self.A = self.decay * self.A + np.abs(v[t][:, :, None] * k[t][:, None, :])
            for h in range(q.shape[1]):
                out[t, h] = self.scale * (self.S[h // self.g] @ q[t, h])
                mag[t, h] = self.scale * (self.A[h // self.g] @ np.abs(q[t, h]))
        self.length += q.shape[0]
        return out, mag


def all_pairs(q, k, v, log_decay, scale):
    """The outputs from all pairs of tokens: sum over j <= i of exp(a (i - j)) (q_i . k_j) v_j."""
    n, hq, _ = q.shape
    g = hq // k.shape[1]
    i = np.arange(n)
    out = np.zeros(q.shape)
    for h in range(hq):
        w = np.where(i[:, None] >= i, np.exp(log_decay[h // g] * np.maximum(i[:, None] - i, 0)), 0.0)
        out[:, h] = scale * ((q[:, h] @ k[:, h // g].T) * w) @ v[:, h // g]
    return out
