"""Int8 KV blocks: what a cache holds of a block of rows under one scale.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

Per-token KV reduction composes with the window (Metronome, arXiv 2607.02640
§4.1 and §6); the paper names no format, so the definition is this one: rows are
bf16 (keys rotated first); a block of rows of one head is quantized when its last
position is appended, with s = max|x| / 127 rounded to fp32 (1 where every row is
zero) and code = x / s rounded to the nearest integer, ties to even; a key of a
complete block reads as code * s, one of the open block as its bf16 row.
Parity: pinned by tests against scalar arithmetic; the GPU kernels are compared
with ``OracleSession(kv_quant="int8_block")``.
"""
from __future__ import annotations

from typing import Tuple

import numpy as np

BLOCK = 16


def bf16(x: np.ndarray) -> np.ndarray:
    """x rounded to bfloat16 (eight significant bits, ties to even; subnormals as
    multiples of 2^-133)."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 8, -133))
    return np.rint(x / step) * step


def scale(rows: np.ndarray) -> float:
    """Scale of a block's rows (one head, one tensor)."""
    top = np.max(np.abs(rows))
    return float(np.float32(top) / np.float32(127.0)) if top > 0 else 1.0


def codes(rows: np.ndarray, s: float) -> np.ndarray:
    return np.clip(np.rint(np.asarray(rows, np.float64) / s), -127, 127)


def roundtrip_block(rows: np.ndarray) -> np.ndarray:
    """Rows [n, D] of one head as their complete block reads."""
    s = scale(rows)
    return codes(rows, s) * s


def block_span(pos: int, n_sink: int) -> Tuple[int, int]:
    """Half-open positions of the block that holds ``pos``: the sinks' blocks
    from 0 on, the last one cut at S, then blocks of 16 from S on."""
    if pos < n_sink:
        lo = pos // BLOCK * BLOCK
        return lo, min(lo + BLOCK, n_sink)
    lo = n_sink + (pos - n_sink) // BLOCK * BLOCK
    return lo, lo + BLOCK
