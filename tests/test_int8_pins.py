"""CPU pins of the int8 block format: the oracle's codec against scalar
arithmetic, its blocks' spans and when they close, and the pool's sizes and
refusals for it (host-only pools)."""
import math
import struct

import numpy as np
import pytest

import paper_2607_02640_amd as mtn
from oracle import int8_kv
from oracle import windowed_attention as wa


def _bf16_bits(x):
    """bf16 by the integer rule on fp32 bits (x is an fp32 value)."""
    b = struct.unpack("<I", struct.pack("<f", x))[0]
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return struct.unpack("<f", struct.pack("<I", b))[0]


def test_bf16_rounding_matches_the_integer_rule():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(2000), np.ldexp(rng.standard_normal(500), rng.integers(-130, 120, 500)),
                        [0.0, 1.0, 1.00390625, 1.01171875, -1.00390625, 2.0 ** -133, 1.5 * 2.0 ** -133]])
    x = x.astype(np.float32)
    assert [_bf16_bits(float(v)) for v in x] == int8_kv.bf16(x).astype(np.float32).tolist()


def test_round_trip_is_within_half_a_step_and_keeps_the_largest():
    rng = np.random.default_rng(1)
    for n in (1, 4, 16):
        rows = int8_kv.bf16(rng.standard_normal((n, 64)) * 3)
        s = int8_kv.scale(rows)
        q = int8_kv.roundtrip_block(rows)
        assert np.max(np.abs(q - rows)) <= s / 2 * (1 + 1e-6)
        assert math.isclose(np.max(np.abs(q)), np.max(np.abs(rows)), rel_tol=1e-6)
        assert np.array_equal(q, np.rint(rows / s) * s)
    assert not int8_kv.roundtrip_block(np.zeros((16, 8))).any()


def test_codes_round_ties_to_even():
    rows = np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5]])
    assert int8_kv.scale(rows) == 1.0
    assert int8_kv.codes(rows, 1.0).tolist() == [[127, 0, 2, 2, 0, -2, 126]]


@pytest.mark.parametrize("S", [0, 1, 4, 16, 20])
def test_spans_partition_the_positions(S):
    at = 0
    while at < 200:
        lo, hi = int8_kv.block_span(at, S)
        assert lo == at and 0 < hi - lo <= 16 and (hi - lo == 16 or hi == S)
        assert all(int8_kv.block_span(p, S) == (lo, hi) for p in range(lo, hi))
        at = hi


def test_what_is_read_does_not_depend_on_the_plans():
    """The same tokens in other chunks: once a block is complete its keys read
    the same; the last rows read as they were appended."""
    rng = np.random.default_rng(2)
    k, v = int8_kv.bf16(rng.standard_normal((2, 45, 2, 16)))
    states = []
    for cuts in ([45], [1] * 45, [7, 20, 18], [16, 16, 13]):
        o = wa.OracleSession(2, 2, 16, 4, 100, kv_quant="int8_block")
        at = 0
        for c in cuts:
            o.begin(c)
            o.layer_step(0, k[at:at + c], k[at:at + c], v[at:at + c], attend=False)
            o.commit()
            at += c
        states.append(o.state[0])
    for s in states[1:]:
        for p in range(45):
            assert np.array_equal(s[p][0], states[0][p][0]) and np.array_equal(s[p][1], states[0][p][1])
    assert np.array_equal(states[0][44][1], v[44])       # position 36 + is open
    assert not np.array_equal(states[0][35][1], v[35])


def _kw(**kw):
    return dict(dict(n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=128, n_sink=4, window=40, max_chunk=9,
                     max_sessions=5, n_blocks=20, dtype="int8"), **kw)


def test_required_bytes():
    assert mtn.Pool.required(**_kw()) == 3 * 20 * (2 * 4096 + 128) + 5 * 2 * 3 * 2 * 8192
    # 17 heads: 17 * 2064 = 35088, padded to 35200; the tails begin at a multiple of 256
    kw = _kw(n_q_heads=17, n_kv_heads=17, head_dim=64, n_layers=1, n_blocks=1)
    assert mtn.Pool.required(**kw) == 35328 + 5 * 2 * 17 * 4096


@pytest.mark.parametrize("change,code", [
    (dict(head_dim=96), mtn.MTN_ERR_UNSUPPORTED),
    (dict(n_q_heads=32), mtn.MTN_ERR_UNSUPPORTED),
    (dict(n_blocks=0), mtn.MTN_ERR_INVALID_ARG),
])
def test_refusals(change, code):
    with pytest.raises(mtn.MtnError) as e:
        mtn.Pool(**_kw(**change), host_only=True)
    assert e.value.code == code


def test_f32_io_and_vector_decode_are_refused():
    pool = mtn.Pool(**_kw(), host_only=True)
    with pytest.raises(mtn.MtnError) as e:
        pool.set_decode_kernel(1)
    assert e.value.code == mtn.MTN_ERR_UNSUPPORTED
    cfg = type(pool.cfg).from_buffer_copy(pool.cfg)
    cfg.io_dtype = 0
    import ctypes as C
    n = C.c_size_t()
    assert mtn.load().mtn_pool_required_bytes(C.byref(cfg), C.byref(n)) == mtn.MTN_ERR_UNSUPPORTED
