"""CPU tests of what Pool.attend_linear checks of its rows before the library is
called: a host-only pool refuses every layer itself (MTN_ERR_BAD_STATE), so another
code is the binding's."""
import pytest
import torch

import paper_2607_02640_amd as mtn

HQ, HKV, D = 4, 2, 64


def _pool(states=True):
    pool = mtn.Pool(n_layers=1, n_q_heads=4, n_kv_heads=1, head_dim=128, n_sink=4, window=32, max_chunk=8,
                    max_sessions=2, n_blocks=16, dtype="bf16", host_only=True)
    shape = mtn.Pool.linear_shape(2, 1, HKV, D)
    pool.set_linear(n_layers=1, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, log_decay=[[-0.1, 0.0]],
                    states=torch.zeros(shape) if states else None)
    return pool, [pool.session_open() for _ in range(2)]


def _rows(t, hq=HQ, hkv=HKV, d=D, dtype=torch.bfloat16):
    return [torch.zeros((t, h, d), dtype=dtype) for h in (hq, hkv, hkv, hq)]


def _code(pool, rows, layer=0):
    with pytest.raises(mtn.MtnError) as e:
        pool.attend_linear(layer, *rows)
    return e.value.code


def test_rows_short_of_the_plan_are_refused():
    pool, sids = _pool()
    pool.plan_begin(sids, [3, 2])
    assert _code(pool, _rows(5)) == mtn.MTN_ERR_BAD_STATE  # the library's
    for i in range(4):
        rows = _rows(5)
        rows[i] = rows[i][:4]
        assert _code(pool, rows) == mtn.MTN_ERR_INVALID_ARG
    pool.plan_abort()
    assert _code(pool, _rows(1)) == mtn.MTN_ERR_BAD_STATE  # no plan: the library's
    pool.plan_begin(sids[:1], [1])
    assert _code(pool, _rows(1)) == mtn.MTN_ERR_BAD_STATE
    assert _code(pool, [r[:0] for r in _rows(1)]) == mtn.MTN_ERR_INVALID_ARG


def test_rows_of_other_heads_or_head_dims_are_refused():
    pool, sids = _pool()
    pool.plan_begin(sids, [3, 2])
    for other in (dict(hq=2), dict(hkv=1), dict(d=32), dict(hq=8), dict(hkv=4), dict(d=128), dict(hq=4, hkv=1, d=128)):
        assert _code(pool, _rows(5, **other)) == mtn.MTN_ERR_INVALID_ARG, other


def test_rows_behind_the_plan_and_other_shapes_of_whole_rows_are_taken():
    pool, sids = _pool()
    pool.plan_begin(sids, [3, 2])
    for rows in (_rows(9), [r[None] for r in _rows(6)], [r.flatten(1) for r in _rows(7)], [r.flatten() for r in _rows(5)]):
        assert _code(pool, rows) == mtn.MTN_ERR_BAD_STATE


def test_rows_of_another_dtype_or_strided_are_refused():
    pool, sids = _pool()
    pool.plan_begin(sids, [3, 2])
    assert _code(pool, _rows(5, dtype=torch.float32)) == mtn.MTN_ERR_INVALID_ARG
    assert _code(pool, [r[..., :D] for r in _rows(5, d=2 * D)]) == mtn.MTN_ERR_INVALID_ARG


def test_nothing_is_checked_against_layers_that_were_taken_away():
    pool, sids = _pool()
    pool.clear_linear()
    pool.plan_begin(sids, [3, 2])
    assert _code(pool, _rows(1, dtype=torch.float32)) == mtn.MTN_ERR_BAD_STATE
    pool.plan_abort()
    pool.set_linear(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=128, log_decay=[[-0.1, 0.0]])
    pool.plan_begin(sids, [3, 2])
    assert _code(pool, _rows(5, hq=2, d=128)) == mtn.MTN_ERR_BAD_STATE


def test_rows_on_another_device_are_refused():
    pool, sids = _pool()
    pool.plan_begin(sids, [1, 1])
    assert _code(pool, [torch.empty_like(r, device="meta") for r in _rows(2)]) == mtn.MTN_ERR_INVALID_ARG


def test_one_tensor_in_two_places_is_held_against_both():
    pool, sids = _pool()
    pool.plan_begin(sids, [3, 2])
    q, k, v, out = _rows(5)
    assert _code(pool, (q, q, v, out)) == mtn.MTN_ERR_INVALID_ARG  # four heads where there are two
    assert _code(pool, (q, k, k, out)) == mtn.MTN_ERR_BAD_STATE
