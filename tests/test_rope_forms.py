"""CPU tests of the rotary forms: the oracle's against their definition, and
the refusals of mtn_pool_set_rope (host-only pools)."""
import math

import numpy as np
import pytest

import paper_2607_02640_amd as mtn
from oracle import windowed_attention as wa


def _pool(d=128, dtype="bf16", **kw):
    return mtn.Pool(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=d, n_sink=4, window=32, max_chunk=8,
                    max_sessions=2, n_blocks=20, dtype=dtype, host_only=True, **kw)


def test_half_whole_rows_are_the_default_form():
    x = np.random.default_rng(0).standard_normal((3, 128))
    assert np.allclose(wa.rope_form(x, 777, 1e6), wa.rope_rotate(x, 777, 1e6), rtol=0, atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "yarn"])
@pytest.mark.parametrize("rd", [16, 48, 128])
def test_scores_depend_on_distance_only(layout, scaling, rd):
    """Rotations of a pair keep q . k a function of the positions' distance, and
    a rotated row's length is m times the original's over the rotated part."""
    rng = np.random.default_rng(rd)
    q, k = rng.standard_normal((2, 128))
    kw = dict(layout=layout, rotary_dim=rd, scaling=scaling, factor=4.0, original_len=256)
    dots = [wa.rope_form(q, p + 37, 1e4, **kw) @ wa.rope_form(k, p, 1e4, **kw) for p in (0, 5, 1000)]
    assert np.allclose(dots, dots[0], rtol=0, atol=1e-9)
    m = 0.1 * math.log(4.0) + 1.0 if scaling == "yarn" else 1.0
    y = wa.rope_form(q, 91, 1e4, **kw)
    assert np.isclose(np.linalg.norm(y[:rd]), m * np.linalg.norm(q[:rd]))
    assert np.array_equal(y[rd:], q[rd:])


def test_scalings_move_the_frequencies_they_name():
    def angle(i, **kw):  # of the unit vector of pair i, one position on
        x = np.zeros(128)
        x[i] = 1.0
        y = wa.rope_form(x, 1, 1e4, **kw)
        return math.atan2(y[i + 64], y[i])
    for i in (0, 20, 63):
        f = 1e4 ** (-i / 64)
        assert math.isclose(angle(i), f)
        assert math.isclose(angle(i, scaling="linear", factor=8.0), f / 8)
    # the fastest pair turns 4096 / 2 pi times over the trained length, the
    # slowest less than once: kept, and divided
    yarn = dict(scaling="yarn", factor=4.0, original_len=4096)
    assert math.isclose(angle(0, **yarn), 1.0)
    assert math.isclose(angle(63, **yarn), 1e4 ** (-63 / 64) / 4)
    assert angle(63, scaling="base", factor=4.0) < 1e4 ** (-63 / 64)
    assert math.isclose(angle(0, scaling="base", factor=4.0), 1.0)


@pytest.mark.parametrize("kw,code", [
    (dict(rotary_dim=24), mtn.MTN_ERR_UNSUPPORTED),
    (dict(rotary_dim=8), mtn.MTN_ERR_UNSUPPORTED),
    (dict(rotary_dim=144), mtn.MTN_ERR_INVALID_ARG),
    (dict(rotary_dim=-16), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="linear", factor=0.5), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="linear", factor=math.nan), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="base", factor=math.inf), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="base", factor=1e300), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="yarn", factor=4.0), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="yarn", factor=4.0, original_len=64, beta_fast=1.0, beta_slow=2.0), mtn.MTN_ERR_INVALID_ARG),
    (dict(scaling="yarn", factor=4.0, original_len=64, beta_slow=-1.0), mtn.MTN_ERR_INVALID_ARG),
    (dict(magnitude=-1.0), mtn.MTN_ERR_INVALID_ARG),
    (dict(magnitude=math.nan), mtn.MTN_ERR_INVALID_ARG),
    (dict(magnitude=1025.0), mtn.MTN_ERR_INVALID_ARG),
])
def test_bad_forms_are_refused(kw, code):
    with pytest.raises(mtn.MtnError) as e:
        _pool().set_rope(**kw)
    assert e.value.code == code


def test_form_is_fixed_while_a_session_holds_tokens():
    pool = _pool(dtype="f32")
    sid = pool.session_open()
    pool.set_rope(layout="interleaved")  # open, but empty
    pool.plan_begin([sid], [3])
    with pytest.raises(mtn.MtnError) as e:
        pool.set_rope()
    assert e.value.code == mtn.MTN_ERR_BAD_STATE
    pool.plan_commit()
    with pytest.raises(mtn.MtnError) as e:
        pool.set_rope()
    assert e.value.code == mtn.MTN_ERR_BAD_STATE
    pool.session_close(sid)
    pool.set_rope(rotary_dim=64, scaling="yarn", factor=2.0, original_len=100)
    lib = mtn.load()
    assert lib.mtn_pool_set_rope(pool.h, None) == mtn.MTN_ERR_INVALID_ARG
    assert lib.mtn_pool_set_rope(None, None) == mtn.MTN_ERR_INVALID_ARG
