"""The tests' own MXFP4 reference, and the refusals of the cache calls that need no device."""
import ctypes

import numpy as np
import pytest

from tests import mx_ref


def test_every_element_and_exponent_is_its_own_rounding():
    for e in range(-23, 14):
        x = np.zeros((1, 32))
        x[0, :8], x[0, 8:16] = mx_ref.MAGNITUDES * 2.0 ** e, -mx_ref.MAGNITUDES * 2.0 ** e
        assert np.array_equal(mx_ref.stored(x), x), e


def test_roundings_are_off_by_at_most_half_a_step():
    """A block's elements are within half the distance to the next one: a quarter of the exponent's unit below 2, half
    of it below 4, one unit up to 6, where the largest of a block is below 7 units."""
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(4000, 128)) * np.exp(rng.uniform(-8, 8, size=(4000, 1)))).astype(np.float32)
    h = x.astype(np.float16).astype(np.float64).reshape(-1, 32)
    y = mx_ref.stored(x).reshape(-1, 32)
    top = np.abs(h).max(-1, keepdims=True)
    unit = 2.0 ** (np.floor(np.log2(top)) - 2)
    unit = np.where(top / unit >= 7, 2 * unit, unit)
    a = np.abs(h) / unit
    assert a.max() < 7
    assert np.all(np.abs(y - h) / unit <= np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0)))


def test_ties_go_to_the_even_element():
    x = np.zeros((1, 32))
    x[0, :9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]
    assert np.array_equal(mx_ref.stored(x)[0, :9], [6, 0, 1, 1, 2, 2, 4, 4, -4])


def test_refusals_before_touching_the_device():
    from paper_2609_34045_amd import stage
    lib = stage.load_library()
    out = ctypes.c_void_p(123)
    assert lib.kf_kv_create_typed(None, 1, 64, 0, 1, ctypes.byref(out)) == 1 and out.value is None
    assert lib.kf_kv_create_typed(ctypes.c_void_p(8), 1, 64, -1, 1, ctypes.byref(out)) == 1
    assert b"n_pages" in lib.kf_last_error()
    assert lib.kf_kv_create_typed(ctypes.c_void_p(8), 1, 64, 0, 2, ctypes.byref(out)) == 1
    assert b"type" in lib.kf_last_error()
    assert lib.kf_kv_create_typed(ctypes.c_void_p(8), 1, 64, 0, 1, None) == 1
    assert lib.kf_kv_format(None, None, None) == 1
    assert lib.kf_kv_copy(None, 0, None, 0, 0, 1) == 1
    assert lib.kf_kv_fork(None, 0, 1, 0) == 1
    assert lib.kf_kv_attend(None, 0, 1, None, None, None, 0, None) == 1
    with pytest.raises(ValueError, match="dtype"):
        stage.KV(None, 1, 64, dtype="int4")
