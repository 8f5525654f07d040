"""Plans of dropit_rotary that dropit_rotary_make_plan did not write: refused before anything is launched (needs no GPU)."""
import ctypes

import pytest

from test_operator_refusals import A, INVALID, NULL, _Rotated, _plan, lib  # noqa: F401


@pytest.mark.parametrize("field, value", [("axes", 0), ("axes", -1), ("axes", 9), ("axes", 1), ("pairs", 0), ("pairs", -3), ("head_dim", 0)])
def test_sizes(lib, field, value):  # noqa: F811
    _, plan = _plan(lib, 16, (8, 8))
    setattr(plan, field, value)
    q = _Rotated(1 << 20, 1 << 20, heads=2)
    assert lib.dropit_rotary(ctypes.byref(plan), 2, 3, ctypes.byref(q), None, A, 0, 6, 2, 1, 0, 0, NULL) == INVALID


@pytest.mark.parametrize("pair", [0, 5, 7])
def test_an_axis_that_positions_do_not_have(lib, pair):  # noqa: F811
    _, plan = _plan(lib, 16, (8, 8))
    plan.axis[pair] = 2
    q = _Rotated(1 << 20, 1 << 20, heads=2)
    assert lib.dropit_rotary(ctypes.byref(plan), 2, 3, ctypes.byref(q), None, A, 0, 6, 2, 1, 0, 0, NULL) == INVALID
    plan.axis[pair], plan.axis[8] = 1, 200                  # behind the last pair it is not looked at
    broken = _Rotated(0, 1 << 20, heads=2)
    assert lib.dropit_rotary(ctypes.byref(plan), 0, 3, ctypes.byref(broken), None, A, 0, 6, 2, 1, 0, 0, NULL) == 0
