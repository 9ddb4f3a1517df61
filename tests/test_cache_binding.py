"""What the cache's operators refuse without a GPU, in the library and in its binding."""
import ctypes
import math

import pytest

from paper_2510_08666_amd import binding as b


def size(**kw):
    return b.lib.dinfer_rotary_table_bytes(ctypes.byref(b.rotary(64, **kw)), 100)


def test_rotary_rules_stay_in_float32s_range():
    """Angles are worked out in double from rules in double: no base or factor may lead them out of it."""
    assert size(theta=1e38) and size(scaling="ntk", theta=1e38, factor=1e38) and size(scaling="linear", factor=1e-37)
    for kw in (dict(theta=1e39), dict(theta=1e-39), dict(scaling="linear", factor=1e39), dict(scaling="linear", factor=1e-39),
               dict(scaling="yarn", factor=2.0, original_positions=64, magnitude=1e39), dict(theta=math.nan), dict(theta=-1.0)):
        assert size(**kw) == 0, kw
        assert b.last_error() != ""
