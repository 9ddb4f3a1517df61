"""What the cache's operators and rotary tables refuse without a GPU."""
import ctypes

import pytest

from paper_2510_08666_amd import binding as b


def size(**kw):
    return b.lib.dinfer_rotary_table_bytes(ctypes.byref(b.rotary(**kw)), 100)


def test_rotary_tables():
    assert size(rotary_dim=64) == 64 * 400 and size(rotary_dim=20, interleaved=True, scaling="ntk", factor=2.0) == 20 * 400
    assert size(rotary_dim=128, scaling="yarn", factor=8.0, original_positions=2048) == 128 * 400
    for kw in (dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=130), dict(rotary_dim=64, theta=0.0), dict(rotary_dim=64, theta=float("inf")),
               dict(rotary_dim=64, scaling="linear", factor=0.0), dict(rotary_dim=64, scaling="linear", factor=float("nan")),
               dict(rotary_dim=2, scaling="ntk", factor=2.0), dict(rotary_dim=64, scaling="yarn", factor=2.0),
               dict(rotary_dim=64, scaling="yarn", factor=2.0, original_positions=64, theta=1.0),
               dict(rotary_dim=64, scaling="yarn", factor=2.0, original_positions=64, beta_fast=1.0, beta_slow=2.0),
               dict(rotary_dim=64, scaling="yarn", factor=2.0, original_positions=64, magnitude=-1.0)):
        assert size(**kw) == 0, kw
        assert b.last_error() != ""
    r = b.rotary(64)
    r.scaling = 4
    assert b.lib.dinfer_rotary_table_bytes(ctypes.byref(r), 100) == 0
    r = b.rotary(64)
    for n in (0, -1, 32769):
        assert b.lib.dinfer_rotary_table_bytes(ctypes.byref(r), n) == 0
    assert b.lib.dinfer_rotary_table_bytes(None, 100) == 0
    assert b.lib.dinfer_rotary_table(ctypes.byref(r), 100, None, 1 << 20, None) == -1
    assert b.lib.dinfer_rotary_table(ctypes.byref(r), 100, 0x1004, 1 << 20, None) == -1 and "aligned" in b.last_error()
    assert b.lib.dinfer_rotary_table(ctypes.byref(r), 100, 0x1000, 64 * 400 - 1, None) == -3


def test_null_contexts():
    use = b.CacheUse()
    assert b.lib.dinfer_kv_append(None, 0, 1, None, None, None, 1, None, 0, None, 0, None, 0, 1, None, None, 0.0, None, None, 0, None,
                                  None, 0, None) == -1
    assert b.lib.dinfer_attend(None, 0, 1, None, None, None, 1, None, 0, 1, None, 0.0, None, 0, None, None) == -1
    assert b.lib.dinfer_kv_score(None, 0, 1, None, None, None, 1, None, 0, 1, None, 0.0, None, 0, 1.0, None, None, 1, None) == -1
    assert b.lib.dinfer_kv_evict(None, 0, 1, 1, 1, 0, 0, None, 1, None, None, 1, None, 1, None, None, None, None) == -1
    assert b.lib.dinfer_step_scored(None, 1, 32, None, None, None, None, 1, None, ctypes.byref(use), None, None, None, None) == -1
    assert b.lib.dinfer_step_scored(None, 1, 32, None, None, None, None, 1, None, None, None, None, None, None) == -1
    assert b.lib.dinfer_refresh_block_scored(None, 1, 32, None, None, None, 1, ctypes.byref(use), None) == -1
