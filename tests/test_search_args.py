"""What the operators of a search refuse without a GPU."""
import ctypes

import pytest
import torch

from paper_2510_08666_amd import binding as b
from test_cache_binding import Host


def test_null_contexts():
    rule = b.AttendRule()
    assert b.lib.dinfer_attend_ruled(None, 0, 1, None, None, None, 1, None, 0, 1, ctypes.byref(rule), 0.0, None, 0, None, None) == -1
    assert b.lib.dinfer_kv_fork(None, 0, 1, None, None, None, None, 0, 0, 0, None, None, None, None, 1, None, None, None, 0, None) == -1
    assert b.lib.dinfer_kv_compact(None, 1, None, None, 1, None, None, None, None, None, None) == -1
    assert b.last_error() == "context is null"


def test_select():
    size = b.lib.dinfer_beam_scratch_bytes
    assert size(1, 1, 1, 1) > 0 and size(8, 64, 157184, 16) >= 8 * 64 * 77 * 8 and size(63, 1024, 100, 64) > 0
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1025, 1, 1), (64, 1024, 1, 1), (1, 1, 0, 1), (1, 1, (1 << 24) + 1, 1), (1, 1, 1, 0), (1, 1, 1, 65)):
        assert size(*bad) == 0 and b.last_error() != "", bad
    good = [0x1000, b.F32, 9, 1, 2, 9, 0x2000, None, 3, 0x3000, 0x4000, 0x5000, 0x6000, 1 << 20, None]
    for at, value in ((0, None), (6, None), (9, None), (10, None), (11, None), (12, None), (1, 2), (2, 8), (3, 0), (4, 1025), (5, 0), (8, 65), (0, 0x1002),
                      (11, 0x2000), (10, 0x3000), (12, 0x6010)):
        args = list(good)
        args[at] = value
        assert b.lib.dinfer_beam_select(*args) == -1, (at, value)
    args = list(good)
    args[13] = size(1, 2, 9, 3) - 1
    assert b.lib.dinfer_beam_select(*args) == -3
    with pytest.raises(b.DinferError):
        b.beam_scratch(1, 1, 1, 65, device="cpu")
    z = torch.zeros(1, 2, 9)
    with pytest.raises(ValueError):      # no tensor of a GPU
        b.beam_select(z, torch.zeros(1, 2), torch.zeros(1, 3, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32), torch.zeros(1, 3), torch.zeros(9, dtype=torch.uint8))


def test_missing_tensors_and_wrong_dimensions():
    c = Host(2, 64)
    c.n_pages = 7
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    rows, table = torch.zeros(3, 128), i(1, 4)
    ruled = dict(layer=0, lens=[3], d_past=None, d_page_table=table, d_q=rows, d_out=rows)
    fork = dict(parent=i(2), d_len=i(1), d_held=i(1), d_page_table=table, refs=i(7), d_new_len=i(2), d_new_held=i(2), d_new_page_table=i(2, 4), new_refs=i(7), short=i(1))
    pack = dict(d_held=i(1), d_page_table=table, refs=i(7), d_new_page_table=i(1, 4), new_refs=i(7), moved=i(2, 7), count=i(2))
    for fn, base in ((c.attend_ruled, ruled), (c.kv_fork, fork), (c.kv_compact, pack)):
        with pytest.raises(b.DinferError):      # what fits reaches the library, which knows no such context
            fn(**base)
        for name, t in base.items():
            if isinstance(t, torch.Tensor) and t.dim() > 1:
                with pytest.raises(ValueError, match=name):
                    fn(**{**base, name: t.reshape(-1)})
            if isinstance(t, torch.Tensor):
                with pytest.raises(ValueError, match=name):
                    fn(**{**base, name: t.double()})
    for bad in (dict(prefix=i(2, 1)), dict(first=i(2)), dict(end=torch.zeros(3)), dict(slope=torch.zeros(1)), dict(lse=torch.zeros(3))):
        with pytest.raises(ValueError, match=list(bad)[0]):
            c.attend_ruled(**ruled, **bad)
    with pytest.raises(ValueError, match="state 0"):
        c.kv_fork(**fork, states=[(i(1, 2), i(2, 3))])
