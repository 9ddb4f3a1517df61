"""What the cache's operators refuse without a GPU, in the library and in its binding."""
import ctypes
import math

import pytest
import torch

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


class Host(b.Context):
    """A context's checks of its arguments on host tensors; nothing of the library behind it."""

    def __init__(self, heads, head_dim, layers=1):
        self.cfg = type("Heads", (), dict(n_heads=heads, head_dim=head_dim, n_layers=layers))
        self.h, self._dtype, self._index = None, torch.float32, -1      # (where host tensors are)

    def _raw_stream(self):
        return 0


def test_missing_tensors_and_wrong_dimensions():
    c = Host(2, 64)
    rows, table = torch.zeros(3, 128), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(b.DinferError):      # what fits reaches the library, which knows no such context
        c.kv_append(0, [3], None, table, rows, rows, rows, rows)
    append = dict(layer=0, lens=[3], d_past=None, d_page_table=table, d_q=rows, d_k=rows, d_v=rows, d_q_out=rows)
    attend = dict(layer=0, lens=[3], d_past=None, d_page_table=table, d_q=rows, d_out=rows)
    score = dict(layer=0, lens=[3], d_past=None, d_page_table=table, d_q=rows, d_score_out=torch.zeros(1, 2, 9))
    evict = dict(first_layer=0, n_layers=1, keep=5, n_sink=0, n_recent=0, d_score=torch.zeros(1, 1, 2, 9), d_len=torch.zeros(1, dtype=torch.int32),
                 d_page_table=table, d_new_page_table=table.clone(), d_kept=torch.zeros(1, 1, 2, 5, dtype=torch.int32),
                 d_new_len=torch.zeros(1, dtype=torch.int32))
    for fn, base, names in ((c.kv_append, append, ("d_page_table", "d_k", "d_v", "d_q_out")), (c.attend, attend, ("d_page_table", "d_q", "d_out")),
                            (c.kv_score, score, ("d_page_table", "d_q", "d_score_out")),
                            (c.kv_evict, evict, ("d_page_table", "d_new_page_table", "d_score"))):
        with pytest.raises(b.DinferError):
            fn(**base)
        for n in names:
            for bad in (None, base[n].reshape(-1)):
                with pytest.raises(ValueError, match=n):
                    fn(**{**base, n: bad})
    with pytest.raises(ValueError, match="rotary_table"):
        c.kv_append(**append, rotary=b.rotary(64), rotary_table=torch.zeros(64))
    with pytest.raises(ValueError, match="score_out"):
        c._cache_use(1, None, None, torch.zeros(9), 1.0)


def test_rotary_table_of_another_gpu(monkeypatch):
    """The table is filled by the GPU that holds it, on that GPU's stream: the library is called with that one current."""
    current, calls = ["cuda:0"], []

    class Current:
        def __init__(self, device):
            self.device, self.old = str(device), None

        def __enter__(self):
            self.old, current[0] = current[0], self.device

        def __exit__(self, *_):
            current[0] = self.old

    class Lib:
        @staticmethod
        def dinfer_rotary_table_bytes(rot, n):
            return 64 * 4 * n

        @staticmethod
        def dinfer_rotary_table(rot, n, table, size, stream):
            calls.append((current[0], stream))
            return 0

    class Table:
        device = "cuda:1"

    monkeypatch.setattr(b, "lib", Lib)
    monkeypatch.setattr(b, "_stream", lambda: "stream of " + current[0])
    monkeypatch.setattr(b, "_ptr", lambda t: 0)
    monkeypatch.setattr(b.torch.cuda, "device", Current)
    monkeypatch.setattr(b.torch, "empty", lambda *a, **kw: Table())
    b.rotary_table(b.rotary(64), 100, "cuda:1")
    assert calls == [("cuda:1", "stream of cuda:1")] and current == ["cuda:0"]
