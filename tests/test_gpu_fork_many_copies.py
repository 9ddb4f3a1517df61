"""A fork that may have to copy more pages than a launch has room for a workgroup each."""
import pytest
import torch

from test_gpu_pages import DEV, I32, Pool

pytestmark = pytest.mark.gpu


def test_all_cached_positions_may_be_written_again():
    import dinfer_inputs as di
    import search_ops as ops
    from paper_2510_08666_amd import binding
    columns = 2049      # 64 sequences of up to 2049 pages of 8 pieces in 16 layers: 16785408 workgroups of 256 threads, more than 2^32 threads
    pool = Pool((di, binding, ops), 150, "bf16", 16, 128, 16, max_pos=32768)
    table, held, length = [[149, 0, 7] + [-1] * (columns - 3)], [3], [33]
    refs = [1] + [0] * 6 + [1] + [0] * 141 + [1]
    parent = [0] * 40 + [-1] * 24
    rows, lens, helds, new_refs, copies, missing = ops.fork(table, held, length, refs, parent, 0, 32768, columns, 32768)
    assert missing == 0 and len(copies) == 39 * 3
    before = pool.kv.clone()
    state, new_state = torch.rand(1, 5000, device=DEV), torch.full((64, 5000), -5.0, device=DEV)
    got = pool.fork(parent, length, held, table, refs, 0, 32768, columns, [(state, new_state)])
    assert got["short"] == [0] and got["d_new_len"] == lens and got["d_new_held"] == helds and got["new_refs"] == new_refs
    assert got["d_new_page_table"] == rows
    for a, z in copies:
        before[:, z] = before[:, a]
    assert torch.equal(pool.kv, before)
    assert torch.equal(new_state[:40], state.expand(40, 5000)) and (new_state[40:] == 0).all()
    pool.close()
