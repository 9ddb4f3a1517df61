"""Workgroups of a fork's second launch (csrc/fork_plan.hpp), compiled for the host."""
import ctypes

import pytest

import host_shim

SHIM = """
#include "fork_plan.hpp"
extern "C" int grid(int n_old, int n_new, const int64_t* rows, int n_states, int columns, int n_layers, int64_t page_bytes, int* out) {
  dinfer::ForkGrid g{};
  const bool fits = dinfer::fork_grid(n_old, n_new, rows, n_states, columns, n_layers, page_bytes, &g);
  out[0] = g.state0, out[1] = g.page0, out[2] = g.pieces, out[3] = g.page_groups;
  for (int k = 0; k < dinfer::MAX_STATES; ++k) out[4 + k] = g.state_pieces[k];
  return fits;
}
"""


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    lib = host_shim.load(tmp_path_factory.mktemp("fork_plan"), SHIM)

    def of(n_old, n_new, rows, columns, n_layers, page_bytes):
        out = (ctypes.c_int * 12)()
        fits = lib.grid(n_old, n_new, (ctypes.c_int64 * 8)(*rows), len(rows), columns, n_layers, ctypes.c_int64(page_bytes), out)
        return bool(fits), list(out)
    return of


def test_small_forks_have_a_workgroup_for_every_piece(grid):
    fits, g = grid(1, 4, [4, 16384, 16385], 2, 1, 131072)
    assert fits and g[:7] == [5, 5 + 4 * 4, 8, 4 * 2 * 8, 1, 1, 2]
    assert grid(0, 1, [], 1, 1, 4096) == (True, [1, 1, 1, 1] + [0] * 8)


def test_no_more_threads_than_a_launch_counts(grid):
    """64 sequences of 2049 pages of 8 pieces in 16 layers are 16785408 pieces, 2^32 threads and more; states alone may be as many."""
    fits, g = grid(64, 64, [], 2049, 16, 131072)
    assert fits and g[3] == 16384
    for row, n, expected in ((2 ** 31 - 4, 1, True), (2 ** 31 - 4, 2, False), (2 ** 31 - 4, 8, False), (2 ** 30, 3, True), (2 ** 30, 4, False)):
        fits, g = grid(64, 64, [row] * n, 2, 16, 131072)
        assert fits == expected == ((g[1] + g[3]) * 256 < 2 ** 32), (row, n)
