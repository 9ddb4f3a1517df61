// Workgroups of a fork's second launch.  Plain host C++.
#pragma once
#include <cstdint>

namespace dinfer {

constexpr int MAX_STATES = 8;
constexpr int PIECE_THREADS = 256, PIECE = PIECE_THREADS * 64;      // bytes that a workgroup moves at once, four loads of 16 per thread under way
// A launch counts its threads in 32 bits (beyond, the runtime starts as many as the lower bits say, without an error).
constexpr int64_t FORK_MOST_GROUPS = UINT32_MAX / PIECE_THREADS;
// Of the pages: the host knows how many pages may have to be copied, not how many there are, so that most of a large number would find nothing
// to do; a workgroup takes every so many pieces.
constexpr int64_t FORK_PAGE_GROUPS = 16384;

struct ForkGrid {
  int state0, page0;          // first workgroups of the states and of the pages (in front: a row of the tables each)
  int state_pieces[MAX_STATES];
  int pieces;                 // of a page
  int page_groups;
};
inline int64_t pieces_of(int64_t bytes) { return (bytes + PIECE - 1) / PIECE; }
// columns: of a sequence that may have to be copied.  False: the states are too many for a launch.
inline bool fork_grid(int n_old, int n_new, const int64_t* row_bytes, int n_states, int columns, int n_layers, int64_t page_bytes, ForkGrid* g) {
  int64_t at = n_old + n_new;
  g->state0 = (int)at;
  for (int k = 0; k < n_states; ++k) {
    g->state_pieces[k] = (int)pieces_of(row_bytes[k]);
    at += pieces_of(row_bytes[k]) * n_new;
  }
  g->page0 = (int)at;
  g->pieces = (int)pieces_of(page_bytes);
  const int64_t most = (int64_t)n_new * columns * n_layers * g->pieces;
  g->page_groups = (int)(most < FORK_PAGE_GROUPS ? most : FORK_PAGE_GROUPS);
  return at + g->page_groups <= FORK_MOST_GROUPS;
}

}  // namespace dinfer
