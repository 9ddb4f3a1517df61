// Operators of a search over several continuations: the best (row, token) pairs of a sequence's rows, sequences that fork from
// parents and share their pages, and the move of the pages in use to the front of the pool.
#pragma once
#include "fork_plan.hpp"
#include "kernels.hpp"

namespace dinfer {

constexpr int MAX_KEEP = 64, MAX_SELECT_ROWS = 1024;
// Bits of a pool's pages in LDS: 8 bytes and a count for every 64 of them.
constexpr int MAX_POOL_PAGES = 12288 * 64;

struct SelectArgs {
  const void* logits;         // [n_seq * n_rows] rows of vocab, row_stride elements apart
  int64_t row_stride;
  int32_t n_seq, n_rows, vocab, n_keep;
  const float* score;         // [n_seq][n_rows], not finite: the row takes no part
  const int32_t* hold;        // [n_seq][n_rows] or null: >= 0: the row's only candidate
  int32_t *row, *token;       // [n_seq][n_keep]
  float* score_out;
  void* scratch;              // select_scratch_bytes
};
size_t select_scratch_bytes(int64_t rows, int vocab);
void launch_select(bool bf16, const SelectArgs& a, hipStream_t st);

// The page pool and the counts of the sequences that hold each page.
struct PagePool {
  char* kv;
  int64_t layer_bytes, page_bytes;
  int32_t n_layers, n_pages;
};
struct StateRows {
  const char* in;
  char* out;
  int64_t row_bytes;
};
// Pages to copy, left by a fork's first launch for its second.
struct CopyList {
  int32_t n, pad[3];
  int2 page[1];               // from, to; n of them
};
size_t fork_copies_bytes(int max_seqs, int max_pos);
struct ForkArgs {
  PagePool pool;
  int32_t n_old, n_new;
  const int32_t *parent, *len, *held;
  const int32_t* table;
  int32_t pt_stride, limit;   // limit: positions that a sequence may have
  int32_t room, rewrite;
  const int32_t* refs;
  int32_t *new_len, *new_held, *new_table;
  int32_t new_stride;
  int32_t *new_refs, *missing;
  StateRows state[MAX_STATES];
  int32_t n_states;
  CopyList* copies;           // fork_copies_bytes
  ForkGrid grid;              // plan_fork
};
// The launch's shape; false: too large.
bool plan_fork(ForkArgs& a);
void launch_fork(const ForkArgs& a, hipStream_t st);

struct CompactArgs {
  PagePool pool;
  int32_t n_seq;
  const int32_t *held, *table;
  int32_t pt_stride;
  const int32_t* refs;
  int32_t *new_table, *new_refs;
  int32_t* moved;             // [2][n_pages]: every page's new id, then the pages that move
  int32_t* count;             // [2]: pages in use, pages that move
};
void launch_compact(const CompactArgs& a, hipStream_t st);
bool configure_search();

}  // namespace dinfer
