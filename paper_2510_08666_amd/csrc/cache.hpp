// Operators on the paged KV cache that work beside the denoising step: the pass that norms, rotates and stores the
// queries, keys and values of new tokens, attention of new tokens over the cache, the weight that cached positions gather,
// and the move of chosen positions into other pages.
#pragma once
#include "kernels.hpp"

namespace dinfer {

constexpr int MAX_GROUP = 64;      // query heads of one cache head

// New tokens of up to MAX_SEQS sequences, packed: sequence s owns tokens [span.off[s], span.off[s+1]) (none is allowed), which
// take the cache positions past[s] .. past[s]+len-1.  limit: positions a sequence may use; a past that would leave it is
// pulled back, as a forward does (token_meta).
struct CacheTokens {
  SeqSpan span;
  const int32_t* past;        // [n_seq] device, or null: 0
  int32_t limit;
  const int32_t* page_table;
  int32_t pt_stride;
};
__device__ inline int cache_base(const CacheTokens& t, int seq, int len) {
  return t.past ? max(0, min(t.past[seq], t.limit - len)) : 0;
}
// The sequence that owns item i of a launch whose items are dealt to the sequences by off (the last one that begins at or
// before i: sequences without items are passed over).
__device__ inline int owner_of(const SeqSpan& s, int i) {
  int q = 0;
#pragma unroll
  for (int step = MAX_SEQS / 2; step > 0; step >>= 1)
    if (q + step < s.n_seq && s.off[q + step] <= i) q += step;
  return q;
}

// Sum of v over the lanes up to this one, by lane-to-lane moves inside the registers (rows of 16 lanes, then across them).
__device__ inline uint32_t lane_scan(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast:31 into rows 2 and 3
  return v;
}
// ---- rotary table: rows of rotary_dim / 2 cosines, then (from row max_pos on) as many of sines
struct RotaryRule {
  int32_t rotary_dim;
  int32_t scaling;            // ROTARY_*
  double theta, factor;
  double low, high;           // ramped frequencies: pairs up to low keep theirs, from high on they are divided by factor
  double magnitude;           // of every cosine and sine
};
enum { ROTARY_PLAIN = 0, ROTARY_LINEAR = 1, ROTARY_NTK = 2, ROTARY_YARN = 3 };
void launch_rotary_table(const RotaryRule& r, int max_pos, float* cos_tab, float* sin_tab, hipStream_t st);

struct AppendArgs {
  CacheTokens tok;
  void* kv_layer;
  KvGeom geom;
  const void *q, *k, *v;      // rows of (n_heads * group | n_heads | n_heads) heads, q null: keys and values only
  int64_t q_stride, k_stride, v_stride;   // elements between rows, rows 16-byte aligned
  int32_t group;              // query heads per cache head
  const float *q_gain, *k_gain;   // [head_dim], null: no norm
  float eps;
  int32_t rotary_dim, interleaved;
  const float *cos_tab, *sin_tab;
  int32_t table_rows;
  const int32_t* positions;   // [T] rotary positions, null: the cache positions
  void* q_out;
  int64_t q_out_stride;
};
void launch_append(bool bf16, const AppendArgs& a, hipStream_t st);

// What the rows of an attention under a rule see (dinfer_attend_rule, its lengths brought into a cache's).
struct AttendRule {
  int32_t block, window;
  const int32_t *prefix;      // [n_seq]
  const int32_t *first, *end; // [T]
  float cap;                  // 0: none
  float cap_ratio, cap_unit, cap_small[4];      // launch_ruled: CapScores
  const float* slope;         // [n_heads * group]
  int32_t least_rows, most_rows;      // of the sequences that a launch takes, set by launch_ruled
  __host__ __device__ bool takes(int rows) const { return rows >= least_rows && rows <= most_rows; }
};

// Queries of one cache head's group are rows of one contraction: row r of a sequence is token r / group, query head
// head * group + r % group.
struct AttendArgs {
  CacheTokens tok;
  const void* kv_layer;
  KvGeom geom;
  const void* q;
  int64_t q_stride, q_plane;  // q_plane: to the low plane of the queries (two-plane forms only)
  int32_t group;
  const uint64_t* visible;    // [T] or null: bit j = the token sees its sequence's new token j
  float scale;
  void* out;                  // [T] rows of n_heads * group heads, or null: normalisers only
  int64_t out_stride;
  float* lse;                 // [T][n_heads * group] natural logarithm of a row's sum of exponentials, or null
  float* part;                // attend_part_bytes
  bool whole;                 // set by the launch: no pair's keys are cut
  AttendRule rule;            // launch_ruled
};
size_t attend_part_bytes(bool bf16, int head_dim, int max_pos);
// planes: of the queries (two: the forward's own bfloat16 queries, normalisers only).
void launch_attend(bool bf16, int planes, const AttendArgs& a, hipStream_t st);
// Under a.rule (a.visible null).
void launch_ruled(bool bf16, AttendArgs a, hipStream_t st);

struct ScoreArgs {
  CacheTokens tok;
  const void* kv_layer;
  KvGeom geom;
  const void* q;
  int64_t q_stride, q_plane;
  int32_t group;
  const uint64_t* visible;
  float scale;
  const float* lse;           // [T][n_heads * group]
  float decay;
  const float* score_in;      // [n_seq][n_heads][score_stride] or null: 0; may be score_out
  float* score_out;
  int32_t score_stride;
};
void launch_score(bool bf16, int planes, const ScoreArgs& a, hipStream_t st);
// The same with normalisers that are worked out on the way and left in lse (= a.lse); part as in AttendArgs.
void launch_normalised_score(bool bf16, int planes, const ScoreArgs& a, float* lse, float* part, hipStream_t st);

struct EvictArgs {
  void* kv;                   // of the first layer
  int64_t kv_layer_bytes;
  KvGeom geom;
  int32_t n_layers, n_seq, keep, n_sink, n_recent, limit;
  const float* score;         // [n_layers][n_seq][n_heads][score_stride]
  int32_t score_stride;
  const int32_t* len;         // [n_seq]
  const int32_t* page_table;
  int32_t pt_stride;
  const int32_t* new_table;
  int32_t new_stride;
  int32_t* kept;              // [n_layers][n_seq][n_heads][keep]
  float* score_out;           // as score, or null
  int32_t* new_len;           // [n_seq]
};
void launch_evict(bool bf16, const EvictArgs& a, hipStream_t st);

bool configure_attend();
bool configure_ruled();

}  // namespace dinfer
