// Attention of new tokens over the paged cache: how a launch deals its work, the kernel of few rows and the one that joins
// the parts of a pair (attend.hip and ruled.hip; what a row sees is a policy of the kernel).
#pragma once
#include <cfloat>
#include <type_traits>

#include "attn_tiles.hpp"
#include "cache.hpp"
#include "gemm.hpp"

namespace dinfer {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

static int rows_of(const AttendArgs& a, int s) { return (a.tok.span.off[s + 1] - a.tok.span.off[s]) * a.group; }
static int most_rows(const AttendArgs& a) {
  int most = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) most = rows_of(a, s) > most ? rows_of(a, s) : most;
  return most;
}

// Bit of a key among the sequence's new tokens: keys in front of them are seen by everybody.
__device__ inline bool sees(uint64_t word, bool masked, int rel) { return rel < 0 || !masked || ((word >> (rel & 63)) & 1); }

// Value operands as words.  Elements of a 16-byte operand from `valid` on become 0; largest magnitude of all of them, as bits (at
// least ODD: one is no finite number).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename E> struct ValueBits;
template <> struct ValueBits<bf16_t> {
  static constexpr uint32_t ODD = 0x7f80u;
  __device__ static uint32_t mask(int j, int valid) { return valid >= 2 * j + 2 ? ~0u : valid == 2 * j + 1 ? 0xffffu : 0u; }
  __device__ static uint32_t larger(uint32_t m, uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
  }
  __device__ static uint32_t largest(uint32_t m) { return max(m & 0xffffu, m >> 16); }
  __device__ static uint32_t finite(uint32_t w) {
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu, hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
    return lo | hi;
  }
};
template <> struct ValueBits<float> {
  static constexpr uint32_t ODD = 0x7f800000u;
  __device__ static uint32_t mask(int j, int valid) { return valid > j ? ~0u : 0u; }
  __device__ static uint32_t larger(uint32_t m, uint32_t w) { return max(m, w & 0x7fffffffu); }
  __device__ static uint32_t largest(uint32_t m) { return m; }
  __device__ static uint32_t finite(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u ? 0u : w; }
};
template <typename E> __device__ inline u32x4 words_of(const typename ET<E>::vec& v) { return __builtin_bit_cast(u32x4, v); }

// A row's running state takes in one tile of scores: p = exp2(s * c2 - m).  A row that has seen nothing yet keeps m = -inf and
// p = 0.  The reference maximum moves only when it is passed by more than SLACK (p <= 2^SLACK).
template <int DT, int NS>
__device__ inline void take_scores(const f32x16 (&s)[NS], float c2, float& m_run, float& l_run, f32x16 (&o)[DT], float (&p)[NS][16]) {
  constexpr float SLACK = 6.f;
  float mx = s[0][0];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[n][v]);
  mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE));
  const float mt = mx * c2;
  const bool moves = mt > m_run + SLACK;
  if (__builtin_amdgcn_ballot_w64(moves)) {
    const float alpha = moves ? __builtin_amdgcn_exp2f(m_run - mt) : 1.f;
    l_run *= alpha;
    m_run = moves ? mt : m_run;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[t][v] *= alpha;
  }
  const float ref = m_run > -INFINITY ? m_run : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[n][v] = __builtin_amdgcn_exp2f(fmaf(s[n][v], c2, -ref));
      sum += p[n][v];
    }
  l_run += sum;
}

// Probabilities of k-step s2 as operands of the product with V.  bfloat16: a plane of the leading eight bits, cut off, and a plane of the
// rest, which is off by 2^-15 of the probability at most.  The rest is never negative, and one step of float32 more than it is, so that it is
// not zero next to a probability that is not: an infinite value times both planes is the infinity.
template <typename E> struct PvWeights;
template <> struct PvWeights<bf16_t> {
  static constexpr int PLANES = 2;
  __device__ static void pair(const float (&p)[16], int s2, int j, u32x4 (&w)[2]) {
    constexpr float STEP = 1.f + 0x1p-23f;
    const float a = p[8 * s2 + 2 * j], b = p[8 * s2 + 2 * j + 1];
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
    w[0][j] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);      // their upper halves
    w[1][j] = __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)fmaf(a, STEP, -__uint_as_float(ua & 0xffff0000u)),
                                                  (bf16_t)fmaf(b, STEP, -__uint_as_float(ub & 0xffff0000u))});
  }
  __device__ static void split(const float (&p)[16], int s2, bf16x8 (&w)[2]) {
    u32x4 x[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) pair(p, s2, j, x);
    w[0] = __builtin_bit_cast(bf16x8, x[0]);
    w[1] = __builtin_bit_cast(bf16x8, x[1]);
  }
};
template <> struct PvWeights<float> {
  static constexpr int PLANES = 1;
  __device__ static void split(const float (&p)[16], int s2, f32x4 (&w)[1]) { w[0] = PvStep<float>::p_vec(p, s2, 0); }
};

// Weight of a partial state (m, l) against the maximum M of all: a state that saw nothing counts nothing, one that is not a
// number (every score NaN: m never moved) makes the sum one.
__device__ inline float state_weight(float m, float l, float M) { return m > -INFINITY ? __builtin_amdgcn_exp2f(m - M) : l; }

// Indicator of a kind of odd value (0: NaN, 1: +inf, 2: -inf) among the first `valid` elements of an operand.
template <typename E> __device__ inline typename ET<E>::vec odd_values(const typename ET<E>::vec& x, int kind, int valid) {
  u32x4 w = words_of<E>(x);
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] &= ValueBits<E>::mask(j, valid);
  const typename ET<E>::vec y = __builtin_bit_cast(typename ET<E>::vec, w);
  typename ET<E>::vec is;
#pragma unroll
  for (int i = 0; i < ET<E>::G; ++i) {
    const float f = to_f32(y[i]);
    is[i] = from_f32<E>((kind == 0 ? f != f : f == (kind == 1 ? INFINITY : -INFINITY)) ? 1.f : 0.f);
  }
  return is;
}
__device__ inline float log_sum(float m, float l) { return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2; }

// How a launch deals its work.  A pair is a cache head with a group of ROWS rows of one sequence; the key tiles of a long pair are cut into
// parts of equal length, a workgroup takes one part, and attend_merge_kernel joins the parts of a pair.  The lengths are on
// the device, so every wave works the plan out for itself, a lane per sequence.  A part has `per` key tiles at most: with few pairs as
// many as leave about as many parts as workgroups run at a time, counting half a part per pair for the rounding (a few
// workgroups more than fit run alone behind the others: 16 sequences of 17 to 32 tokens behind 256 to 2048, 608 of them 44.1 us with the
// join, 496 42.3); with many pairs the workgroups' share of all tiles, the longest parts first, so that the short ones fill the gaps; and at
// least min_part (64 drafts behind 4096 keys: 8 tiles 23.7 us, 12 19.5).  A pair of up to min_cut tiles is left whole: a wave
// has six of them at most to walk, and joining (a launch of 3 to 5 us) costs more than they take.
// In float32 a tile keeps a wave's matrix unit busy for 1.7 us: a pair is cut much earlier (3 sequences behind 64 to 901 keys 20.4 -> 12.3 us).
template <typename E> constexpr int min_cut() { return sizeof(E) == 2 ? 24 : 8; }
template <typename E> constexpr int min_part() { return sizeof(E) == 2 ? 12 : 4; }
constexpr int ATTEND_WAVES = 4;
struct Plan {
  int seq, base, tiles, groups, parts;      // of this lane's sequence
  uint32_t end, slot_end, cut_end;          // sums, up to this lane's sequence, of workgroups, partial results, pairs that were cut
  uint32_t total, cut;
};
// What the rows of attend_kernel see, and what becomes of their scores.
// WordRule: all keys in front of the new tokens, and of those the ones that a visibility word names.
struct WordRule {
  static constexpr bool RANGES = false;
  __host__ __device__ static bool takes(const AttendArgs&, int) { return true; }      // a sequence of so many rows
  __device__ static int first_tile(const AttendArgs&, int) { return 0; }
  __device__ float factor(float c2) const { return c2; }      // of the scores, to units of log 2
};
// RangeRule: the keys of two ranges of cache positions per row (dinfer_attend_rule); scores may be capped and biased by the distance.
struct RowRanges {
  int a0, a1, b0, b1;      // [a0, a1): of the prefix, [b0, b1): near the row, no key in both; joined into [b0, b1) where they touch
};
__device__ inline RowRanges row_ranges(const AttendRule& r, int seq, int tok, int p, int n_keys) {
  const int lo = r.first ? max(0, min(r.first[tok], n_keys)) : 0, hi = r.end ? max(lo, min(r.end[tok], n_keys)) : n_keys;
  const int pre = r.prefix ? max(0, min(r.prefix[seq], n_keys)) : 0;
  RowRanges w{lo, max(lo, min(pre, hi)), lo, hi};
  if (r.block > 0) w.b1 = min(w.b1, p < pre ? pre : pre + ((p - pre) / r.block + 1) * r.block);      // (host: blocks and windows no longer than a cache can be)
  if (r.window > 0) {
    w.b0 = max(w.b0, p - r.window + 1);
    w.b1 = min(w.b1, p + r.window);
  }
  if (w.b0 <= w.a1) {
    w.b0 = w.a0;
    w.b1 = max(w.b1, w.a1);
    w.a1 = w.a0;
  }
  w.b1 = max(w.b0, w.b1);
  return w;
}
// What a group of rows sees together: some_*: keys that a row sees lie in these, all_*: keys that every row sees.
struct GroupRanges {
  int some_a0, some_a1, some_b0, some_b1, all_a0, all_a1, all_b0, all_b1;
  __device__ void take(const RowRanges& w) {
    const bool a = w.a1 > w.a0, b = w.b1 > w.b0;
    some_a0 = a ? w.a0 : INT32_MAX, some_a1 = a ? w.a1 : 0;
    some_b0 = b ? w.b0 : INT32_MAX, some_b1 = b ? w.b1 : 0;
    all_a0 = w.a0, all_a1 = w.a1, all_b0 = w.b0, all_b1 = w.b1;
  }
  __device__ void join(const GroupRanges& o) {
    some_a0 = min(some_a0, o.some_a0), some_a1 = max(some_a1, o.some_a1);
    some_b0 = min(some_b0, o.some_b0), some_b1 = max(some_b1, o.some_b1);
    all_a0 = max(all_a0, o.all_a0), all_a1 = min(all_a1, o.all_a1);
    all_b0 = max(all_b0, o.all_b0), all_b1 = min(all_b1, o.all_b1);
  }
  // over the 32 columns of a wave, whose halves hold the same rows
  __device__ void join_columns() {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      GroupRanges o;
      o.some_a0 = __shfl_xor(some_a0, d, WAVE), o.some_a1 = __shfl_xor(some_a1, d, WAVE);
      o.some_b0 = __shfl_xor(some_b0, d, WAVE), o.some_b1 = __shfl_xor(some_b1, d, WAVE);
      o.all_a0 = __shfl_xor(all_a0, d, WAVE), o.all_a1 = __shfl_xor(all_a1, d, WAVE);
      o.all_b0 = __shfl_xor(all_b0, d, WAVE), o.all_b1 = __shfl_xor(all_b1, d, WAVE);
      join(o);
    }
  }
};
// The key tiles of [kt0, kt1) in which a group sees anything: first those that all its rows see whole, so that these have a loop of
// their own, then the others, as up to six runs of tiles.
struct TileWalk {
  static constexpr int RUNS = 6;
  int run0[RUNS], len[RUNS];
  __device__ static int fixed(int x) { return __builtin_amdgcn_readfirstlane(x); }
  __device__ void set(int r, int t0, int t1) {
    run0[r] = t0;
    len[r] = max(0, t1 - t0);
  }
  // runs of [t0, t1): r: tiles within [all0, all1), then at `rest` those in front of them and behind
  __device__ void split(int r, int rest, int t0, int t1, int all0, int all1, int keys) {
    const int w0 = max(t0, (all0 + keys - 1) / keys), w1 = min(t1, all1 / keys);
    const bool some = w0 < w1;
    set(r, w0, w1);
    set(rest, t0, some ? w0 : t1);
    set(rest + 1, w1, some ? t1 : w1);
  }
  __device__ void start(const GroupRanges& g, int kt0, int kt1, int keys) {      // keys: of a tile
    // (a first range that begins behind the second one, of another document, is widened to it)
    const int a0 = fixed(min(g.some_a0, g.some_b0)), a1 = fixed(g.some_a1), b0 = fixed(g.some_b0), b1 = fixed(g.some_b1);
    const int ta0 = max(kt0, a0 / keys), ta1 = min(kt1, (a1 + keys - 1) / keys);
    const int tb0 = max(max(kt0, a1 > 0 ? ta1 : 0), b0 / keys), tb1 = min(kt1, (b1 + keys - 1) / keys);
    split(0, 2, ta0, max(ta0, ta1), fixed(g.all_a0), fixed(g.all_a1), keys);
    split(1, 4, tb0, max(tb0, tb1), fixed(g.all_b0), fixed(g.all_b1), keys);
  }
  __device__ int whole() const { return len[0] + len[1]; }
  __device__ int tiles() const { return len[0] + len[1] + len[2] + len[3] + len[4] + len[5]; }
  __device__ int tile(int i) const {
    int t = run0[0] + i, before = len[0];
#pragma unroll
    for (int r = 1; r < RUNS; ++r) {
      t = i >= before ? run0[r] + i - before : t;
      before += len[r];
    }
    return t;
  }
};
// cap * tanh(z / cap) of a product s, z = scale * s, in units of log 2, with u = s * ratio = z / cap.  Up to |u| = 1/2 tanh(u) = u S(u^2), 1 in front, so
// that a score far below its cap stays as it is; S's other coefficients make the largest relative error least (2^-26, by Lawson's weighted least
// squares).  Beyond, cap - 2 cap / (exp(2u) + 1), which would cancel near 0.  Either is within 2^-21 of the score.  A score alone decides which one
// it takes (so that no other one reaches it); a wave works out the second form where one of its scores needs it: prompts of 333 to
// 1811 tokens in documents of 301 48.2 us without | 54.3 with it everywhere, 8191 causal tokens with 8 heads of 4 queries 732 | 1000 (uncapped 540).
struct CapScores {
  static constexpr double S[4] = {-0.333331438954662, 0.13325878934223193, -0.0530454923870277, 0.017241486995792973};
  // ratio: of a product to u, neither 0 nor infinite; unit: of a product to scores in log 2; small: S's coefficients, times unit
  static void prepare(AttendRule& r, float scale) {
    const double ratio = (double)scale / r.cap, used = ratio < FLT_MAX ? ratio : FLT_MAX;      // (beyond: every product but 0 is at the cap)
    r.cap_ratio = (float)used > FLT_TRUE_MIN ? (float)used : FLT_TRUE_MIN;
    r.cap_unit = (float)(used * r.cap * (double)LOG2E);
    for (int k = 0; k < 4; ++k) r.cap_small[k] = (float)(S[k] * used * r.cap * (double)LOG2E);
  }
  float cap2, ratio, unit, small[4];
  __device__ float below(float s, float u) const {
    const float y = u * u;
    return s * fmaf(fmaf(fmaf(fmaf(small[3], y, small[2]), y, small[1]), y, small[0]), y, unit);
  }
  __device__ f32x16 scores(f32x16 s) const {
    float top = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(s[v]));      // (NaN stays in either form)
    if (__builtin_amdgcn_ballot_w64(top * ratio > 0.5f)) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float u = s[v] * ratio, t = __builtin_amdgcn_exp2f(u * (2.f * LOG2E));
        const float beyond = fmaf(__builtin_amdgcn_rcpf(t + 1.f), -2.f * cap2, cap2);
        s[v] = fabsf(u) > 0.5f ? beyond : below(s[v], u);
      }
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = below(s[v], s[v] * ratio);
    }
    return s;
  }
};
template <bool CAP, bool BIAS> struct RangeRule {
  static constexpr bool RANGES = true;
  __host__ __device__ static bool takes(const AttendArgs& a, int rows) { return a.rule.takes(rows); }
  // a window without a prefix lets a sequence's walk begin late
  __device__ static int first_tile(const AttendArgs& a, int base) {
    return a.rule.window > 0 && !a.rule.prefix ? max(0, base - a.rule.window + 1) / TILE : 0;
  }
  RowRanges see;
  TileWalk walk;
  float at, slope2;      // (scores are in units of log 2)
  CapScores cap;
  __device__ void start_row(const AttendArgs& a, int seq, int tok, int p, int q_head, int n_keys) {
    see = row_ranges(a.rule, seq, tok, p, n_keys);
    if constexpr (BIAS) at = p, slope2 = a.rule.slope[q_head] * LOG2E;
    if constexpr (CAP) cap = CapScores{a.rule.cap * LOG2E, a.rule.cap_ratio, a.rule.cap_unit, {a.rule.cap_small[0], a.rule.cap_small[1], a.rule.cap_small[2], a.rule.cap_small[3]}};
  }
  __device__ void start(const AttendArgs& a, int seq, int tok, int p, int q_head, int n_keys, int kt0, int kt1) {
    start_row(a, seq, tok, p, q_head, n_keys);
    GroupRanges g;
    g.take(see);
    g.join_columns();
    walk.start(g, kt0, kt1, TILE);
  }
  __device__ bool sees(int key) const {
    return (uint32_t)(key - see.a0) < (uint32_t)(see.a1 - see.a0) || (uint32_t)(key - see.b0) < (uint32_t)(see.b1 - see.b0);
  }
  // Scores of keys that a row does not see become -inf.
  template <typename E> __device__ void hide(f32x16& s, int key0, int half) const {
    const int first = key0 + half * PvStep<E>::key_of_acc(0, 1);
    if (__builtin_amdgcn_ballot_w64(see.a1 > see.a0)) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (!sees(first + PvStep<E>::key_of_acc(v, 0))) s[v] = -INFINITY;
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if ((uint32_t)(first - see.b0 + PvStep<E>::key_of_acc(v, 0)) >= (uint32_t)(see.b1 - see.b0)) s[v] = -INFINITY;
    }
  }
  __device__ float biased(float s, float c2, float key) const {
    const float d = fabsf(at - key);
    return CAP ? fmaf(-slope2, d, s) : fmaf(s, c2, -slope2 * d);
  }
  template <typename E> __device__ __attribute__((always_inline)) void scores(f32x16& s, float c2, int key0, int half) const {      // (a call would keep s in memory)
    if constexpr (CAP) s = cap.scores(s);
    if constexpr (BIAS) {
      const float first = key0 + half * PvStep<E>::key_of_acc(0, 1);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = biased(s[v], c2, first + PvStep<E>::key_of_acc(v, 0));
    }
  }
  __device__ float factor(float c2) const { return CAP || BIAS ? 1.f : c2; }
};

// Workgroups that run at the same time: two per compute unit, one of those with eight row tiles.
constexpr int resident(int rows) { return rows > 128 ? 256 : 512; }
template <typename E, int ROWS, class Rule = WordRule> __device__ inline Plan make_plan(const AttendArgs& a) {
  constexpr int PARTS = resident(ROWS);
  const int lane = threadIdx.x & 63, s = min(lane, a.tok.span.n_seq - 1);
  const int len = lane == s ? a.tok.span.off[s + 1] - a.tok.span.off[s] : 0;
  Plan p;
  p.base = cache_base(a.tok, s, len);
  p.tiles = (p.base + len + TILE - 1) / TILE - Rule::first_tile(a, p.base);
  p.groups = Rule::takes(a, len * a.group) ? (len * a.group + ROWS - 1) / ROWS : 0;
  uint32_t pairs = p.groups * a.geom.n_heads;
  const uint32_t units = __builtin_amdgcn_readlane(lane_scan(pairs * p.tiles), WAVE - 1);      // (host: the sum stays below 2^31)
  const uint32_t all_pairs = __builtin_amdgcn_readlane(lane_scan(pairs), WAVE - 1);
  const bool many = all_pairs > PARTS / 2;
  const uint32_t aim = many ? PARTS : PARTS - all_pairs / 2;
  const int per = max((int)((units + aim - 1) / aim), min_part<E>());
  p.parts = a.whole || p.tiles <= min_cut<E>() ? 1 : (p.tiles + per - 1) / per;
  p.seq = lane;
  if (many && a.tok.span.n_seq > 1) {
    // the longest parts first
    const int mine = (p.tiles + p.parts - 1) / p.parts;
    int rank = 0;
    for (int l = 0; l < a.tok.span.n_seq; ++l) {
      const int other = __builtin_amdgcn_readlane(mine, l);
      rank += other > mine || (other == mine && l < lane) ? 1 : 0;
    }
    const int to = (lane < a.tok.span.n_seq ? rank : lane) * 4;
    p.seq = __builtin_amdgcn_ds_permute(to, p.seq);
    p.base = __builtin_amdgcn_ds_permute(to, p.base);
    p.tiles = __builtin_amdgcn_ds_permute(to, p.tiles);
    p.groups = __builtin_amdgcn_ds_permute(to, p.groups);
    p.parts = __builtin_amdgcn_ds_permute(to, p.parts);
    pairs = p.groups * a.geom.n_heads;
  }
  p.end = lane_scan(pairs * p.parts);
  p.cut_end = lane_scan(p.parts > 1 ? pairs : 0);
  p.slot_end = lane_scan(p.parts > 1 ? pairs * p.parts : 0);
  p.total = __builtin_amdgcn_readlane(p.end, WAVE - 1);
  p.cut = __builtin_amdgcn_readlane(p.cut_end, WAVE - 1);
  return p;
}
// A pair of a sequence and a part of its key tiles.
struct Piece {
  int seq, base, head, group, part, parts, n_tiles;
  uint32_t slot;      // of the pair's first partial result
  uint32_t cut;       // its number among the pairs that were cut
};
// i: a workgroup's index, below plan.total.
__device__ inline Piece piece_at(const Plan& p, uint32_t i, int n_heads) {
  Piece c;
  const int at_lane = __builtin_ctzll(__builtin_amdgcn_ballot_w64(p.end > i));
  c.seq = __builtin_amdgcn_readlane(p.seq, at_lane);
  c.base = __builtin_amdgcn_readlane(p.base, at_lane);
  c.n_tiles = __builtin_amdgcn_readlane(p.tiles, at_lane);
  c.parts = __builtin_amdgcn_readlane(p.parts, at_lane);
  const uint32_t groups = __builtin_amdgcn_readlane(p.groups, at_lane), pairs = groups * n_heads;
  // heads, in them parts, in those row groups: neighbours read the same keys
  uint32_t at = i - (__builtin_amdgcn_readlane(p.end, at_lane) - pairs * c.parts);
  c.group = at % groups;
  at /= groups;
  c.part = at % c.parts;
  c.head = at / c.parts;
  const uint32_t behind = pairs - (c.head * groups + c.group);
  c.slot = __builtin_amdgcn_readlane(p.slot_end, at_lane) - behind * c.parts;
  c.cut = __builtin_amdgcn_readlane(p.cut_end, at_lane) - behind;
  return c;
}
// The same with the heads of a pair's part next to each other, so that each die, to which a launch's workgroups are dealt in turn, reads the keys of
// few heads, and the last rows, which see the most of a causal sequence, first.
__device__ inline Piece piece_by_heads(const Plan& p, uint32_t i, int n_heads) {
  const int at_lane = __builtin_ctzll(__builtin_amdgcn_ballot_w64(p.end > i));
  const uint32_t groups = __builtin_amdgcn_readlane(p.groups, at_lane), parts = __builtin_amdgcn_readlane(p.parts, at_lane);
  const uint32_t first = __builtin_amdgcn_readlane(p.end, at_lane) - groups * n_heads * parts, at = (i - first) / n_heads;
  // (its number in the order of piece_at: heads, in them parts, in those row groups)
  return piece_at(p, first + ((i - first) % n_heads * parts + at % parts) * groups + groups - 1 - at / parts, n_heads);
}
// What the host sizes grids and partial results by.  Every pair that is cut has more than `per` tiles, and per * resident covers all
// tiles: fewer than `resident` pairs are cut, into ceil(tiles / per) < 2 * tiles / per parts each, fewer than
// 2 * resident in all; all workgroups are fewer than `resident` and one more per pair.
// What the joining kernel is told of a pair that was cut, by the workgroup of its first part: it need not work out the plan again.
struct alignas(32) CutPair {
  int32_t seq, row0, head, parts;
  uint32_t slot, pad[3];
};
// In front of the partial results: how many pairs were cut, then their descriptions.
struct CutList {
  int32_t n, pad[7];
  CutPair pair[resident(TILE)];
};
__device__ inline void note_cut(const AttendArgs& a, const Plan& plan, const Piece& c, uint32_t wg, int row0) {
  CutList* list = reinterpret_cast<CutList*>(a.part);
  if (threadIdx.x != 0) return;
  if (wg == 0) list->n = plan.cut;
  if (c.parts > 1 && c.part == 0) list->pair[c.cut] = CutPair{c.seq, row0, c.head, c.parts, c.slot, {}};
}
__device__ inline float* attend_part(const AttendArgs& a, uint32_t slot, int floats) {
  return a.part + sizeof(CutList) / 4 + (int64_t)slot * floats;
}


// Workgroup i of a launch runs on die i mod 8: four neighbours run on one die, the next four on the next, and the workgroups that
// find nothing to do, since the host can only bound their number, come last.  (The launch has a multiple of 32.)
__device__ inline uint32_t near_workgroup() {
  const uint32_t i = blockIdx.x, at = i / 8;
  return at / 4 * 32 + i % 8 * 4 + at % 4;
}

// RG row tiles per workgroup (RG * 32 rows), each walked by 4 / RG waves that deal its key tiles among them (with two row tiles, both
// waves of a team fetch the same tile, the second time out of the compute unit's own cache).  K and V come straight into MFMA operand
// registers, the next tile's as soon as this tile's are used: with a whole tile more in flight a wave takes more than 256 registers and
// its workgroup a compute unit of its own, where nothing covers the latencies between its pieces; two workgroups per
// compute unit cover each other's.
template <typename E, int HD> constexpr int attend_waves_per_simd() { return sizeof(E) * HD > 256 ? 1 : 2; }      // (512-byte rows take the registers of two)
template <typename E, int HD, int NP, int RG, bool PV, class Rule = WordRule>
__global__ __launch_bounds__(ATTEND_WAVES * WAVE, (attend_waves_per_simd<E, HD>())) void attend_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, DT = PV ? HD / TILE : 1, STEPS = PvStep<E>::STEPS;
  constexpr int TEAMS = ATTEND_WAVES / RG, ROWS = RG * TILE;
  constexpr int REGS = PV ? DT * 16 : 0, PW = (REGS + 2) * WAVE, OPL = REGS / TEAMS;      // OPL: output registers a wave finishes
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int rt = wave % RG, team = wave / RG;
  const bool masked = Rule::RANGES || a.visible != nullptr;
  const E* kv = (const E*)a.kv_layer;
  const float c2 = a.scale * LOG2E;
  const int n_q_heads = a.geom.n_heads * a.group;
  extern __shared__ __align__(16) char smem[];
  vec* qs = reinterpret_cast<vec*>(smem) + rt * (DSTEPS * NP * WAVE);                            // [RG][k-step][plane][64 lanes]
  int32_t* pt = reinterpret_cast<int32_t*>(smem + RG * DSTEPS * NP * WAVE * 16);                 // page ids of the piece
  float* lds = reinterpret_cast<float*>(smem);      // behind the key tiles: [ATTEND_WAVES][REGS, then m, l][64 lanes]
  const Plan plan = make_plan<E, ROWS, Rule>(a);
  const uint32_t wg = near_workgroup();
  if (wg >= plan.total) return;
  const Piece c = piece_at(plan, wg, a.geom.n_heads);
  // (a part of a walk may lie anywhere in the sequence)
  const int kt0 = Rule::RANGES ? Rule::first_tile(a, c.base) : c.n_tiles * c.part / c.parts;
  const int kt1 = Rule::RANGES ? kt0 + c.n_tiles : c.n_tiles * (c.part + 1) / c.parts;
  const int tok0 = a.tok.span.off[c.seq], row0 = c.group * ROWS, n_rows = (a.tok.span.off[c.seq + 1] - tok0) * a.group - row0;      // rows from this group on: >= 1
  const int n_keys = c.base + a.tok.span.off[c.seq + 1] - tok0, last_page = (n_keys - 1) / PAGE - 2 * kt0, last_tile = kt1 - 1;
  const int row = row0 + min(rt * TILE + col, n_rows - 1), tok = tok0 + row / a.group, q_head = c.head * a.group + row % a.group;
  if (!a.whole) note_cut(a, plan, c, wg, row0);
  {
    const int32_t* pages = a.tok.page_table + (int64_t)c.seq * a.tok.pt_stride + 2 * kt0;
    for (int i = threadIdx.x; i <= min(2 * (kt1 - kt0) - 1, last_page); i += ATTEND_WAVES * WAVE) pt[i] = safe_page(a.geom, pages[i]);
  }
  const uint64_t word = !Rule::RANGES && masked ? a.visible[tok] : ~0ull;
  Rule rule;
  if constexpr (Rule::RANGES) rule.start(a, c.seq, tok, c.base + tok - tok0, q_head, n_keys, kt0, kt1);
  {
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
    for (int i = team; i < DSTEPS * NP; i += TEAMS) qs[i * WAVE + lane] = load16<E>(qrow + (i % NP) * a.q_plane + (i / NP) * KS);
  }
  __syncthreads();
  vec k[DSTEPS], v[PV ? STEPS : 1][DT];
  auto load_k = [&](int kt) {
    const int key = min(kt * TILE + PvStep<E>::key_of_row(col), n_keys - 1);
    const E* krow = kv + kv_k_index(a.geom, pt[key / PAGE - 2 * kt0], c.head, key % PAGE, 0) + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) k[s] = load16<E>(krow + s * (PAGE * KS));
  };
  auto v_row = [&](int kt, int s2) {
    return kv + kv_v_index(a.geom, pt[min(2 * (kt - kt0) + PvStep<E>::page_of_step(s2), last_page)], c.head, 0, col);
  };
  auto load_v = [&](int kt) {
    if constexpr (PV) {
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) {
        const E* vrow = v_row(kt, s2);
#pragma unroll
        for (int t = 0; t < DT; ++t) v[s2][t] = PvStep<E>::v_vec(vrow + t * (TILE * PAGE), half, s2);
      }
    }
  };
  f32x16 o[DT];
  zero_acc<DT>(o);
  float m_run = -INFINITY, l_run = 0.f;
  uint64_t marks[3] = {0, 0, 0};        // outputs (16 * t + v) that take in a NaN, an infinity, a negative one
  // One key tile; the next one's K loads are issued as soon as the scores have been worked out, its V loads behind the output products
  // (clamped, so that no branch surrounds loads: a wave's last turn repeats its tile).  A tile with new tokens, or the ragged end, is not WHOLE;
  // what is no finite number among its values is looked for if it is ODD.
  enum { WHOLE, PARTLY, ODD };
  auto use_tile = [&](int kt, int next, auto kind) __attribute__((always_inline)) {
    constexpr int KIND = decltype(kind)::value;
    asm volatile("" ::: "memory");      // keeps the query reads inside the loop
    f32x16 s[1];
    zero_acc<1>(s);
    {
      // query fragments are read from LDS QD ahead of the products that take them, no more: the registers are wanted elsewhere
      constexpr int QF = DSTEPS * NP, QD = 3;
      vec ring[QD];
#pragma unroll
      for (int f = 0; f < QD; ++f) ring[f] = qs[f * WAVE + lane];
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        const vec b = ring[f % QD];
        if (f + QD < QF) ring[f % QD] = qs[(f + QD) * WAVE + lane];
        __builtin_amdgcn_sched_barrier(0);
        mfma32(s[0], k[f / NP], b);
      }
    }
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (Rule::RANGES) rule.template scores<E>(s[0], c2, kt * TILE, half);
    bool odd = false;                   // some value of a new token is no finite number
    if constexpr (KIND != WHOLE) {
      // what a row does not see scores -inf, values past the last key (which may hold anything) become 0
      if constexpr (Rule::RANGES) rule.template hide<E>(s[0], kt * TILE, half);
      else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = kt * TILE + PvStep<E>::key_of_acc(i, half);
          if (key >= n_keys || !sees(word, masked, key - c.base)) s[0][i] = -INFINITY;
        }
      }
      if (PV && (KIND == ODD || kt * TILE + TILE > n_keys)) {
        uint32_t most = 0;
#pragma unroll
        for (int s2 = 0; s2 < STEPS; ++s2) {
          const int valid = n_keys - (kt * TILE + PvStep<E>::key_of(s2, half, 0));
          u32x4 m;
#pragma unroll
          for (int j = 0; j < 4; ++j) m[j] = ValueBits<E>::mask(j, valid);
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            const u32x4 w = words_of<E>(v[s2][t]) & m;
            v[s2][t] = __builtin_bit_cast(vec, w);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if constexpr (KIND == ODD) most = ValueBits<E>::larger(most, w[j]);
          }
        }
        odd = KIND == ODD && masked && __builtin_amdgcn_ballot_w64(ValueBits<E>::largest(most) >= ValueBits<E>::ODD) != 0;
      }
    }
    float p[1][16];
    take_scores<DT, 1>(s, rule.factor(c2), m_run, l_run, o, p);
    if constexpr (PV) {
      // (two row tiles under a rule, where the matrix instructions count: one number per weight, rounded to nearest)
      constexpr bool ONE = Rule::RANGES && RG == 2 && sizeof(E) == 2;
      constexpr int PP = ONE ? 1 : PvWeights<E>::PLANES;
      vec pv[STEPS][PP];
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) {
        if constexpr (ONE) pv[s2][0] = PvStep<E>::p_vec(p[0], s2, 0);
        else PvWeights<E>::split(p[0], s2, pv[s2]);
      }
      if (KIND == ODD && odd) {
        // 0 * NaN would reach the rows that do not see the key: the product takes 0 in such a value's place, and the rows with
        // weight on it are found by products with its indicator, one kind (NaN, +inf, -inf) at a time, and marked
#pragma unroll
        for (int s2 = 0; s2 < STEPS; ++s2)
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            u32x4 w = words_of<E>(v[s2][t]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              asm volatile("" : "+v"(w[j]));      // (its test of each word is not to be kept from the one above)
              w[j] = ValueBits<E>::finite(w[j]);
            }
            v[s2][t] = __builtin_bit_cast(vec, w);
          }
#pragma unroll 1
        for (int t = 0; t < DT; ++t)
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {
            f32x16 hit[1];
            zero_acc<1>(hit);
#pragma unroll
            for (int s2 = 0; s2 < STEPS; ++s2) {
              const vec x = PvStep<E>::v_vec(v_row(kt, s2) + t * (TILE * PAGE), half, s2);
              mfma32(hit[0], odd_values<E>(x, kind, n_keys - (kt * TILE + PvStep<E>::key_of(s2, half, 0))), pv[s2][0]);
            }
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) bits |= hit[0][i] != 0.f ? 1u << i : 0u;
            marks[kind] |= (uint64_t)bits << (16 * t);
          }
      }
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2)
#pragma unroll
        for (int pl = 0; pl < PP; ++pl)
#pragma unroll
          for (int t = 0; t < DT; ++t) mfma32(o[t], v[s2][t], pv[s2][pl]);
      __builtin_amdgcn_sched_barrier(0);
      load_v(next);
    }
  };
  if constexpr (Rule::RANGES) {
    const int all = rule.walk.tiles(), n = all * (c.part + 1) / c.parts, whole = min(n, rule.walk.whole()), i0 = all * c.part / c.parts + team;
    if (i0 < n && rt * TILE < n_rows) {
      int i = i0, kt = rule.walk.tile(i);
      load_k(kt);
      load_v(kt);
      auto walk = [&](int end, auto kind) __attribute__((always_inline)) {
        for (; i < end; i += TEAMS) {
          const int next = rule.walk.tile(min(i + TEAMS, n - 1));
          use_tile(kt, next, kind);
          kt = next;
        }
      };
      walk(whole, std::integral_constant<int, WHOLE>{});
      if (i < n) {
        walk(n, std::integral_constant<int, PARTLY>{});
        // Values that are not finite, also where a row does not see them (0 times them is no number), have left outputs that are not: once
        // more with a look for them, which takes half as long again as a partly seen tile without it.
        bool odd = false;
        if constexpr (PV) {
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) odd |= !(fabsf(o[t][v]) < INFINITY);
        }
        if (__builtin_amdgcn_ballot_w64(odd)) {
          zero_acc<DT>(o);
          m_run = -INFINITY, l_run = 0.f;
          i = i0, kt = rule.walk.tile(i);
          load_k(kt);
          load_v(kt);
          walk(n, std::integral_constant<int, ODD>{});
        }
      }
    }
  } else {
    int kt = kt0 + team;
    if (kt <= last_tile && rt * TILE < n_rows) {
      const int full = min(c.base / TILE, kt1);
      load_k(kt);
      load_v(kt);
      for (; kt < full; kt += TEAMS) use_tile(kt, min(kt + TEAMS, last_tile), std::integral_constant<int, WHOLE>{});
      for (; kt <= last_tile; kt += TEAMS) use_tile(kt, min(kt + TEAMS, last_tile), std::integral_constant<int, ODD>{});
    }
  }
  if constexpr (PV) {
    if (__builtin_amdgcn_ballot_w64((marks[0] | marks[1] | marks[2]) != 0)) {
#pragma unroll
      for (int i = 0; i < DT * 16; ++i) {
        if ((marks[1] >> i) & 1) o[i / 16][i % 16] += INFINITY;
        if ((marks[2] >> i) & 1) o[i / 16][i % 16] -= INFINITY;
        if ((marks[0] >> i) & 1) o[i / 16][i % 16] = __builtin_nanf("");
      }
    }
  }
  __syncthreads();      // queries and page ids are done with
  {
    float* pb = lds + wave * PW + lane;      // every wave leaves its state
    if constexpr (PV) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) pb[(t * 16 + i) * WAVE] = o[t][i];
    }
    pb[REGS * WAVE] = m_run;
    pb[(REGS + 1) * WAVE] = l_run + __shfl_xor(l_run, 32, WAVE);
  }
  __syncthreads();
  // and finishes OPL of its row tile's output registers
  float M = -INFINITY, L = 0.f, sum[OPL > 0 ? OPL : 1];
#pragma unroll
  for (int w = 0; w < TEAMS; ++w) M = fmaxf(M, lds[(w * RG + rt) * PW + REGS * WAVE + lane]);
#pragma unroll
  for (int i = 0; i < OPL; ++i) sum[i] = 0.f;
#pragma unroll
  for (int w = 0; w < TEAMS; ++w) {
    const float* pb = lds + (w * RG + rt) * PW + lane;
    const float lw = pb[(REGS + 1) * WAVE], sw = state_weight(pb[REGS * WAVE], lw, M);
    L = fmaf(sw, lw, L);
#pragma unroll
    for (int i = 0; i < OPL; ++i) sum[i] = fmaf(sw, pb[(team * OPL + i) * WAVE], sum[i]);
  }
  if (c.parts == 1) {
    if (rt * TILE + col < n_rows) {
      if (a.lse && team == 0 && half == 0) a.lse[(int64_t)tok * n_q_heads + q_head] = log_sum(M, L);
      const float inv = L == 0.f ? 0.f : 1.f / L;      // a row that sees nothing: zeros
#pragma unroll
      for (int i4 = 0; i4 < OPL / 4; ++i4) {
        const int g = team * OPL + 4 * i4;
        store_elems4<E>((E*)a.out + (int64_t)tok * a.out_stride + q_head * HD + (g / 16) * TILE + acc_row(g % 16, half),
                        f32x4{sum[4 * i4] * inv, sum[4 * i4 + 1] * inv, sum[4 * i4 + 2] * inv, sum[4 * i4 + 3] * inv});
      }
    }
  } else {
    constexpr int PROW = PV ? HD : 0;
    float* part = attend_part(a, c.slot + c.part, ROWS * (PROW + 2));      // [ROWS][HD], then (m, l) [ROWS]
#pragma unroll
    for (int i4 = 0; i4 < OPL / 4; ++i4) {
      const int g = team * OPL + 4 * i4;
      *reinterpret_cast<f32x4*>(part + (rt * TILE + col) * PROW + (g / 16) * TILE + acc_row(g % 16, half)) =
          f32x4{sum[4 * i4], sum[4 * i4 + 1], sum[4 * i4 + 2], sum[4 * i4 + 3]};
    }
    if (team == 0 && half == 0) *reinterpret_cast<float2*>(part + ROWS * PROW + 2 * (rt * TILE + col)) = float2{M, L};
  }
}

// Joins the parts of the pairs that were cut, in key order, each weighted against the maximum of all.  A thread takes four consecutive
// features of a row; a workgroup's rows belong to one pair.  Bound by the latency of its two loads (the pair, its partial
// results), and by the read of these.
constexpr int MERGE_THREADS = 256;
template <int HD, bool PV> constexpr int merge_rows() { return PV ? MERGE_THREADS / (HD / 4) : 32; }      // rows of a pass
template <typename E, int HD, int ROWS, bool PV>
__global__ __launch_bounds__(MERGE_THREADS) void attend_merge_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  constexpr int CHUNKS = PV ? HD / 4 : 1, PROW = PV ? HD : 0, PER = merge_rows<HD, PV>(), PASSES = ROWS > 64 ? 4 : 1;
  constexpr int WGS = ROWS / (PER * PASSES);      // workgroups of a pair
  static_assert(WGS * PER * PASSES == ROWS, "whole passes");
  const CutList* list = reinterpret_cast<const CutList*>(a.part);
  const int pair = blockIdx.x / WGS, n = list->n;
  const CutPair c = list->pair[pair];
  if (pair >= n) return;
  const int n_rows = (a.tok.span.off[c.seq + 1] - a.tok.span.off[c.seq]) * a.group;
  if ((int)threadIdx.x / CHUNKS >= PER) return;
  for (int pass = 0; pass < PASSES; ++pass) {
    const int q = (blockIdx.x % WGS * PASSES + pass) * PER + (int)threadIdx.x / CHUNKS, d = threadIdx.x % CHUNKS * 4, row = c.row0 + q;
    if (row >= n_rows) return;
    const float* part = attend_part(a, c.slot, ROWS * (PROW + 2));
    float M = -INFINITY, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int N = 8;      // parts whose loads are under way together
    for (int p0 = 0; p0 < c.parts; p0 += N) {
      float2 ml[N];
      f32x4 o[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float* from = part + (int64_t)min(p0 + i, c.parts - 1) * (ROWS * (PROW + 2));
        ml[i] = *reinterpret_cast<const float2*>(from + ROWS * PROW + 2 * q);
        if constexpr (PV) o[i] = *reinterpret_cast<const f32x4*>(from + q * PROW + d);
      }
      float top = M;
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, ml[i].x);
      const float old = M > -INFINITY ? __builtin_amdgcn_exp2f(M - top) : 1.f;      // (nothing so far: L and acc are 0, or NaN)
      L *= old;
      if constexpr (PV) acc *= old;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (p0 + i < c.parts) {
          const float w = state_weight(ml[i].x, ml[i].y, top);
          L = fmaf(w, ml[i].y, L);
          if constexpr (PV) {
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] = fmaf(w, o[i][k], acc[k]);
          }
        }
      }
      M = top;
    }
    const int64_t tok = a.tok.span.off[c.seq] + row / a.group;
    const int q_head = c.head * a.group + row % a.group;
    if (a.lse && d == 0) a.lse[tok * (a.geom.n_heads * a.group) + q_head] = log_sum(M, L);
    if constexpr (PV) store_elems4<E>((E*)a.out + tok * a.out_stride + q_head * HD + d, acc * (L == 0.f ? 0.f : 1.f / L));
  }
}

template <typename E, int HD, int NP, int RG, bool PV> constexpr size_t attend_lds() {
  const size_t fold = (size_t)ATTEND_WAVES * ((PV ? HD / TILE * 16 : 0) + 2) * WAVE * 4;
  const size_t walk = (size_t)RG * (HD / ET<E>::KS) * NP * WAVE * 16 + ATTN_MAX_PAGES * 4;
  return fold > walk ? fold : walk;
}


// Grids: workgroups of the first launch, pairs that may have to be joined (none: a.whole).
struct AttendGrid {
  unsigned wgs, cut;
};
template <typename E, int ROWS, class Rule = WordRule> static AttendGrid attend_grid(AttendArgs& a) {
  int64_t pairs = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s)
    if (Rule::takes(a, rows_of(a, s))) pairs += ((int64_t)rows_of(a, s) + ROWS - 1) / ROWS;
  pairs *= a.geom.n_heads;
  a.whole = single_slice() || a.tok.limit <= min_cut<E>() * TILE;
  const int64_t wgs = a.whole ? pairs : pairs + resident(ROWS);
  return AttendGrid{(unsigned)((wgs + 31) / 32 * 32), a.whole ? 0u : (unsigned)(pairs < resident(ROWS) ? pairs : resident(ROWS))};
}
template <typename E, int HD, int ROWS, bool PV> static void launch_merge(const AttendArgs& a, unsigned cut, hipStream_t st) {
  if (cut > 0) attend_merge_kernel<E, HD, ROWS, PV><<<cut * (ROWS / (merge_rows<HD, PV>() * (ROWS > 64 ? 4 : 1))), MERGE_THREADS, 0, st>>>(a, live_word());
}
template <typename E, int HD, int NP, int RG, bool PV, class Rule = WordRule> static void launch_attend_t(AttendArgs a, hipStream_t st) {
  const AttendGrid g = attend_grid<E, RG * TILE, Rule>(a);
  attend_kernel<E, HD, NP, RG, PV, Rule><<<g.wgs, ATTEND_WAVES * WAVE, attend_lds<E, HD, NP, RG, PV>(), st>>>(a, live_word());
  launch_merge<E, HD, RG * TILE, PV>(a, g.cut, st);
}
template <typename E, int HD, int RG, class Rule = WordRule> static bool configure_attend_t() {
  return hipFuncSetAttribute((const void*)attend_kernel<E, HD, 1, RG, true, Rule>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)attend_lds<E, HD, 1, RG, true>()) == hipSuccess;
}

}  // namespace dinfer
