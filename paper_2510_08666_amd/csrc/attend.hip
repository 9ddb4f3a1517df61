// Attention of a sequence's new tokens over its cached positions and, as far as their visibility words allow, over each
// other: softmax(scale * q . K^T) . V in one pass over the keys, with the running maximum and sum of every row in float32.
//
// The queries of all query heads that share a cache head are rows of the same contraction (row = token * group + member), so
// that a tile of 32 rows reads its head's keys once.  MFMA mapping as in attention.hip: S^T[key][row] = K . Q^T, a lane owns
// one row, O^T[d][row] += V^T . P^T from the score registers.  Queries enter as they are (bfloat16 queries are exact), and
// probabilities as two bfloat16 planes (PvWeights), so that an output is rounded once, when it is stored.
#include <type_traits>

#include "attn_tiles.hpp"
#include "cache.hpp"
#include "gemm.hpp"

namespace dinfer {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

static int most_rows(const SeqSpan& span, int group) {
  int most = 0;
  for (int s = 0; s < span.n_seq; ++s) {
    const int rows = (span.off[s + 1] - span.off[s]) * group;
    most = rows > most ? rows : most;
  }
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
// Workgroups that run at the same time: two per compute unit, one of those with eight row tiles.
constexpr int resident(int rows) { return rows > 128 ? 256 : 512; }
template <typename E, int ROWS> __device__ inline Plan make_plan(const AttendArgs& a) {
  constexpr int PARTS = resident(ROWS);
  const int lane = threadIdx.x & 63, s = min(lane, a.tok.span.n_seq - 1);
  const int len = lane == s ? a.tok.span.off[s + 1] - a.tok.span.off[s] : 0;
  Plan p;
  p.base = cache_base(a.tok, s, len);
  p.tiles = (p.base + len + TILE - 1) / TILE;
  p.groups = (len * a.group + ROWS - 1) / ROWS;
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
template <typename E, int HD, int NP, int RG, bool PV>
__global__ __launch_bounds__(ATTEND_WAVES * WAVE, (attend_waves_per_simd<E, HD>())) void attend_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, DT = PV ? HD / TILE : 1, STEPS = PvStep<E>::STEPS;
  constexpr int TEAMS = ATTEND_WAVES / RG, ROWS = RG * TILE;
  constexpr int REGS = PV ? DT * 16 : 0, PW = (REGS + 2) * WAVE, OPL = REGS / TEAMS;      // OPL: output registers a wave finishes
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int rt = wave % RG, team = wave / RG;
  const bool masked = a.visible != nullptr;
  const E* kv = (const E*)a.kv_layer;
  const float c2 = a.scale * LOG2E;
  const int n_q_heads = a.geom.n_heads * a.group;
  extern __shared__ __align__(16) char smem[];
  vec* qs = reinterpret_cast<vec*>(smem) + rt * (DSTEPS * NP * WAVE);                            // [RG][k-step][plane][64 lanes]
  int32_t* pt = reinterpret_cast<int32_t*>(smem + RG * DSTEPS * NP * WAVE * 16);                 // page ids of the piece
  float* lds = reinterpret_cast<float*>(smem);      // behind the key tiles: [ATTEND_WAVES][REGS, then m, l][64 lanes]
  const Plan plan = make_plan<E, ROWS>(a);
  const uint32_t wg = near_workgroup();
  if (wg >= plan.total) return;
  const Piece c = piece_at(plan, wg, a.geom.n_heads);
  const int kt0 = c.n_tiles * c.part / c.parts, kt1 = c.n_tiles * (c.part + 1) / c.parts;
  const int tok0 = a.tok.span.off[c.seq], row0 = c.group * ROWS, n_rows = (a.tok.span.off[c.seq + 1] - tok0) * a.group - row0;      // rows from this group on: >= 1
  const int n_keys = c.base + a.tok.span.off[c.seq + 1] - tok0, last_page = (n_keys - 1) / PAGE - 2 * kt0, last_tile = kt1 - 1;
  const int row = row0 + min(rt * TILE + col, n_rows - 1), tok = tok0 + row / a.group, q_head = c.head * a.group + row % a.group;
  if (!a.whole) note_cut(a, plan, c, wg, row0);
  {
    const int32_t* pages = a.tok.page_table + (int64_t)c.seq * a.tok.pt_stride + 2 * kt0;
    for (int i = threadIdx.x; i <= min(2 * (kt1 - kt0) - 1, last_page); i += ATTEND_WAVES * WAVE) pt[i] = safe_page(a.geom, pages[i]);
  }
  const uint64_t word = masked ? a.visible[tok] : ~0ull;
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
  // (clamped, so that no branch surrounds loads: a wave's last turn repeats its tile).  tail: a tile with new tokens, or the ragged end.
  auto use_tile = [&](int kt, auto tail) {
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
    const int next = min(kt + TEAMS, last_tile);
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    bool odd = false;                   // some value of a new token is no finite number
    if constexpr (decltype(tail)::value) {
      // what a row does not see scores -inf, values past the last key (which may hold anything) become 0
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kt * TILE + PvStep<E>::key_of_acc(i, half);
        if (key >= n_keys || !sees(word, masked, key - c.base)) s[0][i] = -INFINITY;
      }
      if constexpr (PV) {
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
            for (int j = 0; j < 4; ++j) most = ValueBits<E>::larger(most, w[j]);
          }
        }
        odd = masked && __builtin_amdgcn_ballot_w64(ValueBits<E>::largest(most) >= ValueBits<E>::ODD) != 0;
      }
    }
    float p[1][16];
    take_scores<DT, 1>(s, c2, m_run, l_run, o, p);
    if constexpr (PV) {
      constexpr int PP = PvWeights<E>::PLANES;
      vec pv[STEPS][PP];
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) PvWeights<E>::split(p[0], s2, pv[s2]);
      if (decltype(tail)::value && odd) {
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
  int kt = kt0 + team;
  if (kt <= last_tile && rt * TILE < n_rows) {
    const int full = min(c.base / TILE, kt1);
    load_k(kt);
    load_v(kt);
    for (; kt < full; kt += TEAMS) use_tile(kt, std::false_type{});
    for (; kt <= last_tile; kt += TEAMS) use_tile(kt, std::true_type{});
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

// Many rows (grouped query heads): a workgroup takes WAVES row tiles of a head, one per wave, and every key tile goes through LDS
// once for all of them, two tiles a turn, double buffered, the turn after next on its way in registers; in the form above
// each wave would fetch it for itself (48 sequences of 31 to 64 tokens with four query heads per cache head behind 1000 to 8000: 370 us
// with the join).  A wave keeps its queries and output in registers, nothing is folded.  A workgroup takes up to 256 rows, so that K and
// V are read fewer times (four waves and 128 rows, two workgroups per compute unit: 368 us; eight waves 332, 318 without the join).
// What a turn takes now, 2.9 us, is none of its bounds alone (counters: matrix units busy 38 % of the time, vector units 36 %, LDS
// 18 %): scores, exponentials and output are one chain in each wave, and waves wait for each other at every turn.  Without effect, with
// one plane of weights: two turns of loads under way, priorities or half a turn's distance between the waves of a SIMD, output products
// between the second tile's exponentials, deeper rings.  The second plane of weights took 60 us, split in front of its products 69.
template <int HD> constexpr size_t attend_rows_lds() { return (size_t)2 * 4 * (HD / ET<bf16_t>::KS) * WAVE * 16 + ATTN_MAX_PAGES * 4; }
template <int HD, int WAVES>
__global__ __launch_bounds__(WAVES * WAVE, 2) void attend_rows_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef bf16_t E;
  typedef ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, DT = HD / TILE, STEPS = PvStep<E>::STEPS, ROWS = WAVES * TILE;
  constexpr int SHARE = WAVES / 4, WF = DSTEPS, MF = WF / SHARE;      // fragments of a set (K or V of one of a turn's two tiles), and those of it that a wave fetches
  static_assert(DSTEPS == STEPS * DT && STEPS == 2 && (SHARE == 1 || SHARE == 2), "two key tiles have four sets, half a V set is a k-step");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const bool masked = a.visible != nullptr;
  const E* kv_layer = (const E*)a.kv_layer;
  extern __shared__ __align__(16) char smem[];
  auto kv = reinterpret_cast<vec(*)[4][WF][WAVE]>(smem);      // [buffer][K of tile 0, K of tile 1, V of 0, V of 1][fragment][lane]
  int32_t* pt = reinterpret_cast<int32_t*>(smem + (size_t)2 * 4 * WF * WAVE * 16);
  __shared__ int32_t odd_turn[2];      // of a buffer: some value of a new token is no finite number
  const Plan plan = make_plan<E, ROWS>(a);
  const uint32_t wg = near_workgroup();
  if (wg >= plan.total) return;
  const Piece c = piece_at(plan, wg, a.geom.n_heads);
  const int kt0 = c.n_tiles * c.part / c.parts, kt1 = c.n_tiles * (c.part + 1) / c.parts;
  const int tok0 = a.tok.span.off[c.seq], row0 = c.group * ROWS, n_rows = (a.tok.span.off[c.seq + 1] - tok0) * a.group - row0;
  const int n_keys = c.base + a.tok.span.off[c.seq + 1] - tok0, last_page = (n_keys - 1) / PAGE - 2 * kt0;
  const int n_turns = (kt1 - kt0 + 1) / 2;
  const int row = row0 + min(wave * TILE + col, n_rows - 1), tok = tok0 + row / a.group, q_head = c.head * a.group + row % a.group;
  const bool works = wave * TILE < n_rows;      // (every wave fetches)
  if (!a.whole) note_cut(a, plan, c, wg, row0);
  {
    const int32_t* pages = a.tok.page_table + (int64_t)c.seq * a.tok.pt_stride + 2 * kt0;
    for (int i = threadIdx.x; i <= min(2 * (kt1 - kt0) - 1, last_page); i += WAVES * WAVE) pt[i] = safe_page(a.geom, pages[i]);
  }
  const uint64_t word = masked ? a.visible[tok] : ~0ull;
  vec q[DSTEPS];
  {
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) q[s] = load16<E>(qrow + s * KS);
  }
  if (threadIdx.x < 2) odd_turn[threadIdx.x] = 0;
  __syncthreads();
  vec next[MF];
  const int set = wave / SHARE, f0 = wave % SHARE * MF, sub = set & 1;
  const bool fetch_k = set < 2;
  const int last_key = min(n_keys, kt1 * TILE) - 1;      // keys past it are another part's, or none
  auto fetch = [&](int turn) {
    const int key0 = (kt0 + 2 * min(turn, n_turns - 1) + sub) * TILE;
    if (fetch_k) {
      const int key = min(key0 + PvStep<E>::key_of_row(col), last_key);
      const E* krow = kv_layer + kv_k_index(a.geom, pt[key / PAGE - 2 * kt0], c.head, key % PAGE, 0) + half * G + f0 * (PAGE * KS);
#pragma unroll
      for (int j = 0; j < MF; ++j) next[j] = load16<E>(krow + j * (PAGE * KS));
    } else {
#pragma unroll
      for (int h = 0; h < STEPS / SHARE; ++h) {
        const int step = f0 / DT + h;
        const int page = pt[min(key0 + PvStep<E>::page_of_step(step) * PAGE, last_key) / PAGE - 2 * kt0];
        const E* vrow = kv_layer + kv_v_index(a.geom, page, c.head, 0, col);
#pragma unroll
        for (int t = 0; t < DT; ++t) next[h * DT + t] = PvStep<E>::v_vec(vrow + t * (TILE * PAGE), half, step);
      }
    }
  };
  // tail: turns with new tokens or with the end of the part
  auto put = [&](int turn, auto tail) {
    const int key0 = (kt0 + 2 * turn + sub) * TILE;
    if (decltype(tail)::value && !fetch_k) {
      // new tokens, and the end of the part: values past its last key, which may hold anything, become 0, and so does what is
      // no finite number where some row may not see it (the rows that do are found below)
      uint32_t most = 0;
#pragma unroll
      for (int h = 0; h < STEPS / SHARE; ++h) {
        const int valid = last_key + 1 - (key0 + PvStep<E>::key_of(f0 / DT + h, half, 0));
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          u32x4 w = words_of<E>(next[h * DT + t]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] &= ValueBits<E>::mask(j, valid);
            most = ValueBits<E>::larger(most, w[j]);
            if (masked) w[j] = ValueBits<E>::finite(w[j]);
          }
          next[h * DT + t] = __builtin_bit_cast(vec, w);
        }
      }
      if (masked && ValueBits<E>::largest(most) >= ValueBits<E>::ODD) odd_turn[turn & 1] = 1;      // (never taken back: it costs a look)
    }
#pragma unroll
    for (int j = 0; j < MF; ++j) kv[turn & 1][set][f0 + j][lane] = next[j];
  };
  f32x16 o[DT];
  zero_acc<DT>(o);
  float m_run = -INFINITY, l_run = 0.f;
  uint64_t marks[3] = {0, 0, 0};
  const float c2 = a.scale * LOG2E;
  auto take_turn = [&](int turn, auto tail) {
    const auto& tiles = kv[turn & 1];
    // LDS fragments are read RD ahead of the matrix instructions that take them, behind the last ones of K the first of V
    // (pinned by the scheduling barriers: all at once they would take the registers of the queries)
    constexpr int RD = 4, NF = 2 * DSTEPS;
    vec ring[RD];
    f32x16 s[2];
    zero_acc<2>(s);
#pragma unroll
    for (int f = 0; f < RD; ++f) ring[f] = tiles[f & 1][f >> 1][lane];
#pragma unroll
    for (int f = 0; f < NF; ++f) {      // k-step f / 2 of tile f % 2
      const vec k = ring[f % RD];
      const int n = f + RD;
      ring[f % RD] = n < NF ? tiles[n & 1][n >> 1][lane] : tiles[2][n - NF][lane];
      __builtin_amdgcn_sched_barrier(0);
      mfma32(s[f & 1], k, q[f / 2]);
    }
    const int first_key = (kt0 + 2 * turn) * TILE;
    bool odd = false;
    if constexpr (decltype(tail)::value) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = first_key + n * TILE + PvStep<E>::key_of_acc(v, half);
          if (key > last_key || !sees(word, masked, key - c.base)) s[n][v] = -INFINITY;
        }
      odd = odd_turn[turn & 1] != 0;
    }
    float p[2][16];
    take_scores<DT, 2>(s, c2, m_run, l_run, o, p);
    if (decltype(tail)::value && odd) {
      // see attend_kernel: rows with weight on a value that is no finite number are marked
#pragma unroll 1
      for (int t = 0; t < DT; ++t)
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
          f32x16 hit[1];
          zero_acc<1>(hit);
#pragma unroll
          for (int u = 0; u < 2 * STEPS; ++u) {
            const int key0 = first_key + u / STEPS * TILE;
            const int page = pt[min(key0 + PvStep<E>::page_of_step(u % STEPS) * PAGE, last_key) / PAGE - 2 * kt0];
            const vec x = PvStep<E>::v_vec(kv_layer + kv_v_index(a.geom, page, c.head, 0, t * TILE + col), half, u % STEPS);
            mfma32(hit[0], odd_values<E>(x, kind, last_key + 1 - (key0 + PvStep<E>::key_of(u % STEPS, half, 0))), PvStep<E>::p_vec(p[u / STEPS], u % STEPS, 0));
          }
          uint32_t bits = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) bits |= hit[0][i] != 0.f ? 1u << i : 0u;
          marks[kind] |= (uint64_t)bits << (16 * t);
        }
    }
    // (a step's weights are split between the products of the step in front of it)
    u32x4 pv[2][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) PvWeights<E>::pair(p[0], 0, j, pv[0]);
#pragma unroll
    for (int u = 0; u < 2 * STEPS; ++u) {
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const int f = u * DT + t;
        const vec v = ring[f % RD];
        if (f + RD < NF) ring[f % RD] = tiles[2 + (f + RD) / WF][(f + RD) % WF][lane];
        __builtin_amdgcn_sched_barrier(0);
        mfma32(o[t], v, __builtin_bit_cast(vec, pv[u & 1][0]));
        if (u + 1 < 2 * STEPS) {
#pragma unroll
          for (int j = t * 4 / DT; j < (t + 1) * 4 / DT; ++j) PvWeights<E>::pair(p[(u + 1) / STEPS], (u + 1) % STEPS, j, pv[(u + 1) & 1]);
        }
        mfma32(o[t], v, __builtin_bit_cast(vec, pv[u & 1][1]));
      }
    }
  };
  // The turns in front of the tail, and the one before it, whose neighbour has to be masked on its way to LDS.  A turn that was put as one
  // of the tail is taken as one, so that what was replaced on its way is looked for.
  const int full = (min(c.base, last_key + 1) - kt0 * TILE) / (2 * TILE);
  fetch(0);
  if (full > 1) put(0, std::false_type{});
  else put(0, std::true_type{});
  fetch(1);
  int turn = 0;
  for (; turn + 1 < full; ++turn) {
    __syncthreads();      // this turn's tiles are in their buffer, and every wave has done with the other one
    put(turn + 1, std::false_type{});
    fetch(turn + 2);
    if (works) take_turn(turn, std::false_type{});
  }
  for (; turn < n_turns; ++turn) {
    __syncthreads();
    if (turn + 1 < n_turns) {
      put(turn + 1, std::true_type{});
      fetch(turn + 2);
    }
    if (works) take_turn(turn, std::true_type{});
  }
  if (wave * TILE + col >= n_rows) return;
  if (__builtin_amdgcn_ballot_w64((marks[0] | marks[1] | marks[2]) != 0)) {
#pragma unroll
    for (int i = 0; i < DT * 16; ++i) {
      if ((marks[1] >> i) & 1) o[i / 16][i % 16] += INFINITY;
      if ((marks[2] >> i) & 1) o[i / 16][i % 16] -= INFINITY;
      if ((marks[0] >> i) & 1) o[i / 16][i % 16] = __builtin_nanf("");
    }
  }
  const float L = l_run + __shfl_xor(l_run, 32, WAVE);
  if (c.parts == 1) {
    if (a.lse && half == 0) a.lse[(int64_t)tok * (a.geom.n_heads * a.group) + q_head] = log_sum(m_run, L);
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store_elems4<E>((E*)a.out + (int64_t)tok * a.out_stride + q_head * HD + t * TILE + acc_row(4 * g, half),
                        f32x4{o[t][4 * g] * inv, o[t][4 * g + 1] * inv, o[t][4 * g + 2] * inv, o[t][4 * g + 3] * inv});
  } else {
    float* part = attend_part(a, c.slot + c.part, ROWS * (HD + 2));
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(part + (wave * TILE + col) * HD + t * TILE + acc_row(4 * g, half)) =
            f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
    if (half == 0) *reinterpret_cast<float2*>(part + ROWS * HD + 2 * (wave * TILE + col)) = float2{m_run, L};
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
size_t attend_part_bytes(bool bf16, int head_dim, int max_pos) {
  if (max_pos <= (bf16 ? min_cut<bf16_t>() : min_cut<float>()) * TILE) return 0;      // nothing is cut
  const size_t rows = (size_t)2 * resident(8 * TILE) * 8 * TILE, few = (size_t)2 * resident(4 * TILE) * 4 * TILE;
  return (rows > few ? rows : few) * (head_dim + 2) * 4 + sizeof(CutList);
}

// Grids: workgroups of the first launch, pairs that may have to be joined (none: a.whole).
struct AttendGrid {
  unsigned wgs, cut;
};
template <typename E, int ROWS> static AttendGrid attend_grid(AttendArgs& a) {
  int64_t pairs = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) pairs += ((int64_t)(a.tok.span.off[s + 1] - a.tok.span.off[s]) * a.group + ROWS - 1) / ROWS;
  pairs *= a.geom.n_heads;
  a.whole = single_slice() || a.tok.limit <= min_cut<E>() * TILE;
  const int64_t wgs = a.whole ? pairs : pairs + resident(ROWS);
  return AttendGrid{(unsigned)((wgs + 31) / 32 * 32), a.whole ? 0u : (unsigned)(pairs < resident(ROWS) ? pairs : resident(ROWS))};
}
template <typename E, int HD, int ROWS, bool PV> static void launch_merge(const AttendArgs& a, unsigned cut, hipStream_t st) {
  if (cut > 0) attend_merge_kernel<E, HD, ROWS, PV><<<cut * (ROWS / (merge_rows<HD, PV>() * (ROWS > 64 ? 4 : 1))), MERGE_THREADS, 0, st>>>(a, live_word());
}
template <typename E, int HD, int NP, int RG, bool PV> static void launch_attend_t(AttendArgs a, hipStream_t st) {
  const AttendGrid g = attend_grid<E, RG * TILE>(a);
  attend_kernel<E, HD, NP, RG, PV><<<g.wgs, ATTEND_WAVES * WAVE, attend_lds<E, HD, NP, RG, PV>(), st>>>(a, live_word());
  launch_merge<E, HD, RG * TILE, PV>(a, g.cut, st);
}
template <int HD, int WAVES> static void launch_attend_rows(AttendArgs a, hipStream_t st) {
  const AttendGrid g = attend_grid<bf16_t, WAVES * TILE>(a);
  attend_rows_kernel<HD, WAVES><<<g.wgs, WAVES * WAVE, attend_rows_lds<HD>(), st>>>(a, live_word());
  launch_merge<bf16_t, HD, WAVES * TILE, true>(a, g.cut, st);
}
template <typename E, int HD, int RG> static void launch_attend_rg(int planes, const AttendArgs& a, hipStream_t st) {
  if (a.out) launch_attend_t<E, HD, 1, RG, true>(a, st);
  else if (planes == 1) launch_attend_t<E, HD, 1, RG, false>(a, st);
  else if constexpr (sizeof(E) == 2) launch_attend_t<E, HD, 2, RG, false>(a, st);
}
// Meetings of a row tile with a key tile in a call, at most (the lengths are on the device: as if all caches were full).
static int64_t most_meetings(const AttendArgs& a) {
  int64_t row_tiles = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) row_tiles += ((int64_t)(a.tok.span.off[s + 1] - a.tok.span.off[s]) * a.group + TILE - 1) / TILE;
  return row_tiles * a.geom.n_heads * ((a.tok.limit + TILE - 1) / TILE);
}
// Two row tiles per workgroup where a sequence has more than one; more than two: the form whose tiles go through LDS, where there is
// work enough for it.  Its workgroups are few and take 2.9 us a turn, however little there is: of 8 cache heads of 4 queries each, 60
// tokens behind 3000 positions take 38.8 us in it and 20.3 in two row tiles, eight sequences of them (49 thousand meetings) 65 and 63,
// sixteen 98 and 92, 24 (148 thousand) 178 and 153, 32 163 and 202, 48 278 and 298.  How a call's parts fill its 256 places moves the
// crossover: 16 heads of 8 queries and 20 tokens 151 and 133 at 91 thousand, 138 and 154 at 121, 4 heads of 8 and 64 tokens 91 and 95 at 97,
// 183 and 139 at 145, 156 and 165 at 194.  In float32 the matrix instructions are the bound (a sixteenth of the rate), not the reads that row
// tiles could share: one tile per workgroup (3 sequences of 5 to 33 tokens 28.9 -> 20.4 us).
constexpr int64_t ROWS_FORM_MEETINGS = 1 << 17;
template <int HD> static void launch_attend_hd(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  const int most = most_rows(a.tok.span, a.group);
  if (bf16) {
    const bool rows_form = most > 2 * TILE && a.out && most_meetings(a) >= ROWS_FORM_MEETINGS;
    if (rows_form && most > 4 * TILE) launch_attend_rows<HD, 8>(a, st);
    else if (rows_form) launch_attend_rows<HD, 4>(a, st);
    else if (most <= TILE) launch_attend_rg<bf16_t, HD, 1>(planes, a, st);
    else launch_attend_rg<bf16_t, HD, 2>(planes, a, st);
  } else launch_attend_rg<float, HD, 1>(planes, a, st);
}
void launch_attend(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_attend_hd<128>(bf16, planes, a, st);
  else launch_attend_hd<64>(bf16, planes, a, st);
}

template <typename E, int HD, int RG> static bool configure_attend_t() {
  return hipFuncSetAttribute((const void*)attend_kernel<E, HD, 1, RG, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)attend_lds<E, HD, 1, RG, true>()) == hipSuccess;
}
template <int HD, int WAVES> static bool configure_rows() {
  return hipFuncSetAttribute((const void*)attend_rows_kernel<HD, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)attend_rows_lds<HD>()) == hipSuccess;
}
bool configure_attend() {
  const bool ok = configure_attend_t<bf16_t, 128, 1>() && configure_attend_t<bf16_t, 128, 2>() && configure_attend_t<bf16_t, 64, 1>() &&
                  configure_attend_t<bf16_t, 64, 2>() && configure_attend_t<float, 128, 1>() && configure_attend_t<float, 64, 1>() &&
                  configure_rows<128, 4>() &&
                  configure_rows<128, 8>() && configure_rows<64, 4>() && configure_rows<64, 8>();
  (void)hipGetLastError();
  return ok;
}

// ------------------------------------------------------------------------------------------------
// Attention weight that cached positions gather: score[head][key] = decay * score[head][key] + the sum over the rows of the
// head's group of exp(scale * q . k - lse).  Here rows run along the registers and keys along the lanes (A = Q, B = K), so a
// key's sum over 32 rows is an addition of 16 registers and one exchange between the half-waves, and every score has one writer:
// no atomics, the same bits every time.  A wave holds KT key tiles in registers, all their loads under way at once, and meets them with
// one row tile after the other.  Bound by the read of K; with many rows by the matrix instructions and the queries' second
// reads, which KT tiles share (16 KB of keys per wave: what fits the registers beside the queries).  16 sequences of 17 to 32 tokens
// behind 256 to 4096 positions, 150 MB: 35.7 us, 4.2 TB/s with the start of every workgroup (lengths, pages, keys: three dependent loads).
// ------------------------------------------------------------------------------------------------
constexpr int SCORE_WAVES = 4;
// A key's weight over the 16 rows in a lane's registers.  lse: of the tile's rows, times log2(e), infinity for those that weigh nothing;
// words: what they see; tail: the key may be a new token, number rel.
__device__ inline float score_sum(const f32x16& s, float c2, const float* lse, const uint64_t* words, bool tail, int rel, int half) {
  float sum = 0.f;
#pragma unroll
  for (int v4 = 0; v4 < 4; ++v4) {
    const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse + acc_row(4 * v4, half));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float p = __builtin_amdgcn_exp2f(fmaf(s[4 * v4 + j], c2, -l4[j]));
      if (l4[j] == INFINITY) p = 0.f;                                      // (a score that is no number included)
      if (tail && !sees(words[acc_row(4 * v4 + j, half)], true, rel)) p = 0.f;
      sum += p;
    }
  }
  return sum;
}
template <typename E, int HD> constexpr int score_tiles() { return 512 / (sizeof(E) * HD); }
template <typename E, int HD, int NP>
__global__ __launch_bounds__(SCORE_WAVES * WAVE, 2) void score_kernel(ScoreArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, KT = score_tiles<E, HD>();
  const int head = blockIdx.y, seq = blockIdx.z;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0;
  if (len == 0) return;
  const int base = cache_base(a.tok, seq, len), n_keys = min(base + len, a.score_stride);
  const int kt0 = (blockIdx.x * SCORE_WAVES + wave) * KT, n_rows = len * a.group;
  if (kt0 * TILE >= n_keys) return;
  const bool masked = a.visible != nullptr;
  const int n_q_heads = a.geom.n_heads * a.group;
  const int32_t* pages = a.tok.page_table + (int64_t)seq * a.tok.pt_stride;
  int page[KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) page[i] = pages[min((kt0 + i) * TILE + col, n_keys - 1) / PAGE];
  auto row_at = [&](int row0) { return row0 + min(col, n_rows - row0 - 1); };
  auto load_q = [&](int row0, vec (&q)[DSTEPS * NP], float& lse, uint64_t& word) {
    const int row = row_at(row0), tok = tok0 + row / a.group, q_head = head * a.group + row % a.group;
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
#pragma unroll
    for (int i = 0; i < DSTEPS * NP; ++i) q[i] = load16<E>(qrow + (i % NP) * a.q_plane + (i / NP) * KS);
    lse = a.lse[(int64_t)tok * n_q_heads + q_head];
    word = masked ? a.visible[tok] : ~0ull;
  };
  vec q[DSTEPS * NP], k[KT][DSTEPS];
  float lse;
  uint64_t word;
  load_q(0, q, lse, word);
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    const int at = min((kt0 + i) * TILE + col, n_keys - 1);
    const E* krow = (const E*)a.kv_layer + kv_k_index(a.geom, safe_page(a.geom, page[i]), head, at % PAGE, 0) + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) k[i][s] = load16<E>(krow + s * (PAGE * KS));
  }
  __shared__ __align__(16) float s_lse[SCORE_WAVES][TILE];
  __shared__ uint64_t s_word[SCORE_WAVES][TILE];
  const float c2 = a.scale * LOG2E;
  const bool tail = masked && (kt0 + KT) * TILE > base;
  float sum[KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) sum[i] = 0.f;
  for (int row0 = 0; row0 < n_rows; row0 += TILE) {
    if (half == 0) {
      // rows past the last one, and rows that see nothing (lse = -inf), weigh nothing: exp2(x - inf) = 0
      s_lse[wave][col] = row0 + col < n_rows && lse != -INFINITY ? lse * LOG2E : INFINITY;
      s_word[wave][col] = word;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      f32x16 s[1];
      zero_acc<1>(s);
#pragma unroll
      for (int f = 0; f < DSTEPS * NP; ++f) mfma32(s[0], q[f], k[i][f / NP]);
      const int rel = (kt0 + i) * TILE + col - base;
      sum[i] += score_sum(s[0], c2, s_lse[wave], s_word[wave], tail, rel, half);
    }
    if (row0 + TILE < n_rows) load_q(row0 + TILE, q, lse, word);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  const int64_t unit = ((int64_t)seq * a.geom.n_heads + head) * a.score_stride;
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    const float total = sum[i] + __shfl_xor(sum[i], 32, WAVE);
    const int key = (kt0 + i) * TILE + col;
    if (half == 0 && key < n_keys) a.score_out[unit + key] = a.score_in ? fmaf(a.decay, a.score_in[unit + key], total) : total;
  }
}

// Short contexts whose normalisers are not known yet: a workgroup holds all keys of a (sequence, head) in the registers of its eight
// waves, so that they are read once and the normalisers need no launch of their own.  Rows along the lanes for these (A = K, B = Q: the
// same registers), joined over the waves through LDS, then as above.  (One sequence of 32 tokens behind 700 positions: 14.5 ->
// 10.8 us.)
template <typename E, int HD, int NP> constexpr int whole_tiles() { return sizeof(E) * HD == 128 ? 4 : sizeof(E) * HD == 256 ? 4 - NP : 1; }      // what the registers hold
constexpr int WHOLE_WAVES = 8;
template <typename E, int HD, int NP>
__global__ __launch_bounds__(WHOLE_WAVES * WAVE, 2) void score_whole_kernel(ScoreArgs a, float* __restrict__ lse_out, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, KT = whole_tiles<E, HD, NP>();
  const int head = blockIdx.x, seq = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0;
  if (len == 0) return;
  const int base = cache_base(a.tok, seq, len), n_keys = base + len, n_rows = len * a.group;      // n_keys <= 32 * KT * WHOLE_WAVES (host)
  const int kt0 = wave * KT;
  const bool masked = a.visible != nullptr;
  const int n_q_heads = a.geom.n_heads * a.group;
  const int32_t* pages = a.tok.page_table + (int64_t)seq * a.tok.pt_stride;
  vec k[KT][DSTEPS];
  {
    int page[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) page[i] = pages[min((kt0 + i) * TILE + col, n_keys - 1) / PAGE];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const int at = min((kt0 + i) * TILE + col, n_keys - 1);
      const E* krow = (const E*)a.kv_layer + kv_k_index(a.geom, safe_page(a.geom, page[i]), head, at % PAGE, 0) + half * G;
#pragma unroll
      for (int s = 0; s < DSTEPS; ++s) k[i][s] = load16<E>(krow + s * (PAGE * KS));
    }
  }
  __shared__ __align__(16) float s_lse[TILE];
  __shared__ float2 s_state[WHOLE_WAVES][TILE];
  __shared__ uint64_t s_word[TILE];
  const float c2 = a.scale * LOG2E;
  float sum[KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) sum[i] = 0.f;
  for (int row0 = 0; row0 < n_rows; row0 += TILE) {
    const int row = row0 + min(col, n_rows - row0 - 1), tok = tok0 + row / a.group, q_head = head * a.group + row % a.group;
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
    const uint64_t word = masked ? a.visible[tok] : ~0ull;
    vec q[DSTEPS * NP];
#pragma unroll
    for (int i = 0; i < DSTEPS * NP; ++i) q[i] = load16<E>(qrow + (i % NP) * a.q_plane + (i / NP) * KS);
    // (unknown to the compiler, which would work every tile's masks out in front of the loop and keep them in registers)
    int end = n_keys, old = base;
    asm volatile("" : "+s"(end), "+s"(old));
    // normalisers: a lane's row over this wave's keys, then over the waves
    float m = -INFINITY, l = 0.f;
    f32x16 none[1];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if ((kt0 + i) * TILE >= end) break;
      f32x16 s[1];
      zero_acc<1>(s);
#pragma unroll
      for (int f = 0; f < DSTEPS * NP; ++f) mfma32(s[0], k[i][f / NP], q[f]);
      if ((kt0 + i + 1) * TILE > old) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = (kt0 + i) * TILE + acc_row(v, half);      // (keys in order here: no product with V follows)
          if (key >= end || !sees(word, masked, key - old)) s[0][v] = -INFINITY;
        }
      }
      float p[1][16];
      zero_acc<1>(none);
      take_scores<1, 1>(s, c2, m, l, none, p);
    }
    l += __shfl_xor(l, 32, WAVE);
    if (half == 0) s_state[wave][col] = float2{m, l};
    __syncthreads();
    if (wave == 0 && half == 0) {
      float2 st[WHOLE_WAVES];
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < WHOLE_WAVES; ++w) {
        st[w] = s_state[w][col];
        M = fmaxf(M, st[w].x);
      }
#pragma unroll
      for (int w = 0; w < WHOLE_WAVES; ++w) L = fmaf(state_weight(st[w].x, st[w].y, M), st[w].y, L);
      const float lse = log_sum(M, L);
      if (row0 + col < n_rows) lse_out[(int64_t)tok * n_q_heads + q_head] = lse;
      s_lse[col] = row0 + col < n_rows && lse != -INFINITY ? lse * LOG2E : INFINITY;
      s_word[col] = word;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if ((kt0 + i) * TILE >= end) break;
      f32x16 s[1];
      zero_acc<1>(s);
#pragma unroll
      for (int f = 0; f < DSTEPS * NP; ++f) mfma32(s[0], q[f], k[i][f / NP]);
      sum[i] += score_sum(s[0], c2, s_lse, s_word, masked && (kt0 + i + 1) * TILE > old, (kt0 + i) * TILE + col - old, half);
    }
  }
  const int64_t unit = ((int64_t)seq * a.geom.n_heads + head) * a.score_stride;
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    const float total = sum[i] + __shfl_xor(sum[i], 32, WAVE);
    const int key = (kt0 + i) * TILE + col;
    if (half == 0 && key < min(n_keys, a.score_stride))
      a.score_out[unit + key] = a.score_in ? fmaf(a.decay, a.score_in[unit + key], total) : total;
  }
}

template <typename E, int HD, int NP> static void launch_score_t(const ScoreArgs& a, hipStream_t st) {
  const int bound = a.tok.limit < a.score_stride ? a.tok.limit : a.score_stride, keys = SCORE_WAVES * score_tiles<E, HD>() * TILE;
  score_kernel<E, HD, NP><<<dim3((bound + keys - 1) / keys, a.geom.n_heads, a.tok.span.n_seq), SCORE_WAVES * WAVE, 0, st>>>(a, live_word());
}
template <typename E, int HD, int NP> static bool launch_score_whole_t(const ScoreArgs& a, float* lse, hipStream_t st) {
  if (a.tok.limit > WHOLE_WAVES * whole_tiles<E, HD, NP>() * TILE) return false;
  score_whole_kernel<E, HD, NP><<<dim3(a.geom.n_heads, a.tok.span.n_seq), WHOLE_WAVES * WAVE, 0, st>>>(a, lse, live_word());
  return true;
}
template <int HD> static void launch_score_hd(bool bf16, int planes, const ScoreArgs& a, hipStream_t st) {
  if (!bf16) launch_score_t<float, HD, 1>(a, st);
  else if (planes == 1) launch_score_t<bf16_t, HD, 1>(a, st);
  else launch_score_t<bf16_t, HD, 2>(a, st);
}
template <int HD> static bool launch_score_whole_hd(bool bf16, int planes, const ScoreArgs& a, float* lse, hipStream_t st) {
  if (!bf16) return launch_score_whole_t<float, HD, 1>(a, lse, st);
  return planes == 1 ? launch_score_whole_t<bf16_t, HD, 1>(a, lse, st) : launch_score_whole_t<bf16_t, HD, 2>(a, lse, st);
}
void launch_normalised_score(bool bf16, int planes, const ScoreArgs& a, float* lse, float* part, hipStream_t st) {
  if (a.geom.head_dim == 128 ? launch_score_whole_hd<128>(bf16, planes, a, lse, st) : launch_score_whole_hd<64>(bf16, planes, a, lse, st)) return;
  launch_attend(bf16, planes,
                AttendArgs{a.tok, a.kv_layer, a.geom, a.q, a.q_stride, a.q_plane, a.group, a.visible, a.scale, nullptr, 0, lse, part, false}, st);
  launch_score(bf16, planes, a, st);
}
void launch_score(bool bf16, int planes, const ScoreArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_score_hd<128>(bf16, planes, a, st);
  else launch_score_hd<64>(bf16, planes, a, st);
}

}  // namespace dinfer
