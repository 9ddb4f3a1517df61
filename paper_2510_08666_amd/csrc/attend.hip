// Attention of a sequence's new tokens over its cached positions and, as far as their visibility words allow, over each
// other: softmax(scale * q . K^T) . V in one pass over the keys, with the running maximum and sum of every row in float32.
//
// The queries of all query heads that share a cache head are rows of the same contraction (row = token * group + member), so
// that a tile of 32 rows reads its head's keys once.  MFMA mapping as in attention.hip: S^T[key][row] = K . Q^T, a lane owns
// one row, O^T[d][row] += V^T . P^T from the score registers.  Queries enter as they are (bfloat16 queries are exact), and
// probabilities as one bfloat16 plane: their rounding (2^-9 each, independent, weighted by the probabilities themselves) stays below the
// half step of the bfloat16 output.  Sums of probabilities are those of the unrounded ones.
#include <type_traits>

#include "attn_tiles.hpp"
#include "cache.hpp"
#include "gemm.hpp"

namespace dinfer {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

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
template <int DT> __device__ inline void take_scores(const f32x16& s, float c2, float& m_run, float& l_run, f32x16 (&o)[DT], float (&p)[16]) {
  constexpr float SLACK = 6.f;
  float mx = s[0];
#pragma unroll
  for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
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
  for (int v = 0; v < 16; ++v) {
    p[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c2, -ref));
    sum += p[v];
  }
  l_run += sum;
}

// Weight of a partial state (m, l) against the maximum M of all: a state that saw nothing counts nothing, one that is not a
// number (every score NaN: m never moved) makes the sum one.
__device__ inline float state_weight(float m, float l, float M) { return m > -INFINITY ? __builtin_amdgcn_exp2f(m - M) : l; }

__device__ inline float log_sum(float m, float l) { return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2; }

// How a launch deals its work.  A pair is a cache head with a group of ROWS rows of one sequence; the key tiles of a long pair are cut into
// parts of equal length, a workgroup takes one part, and attend_merge_kernel joins the parts of a pair.  The lengths are on
// the device, so every wave works the plan out for itself, a lane per sequence.  A part has `per` key tiles at most: as many as leave
// about ATTEND_PARTS parts, two workgroups on every compute unit, counting half a part per pair for the rounding (a few
// workgroups more than fit run alone behind the others: 608 of them 39.6 us, 16 sequences of 17 to 32 tokens behind 256 to 2048), and at least MIN_PART
// (two per wave).  A pair of up to MIN_CUT tiles is left whole: its waves have most of what they need under way at once, and joining
// costs more than they take.
constexpr int ATTEND_PARTS = 512, ATTEND_MIN_CUT = 24, ATTEND_MIN_PART = 8, ATTEND_WAVES = 4;
struct Plan {
  int base, tiles, groups, parts;      // of this lane's sequence
  uint32_t end, slot_end, cut_end;     // sums, up to this lane's sequence, of workgroups, partial results, pairs that were cut
  uint32_t total, cut;
};
template <int ROWS> __device__ inline Plan make_plan(const AttendArgs& a) {
  const int lane = threadIdx.x & 63, s = min(lane, a.tok.span.n_seq - 1);
  const int len = lane == s ? a.tok.span.off[s + 1] - a.tok.span.off[s] : 0;
  Plan p;
  p.base = cache_base(a.tok, s, len);
  p.tiles = (p.base + len + TILE - 1) / TILE;
  p.groups = (len * a.group + ROWS - 1) / ROWS;
  const uint32_t pairs = p.groups * a.geom.n_heads;
  const uint32_t units = __builtin_amdgcn_readlane(lane_scan(pairs * p.tiles), WAVE - 1);      // (host: the sum stays below 2^31)
  const uint32_t all_pairs = __builtin_amdgcn_readlane(lane_scan(pairs), WAVE - 1);
  const uint32_t aim = max((int)(ATTEND_PARTS - all_pairs / 2), ATTEND_PARTS / 2);
  const int per = max((int)((units + aim - 1) / aim), ATTEND_MIN_PART);
  p.parts = a.whole || p.tiles <= ATTEND_MIN_CUT ? 1 : (p.tiles + per - 1) / per;
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
};
// i: a workgroup's index (below plan.total), or with cut the index of a pair that was cut (below plan.cut).
__device__ inline Piece piece_at(const Plan& p, uint32_t i, int n_heads, bool cut) {
  Piece c;
  c.seq = __builtin_ctzll(__builtin_amdgcn_ballot_w64((cut ? p.cut_end : p.end) > i));
  c.base = __builtin_amdgcn_readlane(p.base, c.seq);
  c.n_tiles = __builtin_amdgcn_readlane(p.tiles, c.seq);
  c.parts = __builtin_amdgcn_readlane(p.parts, c.seq);
  const uint32_t groups = __builtin_amdgcn_readlane(p.groups, c.seq), pairs = groups * n_heads;
  uint32_t pair;
  if (cut) {
    pair = i - (__builtin_amdgcn_readlane(p.cut_end, c.seq) - pairs);
    c.part = 0;
  } else {
    const uint32_t at = i - (__builtin_amdgcn_readlane(p.end, c.seq) - pairs * c.parts);
    pair = at / c.parts;
    c.part = at % c.parts;
  }
  c.slot = __builtin_amdgcn_readlane(p.slot_end, c.seq) - (pairs - pair) * c.parts;
  c.head = pair / groups;      // (the row groups of a head lie next to each other: they read the same keys)
  c.group = pair % groups;
  return c;
}
// What the host sizes grids and partial results by.  Every pair that is cut has more than `per` tiles, per * ATTEND_PARTS covers all
// tiles: fewer than ATTEND_PARTS pairs are cut, into ceil(tiles / per) < 2 * tiles / per parts each, fewer than
// 2 * ATTEND_PARTS in all; all workgroups are fewer than ATTEND_PARTS and one more per pair.
constexpr int ATTEND_SLOTS = 2 * ATTEND_PARTS;

// Neighbouring parts run on one die (workgroup i of a launch runs on die i mod 8), all dies have as many, and the workgroups that find
// nothing to do, since the host can only bound their number, come last.
__device__ inline uint32_t near_workgroup(uint32_t total) {
  const uint32_t each = (total + 7) / 8, at = blockIdx.x / 8;
  return at < each ? blockIdx.x % 8 * each + at : total;
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
  const Plan plan = make_plan<ROWS>(a);
  const uint32_t wg = near_workgroup(plan.total);
  if (wg >= plan.total) return;
  const Piece c = piece_at(plan, wg, a.geom.n_heads, false);
  const int kt0 = c.n_tiles * c.part / c.parts, kt1 = c.n_tiles * (c.part + 1) / c.parts;
  const int tok0 = a.tok.span.off[c.seq], row0 = c.group * ROWS, n_rows = (a.tok.span.off[c.seq + 1] - tok0) * a.group - row0;      // rows from this group on: >= 1
  const int n_keys = c.base + a.tok.span.off[c.seq + 1] - tok0, last_page = (n_keys - 1) / PAGE - 2 * kt0, last_tile = kt1 - 1;
  const int row = row0 + min(rt * TILE + col, n_rows - 1), tok = tok0 + row / a.group, q_head = c.head * a.group + row % a.group;
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
    float p[16];
    take_scores<DT>(s[0], c2, m_run, l_run, o, p);
    if constexpr (PV) {
      vec pv[STEPS];
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) pv[s2] = PvStep<E>::p_vec(p, s2, 0);
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
              vec is;
#pragma unroll
              for (int i = 0; i < G; ++i) {
                const float f = to_f32(x[i]);
                const bool hot = kind == 0 ? f != f : f == (kind == 1 ? INFINITY : -INFINITY);
                is[i] = from_f32<E>(hot && kt * TILE + PvStep<E>::key_of(s2, half, i) < n_keys ? 1.f : 0.f);
              }
              mfma32(hit[0], is, pv[s2]);
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
        for (int t = 0; t < DT; ++t) mfma32(o[t], v[s2][t], pv[s2]);
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
    float* part = a.part + (int64_t)(c.slot + c.part) * (ROWS * (PROW + 2));      // [ROWS][HD], then (m, l) [ROWS]
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
// features of a row; a workgroup's rows belong to one pair.  Bound by the read of the partial results.
constexpr int MERGE_THREADS = 256;
template <typename E, int HD, int ROWS, bool PV>
__global__ __launch_bounds__(MERGE_THREADS) void attend_merge_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  constexpr int CHUNKS = PV ? HD / 4 : 1, PROW = PV ? HD : 0, PER = MERGE_THREADS / CHUNKS < ROWS ? MERGE_THREADS / CHUNKS : ROWS;
  const Plan plan = make_plan<ROWS>(a);
  const int q = blockIdx.x % (ROWS / PER) * PER + (int)threadIdx.x / CHUNKS, d = threadIdx.x % CHUNKS * 4;
  const uint32_t pair = blockIdx.x / (ROWS / PER);
  if (pair >= plan.cut) return;
  const Piece c = piece_at(plan, pair, a.geom.n_heads, true);
  const int row = c.group * ROWS + q, n_rows = (a.tok.span.off[c.seq + 1] - a.tok.span.off[c.seq]) * a.group;
  if ((int)threadIdx.x / CHUNKS >= PER || row >= n_rows) return;
  const float* part = a.part + (int64_t)c.slot * (ROWS * (PROW + 2));
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

template <typename E, int HD, int NP, int RG, bool PV> constexpr size_t attend_lds() {
  const size_t fold = (size_t)ATTEND_WAVES * ((PV ? HD / TILE * 16 : 0) + 2) * WAVE * 4;
  const size_t walk = (size_t)RG * (HD / ET<E>::KS) * NP * WAVE * 16 + ATTN_MAX_PAGES * 4;
  return fold > walk ? fold : walk;
}
size_t attend_part_bytes(int head_dim) { return (size_t)ATTEND_SLOTS * 2 * TILE * (head_dim + 2) * 4; }

template <typename E, int HD, int NP, int RG, bool PV> static void launch_attend_t(AttendArgs a, hipStream_t st) {
  constexpr int ROWS = RG * TILE, PER = MERGE_THREADS / (PV ? HD / 4 : 1) < ROWS ? MERGE_THREADS / (PV ? HD / 4 : 1) : ROWS;
  int64_t pairs = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) pairs += ((int64_t)(a.tok.span.off[s + 1] - a.tok.span.off[s]) * a.group + ROWS - 1) / ROWS;
  pairs *= a.geom.n_heads;
  a.whole = single_slice() || a.tok.limit <= ATTEND_MIN_CUT * TILE;
  const int64_t wgs = a.whole ? pairs : pairs + ATTEND_PARTS;
  attend_kernel<E, HD, NP, RG, PV><<<(unsigned)((wgs + 7) / 8 * 8), ATTEND_WAVES * WAVE, attend_lds<E, HD, NP, RG, PV>(), st>>>(a, live_word());
  if (a.whole) return;
  const int64_t cut = pairs < ATTEND_PARTS ? pairs : ATTEND_PARTS;
  attend_merge_kernel<E, HD, ROWS, PV><<<(unsigned)(cut * (ROWS / PER)), MERGE_THREADS, 0, st>>>(a, live_word());
}
template <typename E, int HD, int RG> static void launch_attend_rg(int planes, const AttendArgs& a, hipStream_t st) {
  if (a.out) launch_attend_t<E, HD, 1, RG, true>(a, st);
  else if (planes == 1) launch_attend_t<E, HD, 1, RG, false>(a, st);
  else if constexpr (sizeof(E) == 2) launch_attend_t<E, HD, 2, RG, false>(a, st);
}
// Two row tiles per workgroup where a sequence has more than one.
template <int HD> static void launch_attend_hd(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  int most = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) {
    const int rows = (a.tok.span.off[s + 1] - a.tok.span.off[s]) * a.group;
    most = rows > most ? rows : most;
  }
  if (bf16) {
    if (most <= TILE) launch_attend_rg<bf16_t, HD, 1>(planes, a, st);
    else launch_attend_rg<bf16_t, HD, 2>(planes, a, st);
  } else {
    if (most <= TILE) launch_attend_rg<float, HD, 1>(planes, a, st);
    else launch_attend_rg<float, HD, 2>(planes, a, st);
  }
}
void launch_attend(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_attend_hd<128>(bf16, planes, a, st);
  else launch_attend_hd<64>(bf16, planes, a, st);
}

template <typename E, int HD, int RG> static bool configure_attend_t() {
  return hipFuncSetAttribute((const void*)attend_kernel<E, HD, 1, RG, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)attend_lds<E, HD, 1, RG, true>()) == hipSuccess;
}
bool configure_attend() {
  const bool ok = configure_attend_t<bf16_t, 128, 1>() && configure_attend_t<bf16_t, 128, 2>() && configure_attend_t<bf16_t, 64, 1>() &&
                  configure_attend_t<bf16_t, 64, 2>() && configure_attend_t<float, 128, 1>() && configure_attend_t<float, 128, 2>() &&
                  configure_attend_t<float, 64, 1>() && configure_attend_t<float, 64, 2>();
  (void)hipGetLastError();
  return ok;
}

// ------------------------------------------------------------------------------------------------
// Attention weight that cached positions gather: score[head][key] = decay * score[head][key] + the sum over the rows of the
// head's group of exp(scale * q . k - lse).  Here rows run along the registers and keys along the lanes (A = Q, B = K), so a
// key's sum over 32 rows is an addition of 16 registers and one exchange between the half-waves, and every score has one writer:
// no atomics, the same bits every time.  Bound by the read of K.
// ------------------------------------------------------------------------------------------------
constexpr int SCORE_WAVES = 4;
template <typename E, int HD, int NP>
__global__ __launch_bounds__(SCORE_WAVES * WAVE) void score_kernel(ScoreArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS;
  const int head = blockIdx.y, seq = blockIdx.z;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0;
  if (len == 0) return;
  const int base = cache_base(a.tok, seq, len), n_keys = min(base + len, a.score_stride);
  const int kt = blockIdx.x * SCORE_WAVES + wave, n_rows = len * a.group;
  if (kt * TILE >= n_keys) return;
  const bool masked = a.visible != nullptr;
  const int key = kt * TILE + col, n_q_heads = a.geom.n_heads * a.group;
  vec k[DSTEPS];
  {
    const int at = min(key, n_keys - 1);
    const int page = safe_page(a.geom, a.tok.page_table[(int64_t)seq * a.tok.pt_stride + at / PAGE]);
    const E* krow = (const E*)a.kv_layer + kv_k_index(a.geom, page, head, at % PAGE, 0) + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) k[s] = load16<E>(krow + s * (PAGE * KS));
  }
  __shared__ float s_lse[SCORE_WAVES][TILE];
  __shared__ uint64_t s_word[SCORE_WAVES][TILE];
  const float c2 = a.scale * LOG2E;
  float sum = 0.f;
  for (int row0 = 0; row0 < n_rows; row0 += TILE) {
    const int row = row0 + min(col, n_rows - row0 - 1), tok = tok0 + row / a.group, q_head = head * a.group + row % a.group;
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
    f32x16 s[1];
    zero_acc<1>(s);
#pragma unroll
    for (int i = 0; i < DSTEPS * NP; ++i) mfma32(s[0], load16<E>(qrow + (i % NP) * a.q_plane + (i / NP) * KS), k[i / NP]);
    if (half == 0) {
      // rows past the last one, and rows that see nothing (lse = -inf), weigh nothing
      const float lse = a.lse[(int64_t)tok * n_q_heads + q_head];
      s_lse[wave][col] = row0 + col < n_rows && lse != -INFINITY ? lse * LOG2E : INFINITY;
      s_word[wave][col] = masked ? a.visible[tok] : ~0ull;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const bool tail = (kt + 1) * TILE > base && masked;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float l = s_lse[wave][acc_row(v, half)];
      float p = __builtin_amdgcn_exp2f(fmaf(s[0][v], c2, -l));
      if (l == INFINITY) p = 0.f;                                             // (a score that is not a number included)
      if (tail && !sees(s_word[wave][acc_row(v, half)], true, key - base)) p = 0.f;
      sum += p;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  sum += __shfl_xor(sum, 32, WAVE);
  if (half == 0 && key < n_keys) {
    const int64_t at = ((int64_t)seq * a.geom.n_heads + head) * a.score_stride + key;
    a.score_out[at] = a.score_in ? fmaf(a.decay, a.score_in[at], sum) : sum;
  }
}

template <int HD> static void launch_score_hd(bool bf16, int planes, const ScoreArgs& a, hipStream_t st) {
  const int bound = a.tok.limit < a.score_stride ? a.tok.limit : a.score_stride;
  const dim3 grid((bound + SCORE_WAVES * TILE - 1) / (SCORE_WAVES * TILE), a.geom.n_heads, a.tok.span.n_seq);
  if (!bf16) score_kernel<float, HD, 1><<<grid, SCORE_WAVES * WAVE, 0, st>>>(a, live_word());
  else if (planes == 1) score_kernel<bf16_t, HD, 1><<<grid, SCORE_WAVES * WAVE, 0, st>>>(a, live_word());
  else score_kernel<bf16_t, HD, 2><<<grid, SCORE_WAVES * WAVE, 0, st>>>(a, live_word());
}
void launch_score(bool bf16, int planes, const ScoreArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_score_hd<128>(bf16, planes, a, st);
  else launch_score_hd<64>(bf16, planes, a, st);
}

}  // namespace dinfer
