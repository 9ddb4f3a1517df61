// Attention of a sequence's new tokens over its cached positions and, as far as their visibility words allow, over each
// other: softmax(scale * q . K^T) . V in one pass over the keys, with the running maximum and sum of every row in float32.
//
// The queries of all query heads that share a cache head are rows of the same contraction (row = token * group + member), so
// that a tile of 32 rows reads its head's keys once.  MFMA mapping as in attention.hip: S^T[key][row] = K . Q^T, a lane owns
// one row, O^T[d][row] += V^T . P^T from the score registers.  Queries enter as they are (bfloat16 queries are exact), and
// probabilities as two bfloat16 planes (PvWeights), so that an output is rounded once, when it is stored.
#include "attend_kernel.hpp"

namespace dinfer {

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

size_t attend_part_bytes(bool bf16, int head_dim, int max_pos) {
  if (max_pos <= (bf16 ? min_cut<bf16_t>() : min_cut<float>()) * TILE) return 0;      // nothing is cut
  const size_t rows = (size_t)2 * resident(8 * TILE) * 8 * TILE, few = (size_t)2 * resident(4 * TILE) * 4 * TILE;
  return (rows > few ? rows : few) * (head_dim + 2) * 4 + sizeof(CutList);
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
  const int most = most_rows(a);
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
