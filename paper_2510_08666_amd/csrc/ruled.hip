// Attention of a sequence's new tokens over its cached positions and over each other under a rule: causal by blocks, windows, a
// prefix that all see, documents, capped scores, a bias by distance.  What a row sees is at most two ranges of cache positions
// (row_ranges), so that a group of rows walks only the key tiles in which it sees anything, and looks at single keys only in
// those that not all of them see whole.
//
// Bound: the matrix instructions of the pairs that are seen (4 * head_dim operations each, at the 1.23 PFLOP/s of a large matrix product) or, for
// few rows, one read of the keys and values.  Few rows take the kernel of attend_kernel.hpp with RangeRule for its words: a token behind
// 511 positions 10.4 us (the chain of dependent loads), 48 tokens behind 1000 to 8000 in a window of 4097 with 8 heads of 4 queries 130 us (5.1 TB/s),
// 512 tokens behind 4096, causal by blocks of 32, 39.2 us (0.47 PFLOP/s), prompts of 333 to 1811 tokens in documents of 301 with capped scores
// 48 us (0.21 PFLOP/s: groups of rows in two documents walk both, all tiles partly seen, and end last).  Two row tiles hold their weights as
// one bfloat16 number (off by 2^-8 at most), which takes half as many matrix instructions out of the product with the values: 47.0 -> 43.2 us and
// 63.6 -> 60.2 with the joins; one row tile waits for memory and keeps two.  In tiles that are partly seen, values that are not finite are looked for only where an output has come out so, in a
// second walk: 60.3 -> 47.6 us for the documents, 43.9 -> 41.9 for the chunk.
#include "attend_kernel.hpp"

namespace dinfer {

// Many rows: a wave takes 32 rows of a cache head, a workgroup of WAVES waves WAVES times as many, and key tiles go through LDS once for
// all of them.  In a turn a wave multiplies (the next tile's keys with its queries, this tile's values with their weights, matrix
// instructions that are fed from LDS without a pause), brings in its share of a later tile and works out the exponentials of the scores that
// it multiplied.  Four buffers: V of tile i, K of tile i + 1, the first fragments of K of tile i + 2, tile i + 3 on its way in.  Weights enter
// the product with the values as one bfloat16 number each, rounded to nearest (off by 2^-8 at most; the sum of a row is that of the
// weights before): a second one would be half as many matrix instructions more.
//
// WAVES = 4: 128 rows, tiles of 32 keys, two workgroups per compute unit, whose waves on a SIMD cover each other as they come; loads are under way
// for two turns.  A workgroup alone on its compute unit takes 1800 cycles a turn, 512 of them its matrix instructions.
// WAVES = 8: 256 rows, tiles of 64 keys, one workgroup per compute unit, and the two waves of a SIMD in two phases by barriers: one multiplies
// while the other one does the rest, then they change places; a wave of the half that is behind still reads tile i while tile i + 3 comes in.
// A causal prompt of 8191 tokens, 8 heads of 4 queries and 128 features: 530 to 550 us, 1.0 PFLOP/s (WAVES = 4: 595), the matrix units busy in 48 %
// of the cycles.  A phase of matrix work takes 1480
// cycles, 1024 of them the instructions' own, LDS gives 119 bytes a cycle, and the clock is 1.88 GHz.  Slower were: 4 waves of 32 rows with
// the products of two tiles woven together (620 to 640 us); 64 rows per wave (842 and more, accumulators move between register files); half of the
// values straight from L1 (813).
constexpr int RULED_BUFFERS = 4;
constexpr int key_tiles(int waves) { return waves / 4; }      // of 32 keys, that go through LDS together
template <int HD, int WAVES> constexpr size_t ruled_rows_lds() {
  return (size_t)RULED_BUFFERS * 2 * key_tiles(WAVES) * (HD / ET<bf16_t>::KS) * WAVE * 16 + (ATTN_MAX_PAGES + 4) * 4;
}
// (NaN if one of them is: a row with such a score is not a number anyway, and the instruction takes matrix results as they are)
__device__ inline float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float both_halves_max(float v) {
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return larger(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
template <class Rule, int HD, int WAVES>
__global__ __launch_bounds__(WAVES * WAVE, 2) void ruled_rows_kernel(AttendArgs a, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef bf16_t E;
  typedef ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, DT = HD / TILE, NT = key_tiles(WAVES), KEYS = NT * TILE, STEPS = KEYS / PAGE, ROWS = WAVES * TILE;
  constexpr bool PHASES = WAVES == 8;
  constexpr int SETS = PHASES ? 1 : 2, AHEAD = 3 + SETS;      // tiles on their way in, and how far in front of its products a tile's loads are issued
  // Fragments of a tile, K and then V, and those that a wave fetches: of K consecutive steps of one row tile, of V feature tiles of one step.
  constexpr int KF = NT * DSTEPS, VF = STEPS * DT, FRAGS = KF + VF, K_MINE = KF / WAVES, V_MINE = VF / WAVES;
  static_assert(K_MINE * WAVES == KF && V_MINE * WAVES == VF && DSTEPS % K_MINE == 0 && DT % V_MINE == 0, "whole fragments");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const E* kv = (const E*)a.kv_layer;
  extern __shared__ __align__(16) char smem[];
  auto tiles = reinterpret_cast<vec(*)[FRAGS][WAVE]>(smem);
  int32_t* pt = reinterpret_cast<int32_t*>(smem + (size_t)RULED_BUFFERS * FRAGS * WAVE * 16);
  __shared__ GroupRanges s_group[WAVES];
  __shared__ int32_t s_odd;      // some value that is not finite was replaced
  const Plan plan = make_plan<E, ROWS, Rule>(a);
  if (blockIdx.x >= plan.total) return;
  const Piece c = piece_by_heads(plan, blockIdx.x, a.geom.n_heads);
  const int tile0 = Rule::first_tile(a, c.base) / NT;      // of KEYS
  const int tok0 = a.tok.span.off[c.seq], row0 = c.group * ROWS, n_rows = (a.tok.span.off[c.seq + 1] - tok0) * a.group - row0;
  const int n_keys = c.base + a.tok.span.off[c.seq + 1] - tok0, last_page = (n_keys - 1) / PAGE - STEPS * tile0;
  if (!a.whole) note_cut(a, plan, c, blockIdx.x, row0);
  {
    const int32_t* pages = a.tok.page_table + (int64_t)c.seq * a.tok.pt_stride + STEPS * tile0;
    for (int i = threadIdx.x; i <= last_page; i += WAVES * WAVE) pt[i] = safe_page(a.geom, pages[i]);
  }
  const int row = row0 + min(wave * TILE + col, n_rows - 1), tok = tok0 + row / a.group, q_head = c.head * a.group + row % a.group;
  vec q[DSTEPS];
  {
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + q_head * HD + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) q[s] = load16<E>(qrow + s * KS);
  }
  Rule rule;
  rule.start_row(a, c.seq, tok, c.base + tok - tok0, q_head, n_keys);
  GroupRanges group;
  group.take(rule.see);
  group.join_columns();
  if (lane == 0) s_group[wave] = group;
  if (threadIdx.x == 0) s_odd = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) group.join(s_group[w]);
  TileWalk walk;
  walk.start(group, tile0, (n_keys + KEYS - 1) / KEYS, KEYS);
  const int all = walk.tiles(), i0 = all * c.part / c.parts, i1 = all * (c.part + 1) / c.parts, whole = walk.whole(), masked = min(whole, i1);

  f32x16 o[DT];
  zero_acc<DT>(o);
  float m_run = -INFINITY, l_run = 0.f, ref = 0.f;
  const float c2 = a.scale * LOG2E, to_log2 = rule.factor(c2);
  if (i0 < i1) {
    struct Fetched {
      vec k[K_MINE], v[V_MINE];
    };
    // Where this lane's pieces of a tile are: a page of its four and the place in it (keys past the last one are read from where they would
    // be, and masked).  A tile's number and pages are looked up a turn before its loads.
    const int k_page = wave * K_MINE / DSTEPS * 2 + PvStep<E>::key_of_row(col) / PAGE, v_page = wave * V_MINE / DT;
    const E* lane_k = kv + kv_k_index(a.geom, 0, c.head, PvStep<E>::key_of_row(col) % PAGE, 0) + half * G + wave * K_MINE % DSTEPS * (PAGE * KS);
    const E* lane_v = kv + kv_v_index(a.geom, 0, c.head, 0, col) + 8 * half + wave * V_MINE % DT * (TILE * PAGE);
    const uint32_t page_elems = (uint32_t)a.geom.page_stride;
    auto tile_at = [&](int i) __attribute__((always_inline)) { return walk.tile(min(i, i1 - 1)); };
    auto page_at = [&](int kt, int page) __attribute__((always_inline)) { return (uint32_t)pt[min(STEPS * (kt - tile0) + page, last_page)]; };
    auto fetch = [&](Fetched& next, uint32_t of_k, uint32_t of_v) __attribute__((always_inline)) {
      const E *k = lane_k + (uint64_t)of_k * page_elems, *v = lane_v + (uint64_t)of_v * page_elems;
#pragma unroll
      for (int j = 0; j < K_MINE; ++j) next.k[j] = load16<E>(k + j * (PAGE * KS));
#pragma unroll
      for (int j = 0; j < V_MINE; ++j) next.v[j] = load16<E>(v + j * (TILE * PAGE));
    };
    auto put = [&](Fetched& next, int i, int kt) __attribute__((always_inline)) {
      if (i >= masked) {
        // Values of a tile that not all rows see whole: those past the last key, which may hold anything, become 0, and so does what is no
        // finite number (rows that see it are found at the end).
        const int valid = i < i1 ? n_keys - (kt * KEYS + v_page * PAGE + 8 * half) : 0;
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < V_MINE; ++j) {
          u32x4 w = words_of<E>(next.v[j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            w[k] &= ValueBits<E>::mask(k, valid);
            most = ValueBits<E>::larger(most, w[k]);
            w[k] = ValueBits<E>::finite(w[k]);
          }
          next.v[j] = __builtin_bit_cast(vec, w);
        }
        if (ValueBits<E>::largest(most) >= ValueBits<E>::ODD) s_odd = 1;
      }
      // K as [row tile][k-step], V as [step][feature tile]
      auto& to = tiles[i & (RULED_BUFFERS - 1)];
#pragma unroll
      for (int j = 0; j < K_MINE; ++j) to[wave * K_MINE + j][lane] = next.k[j];
#pragma unroll
      for (int j = 0; j < V_MINE; ++j) to[KF + wave * V_MINE + j][lane] = next.v[j];
    };
    f32x16 s[NT];
    u32x4 pw[STEPS];
    // Scores of tile i to weights, and the reference maximum moved where a score passes it by more than SLACK.
    auto weigh = [&](int i, int kt) __attribute__((always_inline)) {
      constexpr float SLACK = 6.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) rule.template scores<E>(s[n], c2, kt * KEYS + n * TILE, half);
      if (i >= masked) {
        const int key0 = i < i1 ? kt * KEYS : INT32_MAX / 2;      // (that nobody sees)
#pragma unroll
        for (int n = 0; n < NT; ++n) rule.template hide<E>(s[n], key0 + n * TILE, half);
      }
      float mx = s[0][0];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = larger(mx, s[n][v]);
      const float mt = both_halves_max(mx) * to_log2;
      const bool moves = mt > m_run + SLACK;
      if (__builtin_amdgcn_ballot_w64(moves)) {
        const float alpha = moves ? __builtin_amdgcn_exp2f(m_run - mt) : 1.f;
        l_run *= alpha;
        m_run = moves ? mt : m_run;
        ref = m_run > -INFINITY ? m_run : 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[t][v] *= alpha;
      }
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < STEPS; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
          const float x = __builtin_amdgcn_exp2f(fmaf(s[u / 2][8 * (u % 2) + 2 * j], to_log2, -ref));
          const float y = __builtin_amdgcn_exp2f(fmaf(s[u / 2][8 * (u % 2) + 2 * j + 1], to_log2, -ref));
          sum[j] += x + y;
          pw[u][j] = __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)x, (bf16_t)y});
        }
      l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    int kt[AHEAD + 1];      // of tiles i .. i + AHEAD
#pragma unroll
    for (int k = 0; k <= AHEAD; ++k) kt[k] = tile_at(i0 + k);
    Fetched next[SETS];
    {
      Fetched first[3];      // (all at once: there is no output to hold yet)
#pragma unroll
      for (int k = 0; k < 3; ++k) fetch(first[k], page_at(kt[k], k_page), page_at(kt[k], v_page));
#pragma unroll
      for (int k = 0; k < SETS; ++k) fetch(next[k], page_at(kt[3 + k], k_page), page_at(kt[3 + k], v_page));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 3; ++k) put(first[k], i0 + k, kt[k]);
    }
    uint32_t of_k = page_at(kt[AHEAD], k_page), of_v = page_at(kt[AHEAD], v_page);
    __syncthreads();
    constexpr int RD = 4;
    vec ring[RD];
    auto k_frag = [&](int i, int f) __attribute__((always_inline)) { return tiles[i & (RULED_BUFFERS - 1)][f % NT * DSTEPS + f / NT][lane]; };
    zero_acc<NT>(s);
#pragma unroll
    for (int f = 0; f < KF; ++f) mfma32(s[f % NT], k_frag(i0, f), q[f / NT]);
    weigh(i0, kt[0]);
#pragma unroll
    for (int f = 0; f < RD; ++f) ring[f] = k_frag(i0 + 1, f);
    // the waves of the second half run a phase behind those of the first
    if (PHASES && wave >= WAVES / 2) __builtin_amdgcn_s_barrier();
    auto turn = [&](int i, Fetched& next) __attribute__((always_inline)) {
      zero_acc<NT>(s);
#pragma unroll
      for (int f = 0; f < FRAGS; ++f) {
        const vec x = ring[f % RD];
        const int n = f + RD;
        if (n < FRAGS) ring[f % RD] = n < KF ? k_frag(i + 1, n) : tiles[i & (RULED_BUFFERS - 1)][n][lane];
        __builtin_amdgcn_sched_barrier(0);
        if (f < KF) mfma32(s[f % NT], x, q[f / NT]);
        else mfma32(o[(f - KF) % DT], x, __builtin_bit_cast(vec, pw[(f - KF) / DT]));
      }
      __builtin_amdgcn_sched_barrier(0);
      // (this wave's reads have come in: its matrix instructions took them)
      if constexpr (PHASES) asm volatile("s_barrier" ::: "memory");
      put(next, i + 3, kt[3]);
      fetch(next, of_k, of_v);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) kt[k] = kt[k + 1];
      kt[AHEAD] = tile_at(i + AHEAD + 1);
      of_k = page_at(kt[AHEAD], k_page);
      of_v = page_at(kt[AHEAD], v_page);
      weigh(i + 1, kt[0]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < RD; ++f) ring[f] = k_frag(i + 2, f);
      // (all but the fragments just asked for: what this wave put is there)
      asm volatile("s_waitcnt lgkmcnt(4)\n\ts_barrier" ::: "memory");
      static_assert(RD == 4, "the count above");
    };
    for (int i = i0; i < i1; i += SETS) {
      turn(i, next[0]);
      if (SETS == 2 && i + 1 < i1) turn(i + 1, next[SETS - 1]);
    }
    if (PHASES && wave < WAVES / 2) __builtin_amdgcn_s_barrier();
  }
  // Rows with weight on a value that was replaced: products of the weights with its indicator, one kind (NaN, +inf, -inf) at a time, over
  // the tiles again, 32 keys of them at a time.
  __syncthreads();
  if (i0 < i1 && s_odd != 0) {
#pragma unroll 1
    for (int i = NT * max(i0, whole); i < NT * i1; ++i) {
      const int key0 = walk.tile(i / NT) * KEYS + i % NT * TILE;
      const int key = key0 + PvStep<E>::key_of_row(col), page0 = key0 / PAGE - STEPS * tile0;
      const E* krow = kv + kv_k_index(a.geom, pt[min(page0 + PvStep<E>::key_of_row(col) / PAGE, last_page)], c.head, key % PAGE, 0) + half * G;
      f32x16 x[1];
      zero_acc<1>(x);
#pragma unroll
      for (int f = 0; f < DSTEPS; ++f) mfma32(x[0], load16<E>(krow + f * (PAGE * KS)), q[f]);
      rule.template scores<E>(x[0], c2, key0, half);
      float p[16];
#pragma unroll
      for (int v = 0; v < 16; ++v)
        p[v] = rule.sees(key0 + PvStep<E>::key_of_acc(v, half)) ? __builtin_amdgcn_exp2f(fmaf(x[0][v], to_log2, -ref)) : 0.f;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
          f32x16 hit[1];
          zero_acc<1>(hit);
#pragma unroll
          for (int step = 0; step < 2; ++step) {
            const E* vrow = kv + kv_v_index(a.geom, pt[min(page0 + step, last_page)], c.head, 0, t * TILE + col);
            mfma32(hit[0], odd_values<E>(PvStep<E>::v_vec(vrow, half, step), kind, n_keys - (key0 + PvStep<E>::key_of(step, half, 0))), PvStep<E>::p_vec(p, step, 0));
          }
          const float odd = kind == 0 ? __builtin_nanf("") : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
          for (int v = 0; v < 16; ++v) o[t][v] += hit[0][v] != 0.f ? odd : 0.f;      // (a weight that is not a number: no number)
        }
    }
  }
  const int at = wave * TILE + col;
  const float L = l_run + __shfl_xor(l_run, 32, WAVE);
  if (at >= n_rows) return;
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
        *reinterpret_cast<f32x4*>(part + at * HD + t * TILE + acc_row(4 * g, half)) =
            f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
    if (half == 0) *reinterpret_cast<float2*>(part + ROWS * HD + 2 * at) = float2{m_run, L};
  }
}
template <class Rule, int HD, int WAVES> static void launch_ruled_rows(AttendArgs a, hipStream_t st) {
  const AttendGrid g = attend_grid<bf16_t, WAVES * TILE, Rule>(a);
  ruled_rows_kernel<Rule, HD, WAVES><<<g.wgs, WAVES * WAVE, ruled_rows_lds<HD, WAVES>(), st>>>(a, live_word());
  launch_merge<bf16_t, HD, WAVES * TILE, true>(a, g.cut, st);
}
template <class Rule, int HD, int WAVES> static bool configure_ruled_rows() {
  return hipFuncSetAttribute((const void*)ruled_rows_kernel<Rule, HD, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)ruled_rows_lds<HD, WAVES>()) == hipSuccess;
}

// Meetings of a row tile with a key tile, as far as the host can tell (the lengths are on the device): as if caches were full, half of a
// sequence's own keys seen where there is an order in time, no more than its window.
static int64_t likely_meetings(const AttendArgs& a) {
  int64_t sum = 0;
  for (int s = 0; s < a.tok.span.n_seq; ++s) {
    const int len = a.tok.span.off[s + 1] - a.tok.span.off[s];
    if (!a.rule.takes(len * a.group)) continue;
    int keys = a.tok.limit - (a.rule.block > 0 ? len / 2 : 0);
    if (a.rule.window > 0 && !a.rule.prefix) keys = keys < a.rule.window * (a.rule.block > 0 ? 1 : 2) + TILE ? keys : a.rule.window * (a.rule.block > 0 ? 1 : 2) + TILE;
    sum += ((int64_t)len * a.group + TILE - 1) / TILE * ((keys + TILE - 1) / TILE);
  }
  return sum * a.geom.n_heads / (a.rule.first || a.rule.end ? 8 : 1);      // (documents: most of them are much shorter than the sequence)
}
// The forms of many rows where a call has that many of them (counted in heads of 128 features).  Their workgroups take 9 and 13 us to begin and end,
// those of two row tiles 8, but those are twice as many and read keys twice and four times as often.  Two row tiles | WAVES = 4 | 8, all with
// their joins, 16 heads unless stated, in us (thousands of meetings in front): 8, a causal prompt of 1000 tokens 32 | 37 | 45; 17, 256 tokens behind
// 4096 32 | 42 | 47; 26, four prompts of 1811 in documents of 301 74 | 79 | 98; 32, 2000 causal 54 | 54 | 61; 36, 512 behind 2000, 8 heads of 4
// queries 45 | 48 | 50; 37, 512 behind 4096 44 | 51 | 53; 63, 2000 causal, 8 heads of 4 queries 71 | 61 | 67; 67, 8000 in a window of 512 83 | 82 |
// 98; 74, 1024 behind 4096 74 | 69 | 70; 98, 512 behind 12000 85 | 82 | 82; 126, 4000 causal 141 | 113 | 119; 192, 24 sequences of 17 to 32
// behind 1000 to 8000, 8 heads of 4 queries 148 | 115 | 175; 259, 8000 in a window of 2048 200 | 172 | 178; 282, 6000 causal 256 | 194 | 196; 500, 8000
// causal 404 | 316 | 296; 632, four of 2000 behind 4000 533 | 409 | 384; 1000, 8191 causal, 8 heads of 4 queries 778 | 592 | 552.
constexpr int64_t RULED_FEW = 3 << 14, RULED_MANY = 25 << 14;
// Sequences of at most one row tile keep two numbers per weight, whatever else is in the call.  Beside them longer ones take one row tile per
// workgroup too, or, where they would take a form of many rows, that form in a launch of its own.  All in one tile | two launches | all in the longest
// one's form, with its weights, us, 16 heads unless stated: 8 sequences of 1 to 40 tokens behind 10 to 300 10.6 | 22.1 | 12.0, behind 500 to 2300 29.8 | 45.4 |
// 34.8, 24 of 17 to 40 behind 1000 to 8000 173 | 198 | 219, 48 of 1 to 16, 8 heads of 4 queries 180 | 216 | 215, 4 of 1 to 300 behind 100 to 4000 45.7 | 58.9 |
// 40.5; from RULED_FEW on: 12 of 1 to 500 behind 100 to 3000 119 | 120 | 108, 3 of 1 to 2000 137 | 133 | 121, 24 of 1 to 2000 860 | 595 | 586.
template <class Rule, int HD> static void launch_ruled_t(bool bf16, AttendArgs a, hipStream_t st) {
  const int most = most_rows(a);
  bool few = !bf16 || most <= TILE;      // some sequence takes one row tile
  for (int s = 0; s < a.tok.span.n_seq; ++s) few = few || (rows_of(a, s) > 0 && rows_of(a, s) <= TILE);
  a.rule.least_rows = TILE + 1, a.rule.most_rows = INT32_MAX;
  const int64_t weight = bf16 && most > 2 * TILE ? likely_meetings(a) * HD : 0;
  if (few) {
    a.rule.least_rows = 0, a.rule.most_rows = weight >= RULED_FEW * 128 ? TILE : INT32_MAX;
    if (bf16) launch_attend_t<bf16_t, HD, 1, 1, true, Rule>(a, st);
    else launch_attend_t<float, HD, 1, 1, true, Rule>(a, st);
    if (a.rule.most_rows > TILE) return;
    a.rule.least_rows = TILE + 1, a.rule.most_rows = INT32_MAX;
  }
  if (weight >= RULED_MANY * 128) launch_ruled_rows<Rule, HD, 8>(a, st);
  else if (weight >= RULED_FEW * 128) launch_ruled_rows<Rule, HD, 4>(a, st);
  else launch_attend_t<bf16_t, HD, 1, 2, true, Rule>(a, st);
}
template <class Rule> static void launch_ruled_hd(bool bf16, const AttendArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_ruled_t<Rule, 128>(bf16, a, st);
  else launch_ruled_t<Rule, 64>(bf16, a, st);
}
void launch_ruled(bool bf16, AttendArgs a, hipStream_t st) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slope != nullptr;
  if (cap) CapScores::prepare(a.rule, a.scale);
  if (cap && bias) launch_ruled_hd<RangeRule<true, true>>(bf16, a, st);
  else if (cap) launch_ruled_hd<RangeRule<true, false>>(bf16, a, st);
  else if (bias) launch_ruled_hd<RangeRule<false, true>>(bf16, a, st);
  else launch_ruled_hd<RangeRule<false, false>>(bf16, a, st);
}

template <class Rule, int HD> static bool configure_ruled_t() {
  return configure_attend_t<bf16_t, HD, 1, Rule>() && configure_attend_t<bf16_t, HD, 2, Rule>() && configure_attend_t<float, HD, 1, Rule>() &&
         configure_ruled_rows<Rule, HD, 4>() && configure_ruled_rows<Rule, HD, 8>();
}
template <class Rule> static bool configure_ruled_hd() { return configure_ruled_t<Rule, 64>() && configure_ruled_t<Rule, 128>(); }
bool configure_ruled() {
  const bool ok = configure_ruled_hd<RangeRule<false, false>>() && configure_ruled_hd<RangeRule<true, false>>() &&
                  configure_ruled_hd<RangeRule<false, true>>() && configure_ruled_hd<RangeRule<true, true>>();
  (void)hipGetLastError();
  return ok;
}

}  // namespace dinfer
