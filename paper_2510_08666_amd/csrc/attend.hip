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

constexpr int ATTEND_WAVES = 4;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

size_t attend_part_bytes(int head_dim) { return (size_t)ATTEND_MAX_SHARED * TILE * (head_dim + 2) * 4; }

void fill_tiles(const SeqSpan& span, int group, SeqSpan* tiles) {
  tiles->n_seq = span.n_seq;
  tiles->off[0] = 0;
  for (int s = 0; s < span.n_seq; ++s)
    tiles->off[s + 1] = tiles->off[s] + ((span.off[s + 1] - span.off[s]) * group + TILE - 1) / TILE;
}

// Bit of a key among the sequence's new tokens: keys in front of them are seen by everybody.
__device__ inline bool sees(uint64_t word, bool masked, int rel) { return rel < 0 || !masked || ((word >> (rel & 63)) & 1); }

template <typename E> __device__ inline bool not_finite(E v);
template <> __device__ inline bool not_finite<float>(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
template <> __device__ inline bool not_finite<bf16_t>(bf16_t v) { return (__builtin_bit_cast(uint16_t, v) & 0x7f80u) == 0x7f80u; }

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

template <typename E, int HD, int NP, bool PV>
__global__ __launch_bounds__(ATTEND_WAVES * WAVE) void attend_kernel(AttendArgs a, int n_splits, const int32_t* __restrict__ live) {
  if (step_is_dead(live)) return;
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, KS = ET<E>::KS, DSTEPS = HD / KS, DT = PV ? HD / TILE : 1, STEPS = PvStep<E>::STEPS;
  constexpr int OPL = PV ? HD / TILE * 16 / ATTEND_WAVES : 0;      // output registers a wave finishes
  const int split = blockIdx.z, head = blockIdx.y, tile = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int seq = owner_of(a.tiles, tile);
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0;
  const int row0 = (tile - a.tiles.off[seq]) * TILE, n_rows = len * a.group - row0;      // rows of this tile on: >= 1
  const int base = cache_base(a.tok, seq, len), n_keys = base + len;
  const int my_splits = min(attn_splits_for(n_keys), n_splits);
  if (split >= my_splits) return;
  const bool masked = a.visible != nullptr;
  const E* kv = (const E*)a.kv_layer;

  __shared__ int32_t pt[ATTN_MAX_PAGES];
  {
    const int32_t* row = a.tok.page_table + (int64_t)seq * a.tok.pt_stride;
    const int n_pages = (n_keys + PAGE - 1) / PAGE;        // <= pt_stride, <= ATTN_MAX_PAGES (host checks)
    for (int i = threadIdx.x; i < n_pages; i += blockDim.x) pt[i] = row[i];
  }
  const int row = row0 + min(col, n_rows - 1), tok = tok0 + row / a.group, member = row % a.group;
  const uint64_t word = masked ? a.visible[tok] : ~0ull;
  __shared__ vec qs[DSTEPS * NP * WAVE];
  {
    const E* qrow = (const E*)a.q + (int64_t)tok * a.q_stride + (head * a.group + member) * HD + half * G;
    for (int i = wave; i < DSTEPS * NP; i += ATTEND_WAVES) qs[i * WAVE + lane] = load16<E>(qrow + (i % NP) * a.q_plane + (i / NP) * KS);
  }
  __syncthreads();
  f32x16 o[DT];
  zero_acc<DT>(o);
  float m_run = -INFINITY, l_run = 0.f;
  const int n_tiles = (n_keys + TILE - 1) / TILE, stride = my_splits * ATTEND_WAVES, kt0 = split * ATTEND_WAVES + wave;
  struct TileRegs {
    vec k[DSTEPS];
    vec v[PV ? STEPS : 1][DT];
  };
  auto load_tile = [&](int kt, TileRegs& r) {
    const int key = min(kt * TILE + PvStep<E>::key_of_row(col), n_keys - 1);
    const E* krow = kv + kv_k_index(a.geom, safe_page(a.geom, pt[key / PAGE]), head, key % PAGE, 0) + half * G;
#pragma unroll
    for (int s = 0; s < DSTEPS; ++s) r.k[s] = load16<E>(krow + s * (PAGE * KS));
    if constexpr (PV) {
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) {
        const int pkey = min(kt * TILE + PvStep<E>::page_of_step(s2) * PAGE, n_keys - 1);
        const int page = safe_page(a.geom, pt[pkey / PAGE]);
#pragma unroll
        for (int t = 0; t < DT; ++t)
          r.v[s2][t] = PvStep<E>::v_vec(kv + kv_v_index(a.geom, page, head, 0, t * TILE + col), half, s2);
      }
    }
  };
  const float c2 = a.scale * LOG2E;
  auto use_tile = [&](TileRegs& cur, int kt) {
    asm volatile("" ::: "memory");      // keeps the query reads inside the loop
    f32x16 s[1];
    zero_acc<1>(s);
#pragma unroll
    for (int f = 0; f < DSTEPS * NP; ++f) mfma32(s[0], cur.k[f / NP], qs[f * WAVE + lane]);
    bool odd = false;                   // some value of a new token is no finite number
    if ((kt + 1) * TILE > base) {
      // tiles with new tokens, and the ragged end: what a row does not see scores -inf, values past the last key (which may
      // hold anything) become 0
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = kt * TILE + PvStep<E>::key_of_acc(v, half);
        if (key >= n_keys || !sees(word, masked, key - base)) s[0][v] = -INFINITY;
      }
      if constexpr (PV) {
        bool mine = false;
#pragma unroll
        for (int s2 = 0; s2 < STEPS; ++s2)
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < G; ++i) {
              if (kt * TILE + PvStep<E>::key_of(s2, half, i) >= n_keys) cur.v[s2][t][i] = (E)0.f;
              mine |= not_finite<E>(cur.v[s2][t][i]);
            }
        odd = masked && __builtin_amdgcn_ballot_w64(mine) != 0;
      }
    }
    float p[16];
    take_scores<DT>(s[0], c2, m_run, l_run, o, p);
    if constexpr (PV) {
      vec pv[STEPS];
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2) pv[s2] = PvStep<E>::p_vec(p, s2, 0);
      if (odd) {
        // 0 * NaN would reach the rows that do not see the key: the product takes 0 in such a value's place, and the rows
        // with weight on it are found by products with its indicator, one kind (NaN, +inf, -inf) at a time
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int kind = 0; kind < 3; ++kind) {
            f32x16 hit[1];
            zero_acc<1>(hit);
#pragma unroll
            for (int s2 = 0; s2 < STEPS; ++s2) {
              vec is;
#pragma unroll
              for (int i = 0; i < G; ++i) {
                const float x = (float)cur.v[s2][t][i];
                is[i] = (E)((kind == 0 ? x != x : kind == 1 ? x == INFINITY : x == -INFINITY) ? 1.f : 0.f);
              }
              mfma32(hit[0], is, pv[s2]);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (hit[0][v] != 0.f) o[t][v] += kind == 0 ? __builtin_nanf("") : kind == 1 ? INFINITY : -INFINITY;
          }
#pragma unroll
        for (int s2 = 0; s2 < STEPS; ++s2)
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < G; ++i)
              if (not_finite<E>(cur.v[s2][t][i])) cur.v[s2][t][i] = (E)0.f;
      }
#pragma unroll
      for (int s2 = 0; s2 < STEPS; ++s2)
#pragma unroll
        for (int t = 0; t < DT; ++t) mfma32(o[t], cur.v[s2][t], pv[s2]);
    }
  };
  TileRegs ta, tb;
  if (kt0 < n_tiles) load_tile(kt0, ta);
  for (int kt = kt0; kt < n_tiles; kt += 2 * stride) {
    load_tile(min(kt + stride, n_tiles - 1), tb);
    use_tile(ta, kt);
    if (kt + stride >= n_tiles) break;
    load_tile(min(kt + 2 * stride, n_tiles - 1), ta);
    use_tile(tb, kt + stride);
  }
  // fold the waves through LDS: wave w finishes OPL of the output registers
  extern __shared__ float lds[];        // [ATTEND_WAVES][DT*16 | 0, then m, l][64 lanes]
  constexpr int REGS = PV ? DT * 16 : 0, PW = (REGS + 2) * WAVE;
  {
    float* pb = lds + wave * PW + lane;
    if constexpr (PV) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) pb[(t * 16 + v) * WAVE] = o[t][v];
    }
    pb[REGS * WAVE] = m_run;
    pb[(REGS + 1) * WAVE] = l_run + __shfl_xor(l_run, 32, WAVE);
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f, r[OPL > 0 ? OPL : 1];
#pragma unroll
  for (int w = 0; w < ATTEND_WAVES; ++w) M = fmaxf(M, lds[w * PW + REGS * WAVE + lane]);
#pragma unroll
  for (int i = 0; i < OPL; ++i) r[i] = 0.f;
#pragma unroll
  for (int w = 0; w < ATTEND_WAVES; ++w) {
    const float* pb = lds + w * PW + lane;
    const float lw = pb[(REGS + 1) * WAVE], sw = state_weight(pb[REGS * WAVE], lw, M);
    L = fmaf(sw, lw, L);
#pragma unroll
    for (int i = 0; i < OPL; ++i) r[i] = fmaf(sw, pb[(wave * OPL + i) * WAVE], r[i]);
  }
  const int n_q_heads = a.geom.n_heads * a.group, q_head = head * a.group + member;
  if (my_splits == 1) {
    if (col < n_rows) {
      if (a.lse && wave == 0 && half == 0) a.lse[(int64_t)tok * n_q_heads + q_head] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * LN2;
      const float inv = L == 0.f ? 0.f : 1.f / L;      // a row that sees nothing: zeros
#pragma unroll
      for (int i4 = 0; i4 < OPL / 4; ++i4) {
        const int g = wave * OPL + 4 * i4;
        store_elems4<E>((E*)a.out + (int64_t)tok * a.out_stride + q_head * HD + (g / 16) * TILE + acc_row(g % 16, half),
                        f32x4{r[4 * i4] * inv, r[4 * i4 + 1] * inv, r[4 * i4 + 2] * inv, r[4 * i4 + 3] * inv});
      }
    }
    return;
  }
  // shared keys: partials [32 rows][HD], then (m, l), handed over with device-coherent stores; the last to arrive folds them
  constexpr int PROW = PV ? HD : 0;
  const int pair = tile * a.geom.n_heads + head;
  const buf_rsrc pr = coherent_buffer(a.part);
  const uint32_t part_bytes = TILE * (PROW + 2) * 4, pair_bytes = (uint32_t)pair * n_splits * part_bytes;
  {
    const uint32_t pb = pair_bytes + split * part_bytes;
#pragma unroll
    for (int i4 = 0; i4 < OPL / 4; ++i4) {
      const int g = wave * OPL + 4 * i4;
      const float v4[4] = {r[4 * i4], r[4 * i4 + 1], r[4 * i4 + 2], r[4 * i4 + 3]};
      coherent_store_n<4>(pr, pb + (col * PROW + (g / 16) * TILE + acc_row(g % 16, half)) * 4, v4);
    }
    if (wave == 0 && half == 0) {
      const float ml[2] = {M, L};
      coherent_store_n<2>(pr, pb + (TILE * PROW + 2 * col) * 4, ml);
    }
  }
  __shared__ int32_t s_flag;
  if (!last_arrival(a.tickets + pair, my_splits, &s_flag)) return;
  constexpr int CHUNKS = PV ? HD / 4 : 1;      // a thread takes (row, four consecutive features) items
  for (int item = threadIdx.x; item < TILE * CHUNKS; item += ATTEND_WAVES * WAVE) {
    const int q = item / CHUNKS, d = item % CHUNKS * 4;
    if (q >= n_rows) continue;
    const int srow = row0 + q, stok = tok0 + srow / a.group, shead = head * a.group + srow % a.group;
    float Mx = -INFINITY, Ls = 0.f;
    for (int p = 0; p < my_splits; ++p) {
      float ml[2];
      coherent_load_n<2>(pr, pair_bytes + p * part_bytes + (TILE * PROW + 2 * q) * 4, ml);
      Mx = fmaxf(Mx, ml[0]);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < my_splits; ++p) {
      float ml[2];
      coherent_load_n<2>(pr, pair_bytes + p * part_bytes + (TILE * PROW + 2 * q) * 4, ml);
      const float w = state_weight(ml[0], ml[1], Mx);
      Ls = fmaf(w, ml[1], Ls);
      if constexpr (PV) {
        float op[4];
        coherent_load_n<4>(pr, pair_bytes + p * part_bytes + (q * PROW + d) * 4, op);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = fmaf(w, op[k], acc[k]);
      }
    }
    if (a.lse && d == 0) a.lse[(int64_t)stok * n_q_heads + shead] = Ls == 0.f ? -INFINITY : (Mx + __builtin_amdgcn_logf(Ls)) * LN2;
    if constexpr (PV) store_elems4<E>((E*)a.out + (int64_t)stok * a.out_stride + shead * HD + d, acc * (Ls == 0.f ? 0.f : 1.f / Ls));
  }
}

template <bool PV, int HD> constexpr size_t attend_lds() { return (size_t)ATTEND_WAVES * ((PV ? HD / TILE * 16 : 0) + 2) * WAVE * 4; }

// Key splits the grid offers: as many as the longest possible sequence asks for, but no more than it takes to give every
// compute unit one workgroup.  pairs * splits < 2 * 256 wherever there is more than one.
static int attend_splits(int pairs, int key_bound) {
  const int want = attn_splits_for(key_bound), cover = (256 + pairs - 1) / pairs;
  return want < cover ? want : cover;
}

template <typename E, int HD, int NP, bool PV> static void launch_attend_t(const AttendArgs& a, hipStream_t st) {
  const int n_tiles = a.tiles.off[a.tiles.n_seq];
  const int splits = single_slice() ? 1 : attend_splits(n_tiles * a.geom.n_heads, a.tok.limit);
  attend_kernel<E, HD, NP, PV><<<dim3(n_tiles, a.geom.n_heads, splits), ATTEND_WAVES * WAVE, attend_lds<PV, HD>(), st>>>(a, splits, live_word());
}
template <int HD> static void launch_attend_hd(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  if (!bf16) {
    if (a.out) launch_attend_t<float, HD, 1, true>(a, st);
    else launch_attend_t<float, HD, 1, false>(a, st);
  } else if (a.out) launch_attend_t<bf16_t, HD, 1, true>(a, st);
  else if (planes == 1) launch_attend_t<bf16_t, HD, 1, false>(a, st);
  else launch_attend_t<bf16_t, HD, 2, false>(a, st);
}
void launch_attend(bool bf16, int planes, const AttendArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_attend_hd<128>(bf16, planes, a, st);
  else launch_attend_hd<64>(bf16, planes, a, st);
}

bool configure_attend() {
  const void* fns[4] = {(const void*)attend_kernel<bf16_t, 128, 1, true>, (const void*)attend_kernel<float, 128, 1, true>,
                        (const void*)attend_kernel<bf16_t, 64, 1, true>, (const void*)attend_kernel<float, 64, 1, true>};
  bool ok = true;
  for (const void* fn : fns) ok = ok && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)attend_lds<true, 128>()) == hipSuccess;
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
