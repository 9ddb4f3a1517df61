// Operators of a search over several continuations (search.hpp).
#include <type_traits>

#include "cache.hpp"
#include "search.hpp"

namespace dinfer {

// ---------------------------------------------------------------- select
// Candidates (row, token) with score[row] + z - log(sum of exp z) and the n_keep best of every sequence.  The first launch streams the logits
// once and leaves the maximum and the sum of exponentials of every chunk of 2048.  The second one, a workgroup per sequence, works
// the rows' normalisers out of them, and a threshold: the n_keep-th best of the chunks' best candidates is no better than the n_keep-th
// best candidate, so that only chunks that reach it, about n_keep of them, are read again, and what reaches it there is ranked, in 64 bits.
// Bound: one read of the logits.  8 sequences of 64 rows of 157184 bfloat16, six rows of ten live (98 MB): the stream 20.7 us (4.7 TB/s), the join 16.6 (a chain of short
// steps, 1024 threads: normalisers 4.5, the bound 2.4, the list of chunks 2.1, reading them 3.1, ranking 1.7); one launch that kept every
// row's best ones as it went took 74.7.  4 rows of float32: 3.4 + 10.7.
constexpr int CHUNK_VALUES = 32, CHUNK = WAVE * CHUNK_VALUES;          // logits of a lane, in registers, and of a wave
constexpr int SELECT_THREADS = 256, SELECT_WAVES = SELECT_THREADS / WAVE;
constexpr uint32_t NO_VALUE = 0x007fffffu;                             // order_of(-inf): no candidate

// Order of floats as integers; not a number counts as -inf.
__device__ inline uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return v != v ? NO_VALUE : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

struct ChunkState {
  float m, s;                 // -inf: no candidate
};
static int select_chunks(int vocab) { return (vocab + CHUNK - 1) / CHUNK; }
size_t select_scratch_bytes(int64_t rows, int vocab) { return rows * select_chunks(vocab) * sizeof(ChunkState); }

// A lane's share of a chunk; -inf behind the row and where there is no number.  A lane's tokens are the same for every row, wherever
// it begins in memory (the loads need not be aligned), so that equal rows have equal sums, to the bit, and tie.
template <typename E> struct ChunkOf {
  static constexpr int G = ET<E>::G, N = CHUNK_VALUES / G;
  typename ET<E>::vec v[N];
  __device__ static int token(int chunk, int lane, int r) { return chunk * CHUNK + (r / G * WAVE + lane) * G + r % G; }
  __device__ void load(const E* z, int vocab, int chunk, int lane) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = token(chunk, lane, n * G);
      if (at + G <= vocab) __builtin_memcpy(&v[n], z + at, sizeof(v[n]));
      else {
#pragma unroll
        for (int i = 0; i < G; ++i) v[n][i] = from_f32<E>(-INFINITY);
        if (at < vocab) {      // (one lane, where the row ends)
#pragma unroll
          for (int i = 0; i < G - 1; ++i)
            if (at + i < vocab) v[n][i] = z[at + i];
        }
      }
    }
  }
  __device__ float raw(int r) const { return to_f32(v[r / G][r % G]); }
  __device__ float value(int r) const {
    const float x = raw(r);
    return x != x ? -INFINITY : x;
  }
};

// Largest and sum over a wave, in every lane, by moves inside the registers up to rows of 16 lanes.
template <int CTRL> __device__ inline float from_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ inline float wave_largest(float v) {
  v = fmaxf(v, from_lane<0x128>(v));      // row_ror:8, 4, 2, 1
  v = fmaxf(v, from_lane<0x124>(v));
  v = fmaxf(v, from_lane<0x122>(v));
  v = fmaxf(v, from_lane<0x121>(v));
  v = fmaxf(v, __shfl_xor(v, 16, WAVE));
  return fmaxf(v, __shfl_xor(v, 32, WAVE));
}
__device__ inline float wave_total(float v) {
  v += from_lane<0x128>(v);
  v += from_lane<0x124>(v);
  v += from_lane<0x122>(v);
  v += from_lane<0x121>(v);
  v += __shfl_xor(v, 16, WAVE);
  return v + __shfl_xor(v, 32, WAVE);
}

// A wave takes PER chunks of a row, the next one's loads under way while it works on one.
template <typename E, int PER>
__global__ __launch_bounds__(SELECT_THREADS) void select_chunk_kernel(SelectArgs a, ChunkState* state, int chunks) {
  const int64_t row = blockIdx.y;
  const int chunk0 = (blockIdx.x * SELECT_WAVES + (threadIdx.x >> 6)) * PER, lane = threadIdx.x & 63;
  if (chunk0 >= chunks || !(fabsf(a.score[row]) < INFINITY) || (a.hold && a.hold[row] >= 0)) return;
  const E* z = (const E*)a.logits + row * a.row_stride;
  ChunkOf<E> x, next;
  x.load(z, a.vocab, chunk0, lane);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int chunk = chunk0 + i;
    if (i + 1 < PER && chunk + 1 < chunks) next.load(z, a.vocab, chunk + 1, lane);
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < CHUNK_VALUES; ++r) top = fmaxf(top, x.raw(r));      // (the larger of a number and NaN is the number)
    // (the maximum is taken off first: the largest term is 1 whatever the logits' size, and the sum between 1 and CHUNK)
    const float M = wave_largest(top), away = M > -INFINITY ? M : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < CHUNK_VALUES; ++r) sum += __builtin_amdgcn_exp2f((x.raw(r) - away) * 1.44269504088896341f);
    sum = wave_total(sum);
    if (!(sum < INFINITY)) {      // NaN among them, or infinities, which count one each
      sum = 0.f;
#pragma unroll
      for (int r = 0; r < CHUNK_VALUES; ++r)
        sum += M < INFINITY ? __builtin_amdgcn_exp2f((x.value(r) - away) * 1.44269504088896341f) : x.value(r) == M ? 1.f : 0.f;
      sum = wave_total(sum);
    }
    if (lane == 0) state[row * chunks + chunk] = ChunkState{M, sum};
    if (chunk + 1 >= chunks) return;
    x = next;
  }
}

// A candidate of a sequence: its score, then the lower (row, token).
struct Candidate {
  double score;
  uint64_t at;                // row << 32 | token
};
__device__ inline bool better(const Candidate& x, const Candidate& y) { return x.score > y.score || (x.score == y.score && x.at < y.at); }

constexpr int JOIN_THREADS = 1024, JOIN_WAVES = JOIN_THREADS / WAVE;
constexpr int JOIN_CHUNKS = 1024, JOIN_LIST = 2048, JOIN_FEW = 256, JOIN_ALL = 64;    // chunks that are read again, candidates that are ranked together, and without another look
constexpr int JOIN_ROWS = 4;                                           // rows of a wave whose chunks are under way together
template <typename E>
__global__ __launch_bounds__(JOIN_THREADS) void select_join_kernel(SelectArgs a, const ChunkState* state, int chunks) {
  const int seq = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, K = a.n_keep, R = a.n_rows;
  const int64_t row0 = (int64_t)seq * R;
  state += row0 * chunks;
  // score - log(sum of exp(z - peak)), which a candidate's z - peak is added to (peak itself may be so large that 64 bits lose the rest next to
  // it); of rows that hold: the score
  __shared__ double norm[MAX_SELECT_ROWS];
  __shared__ float peak[MAX_SELECT_ROWS];       // largest logit of the row, -inf: no candidate, NaN: one that is held
  __shared__ float row_sum[MAX_SELECT_ROWS];
  __shared__ __align__(16) Candidate list[JOIN_LIST];
  __shared__ int chunk_row[JOIN_CHUNKS], chunk_at[JOIN_CHUNKS];
  __shared__ int n_list, n_chunks, n_top;
  __shared__ uint32_t reach[JOIN_WAVES], least_of_all;
  uint32_t* tops = reinterpret_cast<uint32_t*>(list);      // (before the list is used)
  static_assert(sizeof(list) >= JOIN_THREADS * sizeof(uint32_t), "a value per thread");
  if (threadIdx.x == 0) n_list = n_chunks = n_top = 0;
  // the best candidate's score of a chunk with the largest logit m, rounded to a float (-inf: none)
  auto head = [](double n, float p, float m, bool first) {
    if (p != p) return first ? (float)n : -INFINITY;
    if (!(p > -INFINITY) || !(m > -INFINITY)) return -INFINITY;
    return p < INFINITY ? (float)(n + ((double)m - (double)p)) : m == INFINITY ? (float)n : -INFINITY;
  };
  // A batch of rows: maximum and sum of each (a wave has JOIN_ROWS of them), the normalisers a lane per row.
  for (int b0 = 0; b0 < R; b0 += JOIN_WAVES * JOIN_ROWS) {
    const int r0 = b0 + wave;
    float M[JOIN_ROWS], s[JOIN_ROWS];
#pragma unroll
    for (int u = 0; u < JOIN_ROWS; ++u) M[u] = -INFINITY, s[u] = 0.f;
    const int mine = min(b0 + (int)threadIdx.x, R - 1);
    const float base = a.score[row0 + mine];
    const int hold = *(a.hold ? a.hold + row0 + mine : a.row);      // (some readable word)
    for (int c0 = 0; c0 < chunks; c0 += 2 * WAVE) {
      ChunkState st[JOIN_ROWS][2];
#pragma unroll
      for (int u = 0; u < JOIN_ROWS; ++u)
#pragma unroll
        for (int v = 0; v < 2; ++v)      // (of rows that take no part: anything)
          st[u][v] = state[(int64_t)min(r0 + u * JOIN_WAVES, R - 1) * chunks + min(c0 + v * WAVE + lane, chunks - 1)];
#pragma unroll
      for (int u = 0; u < JOIN_ROWS; ++u)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const bool is = c0 + v * WAVE + lane < chunks && st[u][v].m > -INFINITY;
          const float m = is ? st[u][v].m : -INFINITY, both = fmaxf(M[u], m);
          const float keep = M[u] == both ? 1.f : __builtin_amdgcn_exp2f((M[u] - both) * 1.44269504088896341f);
          const float take = m == both ? 1.f : __builtin_amdgcn_exp2f((m - both) * 1.44269504088896341f);
          s[u] = s[u] * keep + (is ? st[u][v].s * take : 0.f);
          M[u] = both;
        }
    }
#pragma unroll
    for (int u = 0; u < JOIN_ROWS; ++u) {
      const float p = wave_largest(M[u]);
      const float sum = wave_total(M[u] == p ? s[u] : s[u] * __builtin_amdgcn_exp2f((M[u] - p) * 1.44269504088896341f));
      if (lane == 0 && r0 + u * JOIN_WAVES < R) {
        peak[r0 + u * JOIN_WAVES] = p;
        row_sum[r0 + u * JOIN_WAVES] = sum;
      }
    }
    __syncthreads();
    if (threadIdx.x < JOIN_WAVES * JOIN_ROWS && b0 + (int)threadIdx.x < R) {
      const float p = peak[mine];
      const bool live = fabsf(base) < INFINITY, held = live && a.hold && hold >= 0, some = live && !held && p > -INFINITY;
      peak[mine] = held ? __builtin_nanf("") : some ? p : -INFINITY;
      // (infinite logits share the row's weight: log(1 / their number) each)
      norm[mine] = held ? (double)base : some ? (double)base - log((double)row_sum[mine]) : 0.0;
    }
    __syncthreads();
  }
  // The K-th largest of the threads' values, or a little less, NO_VALUE + 1 where fewer than K have one: a bound from below by every wave's own,
  // then among those that reach it.
  auto kth = [&](float value) {
    const uint32_t mine = order_of(value);
    if (threadIdx.x == 0) n_top = 0;
    uint32_t t = 0;
    for (int b = 31; b >= 16; --b) {
      const uint32_t up = t | 1u << b;
      if (__popcll(__builtin_amdgcn_ballot_w64(mine >= up)) >= K) t = up;
    }
    if (lane == 0) reach[wave] = t;
    __syncthreads();
    t = 0;
#pragma unroll
    for (int v = 0; v < JOIN_WAVES; ++v) t = max(t, reach[v]);
    if (mine >= t && mine > NO_VALUE) tops[atomicAdd(&n_top, 1)] = mine;
    __syncthreads();
    if (wave == 0) {
      const int n = n_top;
      auto search = [&](auto most) __attribute__((always_inline)) {
        constexpr int U = decltype(most)::value;
        uint32_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = u * WAVE + lane < n ? tops[u * WAVE + lane] : 0;
        t = 0;
        for (int b = 31; b >= 10; --b) {
          const uint32_t up = t | 1u << b;
          int reached = 0;
#pragma unroll
          for (int u = 0; u < U; ++u) reached += __popcll(__builtin_amdgcn_ballot_w64(x[u] >= up));
          if (reached >= K) t = up;
        }
      };
      if (n >= K && n <= 4 * WAVE) search(std::integral_constant<int, 4>{});
      else if (n >= K) search(std::integral_constant<int, JOIN_WAVES>{});
      if (lane == 0) least_of_all = n >= K ? max(t, NO_VALUE + 1) : NO_VALUE + 1;
    }
    __syncthreads();
    return least_of_all;
  };
  // (of 64 chunks or less all are read again: the bound comes from what is in them, below)
  const int units = R * chunks;
  float top = -INFINITY;
  for (int l0 = threadIdx.x; l0 < units && units > JOIN_ALL; l0 += 4 * JOIN_THREADS) {
    float m[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) m[u] = state[min(l0 + u * JOIN_THREADS, units - 1)].m;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int l = l0 + u * JOIN_THREADS;
      if (l < units) top = fmaxf(top, head(norm[l / chunks], peak[l / chunks], m[u], l % chunks == 0));
    }
  }
  uint32_t least = units > JOIN_ALL ? kth(top) : NO_VALUE + 1;
  // every chunk whose best candidate reaches it
  auto each_chunk = [&](auto use) {
    for (int r0 = wave; r0 < R; r0 += JOIN_WAVES * JOIN_ROWS)
      for (int c0 = 0; c0 < chunks; c0 += WAVE) {
        float m[JOIN_ROWS];
#pragma unroll
        for (int u = 0; u < JOIN_ROWS; ++u) m[u] = state[(int64_t)min(r0 + u * JOIN_WAVES, R - 1) * chunks + min(c0 + lane, chunks - 1)].m;
#pragma unroll
        for (int u = 0; u < JOIN_ROWS; ++u) {
          const int r = r0 + u * JOIN_WAVES;
          if (r < R) use(r, c0, c0 + lane < chunks && order_of(head(norm[r], peak[r], m[u], c0 + lane == 0)) >= least);
        }
      }
  };
  each_chunk([&](int r, int c0, bool reaches) {
    if (reaches) {
      const int at = atomicAdd(&n_chunks, 1);
      if (at < JOIN_CHUNKS) {
        chunk_row[at] = r;
        chunk_at[at] = c0 + lane;
      }
    }
  });
  __syncthreads();
  const int64_t out = (int64_t)seq * K;
  auto put = [&](int k, const Candidate& c) {
    a.row[out + k] = (int32_t)(c.at >> 32);
    a.token[out + k] = (int32_t)c.at;
    a.score_out[out + k] = (float)c.score;
  };
  // The candidates of a chunk that reach it, in this wave: take(is one, candidate) in all lanes together.
  auto load = [&](int r, int chunk, ChunkOf<E>& x) __attribute__((always_inline)) {
    x.load((const E*)a.logits + (row0 + r) * a.row_stride, peak[r] != peak[r] ? 0 : a.vocab, chunk, lane);
  };
  auto scan = [&](int r, int chunk, const ChunkOf<E>& x, auto take) __attribute__((always_inline)) {
    const float p = peak[r];
    const double n = norm[r], bound = (double)__uint_as_float(least & 0x80000000u ? least ^ 0x80000000u : ~least);
    if (p != p) {
      take(lane == 0, Candidate{n, (uint64_t)r << 32 | (uint32_t)a.hold[row0 + r]});
      return;
    }
    // (a logit below `cut` cannot; those above it are looked at)
    const float cut = p < INFINITY ? (float)((double)p + (bound - n) - (fabs(bound) + fabs(n) + fabs((double)p) + 1.0) * 0x1p-20) : INFINITY;
#pragma unroll
    for (int v = 0; v < CHUNK_VALUES; ++v) {
      const float z = x.value(v);
      const bool may = z >= cut && z > -INFINITY;
      if (__builtin_amdgcn_ballot_w64(may)) {
        const double score = p < INFINITY ? n + ((double)z - (double)p) : n;
        take(may && order_of((float)score) >= least, Candidate{score, (uint64_t)r << 32 | (uint32_t)ChunkOf<E>::token(chunk, lane, v)});
      }
    }
  };
  // Candidates into the list.  Where fewer than K chunks have one (turn 0), and where the list gets long, as the best rows' do that have many better
  // than others' best (turn 2), the bound is first raised to that of the lanes' best ones in the listed chunks.  (If fewer than K lanes have
  // one, all candidates together are no more than 32 * K.)
  if (n_chunks <= JOIN_CHUNKS) {
    ChunkOf<E> kept;      // a wave's first one
    if (wave < n_chunks) load(__builtin_amdgcn_readfirstlane(chunk_row[wave]), __builtin_amdgcn_readfirstlane(chunk_at[wave]), kept);
    for (int turn = least == NO_VALUE + 1 ? 0 : 1; turn < 4; ++turn) {
      const bool raise = turn % 2 == 0;
      float best = -INFINITY;
      for (int i = wave; i < n_chunks; i += JOIN_WAVES) {
        const int r = __builtin_amdgcn_readfirstlane(chunk_row[i]), chunk = __builtin_amdgcn_readfirstlane(chunk_at[i]);
        ChunkOf<E> x = kept;
        if (i != wave) load(r, chunk, x);
        if (raise) {
          float z = -INFINITY;
#pragma unroll
          for (int v = 0; v < CHUNK_VALUES; ++v) z = fmaxf(z, x.value(v));
          best = fmaxf(best, head(norm[r], peak[r], z, lane == 0));      // (the larger logit, the better)
          continue;
        }
        scan(r, chunk, x, [&](bool is, const Candidate& c) __attribute__((always_inline)) {
          const uint64_t all = __builtin_amdgcn_ballot_w64(is);
          if (all == 0) return;
          int at = 0;
          if (lane == 0) at = atomicAdd(&n_list, (int)__popcll(all));
          at = __builtin_amdgcn_readfirstlane(at) + __popcll(all & (lane ? ~0ull >> (64 - lane) : 0ull));
          if (is && at < JOIN_LIST) list[at] = c;
        });
      }
      if (raise) {
        least = kth(best);
        continue;
      }
      __syncthreads();
      if (turn == 3 || n_list <= JOIN_FEW) break;
      __syncthreads();      // (all have looked)
      if (threadIdx.x == 0) n_list = 0;
    }
  }
  __syncthreads();
  const int n = n_list;
  int filled = min(n, K);
  if (n_chunks <= JOIN_CHUNKS && n <= JOIN_LIST) {
    for (int i = threadIdx.x; i < n; i += JOIN_THREADS) {
      const Candidate mine = list[i];
      int rank = 0;
      constexpr int U = 8;
      for (int j0 = 0; j0 < n; j0 += U) {
        Candidate c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = list[min(j0 + u, n - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) rank += j0 + u < n && better(c[u], mine);
      }
      if (rank < K) put(rank, mine);
    }
  } else {
    // thousands of candidates reach the threshold, as equal ones do: the best one behind the last, K times
    __shared__ Candidate found[JOIN_WAVES];
    Candidate last{INFINITY, 0};
    bool begun = false;
    for (filled = 0; filled < K; ++filled) {
      Candidate mine{-INFINITY, ~0ull};
      each_chunk([&](int r, int c0, bool reaches) {
        for (uint64_t left = __builtin_amdgcn_ballot_w64(reaches); left; left &= left - 1) {
          ChunkOf<E> x;
          load(r, c0 + __builtin_ctzll(left), x);
          scan(r, c0 + __builtin_ctzll(left), x, [&](bool is, const Candidate& c) __attribute__((always_inline)) {
            if (is && (!begun || better(last, c)) && better(c, mine)) mine = c;
          });
        }
      });
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const Candidate other{__shfl_xor(mine.score, d, WAVE), __shfl_xor((unsigned long long)mine.at, d, WAVE)};
        if (better(other, mine)) mine = other;
      }
      if (lane == 0) found[wave] = mine;
      __syncthreads();
      for (int v = 0; v < JOIN_WAVES; ++v)
        if (better(found[v], mine)) mine = found[v];
      __syncthreads();
      if (mine.at == ~0ull) break;
      if (threadIdx.x == 0) put(filled, mine);
      last = mine;
      begun = true;
    }
  }
  for (int k = filled + threadIdx.x; k < K; k += JOIN_THREADS) {
    a.row[out + k] = a.token[out + k] = -1;
    a.score_out[out + k] = -INFINITY;
  }
}

constexpr int SELECT_MANY = 4 * 8192;
template <typename E> static void launch_select_t(const SelectArgs& a, hipStream_t st) {
  const int chunks = select_chunks(a.vocab);
  ChunkState* state = (ChunkState*)a.scratch;
  const int64_t rows = (int64_t)a.n_seq * a.n_rows;
  if (rows * chunks >= SELECT_MANY) select_chunk_kernel<E, 4><<<dim3((chunks + 4 * SELECT_WAVES - 1) / (4 * SELECT_WAVES), rows), SELECT_THREADS, 0, st>>>(a, state, chunks);
  else select_chunk_kernel<E, 1><<<dim3((chunks + SELECT_WAVES - 1) / SELECT_WAVES, rows), SELECT_THREADS, 0, st>>>(a, state, chunks);
  select_join_kernel<E><<<a.n_seq, JOIN_THREADS, 0, st>>>(a, state, chunks);
}
void launch_select(bool bf16, const SelectArgs& a, hipStream_t st) {
  if (bf16) launch_select_t<bf16_t>(a, st);
  else launch_select_t<float>(a, st);
}

// ---------------------------------------------------------------- pages
// One bit per page of the pool, in LDS, with the number of bits in front of every 64 of them: the k-th page of a kind is found
// there, and what a page's place among its kind is.
constexpr int POOL_THREADS = 1024, POOL_WAVES = POOL_THREADS / WAVE;
struct PageBits {
  uint64_t* word;
  int32_t* before;            // [words + 1]
  int words;
  static constexpr int U = 8;
  int first[U];               // counts of this thread's first pages: asked for early, and kept
  __device__ static int page_of(int u) { return u * POOL_THREADS + threadIdx.x; }
  __device__ void load(const int32_t* refs, int n_pages) {
#pragma unroll
    for (int u = 0; u < U; ++u) first[u] = refs[min(page_of(u), n_pages - 1)];
  }
  // Bits of the pages whose count is (not) positive (every thread of the workgroup calls; ends with a barrier).
  template <bool Used> __device__ void build(const int32_t* refs, int n_pages, char* lds) {
    words = (n_pages + 63) / 64;
    word = reinterpret_cast<uint64_t*>(lds);
    before = reinterpret_cast<int32_t*>(lds + (size_t)words * 8);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int w0 = wave; w0 < words; w0 += POOL_WAVES * U) {
      int n[U];
#pragma unroll
      for (int u = 0; u < U; ++u) n[u] = w0 == wave ? first[u] : refs[min((w0 + u * POOL_WAVES) * 64 + lane, n_pages - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int w = w0 + u * POOL_WAVES;
        const uint64_t b = __builtin_amdgcn_ballot_w64((n[u] > 0) == Used && w * 64 + lane < n_pages);
        if (lane == 0 && w < words) word[w] = b;
      }
    }
    __shared__ int sums[POOL_WAVES];
    __syncthreads();
    const int per = (words + POOL_THREADS - 1) / POOL_THREADS, w0 = min((int)threadIdx.x * per, words), w1 = min(w0 + per, words);
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popcll(word[w]);
    const int upto = lane_scan(mine);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int at = upto - mine;
    for (int v = 0; v < wave; ++v) at += sums[v];
    for (int w = w0; w < w1; ++w) {
      before[w] = at;
      at += __popcll(word[w]);
    }
    if (threadIdx.x == POOL_THREADS - 1) before[words] = at;
    __syncthreads();
  }
  __device__ int total() const { return before[words]; }
  __device__ bool has(int page) const { return (word[page >> 6] >> (page & 63)) & 1; }
  __device__ int in_front(int page) const { return before[page >> 6] + (page & 63 ? __popcll(word[page >> 6] << (64 - (page & 63))) : 0); }
  // The k-th page (from 0) whose bit is `Set`; there are that many.
  template <bool Set> __device__ int find(int k) const {
    int lo = 0, hi = words;      // the word with lo: no more than k in front of it
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2, front = Set ? before[mid] : mid * 64 - before[mid];
      if (front <= k) lo = mid;
      else hi = mid;
    }
    k -= Set ? before[lo] : lo * 64 - before[lo];
    uint64_t bits = Set ? word[lo] : ~word[lo];
    int at = 0;
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) {
      const int n = __popcll(bits & ((1ull << step) - 1));
      if (k >= n) {
        k -= n;
        bits >>= step;
        at += step;
      }
    }
    return lo * 64 + at;
  }
};
static size_t page_bits_bytes(int n_pages) { return (size_t)((n_pages + 63) / 64) * 12 + 16; }

__device__ inline void move_piece(const char* from, char* to, int64_t bytes) {      // bytes: a multiple of 16
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = (int64_t)(i * PIECE_THREADS + threadIdx.x) * 16;
    if (at < bytes) v[i] = *reinterpret_cast<const u32x4*>(from + at);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = (int64_t)(i * PIECE_THREADS + threadIdx.x) * 16;
    if (at < bytes) *reinterpret_cast<u32x4*>(to + at) = v[i];
  }
}
__device__ inline void move_page_piece(const PagePool& p, int from, int to, int layer, int piece) {
  char* at = p.kv + layer * p.layer_bytes + (int64_t)piece * PIECE;
  move_piece(at + from * p.page_bytes, at + to * p.page_bytes, min((int64_t)PIECE, p.page_bytes - (int64_t)piece * PIECE));
}

// ---------------------------------------------------------------- fork
// What becomes of sequence i: columns below `own` are its parent's pages, shared; those below `need` are its own.
struct Fork {
  int parent, len, own, have, need, held;
  bool first;                 // of its parent's children: it takes over the pages that nobody else holds
};
__device__ inline Fork fork_of(const ForkArgs& a, int i) {      // i: the same in a whole wave
  const int all = a.parent[min((int)threadIdx.x & 63, a.n_new - 1)];
  Fork f;
  f.parent = __builtin_amdgcn_readlane(all, i);
  if (f.parent < 0 || f.parent >= a.n_old) f.parent = -1;
  f.len = f.held = 0;
  if (a.n_old > 0) {
    const int p = max(f.parent, 0), n = a.len[p], h = a.held[p];      // (no branch on the parent: several sequences' loads go together)
    f.len = f.parent < 0 ? 0 : max(0, min(n, a.limit));
    f.held = f.parent < 0 ? 0 : max(0, min(h, a.pt_stride));
  }
  f.own = max(0, f.len - a.rewrite) / PAGE;
  f.have = (f.len + PAGE - 1) / PAGE;
  f.need = (int)min(((int64_t)f.len + a.room + PAGE - 1) / PAGE, (int64_t)a.new_stride);
  f.first = f.parent >= 0 && (__builtin_amdgcn_ballot_w64(all == f.parent) & ((1ull << i) - 1)) == 0;
  return f;
}
__device__ inline int old_page(const ForkArgs& a, const Fork& f, int c) {      // -1: none
  const int page = c < f.held ? a.table[(int64_t)f.parent * a.pt_stride + c] : -1;
  return page >= 0 && page < a.pool.n_pages ? page : -1;
}

// The first launch, one workgroup: who gets which free page, the lowest ones in the order of sequences and columns, and the list of the
// pages to copy.  A wave takes every POOL_WAVES-th sequence; what it finds out about the first 64 columns of their own it keeps.  Bound by its
// chain of loads (parents, lengths, pages, counts) and, in pools of many pages, by one workgroup's reads of the counts.  4 sequences 5.4 us, 64 of them
// behind up to 4001 positions 10.5.
constexpr int FORK_SEQS = MAX_SEQS / POOL_WAVES;
__global__ __launch_bounds__(POOL_THREADS) void fork_plan_kernel(ForkArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ int wanted[MAX_SEQS], n_copies;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (threadIdx.x == 0) n_copies = 0;
  auto look = [&](const Fork& f, int c, int& page) {      // does column c need another page than the parent's `page`
    page = c < f.need ? old_page(a, f, c) : -1;
    return c < f.need && !(f.first && page >= 0 && a.refs[max(page, 0)] == 1);
  };
  PageBits free;
  free.load(a.refs, a.pool.n_pages);
  Fork f[FORK_SEQS];
  int page[FORK_SEQS];
  uint64_t fresh[FORK_SEQS];
#pragma unroll
  for (int u = 0; u < FORK_SEQS; ++u) f[u] = fork_of(a, min(wave + u * POOL_WAVES, a.n_new - 1));
#pragma unroll
  for (int u = 0; u < FORK_SEQS; ++u) fresh[u] = __builtin_amdgcn_ballot_w64(look(f[u], f[u].own + lane, page[u]));
#pragma unroll
  for (int u = 0; u < FORK_SEQS; ++u) {
    int n = __popcll(fresh[u]), other;
    for (int c0 = f[u].own + WAVE; c0 < f[u].need; c0 += WAVE) n += __popcll(__builtin_amdgcn_ballot_w64(look(f[u], c0 + lane, other)));
    if (lane == 0 && wave + u * POOL_WAVES < a.n_new) wanted[wave + u * POOL_WAVES] = n;
  }
  free.build<false>(a.refs, a.pool.n_pages, lds);
  const int upto = lane_scan(lane < a.n_new ? wanted[lane] : 0);      // (n_new <= 64)
  const int missing = max(0, __builtin_amdgcn_readlane(upto, 63) - free.total());
  if (threadIdx.x == 0) {
    *a.missing = missing;
    if (missing > 0) a.copies->n = 0;
  }
  if (missing > 0) return;
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
#pragma unroll
  for (int u = 0; u < FORK_SEQS; ++u) {
    const int i = wave + u * POOL_WAVES;
    if (i >= a.n_new) break;
    int at = __builtin_amdgcn_readlane(upto, i) - wanted[i];
    int32_t* row = a.new_table + (int64_t)i * a.new_stride;
    for (int c0 = f[u].own; c0 < f[u].need; c0 += WAVE) {
      const int c = c0 + lane;
      if (c0 > f[u].own) fresh[u] = __builtin_amdgcn_ballot_w64(look(f[u], c, page[u]));
      if (fresh[u] >> lane & 1) {
        const int to = free.find<true>(at + __popcll(fresh[u] & below));
        row[c] = to;
        if (c < f[u].have && page[u] >= 0) a.copies->page[atomicAdd(&n_copies, 1)] = int2{page[u], to};
      } else if (c < f[u].need) row[c] = page[u];
      at += __popcll(fresh[u]);
    }
    if (lane == 0) {
      a.new_len[i] = f[u].len;
      a.new_held[i] = f[u].need;
    }
  }
#pragma unroll
  for (int u = 0; u < PageBits::U; ++u)
    if (PageBits::page_of(u) < a.pool.n_pages) a.new_refs[PageBits::page_of(u)] = free.first[u];
  for (int p = PageBits::U * POOL_THREADS + threadIdx.x; p < a.pool.n_pages; p += POOL_THREADS) a.new_refs[p] = a.refs[p];
  __syncthreads();
  if (threadIdx.x == 0) a.copies->n = n_copies;
}

// The second: shared columns and the counts of all pages, the sequences' states, and the pages that are copied.  Bound by their bytes,
// once each way: 64 sequences, 69 MB, 12.3 us.  (Workgroups that looked for themselves what to copy: 28.7 us both launches, with the list 25.0.)
__global__ __launch_bounds__(PIECE_THREADS) void fork_apply_kernel(ForkArgs a) {
  if (*a.missing > 0) return;
  const ForkGrid& g = a.grid;
  int b = blockIdx.x;
  if (b < a.n_new) {
    const Fork f = fork_of(a, b);
    int32_t* row = a.new_table + (int64_t)b * a.new_stride;
    for (int c = threadIdx.x; c < a.new_stride; c += PIECE_THREADS) {
      int page = -1;
      if (c < min(f.own, f.need)) row[c] = page = old_page(a, f, c);
      else if (c < f.need) page = row[c];
      else row[c] = -1;
      if (page >= 0) atomicAdd(&a.new_refs[page], 1);
    }
    return;
  }
  if (b < g.state0) {
    const int s = b - a.n_new, held = max(0, min(a.held[s], a.pt_stride));
    for (int c = threadIdx.x; c < held; c += PIECE_THREADS) {
      const int page = a.table[(int64_t)s * a.pt_stride + c];
      if (page >= 0 && page < a.pool.n_pages) atomicAdd(&a.new_refs[page], -1);
    }
    return;
  }
  if (b < g.page0) {
    b -= g.state0;
    int k = 0;
    while (b >= g.state_pieces[k] * a.n_new) b -= g.state_pieces[k++] * a.n_new;
    const StateRows st = a.state[k];
    const int i = b / g.state_pieces[k], parent = a.parent[i];
    const int64_t at = (int64_t)(b % g.state_pieces[k]) * PIECE, n = min((int64_t)PIECE, st.row_bytes - at);
    char* to = st.out + i * st.row_bytes + at;
    const bool none = parent < 0 || parent >= a.n_old;
    const char* from = st.in + (none ? 0 : parent) * st.row_bytes + at;
    if (!none && (((uintptr_t)to | (uintptr_t)from | n) & 15) == 0) move_piece(from, to, n);
    else
      for (int64_t j = threadIdx.x * 4; j < n; j += PIECE_THREADS * 4) *reinterpret_cast<uint32_t*>(to + j) = none ? 0u : *reinterpret_cast<const uint32_t*>(from + j);
    return;
  }
  const int per = g.pieces * a.pool.n_layers;
  int item = b - g.page0;
  int2 p = a.copies->page[item / per];      // (there are as many as workgroups; beyond n: anything)
  const int items = a.copies->n * per;      // (of different pages of the pool, at least 4 KiB each: below 2^31)
  while (item < items) {
    move_page_piece(a.pool, p.x, p.y, item / g.pieces % a.pool.n_layers, item % g.pieces);
    item += g.page_groups;
    if (item < items) p = a.copies->page[item / per];
  }
}

// Columns of a sequence that hold something and are written: from (len - rewrite) / PAGE on.
static int fork_columns(int rewrite, int stride) {
  const int n = (rewrite + PAGE - 1) / PAGE + 1;
  return n < stride ? n : stride;
}
size_t fork_copies_bytes(int max_seqs, int max_pos) { return sizeof(CopyList) + (size_t)max_seqs * fork_columns(max_pos, INT32_MAX) * sizeof(int2); }
bool plan_fork(ForkArgs& a) {
  int64_t row_bytes[MAX_STATES];
  for (int k = 0; k < a.n_states; ++k) row_bytes[k] = a.state[k].row_bytes;
  return fork_grid(a.n_old, a.n_new, row_bytes, a.n_states, fork_columns(a.rewrite, a.new_stride), a.pool.n_layers, a.pool.page_bytes, &a.grid);
}
void launch_fork(const ForkArgs& a, hipStream_t st) {
  fork_plan_kernel<<<1, POOL_THREADS, page_bits_bytes(a.pool.n_pages), st>>>(a);
  fork_apply_kernel<<<a.grid.page0 + a.grid.page_groups, PIECE_THREADS, 0, st>>>(a);
}

// ---------------------------------------------------------------- compact
// The k-th page in use behind the front goes to the k-th free page in the front, the front being as long as there are pages in use, so that no
// page is moved twice and none is overwritten that is still to be read.  Plan: bound by its loads in turn (3.0 us; 6.3 with 48 sequences; counts
// that were read again for every use took 10.5).  Move: bound by its bytes, 131 us for 665 MB both ways, 5.08 TB/s, the rate of a copy.
__global__ __launch_bounds__(POOL_THREADS) void compact_plan_kernel(CompactArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int n = a.pool.n_pages;
  PageBits used;
  used.load(a.refs, n);
  used.build<true>(a.refs, n, lds);
  const int front = used.total(), stay = front < n ? used.in_front(front) : front, moves = front - stay;
  if (threadIdx.x == 0) {
    a.count[0] = front;
    a.count[1] = moves;
  }
  auto settle = [&](int p, int refs) {
    int to = -1;
    if (used.has(p)) {
      to = p;
      if (p >= front) {
        const int k = used.in_front(p) - stay;
        to = used.find<false>(k);
        a.moved[n + k] = p;
      }
      a.new_refs[to] = refs;
    }
    a.moved[p] = to;
    if (p >= front) a.new_refs[p] = 0;
    if (p >= moves) a.moved[n + p] = -1;
  };
#pragma unroll
  for (int u = 0; u < PageBits::U; ++u)
    if (PageBits::page_of(u) < n) settle(PageBits::page_of(u), used.first[u]);
  for (int p = PageBits::U * POOL_THREADS + threadIdx.x; p < n; p += POOL_THREADS) settle(p, a.refs[p]);
}
__global__ __launch_bounds__(PIECE_THREADS) void compact_move_kernel(CompactArgs a, int pieces) {
  if ((int)blockIdx.x < a.n_seq) {
    const int s = blockIdx.x, held = max(0, min(a.held[s], a.pt_stride));
    for (int c = threadIdx.x; c < a.pt_stride; c += PIECE_THREADS) {
      const int page = c < held ? a.table[(int64_t)s * a.pt_stride + c] : -1;
      a.new_table[(int64_t)s * a.pt_stride + c] = page >= 0 && page < a.pool.n_pages ? a.moved[page] : -1;
    }
    return;
  }
  const int64_t items = (int64_t)a.count[1] * a.pool.n_layers * pieces;
  for (int64_t b = blockIdx.x - a.n_seq; b < items; b += gridDim.x - a.n_seq) {
    const int from = a.moved[a.pool.n_pages + b / (a.pool.n_layers * pieces)];
    move_page_piece(a.pool, from, a.moved[from], (int)(b / pieces % a.pool.n_layers), (int)(b % pieces));
  }
}
constexpr int MOVE_GROUPS = 4096;
void launch_compact(const CompactArgs& a, hipStream_t st) {
  const int pieces = (int)pieces_of(a.pool.page_bytes);
  const int64_t most = (int64_t)(a.pool.n_pages / 2 + 1) * a.pool.n_layers * pieces;
  compact_plan_kernel<<<1, POOL_THREADS, page_bits_bytes(a.pool.n_pages), st>>>(a);
  compact_move_kernel<<<a.n_seq + (int)(most < MOVE_GROUPS ? most : MOVE_GROUPS), PIECE_THREADS, 0, st>>>(a, pieces);
}

bool configure_search() {
  const int most = (int)page_bits_bytes(MAX_POOL_PAGES);
  const bool ok = hipFuncSetAttribute((const void*)fork_plan_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most) == hipSuccess &&
                  hipFuncSetAttribute((const void*)compact_plan_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most) == hipSuccess;
  (void)hipGetLastError();
  return ok;
}

}  // namespace dinfer
