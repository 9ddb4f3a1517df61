// Operators of a search over several continuations (search.hpp).
#include "cache.hpp"
#include "search.hpp"

namespace dinfer {

// ---------------------------------------------------------------- select
// Candidates (row, token) with score[row] + z - log(sum of exp z) and the n_keep best of every sequence.  Within a row the order is that of
// the logits, so the first launch, a workgroup per slice of a row, leaves the slice's n_keep best logits and its (maximum, sum of exponentials), and
// the second one, a workgroup per sequence, the rows' normalisers and the best of what is left, in 64 bits.  Only what could be
// among the best is sorted: the n_keep-th largest of the lanes' own maxima is no larger than the n_keep-th largest value.
constexpr int SELECT_THREADS = 256, SELECT_WAVES = SELECT_THREADS / WAVE;
constexpr int LANE_VALUES = 32;                                        // logits of a lane, in registers
constexpr int SLICE = SELECT_THREADS * LANE_VALUES;
constexpr int WAVE_LIST = 512;                                         // candidates of a wave that are ranked together
constexpr uint32_t NO_VALUE = 0x007fffffu;                             // order_of(-inf): no candidate

// Order of floats as integers; not a number counts as -inf.
__device__ inline uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return v != v ? NO_VALUE : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
// Best first: the larger value, then the lower token.
__device__ inline uint64_t key_of(uint32_t order, uint32_t token) { return (uint64_t)order << 32 | (uint32_t)~token; }
__device__ inline uint32_t key_order(uint64_t k) { return (uint32_t)(k >> 32); }
__device__ inline uint32_t key_token(uint64_t k) { return ~(uint32_t)k; }

// The largest t of `bits` leading bits that at least `want` lanes reach.
__device__ inline uint32_t reached_by(uint32_t order, int want, int bits) {
  uint32_t t = 0;
  for (int b = 31; b > 31 - bits; --b) {
    const uint32_t up = t | 1u << b;
    if (__popcll(__builtin_amdgcn_ballot_w64(order >= up)) >= want) t = up;
  }
  return t;
}

struct SliceState {
  float m, s;
};
struct SelectScratch {
  SliceState* state;          // [row][slice]
  uint64_t* key;              // [row][slice][n_keep], best first, 0 behind the last
};
static size_t state_bytes(int64_t lists) { return (lists * sizeof(SliceState) + 255) / 256 * 256; }
static int select_slices(int vocab) { return (vocab + SLICE - 1) / SLICE; }
static SelectScratch scratch_of(const SelectArgs& a) {
  const int64_t lists = (int64_t)a.n_seq * a.n_rows * select_slices(a.vocab);
  return SelectScratch{(SliceState*)a.scratch, (uint64_t*)((char*)a.scratch + state_bytes(lists))};
}
size_t select_scratch_bytes(int64_t rows, int vocab, int n_keep) {
  const int64_t lists = rows * select_slices(vocab);
  return state_bytes(lists) + lists * n_keep * sizeof(uint64_t);
}

template <typename E>
__global__ __launch_bounds__(SELECT_THREADS) void select_slice_kernel(SelectArgs a, SelectScratch w) {
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, N = LANE_VALUES / G;
  const int64_t row = blockIdx.y;
  if (!(a.score[row] > -INFINITY) || (a.hold && a.hold[row] >= 0)) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, K = a.n_keep;
  const E* z = (const E*)a.logits + row * a.row_stride;
  // A lane's tokens are the same for every row, wherever it begins in memory (the loads need not be aligned), so that equal rows have
  // equal sums, to the bit, and tie.
  const int first = (int)blockIdx.x * SLICE + wave * (WAVE * LANE_VALUES);
  float x[LANE_VALUES];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int at = first + (n * WAVE + lane) * G;
    if (at + G <= a.vocab) {
      vec v;
      __builtin_memcpy(&v, z + at, sizeof(v));
#pragma unroll
      for (int i = 0; i < G; ++i) x[n * G + i] = to_f32(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i) x[n * G + i] = at + i < a.vocab ? to_f32(z[at + i]) : -INFINITY;
    }
  }
  auto token_at = [&](int r) { return first + (r / G * WAVE + lane) * G + r % G; };
  float top = -INFINITY;
#pragma unroll
  for (int r = 0; r < LANE_VALUES; ++r) {
    x[r] = x[r] != x[r] ? -INFINITY : x[r];
    top = fmaxf(top, x[r]);
  }
  const float M = wave_max(top);
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < LANE_VALUES; ++r) sum += x[r] == M ? 1.f : __builtin_amdgcn_exp2f((x[r] - M) * 1.44269504088896341f);
  sum = M > -INFINITY ? wave_sum(sum) : 0.f;

  __shared__ uint64_t list[SELECT_WAVES][WAVE_LIST];
  __shared__ uint64_t best[SELECT_WAVES][MAX_KEEP];
  __shared__ SliceState state[SELECT_WAVES];
  if (lane == 0) state[wave] = SliceState{M, sum};
  const uint32_t least = max(reached_by(order_of(top), K, 20), NO_VALUE + 1);
  int n = 0;
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
#pragma unroll
  for (int r = 0; r < LANE_VALUES; ++r) {
    const uint32_t o = order_of(x[r]);
    const uint64_t in = __builtin_amdgcn_ballot_w64(o >= least);
    const int at = n + __popcll(in & below);
    if (o >= least && at < WAVE_LIST) list[wave][at] = key_of(o, token_at(r));
    n += __popcll(in);
  }
  if (lane < K) best[wave][lane] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (n <= WAVE_LIST) {
    for (int i = lane; i < n; i += WAVE) {
      const uint64_t mine = list[wave][i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += list[wave][j] > mine;
      if (rank < K) best[wave][rank] = mine;
    }
  } else {
    // hundreds of equal values: one after the other
    uint64_t last = ~0ull;
    for (int k = 0; k < K; ++k) {
      uint64_t mine = 0;
#pragma unroll
      for (int r = 0; r < LANE_VALUES; ++r) {
        const uint32_t o = order_of(x[r]);
        const uint64_t key = o > NO_VALUE ? key_of(o, token_at(r)) : 0;
        mine = key < last && key > mine ? key : mine;
      }
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)mine, d, WAVE);
        mine = other > mine ? other : mine;
      }
      if (mine == 0) break;
      if (lane == 0) best[wave][k] = mine;
      last = mine;
    }
  }
  __syncthreads();
  // the waves' lists joined
  const int64_t unit = row * gridDim.x + blockIdx.x;
  uint64_t* out = w.key + unit * K;
  __shared__ int filled;
  if (threadIdx.x == 0) filled = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < SELECT_WAVES * K; i += SELECT_THREADS) {
    const uint64_t mine = best[i / K][i % K];
    if (mine == 0) continue;
    int rank = 0;
    for (int v = 0; v < SELECT_WAVES; ++v)
      for (int j = 0; j < K; ++j) rank += best[v][j] > mine;
    if (rank < K) {
      out[rank] = mine;
      atomicAdd(&filled, 1);
    }
  }
  __syncthreads();
  for (int i = filled + threadIdx.x; i < K; i += SELECT_THREADS) out[i] = 0;
  if (threadIdx.x == 0) {
    float top_m = -INFINITY, s = 0.f;
    for (int v = 0; v < SELECT_WAVES; ++v) top_m = fmaxf(top_m, state[v].m);
    for (int v = 0; v < SELECT_WAVES; ++v)
      s += state[v].m == top_m ? state[v].s : state[v].s * __builtin_amdgcn_exp2f((state[v].m - top_m) * 1.44269504088896341f);
    w.state[unit] = SliceState{top_m, top_m > -INFINITY ? s : 0.f};
  }
}

// A candidate of a sequence: its score, then the lower (row, token).
struct Candidate {
  double score;
  uint64_t at;                // row << 32 | token
};
__device__ inline bool better(const Candidate& x, const Candidate& y) { return x.score > y.score || (x.score == y.score && x.at < y.at); }

constexpr int JOIN_THREADS = 1024, JOIN_WAVES = JOIN_THREADS / WAVE, JOIN_LIST = 2048;
__global__ __launch_bounds__(JOIN_THREADS) void select_join_kernel(SelectArgs a, SelectScratch w, int slices) {
  const int seq = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, K = a.n_keep, R = a.n_rows;
  const int64_t row0 = (int64_t)seq * R;
  __shared__ double norm[MAX_SELECT_ROWS];      // score - log(sum of exp z); for rows that hold: the score
  __shared__ float peak[MAX_SELECT_ROWS];       // largest logit of the row, -inf: no candidate, NaN: one that is held
  for (int r = wave; r < R; r += JOIN_WAVES) {
    const float base = a.score[row0 + r];
    const bool live = base > -INFINITY, held = live && a.hold && a.hold[row0 + r] >= 0;
    float M = -INFINITY;
    double s = 0.0;
    if (live && !held) {
      const SliceState* st = w.state + (row0 + r) * slices;
      for (int i = lane; i < slices; i += WAVE) M = fmaxf(M, st[i].m);
      M = wave_max(M);
      for (int i = lane; i < slices; i += WAVE)
        if (st[i].m > -INFINITY) s += st[i].m == M ? (double)st[i].s : (double)st[i].s * exp((double)st[i].m - (double)M);
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, WAVE);
    }
    if (lane == 0) {
      peak[r] = held ? __builtin_nanf("") : M;
      // (infinite logits share the row's weight: log(1 / their number) each)
      norm[r] = held ? (double)base : M > -INFINITY ? (double)base - ((M < INFINITY ? (double)M : 0.0) + log(s)) : 0.0;
    }
  }
  __shared__ Candidate list[JOIN_LIST];
  __shared__ int n_list;
  __shared__ uint32_t reach[JOIN_WAVES];
  if (threadIdx.x == 0) n_list = 0;
  __syncthreads();
  const int lists = R * slices;
  // candidate k of a list; false: there is none
  auto look = [&](int l, int k, Candidate& c) {
    const int r = l / slices;
    const float p = peak[r];
    if (p != p) {
      c = Candidate{norm[r], (uint64_t)r << 32 | (uint32_t)a.hold[row0 + r]};
      return l % slices == 0 && k == 0;
    }
    if (!(p > -INFINITY)) return false;
    const uint64_t key = w.key[(row0 * slices + l) * K + k];
    const float z = value_of(key_order(key));
    c = Candidate{norm[r] + (p < INFINITY ? (double)z : 0.0), (uint64_t)r << 32 | key_token(key)};
    return key != 0 && (p < INFINITY || z == INFINITY);
  };
  // no candidate below the K-th largest first one of any wave's lanes is wanted (scores as floats, rounded: what is as large, is looked at)
  float top = -INFINITY;
  for (int l = threadIdx.x; l < lists; l += JOIN_THREADS) {
    Candidate c;
    if (look(l, 0, c)) top = fmaxf(top, (float)c.score);
  }
  const uint32_t t = reached_by(order_of(top), K, 32);
  if (lane == 0) reach[wave] = t;
  __syncthreads();
  uint32_t least = NO_VALUE;
  for (int v = 0; v < JOIN_WAVES; ++v) least = max(least, reach[v]);
  for (int l = threadIdx.x; l < lists; l += JOIN_THREADS)
    for (int k = 0; k < K; ++k) {
      Candidate c;
      if (!look(l, k, c) || order_of((float)c.score) < least) break;
      const int at = atomicAdd(&n_list, 1);
      if (at < JOIN_LIST) list[at] = c;
    }
  __syncthreads();
  const int n = n_list;
  const int64_t out = (int64_t)seq * K;
  auto put = [&](int k, const Candidate& c) {
    a.row[out + k] = (int32_t)(c.at >> 32);
    a.token[out + k] = (int32_t)c.at;
    a.score_out[out + k] = (float)c.score;
  };
  int filled = n;
  if (n <= JOIN_LIST) {
    for (int i = threadIdx.x; i < n; i += JOIN_THREADS) {
      const Candidate mine = list[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += better(list[j], mine);
      if (rank < K) put(rank, mine);
    }
  } else {
    // thousands of equal scores: one after the other
    __shared__ Candidate found[JOIN_WAVES];
    Candidate last{INFINITY, 0};
    bool begun = false;
    for (filled = 0; filled < K; ++filled) {
      Candidate mine{-INFINITY, ~0ull};
      for (int l = threadIdx.x; l < lists; l += JOIN_THREADS)
        for (int k = 0; k < K; ++k) {
          Candidate c;
          if (!look(l, k, c)) break;
          if ((!begun || better(last, c)) && better(c, mine)) mine = c;
        }
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
  for (int k = min(filled, K) + threadIdx.x; k < K; k += JOIN_THREADS) {
    a.row[out + k] = a.token[out + k] = -1;
    a.score_out[out + k] = -INFINITY;
  }
}

void launch_select(bool bf16, const SelectArgs& a, hipStream_t st) {
  const SelectScratch w = scratch_of(a);
  const int slices = select_slices(a.vocab);
  const dim3 grid(slices, a.n_seq * a.n_rows);
  if (bf16) select_slice_kernel<bf16_t><<<grid, SELECT_THREADS, 0, st>>>(a, w);
  else select_slice_kernel<float><<<grid, SELECT_THREADS, 0, st>>>(a, w);
  select_join_kernel<<<a.n_seq, JOIN_THREADS, 0, st>>>(a, w, slices);
}

// ---------------------------------------------------------------- pages
// One bit per page of the pool, in LDS, with the number of bits in front of every 64 of them: the k-th page of a kind is found
// there, and what a page's place among its kind is.
constexpr int POOL_THREADS = 1024, POOL_WAVES = POOL_THREADS / WAVE;
struct PageBits {
  uint64_t* word;
  int32_t* before;            // [words + 1]
  int words;
  // Bits of the pages that `in` says yes to (every thread of the workgroup calls; ends with a barrier).
  template <class In> __device__ void build(int n_pages, char* lds, In in) {
    words = (n_pages + 63) / 64;
    word = reinterpret_cast<uint64_t*>(lds);
    before = reinterpret_cast<int32_t*>(lds + (size_t)words * 8);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int U = 8;
    for (int w0 = wave * U; w0 < words; w0 += POOL_WAVES * U) {
      bool is[U];
#pragma unroll
      for (int u = 0; u < U; ++u) is[u] = in(min((w0 + u) * 64 + lane, n_pages - 1));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t b = __builtin_amdgcn_ballot_w64(is[u] && (w0 + u) * 64 + lane < n_pages);
        if (lane == 0 && w0 + u < words) word[w0 + u] = b;
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

constexpr int PIECE_THREADS = 256, PIECE = PIECE_THREADS * 64;      // bytes that a workgroup moves at once, four loads of 16 per thread under way
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
static int page_pieces(const PagePool& p) { return (int)((p.page_bytes + PIECE - 1) / PIECE); }

// ---------------------------------------------------------------- fork
// What becomes of sequence i: columns below `own` are its parent's pages, shared; those below `need` are its own.
struct Fork {
  int parent, len, own, have, need, held;
  bool first;                 // of its parent's children: it takes over the pages that nobody else holds
};
__device__ inline Fork fork_of(const ForkArgs& a, int i) {      // i: the same in a whole wave
  const int all = a.parent[min((int)threadIdx.x & 63, a.n_new - 1)];
  Fork f;
  f.parent = a.parent[i];
  if (f.parent < 0 || f.parent >= a.n_old) f.parent = -1;
  f.len = f.parent < 0 ? 0 : max(0, min(a.len[f.parent], a.limit));
  f.held = f.parent < 0 ? 0 : max(0, min(a.held[f.parent], a.pt_stride));
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

// The first launch, one workgroup: who gets which free page, the lowest ones in the order of sequences and columns.
__global__ __launch_bounds__(POOL_THREADS) void fork_plan_kernel(ForkArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ int wanted[MAX_SEQS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  PageBits free;
  free.build(a.pool.n_pages, lds, [&](int page) { return a.refs[page] <= 0; });
  auto fresh_at = [&](const Fork& f, int c) {
    if (c >= f.need) return false;
    const int page = f.first ? old_page(a, f, c) : -1;
    return page < 0 || a.refs[page] != 1;
  };
  for (int i = wave; i < a.n_new; i += POOL_WAVES) {
    const Fork f = fork_of(a, i);
    int n = 0;
    for (int c0 = f.own; c0 < f.need; c0 += WAVE) n += __popcll(__builtin_amdgcn_ballot_w64(fresh_at(f, c0 + lane)));
    if (lane == 0) wanted[i] = n;
  }
  __syncthreads();
  const int upto = lane_scan(lane < a.n_new ? wanted[lane] : 0);      // (n_new <= 64)
  const int missing = max(0, __builtin_amdgcn_readlane(upto, 63) - free.total());
  if (threadIdx.x == 0) *a.missing = missing;
  if (missing > 0) return;
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
  for (int i = wave; i < a.n_new; i += POOL_WAVES) {
    const Fork f = fork_of(a, i);
    int at = __builtin_amdgcn_readlane(upto, i) - wanted[i];
    int32_t* row = a.new_table + (int64_t)i * a.new_stride;
    for (int c0 = f.own; c0 < f.need; c0 += WAVE) {
      const int c = c0 + lane;
      const bool fresh = fresh_at(f, c);
      const uint64_t all = __builtin_amdgcn_ballot_w64(fresh);
      if (fresh) row[c] = free.find<true>(at + __popcll(all & below));
      else if (c < f.need) row[c] = old_page(a, f, c);
      at += __popcll(all);
    }
    if (lane == 0) {
      a.new_len[i] = f.len;
      a.new_held[i] = f.need;
    }
  }
  for (int p = threadIdx.x; p < a.pool.n_pages; p += POOL_THREADS) a.new_refs[p] = a.refs[p];
}

// The second: shared columns and the counts of all pages, the sequences' states, and the pages that are copied.
struct ForkGrid {
  int state0, page0;          // first workgroups of the states and of the pages (in front: a row of the tables each)
  int state_pieces[MAX_STATES];
  int columns, pieces;
};
__global__ __launch_bounds__(PIECE_THREADS) void fork_apply_kernel(ForkArgs a, ForkGrid g) {
  if (*a.missing > 0) return;
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
  b -= g.page0;
  const int piece = b % g.pieces, layer = b / g.pieces % a.pool.n_layers;
  b /= g.pieces * a.pool.n_layers;
  const Fork f = fork_of(a, b / g.columns);
  const int c = f.own + b % g.columns;
  if (c >= min(f.have, f.need)) return;
  const int from = old_page(a, f, c), to = a.new_table[(int64_t)(b / g.columns) * a.new_stride + c];
  if (from >= 0 && from != to) move_page_piece(a.pool, from, to, layer, piece);
}

void launch_fork(const ForkArgs& a, hipStream_t st) {
  ForkGrid g{};
  g.state0 = a.n_new + a.n_old;
  g.page0 = g.state0;
  for (int k = 0; k < a.n_states; ++k) {
    g.state_pieces[k] = (int)((a.state[k].row_bytes + PIECE - 1) / PIECE);
    g.page0 += g.state_pieces[k] * a.n_new;
  }
  g.columns = (a.rewrite + PAGE - 1) / PAGE + 1;      // that hold something and are written: from (len - rewrite) / PAGE on
  if (g.columns > a.new_stride) g.columns = a.new_stride;
  g.pieces = page_pieces(a.pool);
  fork_plan_kernel<<<1, POOL_THREADS, page_bits_bytes(a.pool.n_pages), st>>>(a);
  fork_apply_kernel<<<g.page0 + a.n_new * g.columns * a.pool.n_layers * g.pieces, PIECE_THREADS, 0, st>>>(a, g);
}

// ---------------------------------------------------------------- compact
// The k-th page in use behind the front goes to the k-th free page in the front, the front being as long as there are pages in use.
__global__ __launch_bounds__(POOL_THREADS) void compact_plan_kernel(CompactArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int n = a.pool.n_pages;
  PageBits used;
  used.build(n, lds, [&](int page) { return a.refs[page] > 0; });
  const int front = used.total(), stay = front < n ? used.in_front(front) : front, moves = front - stay;
  if (threadIdx.x == 0) {
    a.count[0] = front;
    a.count[1] = moves;
  }
  for (int p = threadIdx.x; p < n; p += POOL_THREADS) {
    int to = -1;
    if (used.has(p)) {
      to = p;
      if (p >= front) {
        const int k = used.in_front(p) - stay;
        to = used.find<false>(k);
        a.moved[n + k] = p;
      }
      a.new_refs[to] = a.refs[p];
    }
    a.moved[p] = to;
    if (p >= front) a.new_refs[p] = 0;
    if (p >= moves) a.moved[n + p] = -1;
  }
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
  const int pieces = page_pieces(a.pool);
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
