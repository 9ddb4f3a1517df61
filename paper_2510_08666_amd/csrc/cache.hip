// The paged cache's writer and its evictor: norms per head, rotation and page layout of new tokens in one pass, and the move
// of chosen positions into other pages.
#include "cache.hpp"

namespace dinfer {

// ---------------------------------------------------------------- rotary tables
// cos / sin of pos * f_j times the rule's magnitude, worked out in double and stored as float: a float32 angle of position
// 32767 is off by up to 2e-3.
__global__ __launch_bounds__(256) void rotary_table_kernel(RotaryRule r, int max_pos, float* __restrict__ cos_tab, float* __restrict__ sin_tab) {
  const int half = r.rotary_dim / 2;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (int64_t)max_pos * half) return;
  const int pos = (int)(i / half), j = (int)(i % half);
  double f = pow(r.theta, -2.0 * j / r.rotary_dim);
  if (r.scaling == ROTARY_LINEAR) f /= r.factor;
  if (r.scaling == ROTARY_YARN) {
    const double ramp = fmin(fmax((j - r.low) / (r.high - r.low), 0.0), 1.0);
    f = f * (1.0 - ramp) + f / r.factor * ramp;
  }
  cos_tab[i] = (float)(cos(pos * f) * r.magnitude);
  sin_tab[i] = (float)(sin(pos * f) * r.magnitude);
}
void launch_rotary_table(const RotaryRule& r, int max_pos, float* cos_tab, float* sin_tab, hipStream_t st) {
  const int64_t n = (int64_t)max_pos * (r.rotary_dim / 2);
  rotary_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(r, max_pos, cos_tab, sin_tab);
}

// ---------------------------------------------------------------- append
// y = x / sqrt(mean(x^2) + eps) * gain over a head, then the pairs (j, j + r/2), or (2j, 2j + 1), of its first r features
// turned by the position's angles, all in float32 and rounded once.  A workgroup takes the tokens of one page (up to 16 slots)
// and either a cache head's keys and values or a query head; LANES lanes hold a row, 16 bytes each, so the norm is a
// reduction over lanes.  Keys go out in 32-byte blocks as the page has them; values are turned in LDS so that full half pages leave as
// 16-byte stores of eight slots.  Bound by its traffic.
constexpr int APPEND_THREADS = 256;
template <typename E, int HD>
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(AppendArgs a, SeqSpan groups) {
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, LANES = HD / G, ROWS = APPEND_THREADS / LANES;      // rows of a pass
  const int seq = owner_of(groups, blockIdx.x);
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0, base = cache_base(a.tok, seq, len);
  const int page_index = base / PAGE + ((int)blockIdx.x - groups.off[seq]);
  const int first = max(base, page_index * PAGE), last = min(base + len, (page_index + 1) * PAGE);   // cache positions [first, last)
  if (first >= last) return;
  const bool keys = (int)blockIdx.y < a.geom.n_heads;
  const int head = keys ? blockIdx.y : blockIdx.y - a.geom.n_heads;
  const int row = threadIdx.x / LANES, chunk = threadIdx.x % LANES, c0 = chunk * G;
  const float* gain = keys ? a.k_gain : a.q_gain;
  const int r = a.rotary_dim, h = r / 2;
  __shared__ float turn[ROWS][HD + 4];
  __shared__ E vt[PAGE][HD + 4];
  const int page = keys ? safe_page(a.geom, a.tok.page_table[(int64_t)seq * a.tok.pt_stride + page_index]) : 0;
  E* kv = (E*)a.kv_layer;
  for (int r0 = 0; r0 < PAGE; r0 += ROWS) {
    const int slot = r0 + row, pos = page_index * PAGE + slot;
    const bool valid = slot < PAGE && pos >= first && pos < last;
    const int64_t tok = tok0 + min(max(pos, first), last - 1) - base;      // rows that are none of the call's repeat one
    const vec x = load16<E>((keys ? (const E*)a.k + tok * a.k_stride : (const E*)a.q + tok * a.q_stride) + head * HD + c0);
    vec vv;
    if (keys) vv = load16<E>((const E*)a.v + tok * a.v_stride + head * HD + c0);
    const int where = a.positions ? a.positions[tok] : (int)(tok - tok0) + base;
    const int64_t angles = (int64_t)min(max(where, 0), a.table_rows - 1) * h;
    float f[G];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      f[i] = to_f32(x[i]);
      ss = fmaf(f[i], f[i], ss);
    }
    if (gain) {
#pragma unroll
      for (int d = LANES / 2; d > 0; d >>= 1) ss += __shfl_xor(ss, d, WAVE);
      const float inv = rsqrtf(ss * (1.f / HD) + a.eps);
#pragma unroll
      for (int i = 0; i < G; ++i) f[i] = f[i] * inv * gain[c0 + i];
    }
    if (!a.interleaved) {
#pragma unroll
      for (int i = 0; i < G; ++i) turn[row][c0 + i] = f[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int c = c0 + i;
        if (c < r) {
          const int j = c < h ? c : c - h;
          const float cs = a.cos_tab[angles + j], sn = a.sin_tab[angles + j], other = turn[row][c < h ? c + h : c - h];
          f[i] = c < h ? f[i] * cs - other * sn : f[i] * cs + other * sn;
        }
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        if (c0 + i < r) {
          const int j = (c0 + i) / 2;
          const float cs = a.cos_tab[angles + j], sn = a.sin_tab[angles + j], u = f[i], w = f[i + 1];
          f[i] = u * cs - w * sn;
          f[i + 1] = w * cs + u * sn;
        }
      }
    }
    vec y;
#pragma unroll
    for (int i = 0; i < G; ++i) y[i] = from_f32<E>(f[i]);
    if (keys) {
      if (valid) *reinterpret_cast<vec*>(kv + kv_k_index(a.geom, page, head, slot, c0)) = y;
      if (slot < PAGE) {
#pragma unroll
        for (int i = 0; i < G; ++i) vt[slot][c0 + i] = vv[i];
      }
    } else if (valid) {
      *reinterpret_cast<vec*>((E*)a.q_out + tok * a.q_out_stride + head * HD + c0) = y;
    }
  }
  if (!keys) return;
  __syncthreads();
  // values: a thread takes G slots of one feature
  const int s_lo = first - page_index * PAGE, s_hi = last - page_index * PAGE;
  for (int item = threadIdx.x; item < HD * (PAGE / G); item += APPEND_THREADS) {
    const int d = item / (PAGE / G), s0 = item % (PAGE / G) * G;
    E* dst = kv + kv_v_index(a.geom, page, head, s0, d);
    if (s0 >= s_lo && s0 + G <= s_hi) {
      vec y;
#pragma unroll
      for (int i = 0; i < G; ++i) y[i] = vt[s0 + i][d];
      *reinterpret_cast<vec*>(dst) = y;
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (s0 + i >= s_lo && s0 + i < s_hi) dst[i] = vt[s0 + i][d];
    }
  }
}

template <typename E, int HD> static void launch_append_t(const AppendArgs& a, const SeqSpan& groups, hipStream_t st) {
  const int heads = a.geom.n_heads * (1 + (a.q ? a.group : 0));
  append_kernel<E, HD><<<dim3(groups.off[groups.n_seq], heads), APPEND_THREADS, 0, st>>>(a, groups);
}
void launch_append(bool bf16, const AppendArgs& a, hipStream_t st) {
  SeqSpan groups;      // pages that a sequence's tokens may touch, wherever its first one falls
  groups.n_seq = a.tok.span.n_seq;
  groups.off[0] = 0;
  for (int s = 0; s < groups.n_seq; ++s) {
    const int len = a.tok.span.off[s + 1] - a.tok.span.off[s];
    groups.off[s + 1] = groups.off[s] + (len > 0 ? (len + PAGE - 2) / PAGE + 1 : 0);
  }
  if (bf16) {
    if (a.geom.head_dim == 128) launch_append_t<bf16_t, 128>(a, groups, st);
    else launch_append_t<bf16_t, 64>(a, groups, st);
  } else {
    if (a.geom.head_dim == 128) launch_append_t<float, 128>(a, groups, st);
    else launch_append_t<float, 64>(a, groups, st);
  }
}

// ---------------------------------------------------------------- evict
// Which positions stay: the best `m` of a head's n scores, ties to the lower position, the first n_sink and the last n_recent
// whatever they score.  One workgroup per (layer, sequence, head) holds the scores in registers as order-preserving integers; the m-th largest
// is found bit by bit from the top (a bit stays if at least m scores reach the value with it set), by counting: ties and
// repeated scores cost nothing, and no order of arrival matters.  Positions keep their order: a position's place is the number of
// chosen ones in front of it, from ballots and one prefix sum over the waves' counts.
constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / WAVE;

__device__ inline uint32_t score_order(float v) {
  if (v != v) return 0;                                // not a number: below everything
  const uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;       // (-inf maps to 0x007fffff: nothing but NaN reaches 0)
}

template <int PER>
__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(EvictArgs a) {
  const int head = blockIdx.x, seq = blockIdx.y, layer = blockIdx.z;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = min(max(a.len[seq], 0), min(a.limit, a.score_stride)), m = min(n, a.keep);
  const int64_t unit = ((int64_t)layer * a.n_seq + seq) * a.geom.n_heads + head;
  const float* score = a.score + unit * a.score_stride;
  int32_t* kept = a.kept + unit * a.keep;
  float* out = a.score_out ? a.score_out + unit * a.score_stride : nullptr;
  if (layer == 0 && head == 0 && tid == 0) a.new_len[seq] = m;
  float val[PER];
  uint32_t ord[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * EVICT_THREADS + tid;
    val[j] = i < n ? score[i] : 0.f;
    ord[j] = i < a.n_sink || i >= n - a.n_recent ? 0xffffffffu : score_order(val[j]);
  }
  __shared__ int count[2][EVICT_WAVES];
  // largest t with at least m scores >= t (t = 0 always has)
  uint32_t t = 0;
  int turn = 0;
  for (int bit = 31; bit >= 0; --bit, turn ^= 1) {
    const uint32_t c = t | (1u << bit);
    int mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      mine += __popcll(__builtin_amdgcn_ballot_w64(j * EVICT_THREADS + tid < n && ord[j] >= c));
    if (lane == 0) count[turn][wave] = mine;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < EVICT_WAVES; ++w) total += count[turn][w];
    if (total >= m) t = c;
  }
  // places: chosen are all above t, and the first of those equal to it until m are full
  __shared__ int above[PER][EVICT_WAVES], equal[PER][EVICT_WAVES];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bool in = j * EVICT_THREADS + tid < n;
    const uint64_t gt = __builtin_amdgcn_ballot_w64(in && ord[j] > t), eq = __builtin_amdgcn_ballot_w64(in && ord[j] == t);
    if (lane == 0) {
      above[j][wave] = __popcll(gt);
      equal[j][wave] = __popcll(eq);
    }
  }
  __syncthreads();
  __shared__ int total_above;
  if (wave == 0) {
    // prefix sums over the PER * EVICT_WAVES counts, in position order
    int run_gt = 0, run_eq = 0;
    for (int i0 = 0; i0 < PER * EVICT_WAVES; i0 += WAVE) {
      const int i = i0 + lane;
      const bool in = i < PER * EVICT_WAVES;
      int g = in ? above[i / EVICT_WAVES][i % EVICT_WAVES] : 0, e = in ? equal[i / EVICT_WAVES][i % EVICT_WAVES] : 0;
      const int g0 = g, e0 = e;
#pragma unroll
      for (int d = 1; d < WAVE; d <<= 1) {
        const int ug = __shfl_up(g, d, WAVE), ue = __shfl_up(e, d, WAVE);
        if (lane >= d) {
          g += ug;
          e += ue;
        }
      }
      if (in) {
        above[i / EVICT_WAVES][i % EVICT_WAVES] = run_gt + g - g0;
        equal[i / EVICT_WAVES][i % EVICT_WAVES] = run_eq + e - e0;
      }
      run_gt += __shfl(g, WAVE - 1, WAVE);
      run_eq += __shfl(e, WAVE - 1, WAVE);
    }
    if (lane == 0) total_above = run_gt;
  }
  __syncthreads();
  const int ties = m - total_above;      // of those equal to t
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * EVICT_THREADS + tid;
    const bool in = i < n, gt = in && ord[j] > t, eq = in && ord[j] == t;
    const int g = above[j][wave] + __popcll(__builtin_amdgcn_ballot_w64(gt) & below);
    const int e = equal[j][wave] + __popcll(__builtin_amdgcn_ballot_w64(eq) & below);
    if (gt || (eq && e < ties)) {
      const int at = g + min(e, ties);
      kept[at] = i;
      if (out) out[at] = val[j];
    }
  }
  for (int i = m + tid; i < a.keep; i += EVICT_THREADS) kept[i] = -1;
  if (out)
    for (int i = m + tid; i < a.score_stride; i += EVICT_THREADS) out[i] = 0.f;
}

// The chosen rows of one head into one new page: keys in 16-byte pieces, values slot by slot.
constexpr int MOVE_THREADS = 256;
template <typename E, int HD>
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictArgs a, int n_new_pages) {
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, LANES = HD / G;
  const int seq = blockIdx.y, layer = blockIdx.z, head = blockIdx.x % a.geom.n_heads, new_page = blockIdx.x / a.geom.n_heads;
  const int64_t unit = ((int64_t)layer * a.n_seq + seq) * a.geom.n_heads + head;
  const int n = min(max(a.len[seq], 0), min(a.limit, a.score_stride)), m = min(n, a.keep), slots = min(PAGE, m - new_page * PAGE);
  if (slots <= 0) return;
  E* kv = (E*)((char*)a.kv + layer * a.kv_layer_bytes);
  __shared__ int32_t s_page[PAGE], s_slot[PAGE];
  if (threadIdx.x < PAGE) {
    const int pos = a.kept[unit * a.keep + new_page * PAGE + min((int)threadIdx.x, slots - 1)];
    s_page[threadIdx.x] = safe_page(a.geom, a.page_table[(int64_t)seq * a.pt_stride + pos / PAGE]);
    s_slot[threadIdx.x] = pos % PAGE;
  }
  const int to = safe_page(a.geom, a.new_table[(int64_t)seq * a.new_stride + new_page]);
  __syncthreads();
  for (int item = threadIdx.x; item < slots * LANES; item += MOVE_THREADS) {
    const int slot = item / LANES, c0 = item % LANES * G;
    *reinterpret_cast<vec*>(kv + kv_k_index(a.geom, to, head, slot, c0)) =
        load16<E>(kv + kv_k_index(a.geom, s_page[slot], head, s_slot[slot], c0));
  }
  for (int item = threadIdx.x; item < HD * (PAGE / G); item += MOVE_THREADS) {
    const int d = item / (PAGE / G), s0 = item % (PAGE / G) * G;
    vec y;
#pragma unroll
    for (int i = 0; i < G; ++i) y[i] = kv[kv_v_index(a.geom, s_page[s0 + i], head, s_slot[s0 + i], d)];
    E* dst = kv + kv_v_index(a.geom, to, head, s0, d);
    if (s0 + G <= slots) *reinterpret_cast<vec*>(dst) = y;
    else
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (s0 + i < slots) dst[i] = y[i];
  }
}

template <typename E, int HD> static void launch_move(const EvictArgs& a, hipStream_t st) {
  const int pages = (a.keep + PAGE - 1) / PAGE;
  evict_move_kernel<E, HD><<<dim3(pages * a.geom.n_heads, a.n_seq, a.n_layers), MOVE_THREADS, 0, st>>>(a, pages);
}
void launch_evict(bool bf16, const EvictArgs& a, hipStream_t st) {
  const dim3 grid(a.geom.n_heads, a.n_seq, a.n_layers);
  const int bound = a.limit < a.score_stride ? a.limit : a.score_stride;
  if (bound <= 4 * EVICT_THREADS) evict_select_kernel<4><<<grid, EVICT_THREADS, 0, st>>>(a);
  else if (bound <= 8 * EVICT_THREADS) evict_select_kernel<8><<<grid, EVICT_THREADS, 0, st>>>(a);
  else evict_select_kernel<32><<<grid, EVICT_THREADS, 0, st>>>(a);
  if (bf16) {
    if (a.geom.head_dim == 128) launch_move<bf16_t, 128>(a, st);
    else launch_move<bf16_t, 64>(a, st);
  } else {
    if (a.geom.head_dim == 128) launch_move<float, 128>(a, st);
    else launch_move<float, 64>(a, st);
  }
}

}  // namespace dinfer
