// The paged cache's writer and its evictor: norms per head, rotation and page layout of new tokens in one pass, and the move
// of chosen positions into other pages.
#include "cache.hpp"

namespace dinfer {

// ---------------------------------------------------------------- rotary tables
// cos / sin of pos * f_j times the rule's magnitude, worked out in double from a rule in double and stored as float: a float32 angle of
// position 32767 is off by up to 2e-3, and a base or factor that was rounded to float32 turns it as far.
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
// turned by the position's angles, all in float32 and rounded once.  Bound by its traffic.  A workgroup takes the tokens of one page (up
// to 16 slots) and the keys and values of HB cache heads, or HB query heads: all its rows are under way at once, and a token's angles
// and the gains are fetched once for them.  LANES lanes hold a row, 16 bytes each, so a norm is a reduction over lanes and
// a pair's other half comes from the lane that holds it.  Keys go out in 32-byte blocks as the page has them; values are
// turned in LDS so that full half pages leave as 16-byte stores.  ALIGNED: r is a multiple of two lanes' features (whole heads,
// halves, quarters): angles come as 16-byte loads, other halves as whole registers; otherwise feature by feature.
constexpr int APPEND_THREADS = 256;
template <typename E, int HD, int HB, bool ALIGNED>
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(AppendArgs a, SeqSpan groups) {
  typedef typename ET<E>::vec vec;
  constexpr int G = ET<E>::G, LANES = HD / G, ROWS = APPEND_THREADS / LANES;      // rows of a pass
  constexpr int HALVES = ROWS < PAGE ? PAGE / ROWS : 1, AT_ONCE = ROWS > PAGE ? ROWS / PAGE : 1, PASSES = HB / AT_ONCE;
  static_assert(HB % AT_ONCE == 0, "a pass takes whole heads");
  const int seq = owner_of(groups, blockIdx.x);
  const int tok0 = a.tok.span.off[seq], len = a.tok.span.off[seq + 1] - tok0, base = cache_base(a.tok, seq, len);
  const int page_index = base / PAGE + ((int)blockIdx.x - groups.off[seq]);
  const int first = max(base, page_index * PAGE), last = min(base + len, (page_index + 1) * PAGE);   // cache positions [first, last)
  if (first >= last) return;
  const int key_blocks = (a.geom.n_heads + HB - 1) / HB;
  const bool keys = (int)blockIdx.y < key_blocks;
  const int head0 = (keys ? blockIdx.y : blockIdx.y - key_blocks) * HB, n_heads = keys ? a.geom.n_heads : a.geom.n_heads * a.group;
  const int row = threadIdx.x / LANES, chunk = threadIdx.x % LANES, c0 = chunk * G;
  const float* gain = keys ? a.k_gain : a.q_gain;
  const int r = a.rotary_dim, h = r / 2;
  __shared__ float turn[ALIGNED ? 1 : ROWS][HD + 4];
  __shared__ __align__(16) E vt[HB][PAGE][HD + 16 / sizeof(E)];
  const int page = keys ? safe_page(a.geom, a.tok.page_table[(int64_t)seq * a.tok.pt_stride + page_index]) : 0;
  E* kv = (E*)a.kv_layer;
  f32x4 g4[G / 4];
#pragma unroll
  for (int i = 0; i < G / 4; ++i) g4[i] = gain ? *reinterpret_cast<const f32x4*>(gain + c0 + 4 * i) : f32x4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
  for (int half = 0; half < HALVES; ++half) {
    const int slot = half * ROWS + row % PAGE, pos = page_index * PAGE + slot;
    const bool valid = pos >= first && pos < last;
    const int64_t tok = tok0 + min(max(pos, first), last - 1) - base;      // slots that are none of the call's repeat a token
    vec x[PASSES], vv[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int head = min(head0 + p * AT_ONCE + row / PAGE, n_heads - 1);
      x[p] = load16<E>((keys ? (const E*)a.k + tok * a.k_stride : (const E*)a.q + tok * a.q_stride) + head * HD + c0);
      if (keys) vv[p] = load16<E>((const E*)a.v + tok * a.v_stride + head * HD + c0);
    }
    const int where = a.positions ? a.positions[tok] : (int)(tok - tok0) + base;
    const int64_t angles = (int64_t)min(max(where, 0), a.table_rows - 1) * h;
    const bool turns = c0 < r, low = c0 < h;      // (aligned: the whole 16 bytes are)
    float cs[G], sn[G];
    if constexpr (ALIGNED) {
      if (!a.interleaved) {
        const int64_t at = angles + (turns ? low ? c0 : c0 - h : 0);
#pragma unroll
        for (int i = 0; i < G; i += 4) {
          const f32x4 c4 = *reinterpret_cast<const f32x4*>(a.cos_tab + at + i), s4 = *reinterpret_cast<const f32x4*>(a.sin_tab + at + i);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            cs[i + j] = c4[j];
            sn[i + j] = low ? -s4[j] : s4[j];
          }
        }
      } else {
        const int64_t at = angles + (turns ? c0 / 2 : 0);
#pragma unroll
        for (int i = 0; i < G / 2; i += 2) {
          const float2 c2 = *reinterpret_cast<const float2*>(a.cos_tab + at + i), s2 = *reinterpret_cast<const float2*>(a.sin_tab + at + i);
          cs[2 * i] = cs[2 * i + 1] = c2.x;
          cs[2 * i + 2] = cs[2 * i + 3] = c2.y;
          sn[2 * i] = -s2.x, sn[2 * i + 1] = s2.x;
          sn[2 * i + 2] = -s2.y, sn[2 * i + 3] = s2.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int c = c0 + i, j = a.interleaved ? c / 2 : c < h ? c : c - h;
        const float s = c < r ? a.sin_tab[angles + j] : 0.f;
        cs[i] = c < r ? a.cos_tab[angles + j] : 1.f;
        sn[i] = (a.interleaved ? c % 2 == 0 : c < h) ? -s : s;
      }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int head = head0 + p * AT_ONCE + row / PAGE;
      float f[G], o[G];
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        f[i] = to_f32(x[p][i]);
        ss = fmaf(f[i], f[i], ss);
      }
      if (gain) {
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) ss += __shfl_xor(ss, d, WAVE);
        const float inv = rsqrtf(ss * (1.f / HD) + a.eps);
#pragma unroll
        for (int i = 0; i < G; ++i) f[i] = f[i] * inv * g4[i / 4][i % 4];
      }
      // the other halves of this lane's pairs
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < G; ++i) o[i] = f[i ^ 1];
      } else if constexpr (ALIGNED) {
        const int from = (threadIdx.x & 63) + (turns ? low ? h / G : -(h / G) : 0);
#pragma unroll
        for (int i = 0; i < G; ++i) o[i] = __shfl(f[i], from, WAVE);
      } else {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G; ++i) turn[row][c0 + i] = f[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G; ++i) o[i] = c0 + i < r ? turn[row][c0 + i < h ? c0 + i + h : c0 + i - h] : 0.f;
      }
      vec y;
#pragma unroll
      for (int i = 0; i < G; ++i) y[i] = from_f32<E>((ALIGNED ? turns : c0 + i < r) ? f[i] * cs[i] + o[i] * sn[i] : f[i]);
      if (keys) {
        if (valid && head < n_heads) *reinterpret_cast<vec*>(kv + kv_k_index(a.geom, page, head, slot, c0)) = y;
        *reinterpret_cast<vec*>(&vt[p * AT_ONCE + row / PAGE][slot][c0]) = vv[p];
      } else if (valid && head < n_heads) {
        *reinterpret_cast<vec*>((E*)a.q_out + tok * a.q_out_stride + head * HD + c0) = y;
      }
    }
  }
  if (!keys) return;
  __syncthreads();
  // values: a thread takes G slots of one feature
  const int s_lo = first - page_index * PAGE, s_hi = last - page_index * PAGE;
  constexpr int ITEMS = HD * (PAGE / G);
#pragma unroll
  for (int i0 = 0; i0 < HB * ITEMS; i0 += APPEND_THREADS) {
    const int item = i0 + threadIdx.x, b = item / ITEMS, d = item % ITEMS / (PAGE / G), s0 = item % (PAGE / G) * G;
    if (item >= HB * ITEMS || head0 + b >= n_heads) break;
    E* dst = kv + kv_v_index(a.geom, page, head0 + b, s0, d);
    if (s0 >= s_lo && s0 + G <= s_hi) {
      vec y;
#pragma unroll
      for (int i = 0; i < G; ++i) y[i] = vt[b][s0 + i][d];
      *reinterpret_cast<vec*>(dst) = y;
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (s0 + i >= s_lo && s0 + i < s_hi) dst[i] = vt[b][s0 + i][d];
    }
  }
}

template <typename E, int HD, int HB> static void launch_append_hb(const AppendArgs& a, const SeqSpan& groups, hipStream_t st) {
  const int blocks = (a.geom.n_heads + HB - 1) / HB + (a.q ? (a.geom.n_heads * a.group + HB - 1) / HB : 0);
  const dim3 grid(groups.off[groups.n_seq], blocks);
  if (a.rotary_dim % (2 * ET<E>::G) == 0) append_kernel<E, HD, HB, true><<<grid, APPEND_THREADS, 0, st>>>(a, groups);
  else append_kernel<E, HD, HB, false><<<grid, APPEND_THREADS, 0, st>>>(a, groups);
}
// Four heads per workgroup once that leaves the chip full of workgroups, else as few as a pass takes (16 heads of 128: a block of 32
// tokens 4.4 us against 6.5 with four heads, 16 sequences of 1 to 64 tokens 6.9 against 9.4; four prompts of 333 to 1811 tokens, 108 MB,
// 27 with four heads, 4.0 TB/s, a microsecond more with one).
constexpr int APPEND_FULL = 2048;
template <typename E, int HD> static void launch_append_t(const AppendArgs& a, const SeqSpan& groups, hipStream_t st) {
  constexpr int LEAST = sizeof(E) * HD == 128 ? 2 : 1;
  const int64_t heads = (int64_t)groups.off[groups.n_seq] * a.geom.n_heads * (1 + (a.q ? a.group : 0));
  if (heads >= 4 * APPEND_FULL) launch_append_hb<E, HD, 4>(a, groups, st);
  else launch_append_hb<E, HD, LEAST>(a, groups, st);
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
// whatever they score.  One workgroup per (layer, sequence, head) holds the scores in registers as order-preserving integers and finds the
// m-th largest digit by digit (8 bits) from the top: a histogram in LDS of the scores that share the digits found so far, and the
// digit where its sums from above reach what is still wanted; the search ends where a digit is taken whole.  The counts are
// whole numbers, so the order of the atomics does not matter.  Positions keep their order: a position's place is the number of
// chosen ones in front of it, from ballots and one prefix sum over the waves' counts.  Bound by the latency of these
// turns (512 heads of up to 4096 scores 15.1 us; a search two bits at a time by ballots took 16 turns, 35 us).
__device__ inline uint32_t score_order(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);                           // (-0 + 0 is 0)
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return v != v ? 0u : o;                                                // not a number: below everything (-inf maps to 0x007fffff)
}

template <int EVICT_THREADS, int PER>
__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(EvictArgs a) {
  constexpr int EVICT_WAVES = EVICT_THREADS / WAVE;
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
  for (int j = 0; j < PER; ++j) val[j] = score[max(0, min(j * EVICT_THREADS + tid, n - 1))];      // no branch: all under way together
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * EVICT_THREADS + tid;
    ord[j] = i >= n ? 0 : i < a.n_sink || i >= n - a.n_recent ? 0xffffffffu : score_order(val[j]);      // (0 reaches no value asked for)
  }
  __shared__ __align__(16) int hist[256];      // by digit, the largest first
  __shared__ int found[3];                     // digit, how many of it are wanted, how many there are
  uint32_t t = 0;                              // the digits found; at the end the m-th largest score, or less where all that share its digits are taken
  int want = m;
  for (int shift = 24; shift >= 0 && n > 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (j * EVICT_THREADS + tid < n && (shift == 24 || (ord[j] ^ t) >> (shift + 8) == 0)) atomicAdd(&hist[255 - (ord[j] >> shift & 255)], 1);
    __syncthreads();
    if (wave == 0) {
      const int4 h = reinterpret_cast<const int4*>(hist)[lane];
      const int sum = lane_scan(h.x + h.y + h.z + h.w), front = sum - (h.x + h.y + h.z + h.w);
      if (front < want && sum >= want) {       // exactly one lane
        int before = front, size = h.x, d = 4 * lane;
        if (before + size < want) before += size, size = h.y, ++d;
        if (before + size < want) before += size, size = h.z, ++d;
        if (before + size < want) before += size, size = h.w, ++d;
        found[0] = 255 - d;
        found[1] = want - before;
        found[2] = size;
      }
    }
    __syncthreads();
    t |= (uint32_t)found[0] << shift;
    want = found[1];
    if (want == found[2]) break;
  }
  // places: chosen are all above t, and the first of those equal to it until m are full
  __shared__ int above[PER][EVICT_WAVES], equal[PER][EVICT_WAVES];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const uint64_t gt = __builtin_amdgcn_ballot_w64(ord[j] > t), eq = __builtin_amdgcn_ballot_w64(j * EVICT_THREADS + tid < n && ord[j] == t);
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
#pragma unroll
    for (int i0 = 0; i0 < PER * EVICT_WAVES; i0 += WAVE) {
      const int i = i0 + lane;
      const bool in = i < PER * EVICT_WAVES;
      const int g = in ? above[i / EVICT_WAVES][i % EVICT_WAVES] : 0, e = in ? equal[i / EVICT_WAVES][i % EVICT_WAVES] : 0;
      const int sg = lane_scan(g), se = lane_scan(e);
      if (in) {
        above[i / EVICT_WAVES][i % EVICT_WAVES] = run_gt + sg - g;
        equal[i / EVICT_WAVES][i % EVICT_WAVES] = run_eq + se - e;
      }
      run_gt += __builtin_amdgcn_readlane(sg, WAVE - 1);
      run_eq += __builtin_amdgcn_readlane(se, WAVE - 1);
    }
    if (lane == 0) total_above = run_gt;
  }
  __syncthreads();
  const int ties = m - total_above;      // of those equal to t
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * EVICT_THREADS + tid;
    const bool gt = ord[j] > t, eq = i < n && ord[j] == t;
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

// The chosen rows of one head into one new page: keys in 16-byte pieces, values slot by slot.  Bound by the traffic: a cache line of
// values holds all 16 positions of a page, and what of it is not kept is fetched too (512 heads, 1024 kept of 900 to 4096
// positions: 171 us; by the memory counters 596 MB fetched for 266 MB of rows and as many written, 5.0 TB/s).
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
  if (bound <= 1024) evict_select_kernel<256, 4><<<grid, 256, 0, st>>>(a);
  else if (bound <= 4096) evict_select_kernel<256, 16><<<grid, 256, 0, st>>>(a);
  else if (bound <= 8192) evict_select_kernel<512, 16><<<grid, 512, 0, st>>>(a);
  else evict_select_kernel<1024, 32><<<grid, 1024, 0, st>>>(a);
  if (bf16) {
    if (a.geom.head_dim == 128) launch_move<bf16_t, 128>(a, st);
    else launch_move<bf16_t, 64>(a, st);
  } else {
    if (a.geom.head_dim == 128) launch_move<float, 128>(a, st);
    else launch_move<float, 64>(a, st);
  }
}

}  // namespace dinfer
