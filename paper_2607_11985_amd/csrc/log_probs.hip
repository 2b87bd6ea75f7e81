// log_probs.hip -- log probabilities of given outcomes, entropy and the most probable
// outcomes of a row of scores, and the gradient with respect to logits.
//
//   logits   d_j = (z_j - m) / T with m = max z;  S = sum e^d_j,  U = sum e^d_j d_j
//            log p_j = d_j - ln S,  H = ln S - U / S
//   weights  v_j = w_j / m with m a power of two near the largest weight;  S = sum v_j,
//            U = sum v_j ln v_j,  log p_j = ln v_j - ln S,  H = ln S - U / S
//   dz_j = (sum_{t_s = j} g_s - p_j sum g_s - gH p_j (log p_j + H)) / T
//
// Memory-bound: the forward reads the scores once, the backward reads them and writes the
// gradient once.  One pass keeps a running m, S and U per thread (rescaled when m grows) and
// the row's largest scores: every wave holds its 64 best as a sorted list, one key per lane,
// and a threshold below which a score cannot be among the wanted ones.  A score above it goes
// to a small buffer in LDS; 64 of those are sorted across the lanes and merged into the list.
// After steps 1, 4, 16, ... the threshold is raised to what n of the lanes' maxima reach, so
// that some n scores pass each time: one comparison per pack and one sort per row.
//
// bf16 4096 x 32768: forward 58 us without a ranking, 77 with the 5 best (268 MB, 3.5 TB/s: 11
// instructions a score, one an exponential, bind as much as memory does); backward 96 us (537 MB,
// 5.6 TB/s).  fp32: forward 98 and 108 us (5.5 and 5.0 TB/s), at memory's rate.  256 x 65536
// weights with the 8 best 22 us, 12.5 without (67 MB, 5.4 TB/s).  One row of 2^20 with the 16
// best 18 us, in two launches, where chains of dependent steps bind.
#include <algorithm>
#include <type_traits>

#include "layers.h"
#include "layers_device.h"

namespace vqc {
namespace {

constexpr int kMaxParts = 64;  // of a split row
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeastNormal = 0x1p-126f;

// ------------------------------------------------------------ keys and lists

// Scores as integers in their order: NaN above all, -0 equal to +0.  A key holds the score
// above the complement of its column, so that equal scores order from the lowest column.
// 0 is no entry.
__device__ __forceinline__ uint32_t score_key(float z) {
  if (z != z) return 0xFFFFFFFFu;
  const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
  if (k == 0xFFFFFFFFu) return __builtin_nanf("");
  return __builtin_bit_cast(float, k ^ ((k & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu));
}
// Columns fit 31 bits: a longer row is refused.
__device__ __forceinline__ uint64_t make_key(float z, uint32_t col) {
  return ((uint64_t)score_key(z) << 32) | (uint32_t)~col;
}

template <int N>
__device__ __forceinline__ uint64_t lane_xor_key(uint64_t x) {
  return ((uint64_t)lane_xor<N>((uint32_t)(x >> 32)) << 32) | lane_xor<N>((uint32_t)x);
}

// Compare-exchange with lane ^ N: the larger key goes to the lane with bit N clear where
// `falling`, else to the other.
template <int N>
__device__ __forceinline__ uint64_t exchange_keys(uint64_t x, int lane, bool falling) {
  const uint64_t o = lane_xor_key<N>(x);
  const bool want_max = ((lane & N) == 0) == falling;
  return (x > o) == want_max ? x : o;
}

// A bitonic sequence over 64 lanes into falling order.
__device__ __forceinline__ uint64_t merge_lanes(uint64_t x, int lane) {
  x = exchange_keys<32>(x, lane, true);
  x = exchange_keys<16>(x, lane, true);
  x = exchange_keys<8>(x, lane, true);
  x = exchange_keys<4>(x, lane, true);
  x = exchange_keys<2>(x, lane, true);
  return exchange_keys<1>(x, lane, true);
}

// Falling order over 64 lanes.
__device__ __forceinline__ uint64_t sort_lanes(uint64_t x, int lane) {
  x = exchange_keys<1>(x, lane, !(lane & 2));
  x = exchange_keys<2>(x, lane, !(lane & 4));
  x = exchange_keys<1>(x, lane, !(lane & 4));
  x = exchange_keys<4>(x, lane, !(lane & 8));
  x = exchange_keys<2>(x, lane, !(lane & 8));
  x = exchange_keys<1>(x, lane, !(lane & 8));
  x = exchange_keys<8>(x, lane, !(lane & 16));
  x = exchange_keys<4>(x, lane, !(lane & 16));
  x = exchange_keys<2>(x, lane, !(lane & 16));
  x = exchange_keys<1>(x, lane, !(lane & 16));
  x = exchange_keys<16>(x, lane, !(lane & 32));
  x = exchange_keys<8>(x, lane, !(lane & 32));
  x = exchange_keys<4>(x, lane, !(lane & 32));
  x = exchange_keys<2>(x, lane, !(lane & 32));
  x = exchange_keys<1>(x, lane, !(lane & 32));
  return merge_lanes(x, lane);
}

// The largest of aligned groups of G lanes, in every lane.
template <int G>
__device__ __forceinline__ float lanes_max(float x) {
  if constexpr (G > 1) x = fmaxf(x, lane_xor<1>(x));
  if constexpr (G > 2) x = fmaxf(x, lane_xor<2>(x));
  if constexpr (G > 4) x = fmaxf(x, lane_xor<4>(x));
  if constexpr (G > 8) x = fmaxf(x, lane_xor<8>(x));
  if constexpr (G > 16) x = fmaxf(x, lane_xor<16>(x));
  if constexpr (G > 32) x = fmaxf(x, lane_xor<32>(x));
  return x;
}

template <int N>
__device__ __forceinline__ void lanes_range(float& lo, float& hi) {
  lo = fminf(lo, lane_xor<N>(lo));
  hi = fmaxf(hi, lane_xor<N>(hi));
}

// A number that at least n of the lanes' numbers reach (none of them NaN; -inf: not there), near
// the n-th best; false if there are fewer.  By bisection: 5 instructions a step, and a bound a
// little low only lets a few more scores pass.
__device__ __forceinline__ bool lanes_bound(float x, int n, float& bound) {
  if (__popcll(__ballot(x > -INFINITY)) < n) return false;
  float lo = x > -INFINITY ? x : INFINITY, hi = x;
  lanes_range<1>(lo, hi);
  lanes_range<2>(lo, hi);
  lanes_range<4>(lo, hi);
  lanes_range<8>(lo, hi);
  lanes_range<16>(lo, hi);
  lanes_range<32>(lo, hi);
  if (__popcll(__ballot(x >= hi)) >= n) {
    bound = hi;
    return true;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float mid = 0.5f * lo + 0.5f * hi;
    const bool reached = __popcll(__ballot(x >= mid)) >= n;
    lo = reached ? mid : lo;
    hi = reached ? hi : mid;
  }
  bound = lo;
  return __popcll(__ballot(x >= lo)) >= n;
}

__device__ __forceinline__ uint64_t shuffle_key(uint64_t x, int lane) {
  const uint32_t hi = (uint32_t)__shfl((int)(x >> 32), lane), lo = (uint32_t)__shfl((int)x, lane);
  return ((uint64_t)hi << 32) | lo;
}

// The best 64 of two lists in falling order, as one.
__device__ __forceinline__ uint64_t merge_lists(uint64_t a, uint64_t b, int lane) {
  const uint64_t r = shuffle_key(b, 63 - lane);
  return merge_lanes(a > r ? a : r, lane);
}

__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's list of its best scores.  buf: 128 keys of LDS of this wave's own.
struct TopList {
  uint64_t list = 0;   // this lane's entry, falling over the lanes
  uint64_t bar = 0;    // the n-th entry
  float threshold;     // a score at or below it is not wanted, in a column beyond the list's
  int count = 0;       // keys in buf (the same in all lanes)
  bool filled = false; // the list has entries
  uint64_t* buf;
  int n, lane;

  __device__ void init(uint64_t* b, int top) {
    buf = b;
    n = top;
    lane = threadIdx.x & 63;
    threshold = __builtin_nanf("");  // everything passes
  }
  // A threshold from the largest score of each lane so far (-inf: none): just below one that n
  // of them reach, which must itself still pass.
  __device__ void raise(float most) {
    float t;
    if (!lanes_bound(most, n, t)) return;
    const uint32_t k = score_key(t);
    // (the key below +0 is -0, which compares equal: one further)
    const float below = key_score(k - (k == 0x80000000u ? 2 : 1));
    threshold = threshold >= below ? threshold : below;
  }
  __device__ void flush() {
    if (count == 0) return;
    wave_lds_fence();
    const int m = count < 64 ? count : 64;
    uint64_t x = lane < m ? buf[lane] : 0;
    const uint64_t rest = lane + 64 < count ? buf[lane + 64] : 0;
    wave_lds_fence();
    buf[lane] = rest;
    count -= m;
    x = sort_lanes(x, lane);
    list = filled ? merge_lists(list, x, lane) : x;
    filled = true;
    bar = shuffle_key(list, n - 1);
    if (bar) {  // with fewer than n entries everything passes
      const float t = key_score((uint32_t)(bar >> 32));
      threshold = threshold > t ? threshold : t;
    }
  }
  // The list once the row is through, by this wave alone.  Usually nothing has been sorted yet
  // and a few keys wait: a key's place is the number of keys above it.
  __device__ void finish() {
    if (filled || count > 32) {
      flush();
      return;
    }
    wave_lds_fence();
    const uint64_t x = lane < count ? buf[lane] : 0;
    int above = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) above += buf[j] > x;
    wave_lds_fence();
    if (x) buf[64 + above] = x;
    wave_lds_fence();
    list = lane < count ? buf[64 + lane] : 0;
    count = 0;
  }
  // One score per lane.  The columns of a pack's scores do not come in their order, so that
  // whole keys are compared here.
  __device__ void push(float z, uint32_t col, bool wanted) {
    const uint64_t key = make_key(z, col);
    const bool want = wanted && key > bar;
    const uint64_t mask = __ballot(want);
    if (mask == 0) return;
    if (want) buf[count + __popcll(mask & ((1ull << lane) - 1))] = key;
    count += __popcll(mask);
    if (count >= 64) flush();
  }
};

// The entries of several waves that can be among the row's n best, gathered in LDS: each wave
// has n scores at or above its own threshold, so none below the largest of these counts.
// Their places depend on which wave comes first; the order does not, once they are sorted.
struct Gathered {
  uint64_t* keys;
  int* count;

  __device__ void add(uint64_t key, float least, int lane) const {
    const bool want = key != 0 && !(key_score((uint32_t)(key >> 32)) < least);
    const uint64_t mask = __ballot(want);
    if (mask == 0) return;
    int base = 0;
    if (lane == 0) base = atomicAdd(count, (int)__popcll(mask));
    base = __shfl(base, 0);
    if (want) keys[base + __popcll(mask & ((1ull << lane) - 1))] = key;
  }
};

// The n best of `count` keys, in falling order over the first lanes of the first wave.  All
// THREADS threads of the workgroup, behind a barrier; keys is overwritten.
// Up to 256 keys: a key's place is the number of keys above it, groups of threads sharing the
// counting where the keys are few.  More: every wave sorts and merges its share, then the waves'
// lists are merged by halves.
template <int THREADS>
__device__ __forceinline__ uint64_t ranked(uint64_t* keys, int count, int* ranks, uint64_t* best,
                                           int n) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if (count > 256) {
    uint64_t list = 0;
    for (int i = wave * 64; i < count; i += THREADS) {
      const uint64_t x = sort_lanes(i + lane < count ? keys[i + lane] : 0, lane);
      list = i < THREADS ? x : merge_lists(list, x, lane);
    }
    __syncthreads();
    keys[t] = list;
    __syncthreads();
#pragma unroll
    for (int h = THREADS / 128; h > 0; h /= 2) {
      if (wave < h) {
        list = merge_lists(list, keys[t + 64 * h], lane);
        keys[t] = list;
      }
      __syncthreads();
    }
    return list;
  }
  int slots = 64;
  while (slots < count) slots *= 2;
  const int shares = THREADS / slots, share = t / slots, i = t % slots;
  if (t < count) ranks[t] = 0;
  if (t < 64) best[t] = 0;
  __syncthreads();
  const uint64_t key = i < count ? keys[i] : 0;
  int above = 0;
#pragma unroll 8
  for (int j = share; j < count; j += shares) above += keys[j] > key;
  if (key && above) atomicAdd(&ranks[i], above);
  __syncthreads();
  if (t < count && ranks[t] < n) best[ranks[t]] = keys[t];
  __syncthreads();
  return best[lane];
}

// ------------------------------------------------------------ running sums

struct Sums {
  float m, s, u;
};

// Weights are summed in units of a power of two near the largest one: large ones do not add up
// beyond fp32, and the logarithm instruction, which has no numbers below 2^-126, gets none that
// count.  Units and their inverses are normal numbers.
constexpr float kLeastUnit = 0x1p-120f, kMostUnit = 0x1p126f;
__device__ __forceinline__ float unit_of(float w) {
  const float u = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, w) & 0x7F800000u);
  return fminf(fmaxf(u, kLeastUnit), kMostUnit);
}
__device__ __forceinline__ float inverse_unit(float m) {
  return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, m));
}
__device__ __forceinline__ float log2_units(float a, float b) {  // log2(a / b)
  return (float)((int)(__builtin_bit_cast(uint32_t, a) >> 23) -
                 (int)(__builtin_bit_cast(uint32_t, b) >> 23));
}
// The same sums in units of m >= x.m (0 where nothing of them is left).
__device__ __forceinline__ Sums in_units(const Sums& x, float m) {
  const float e = x.m * inverse_unit(m);
  return {m, e * x.s, e > 0.f ? e * (x.u + x.s * log2_units(x.m, m)) : 0.f};
}

// No score yet (S = U = 0).
template <bool LOGITS>
__device__ __forceinline__ Sums no_sums() {
  return {LOGITS ? -INFINITY : kLeastUnit, 0.f, 0.f};
}

// From differences of logits to exponents of 2; finite at the largest 1 / T too, where 0 times
// infinity would be the largest logit's exponent.
__device__ __forceinline__ float exponent_scale(float inv_t) {
  return fminf(inv_t * kLog2e, 3.4028234e38f);
}

// (m, S, U) of two sets of logits; m = -inf: no score yet.
__device__ __forceinline__ Sums join_logits(const Sums& a, const Sums& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float ref = m == -INFINITY ? 0.f : m;
  const float da = a.m == -INFINITY ? 0.f : (a.m - ref) * c;
  const float db = b.m == -INFINITY ? 0.f : (b.m - ref) * c;
  const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
  // an m far below the other's: nothing is left of its sums, whatever da is
  const float ua = ea > 0.f ? ea * (a.u + a.s * da) : 0.f;
  const float ub = eb > 0.f ? eb * (b.u + b.s * db) : 0.f;
  return {m, ea * a.s + eb * b.s, ua + ub};
}

template <int N>
__device__ __forceinline__ void join_logits_lanes(Sums& x, float c) {
  x = join_logits(x, {lane_xor<N>(x.m), lane_xor<N>(x.s), lane_xor<N>(x.u)}, c);
}

// The sums of aligned groups of G lanes, in every lane.
template <int G, bool LOGITS>
__device__ __forceinline__ void join_lanes(Sums& x, float c) {
  if constexpr (LOGITS) {
    join_logits_lanes<1>(x, c);
    join_logits_lanes<2>(x, c);
    if constexpr (G > 4) {
      join_logits_lanes<4>(x, c);
      join_logits_lanes<8>(x, c);
    }
    if constexpr (G > 16) {
      join_logits_lanes<16>(x, c);
      join_logits_lanes<32>(x, c);
    }
  } else {
    x = in_units(x, lanes_max<G>(x.m));
    x.s = lanes_sum<G>(x.s);
    x.u = lanes_sum<G>(x.u);
  }
}

// The sums of NW waves, in LDS behind a barrier, as one; the same in all lanes.
template <int NW, bool LOGITS>
__device__ __forceinline__ Sums join_waves(const Sums* sums, int lane, float c) {
  Sums x = sums[lane % NW];
  join_lanes<NW, LOGITS>(x, c);
  return {__shfl(x.m, 0), __shfl(x.s, 0), __shfl(x.u, 0)};
}

// The pack's scores into a thread's running sums (U in units of log2); returns the largest of
// them (NaN left out: it shows in the sum).
template <typename T, bool LOGITS>
__device__ __forceinline__ float add_pack(Sums& x, const Pack<T>& p, float c) {
  constexpr int V = kPack<T>;
  float top = (float)p.v[0];
#pragma unroll
  for (int i = 1; i < V; ++i) top = fmaxf(top, (float)p.v[i]);
  if constexpr (LOGITS) {
    if (top > x.m) {
      const float d = x.m == -INFINITY ? 0.f : (x.m - top) * c;
      const float e = __builtin_amdgcn_exp2f(d);
      x.u = e > 0.f ? e * (x.u + x.s * d) : 0.f;
      x.s *= e;
      x.m = top;
    }
    const float ref = x.m == -INFINITY ? 0.f : x.m;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = ((float)p.v[i] - ref) * c;  // -inf where ruled out, NaN where it is NaN
      const float e = __builtin_amdgcn_exp2f(d);
      x.s += e;
      x.u += e * fmaxf(d, -3.e38f);  // 0 * -inf would be NaN
    }
  } else {
    if (top >= 0x1p32f * x.m) x = in_units(x, unit_of(top));  // the first ones, then hardly ever
    const float inv = inverse_unit(x.m);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float w = (float)p.v[i] * inv;
      x.s += w;
      x.u += w * __builtin_amdgcn_logf(fmaxf(w, kLeastNormal));  // w log2 w; 0 for 0
    }
  }
  return top;
}

__device__ __forceinline__ float entropy_of(const Sums& x) {
  return x.s == 0.f ? 0.f : logf(x.s) - x.u * kLn2 / x.s;
}

// log p of a score in a row with these sums.
template <bool LOGITS>
__device__ __forceinline__ float log_p(float z, const Sums& x, float inv_t) {
  if (x.s == 0.f) return -INFINITY;
  if constexpr (LOGITS) return (z - x.m) * inv_t - logf(x.s);
  const float w = z * inverse_unit(x.m);
  if (w >= kLeastNormal) return logf(w) - logf(x.s);
  return logf(z) - (logf(x.s) + kLn2 * log2_units(x.m, 1.f));
}

// ------------------------------------------------------------ forward

// A row's outputs by `threads` threads; list: thread t's entry of the row's list.
template <typename T, bool LOGITS>
__device__ void write_row(const ScoreArgs& A, int64_t r, const Sums& x, uint64_t list, int t,
                          int threads) {
  const T* z = static_cast<const T*>(A.scores) + r * A.lds;
  if (t == 0) {
    if (A.entropy) A.entropy[r] = entropy_of(x);
    if (A.stats) {
      A.stats[2 * r] = x.m;
      A.stats[2 * r + 1] = x.s;
    }
  }
  if (t < A.n_top) {  // n_top <= cols: the list is full
    const uint32_t col = ~(uint32_t)list;
    A.top_index[r * A.n_top + t] = col;
    A.top_logp[r * A.n_top + t] = log_p<LOGITS>(key_score((uint32_t)(list >> 32)), x, A.inv_t);
  }
  for (int64_t s = t; s < A.n_targets; s += threads) {
    const int64_t j = A.targets[r * A.n_targets + s];
    float v = 0.f;
    if (j != -1)
      v = j < 0 || j >= A.cols ? __builtin_nanf("") : log_p<LOGITS>((float)z[j], x, A.inv_t);
    A.logp[r * A.n_targets + s] = v;
  }
}

// A split row's parts in the workspace: [rows][parts] sums, then [rows][parts][n_top] keys.
struct SplitWs {
  Sums* sums;
  uint64_t* keys;
};
__host__ __device__ inline SplitWs split_ws(unsigned char* ws, int64_t rows, int64_t parts) {
  const int64_t head = (rows * parts * (int64_t)sizeof(Sums) + 255) / 256 * 256;
  return {reinterpret_cast<Sums*>(ws), reinterpret_cast<uint64_t*>(ws + head)};
}

// NW waves per row (or per part of one), RW rows per workgroup.  parts > 1: blockIdx.x =
// row * parts + part, and the part goes to the workspace.  SHORT: rows of less than a pack.
template <typename T, bool LOGITS, bool TOP, int NW, int RW, bool SHORT>
__global__ void __launch_bounds__(64 * NW * RW, 4) score_kernel(const ScoreArgs A, int64_t parts,
                                                             int64_t part_cols) {
  constexpr int V = kPack<T>, U = 2;
  __shared__ uint64_t bufs[TOP ? NW * RW * 128 : 1];
  __shared__ uint64_t gathered[TOP && NW > 1 ? NW * 128 : 1];
  __shared__ uint64_t best64[TOP && NW > 1 ? 64 : 1];
  __shared__ int ranks[TOP && NW > 1 ? 256 : 1];
  __shared__ Sums sums[NW * RW];
  __shared__ float bounds[NW * RW];
  __shared__ int found;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mine = wave / NW, wr = wave % NW;
  const float c = LOGITS ? exponent_scale(A.inv_t) : 1.f;
  const int64_t work = A.rows * parts;
  for (int64_t base = (int64_t)blockIdx.x * RW; base < work; base += (int64_t)gridDim.x * RW) {
    if constexpr (NW > 1) __syncthreads();  // the last row's readers are done with sums and bufs
    const int64_t item = base + mine < work ? base + mine : work - 1;
    const int64_t r = parts > 1 ? item / parts : item;
    const int64_t c0 = parts > 1 ? (item - r * parts) * part_cols : 0;
    const int64_t c1 = parts > 1 && c0 + part_cols < A.cols ? c0 + part_cols : A.cols;
    const T* z = static_cast<const T*>(A.scores) + r * A.lds;
    Sums x = no_sums<LOGITS>();
    TopList top;
    if constexpr (TOP) top.init(bufs + wave * 128, A.n_top);
    float most = -INFINITY;   // this lane's largest score so far
    int step = 0, again = 1;  // the threshold is raised after steps 1, 4, 16, ...
    // a step covers U * 64 * V columns of this wave; the next step's packs are on their way
    // while one is worked on
    constexpr int64_t kStep = U * 64 * V;
    Raw next[U];
    auto load = [&](Raw(&to)[U], int64_t at) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        to[u] = load_raw<T, SHORT>(z, at + (u * 64 + lane) * V, c1);
    };
    int64_t at = c0 + (int64_t)wr * kStep;
    if (at < c1) load(next, at);
    for (; at < c1; at += NW * kStep) {
      Pack<T> p[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        p[u] = taken<T, SHORT>(next[u], at + (u * 64 + lane) * V, c1,
                               LOGITS ? (T)-INFINITY : (T)0.f);
      if (at + NW * kStep < c1) load(next, at + NW * kStep);
      float best[U];
#pragma unroll
      for (int u = 0; u < U; ++u) best[u] = add_pack<T, LOGITS>(x, p[u], c);
      if constexpr (TOP) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (LOGITS || at + (u * 64 + lane + 1) * V <= c1) {
            most = fmaxf(most, best[u]);
          } else {  // (zeros are filled in behind the end)
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (at + (u * 64 + lane) * V + i < c1) most = fmaxf(most, (float)p[u].v[i]);
          }
        }
        if (++step == again) {
          top.raise(most);
          again *= 4;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t col = at + (u * 64 + lane) * V;
          const float least = top.threshold;
          // a sum of NaN: the pack may hold one, which best[u] left out
          if (__ballot((!(best[u] <= least) || x.s != x.s) && col < c1) == 0) continue;
          uint32_t left = 0;  // this lane's wanted scores
#pragma unroll
          for (int i = 0; i < V; ++i)
            left |= (!((float)p[u].v[i] <= least) && col + i < c1 ? 1u : 0u) << i;
          while (__ballot(left != 0)) {
            const int i = left ? __builtin_ctz(left) : 0;
            float zi = (float)p[u].v[0];
#pragma unroll
            for (int k = 1; k < V; ++k) zi = i == k ? (float)p[u].v[k] : zi;
            top.push(zi, (uint32_t)(col + i), left != 0);
            left &= left - 1;
          }
        }
      }
    }
    if constexpr (TOP && NW == 1) top.finish();
    join_lanes<64, LOGITS>(x, c);
    if constexpr (NW > 1) {
      if (lane == 0) {
        sums[wave] = x;
        if constexpr (TOP)
          bounds[wave] = top.threshold == top.threshold ? top.threshold : -INFINITY;
      }
      if (threadIdx.x == 0) found = 0;
      __syncthreads();
      x = join_waves<NW, LOGITS>(sums, lane, c);
      if constexpr (TOP) {
        float least = bounds[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) least = fmaxf(least, bounds[w]);
        const Gathered all = {gathered, &found};
        all.add(lane < top.count ? top.buf[lane] : 0, least, lane);  // count < 64
        all.add(top.list, least, lane);
        __syncthreads();
        top.list = ranked<64 * NW>(gathered, found, ranks, best64, A.n_top);
      }
    }
    if (base + mine >= work) continue;
    const int t = wr * 64 + lane;
    if (parts > 1) {
      const SplitWs ws = split_ws(A.ws, A.rows, parts);
      if (t == 0) ws.sums[item] = x;
      if constexpr (TOP)
        if (t < A.n_top) ws.keys[item * A.n_top + t] = top.list;
    } else {
      write_row<T, LOGITS>(A, r, x, TOP ? top.list : 0, t, NW * 64);
    }
  }
}

// The parts of a split row, joined by one workgroup: a launch's latency and 1 to 3 us.
template <typename T, bool LOGITS, bool TOP>
__global__ void __launch_bounds__(1024) score_join_kernel(const ScoreArgs A, int64_t parts) {
  constexpr int NW = 16;
  __shared__ uint64_t gathered[TOP ? kMaxParts * 64 : 1];
  __shared__ uint64_t best64[TOP ? 64 : 1];
  __shared__ int ranks[TOP ? 256 : 1];
  __shared__ Sums sums[NW];
  __shared__ float bounds[NW];
  __shared__ int found;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float c = LOGITS ? exponent_scale(A.inv_t) : 1.f;
  const SplitWs ws = split_ws(A.ws, A.rows, parts);
  const int64_t r = blockIdx.x;
  Sums x = no_sums<LOGITS>();
  float least = -INFINITY;  // the largest n-th entry of a part
  for (int64_t p = threadIdx.x; p < parts; p += 64 * NW) {
    const Sums o = ws.sums[r * parts + p];
    if constexpr (LOGITS) {
      x = join_logits(x, o, c);
    } else {
      const float m = fmaxf(x.m, o.m);
      const Sums a = in_units(x, m), b = in_units(o, m);
      x = {m, a.s + b.s, a.u + b.u};
    }
    if constexpr (TOP) {
      const uint64_t last = ws.keys[(r * parts + p) * A.n_top + A.n_top - 1];
      if (last) least = fmaxf(least, key_score((uint32_t)(last >> 32)));
    }
  }
  join_lanes<64, LOGITS>(x, c);
  float unused = 0.f;
  lanes_range<1>(unused, least);
  lanes_range<2>(unused, least);
  lanes_range<4>(unused, least);
  lanes_range<8>(unused, least);
  lanes_range<16>(unused, least);
  lanes_range<32>(unused, least);
  if (lane == 0) {
    sums[wave] = x;
    bounds[wave] = least;
  }
  if (threadIdx.x == 0) found = 0;
  __syncthreads();
  x = join_waves<NW, LOGITS>(sums, lane, c);
  least = bounds[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) least = fmaxf(least, bounds[w]);
  uint64_t best = 0;
  if constexpr (TOP) {
    const Gathered all = {gathered, &found};
    for (int64_t p = wave; p < parts; p += NW)
      all.add(lane < A.n_top ? ws.keys[(r * parts + p) * A.n_top + lane] : 0, least, lane);
    __syncthreads();
    best = ranked<64 * NW>(gathered, found, ranks, best64, A.n_top);
  }
  write_row<T, LOGITS>(A, r, x, best, threadIdx.x, 64 * NW);
}

// ------------------------------------------------------------ backward

// One row's constants of the gradient.
struct RowGrad {
  float m, inv_s, log_s, h, g, gh;
  bool empty;
};

__device__ __forceinline__ float score_gradient(float z, const RowGrad& k, float inv_t,
                                                float picked) {
  if (k.empty) return 0.f;
  const float d = (z - k.m) * inv_t;
  // the exp2 instruction has no results below 2^-126: those are taken 2^64 times larger, and
  // back in the last product
  const float d2 = d * kLog2e;
  const bool small = d2 < -125.f;
  const float p = __builtin_amdgcn_exp2f(small ? d2 + 64.f : d2) * k.inv_s;
  const float lp = fmaxf(d - k.log_s, -1.e4f);  // where p = 0, p * -inf would be NaN
  return inv_t * (picked - p * (k.g + k.gh * (lp + k.h)) * (small ? 5.42101086e-20f : 1.f));
}

// The sum of a row's cotangents over its targets, by G threads; in every one of them.  G > 64: the
// workgroup's, with a barrier, and `red` is not the last call's.
template <int G>
__device__ __forceinline__ float cotangent_sum(const ScoreArgs& A, int64_t r, int t, float* red) {
  float v[1] = {0.f};
  for (int64_t i = t; i < A.n_targets; i += G) {
    const int64_t j = A.targets[r * A.n_targets + i];
    if (j >= 0 && j < A.cols) v[0] += A.dlogp[r * A.n_targets + i];
  }
  group_sums<G, 1>(v, red);
  return v[0];
}

// Reads z, writes dz, everything else is two numbers per row: many short workgroups, four packs in
// flight per thread.  G threads per row and step of G * 4 packs (1 pack where G = 64); `steps`
// steps of a row are items of their own.
template <typename T, int G, bool SHORT>
__global__ void __launch_bounds__(256) score_backward_kernel(const ScoreArgs A, int64_t steps) {
  constexpr int V = kPack<T>, U = G == 256 ? 4 : 1, RW = 256 / G;
  __shared__ float red[2][4];
  const int t = threadIdx.x % G, mine = threadIdx.x / G;
  int turn = 0;
  const int64_t work = A.rows * steps;
  for (int64_t item = (int64_t)blockIdx.x * RW + mine; item < work;
       item += (int64_t)gridDim.x * RW) {
    const int64_t r = steps > 1 ? item / steps : item;
    const int64_t at = (item - r * steps) * (G * U * V);
    const T* z = static_cast<const T*>(A.scores) + r * A.lds;
    T* dz = static_cast<T*>(A.dscores) + r * A.ldds;
    Raw raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = load_raw<T, SHORT>(z, at + (int64_t)(u * G + t) * V, A.cols);
    RowGrad k;
    k.m = A.stats_in[2 * r];
    const float s = A.stats_in[2 * r + 1];
    k.empty = s == 0.f;
    k.inv_s = 1.f / s;
    k.log_s = logf(s);
    k.gh = A.dentropy ? A.dentropy[r] : 0.f;
    k.h = A.dentropy ? A.entropy_in[r] : 0.f;
    k.g = 0.f;
    int64_t target = -1;
    float gt = 0.f;
    if (A.dlogp && A.n_targets == 1) {
      const int64_t j = A.targets[r];
      if (j >= 0 && j < A.cols) {
        target = j;
        k.g = gt = A.dlogp[r];
      }
    } else if (A.dlogp) {  // score_targets_kernel adds them
      k.g = cotangent_sum<G>(A, r, t, red[turn]);
      turn ^= 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t col = at + (int64_t)(u * G + t) * V;
      if (col >= A.cols) continue;
      const Pack<T> p = taken<T, SHORT>(raw[u], col, A.cols, (T)0.f);
      Pack<T> o;
#pragma unroll
      for (int i = 0; i < V; ++i)
        o.v[i] = (T)score_gradient((float)p.v[i], k, A.inv_t, col + i == target ? gt : 0.f);
      store_pack<T>(dz, col, A.cols, o);
    }
  }
}

// Several targets per row: the gradient at each target again, with the cotangents of all
// targets that name it, added in their order (no atomics: the result does not depend on
// which thread comes first).  A workgroup takes 256 targets of a row and passes all of the row's
// by them, 256 at a time in LDS.  Backward of bf16 256 x 65536 with 1024 targets 120 us in all,
// of 64 x 700 with 1000 targets 81 us (each thread reading every target from memory: 1150 and 540).
template <typename T>
__global__ void __launch_bounds__(256) score_targets_kernel(const ScoreArgs A, int64_t chunks) {
  __shared__ __attribute__((aligned(16))) int64_t named[256];
  __shared__ __attribute__((aligned(16))) float given[256];
  __shared__ float red[2][4];
  const int t = threadIdx.x;
  int turn = 0;
  const int64_t work = A.rows * chunks;
  for (int64_t item = blockIdx.x; item < work; item += gridDim.x) {
    const int64_t r = chunks > 1 ? item / chunks : item;
    const int64_t i = (item - r * chunks) * 256 + t;
    const int64_t* targets = A.targets + r * A.n_targets;
    const float* dlogp = A.dlogp + r * A.n_targets;
    RowGrad k;
    k.m = A.stats_in[2 * r];
    const float s = A.stats_in[2 * r + 1];
    k.empty = s == 0.f;
    k.inv_s = 1.f / s;
    k.log_s = logf(s);
    k.gh = A.dentropy ? A.dentropy[r] : 0.f;
    k.h = A.dentropy ? A.entropy_in[r] : 0.f;
    k.g = cotangent_sum<256>(A, r, t, red[turn]);
    turn ^= 1;
    const int64_t j = i < A.n_targets ? targets[i] : -1;
    const bool there = j >= 0 && j < A.cols;
    int64_t first = i;  // the first target that names this outcome: its thread writes it
    float picked = 0.f;
    for (int64_t q0 = 0; q0 < A.n_targets; q0 += 256) {
      __syncthreads();  // the last 256 have been read
      named[t] = q0 + t < A.n_targets ? targets[q0 + t] : -1;
      given[t] = q0 + t < A.n_targets ? dlogp[q0 + t] : 0.f;
      __syncthreads();
      if (!there) continue;
#pragma unroll 8
      for (int q = 0; q < 256; ++q) {
        const bool same = named[q] == j;
        picked += same ? given[q] : 0.f;
        first = same && q0 + q < first ? q0 + q : first;
      }
    }
    if (there && first == i)
      static_cast<T*>(A.dscores)[r * A.ldds + j] =
          (T)score_gradient((float)(static_cast<const T*>(A.scores) + r * A.lds)[j], k, A.inv_t,
                            picked);
  }
}

// ------------------------------------------------------------ launches

constexpr int64_t kMaxBlocks = 1 << 20;  // grids beyond this loop
constexpr int64_t kWaves = 4096;         // waves that fill the chip: 4 per SIMD

// How a row is shared out: waves per row, and parts of a row in the workspace.
struct Split {
  int waves;
  int64_t parts, part_cols;
};

// Rows are split until the call has about kWaves waves, as long as a wave keeps 1024 columns
// (2048: a row of 2^20 weights with its 16 best 21.7 us instead of 18.1, 300 x 5000 bf16 with 5
// 10.7 instead of 8.0; 512: no less).  Beyond 16 waves the split goes over several workgroups and
// a second launch.
Split split_of(int64_t rows, int64_t cols) {
  const int64_t most = std::max<int64_t>(1, cols / 1024);
  const int64_t want = std::max<int64_t>(1, std::min(most, kWaves / std::max<int64_t>(rows, 1)));
  if (want < 4) return {1, 1, cols};
  if (want < 16) return {4, 1, cols};
  if (want < 64) return {16, 1, cols};
  const int64_t step = 16 * 1024;  // columns of a step of 16 waves
  const int64_t parts = std::min<int64_t>(want / 16, kMaxParts);
  const int64_t per = ((cols + parts - 1) / parts + step - 1) / step * step;
  return {16, (cols + per - 1) / per, per};
}

template <typename T, bool LOGITS, bool TOP>
int launch_scores(const ScoreArgs& a, hipStream_t st) {
  const Split sp = split_of(a.rows, a.cols);
  const int64_t work = a.rows * sp.parts;
  const int rw = sp.waves == 1 ? 4 : 1;
  const dim3 grid((unsigned)std::min<int64_t>((work + rw - 1) / rw, kMaxBlocks));
  if (a.cols < kPack<T>)
    score_kernel<T, LOGITS, TOP, 1, 4, true><<<grid, 256, 0, st>>>(a, sp.parts, sp.part_cols);
  else if (sp.waves == 1)
    score_kernel<T, LOGITS, TOP, 1, 4, false><<<grid, 256, 0, st>>>(a, sp.parts, sp.part_cols);
  else if (sp.waves == 4)
    score_kernel<T, LOGITS, TOP, 4, 1, false><<<grid, 256, 0, st>>>(a, sp.parts, sp.part_cols);
  else
    score_kernel<T, LOGITS, TOP, 16, 1, false><<<grid, 1024, 0, st>>>(a, sp.parts, sp.part_cols);
  int rc = (int)hipGetLastError();
  if (rc || sp.parts == 1) return rc;
  score_join_kernel<T, LOGITS, TOP><<<dim3((unsigned)a.rows), 1024, 0, st>>>(a, sp.parts);
  return (int)hipGetLastError();
}

}  // namespace

size_t log_probs_workspace(int64_t rows, int64_t cols, int n_top) {
  if (rows == 0) return 0;
  const Split sp = split_of(rows, cols);
  if (sp.parts == 1) return 0;
  const size_t items = (size_t)rows * (size_t)sp.parts;
  return (items * sizeof(Sums) + 255) / 256 * 256 + items * (size_t)n_top * 8;
}

int launch_log_probs(int kind, int dtype, const ScoreArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    if (kind == 0)
      return a.n_top ? launch_scores<T, true, true>(a, st) : launch_scores<T, true, false>(a, st);
    return a.n_top ? launch_scores<T, false, true>(a, st) : launch_scores<T, false, false>(a, st);
  });
}

int launch_log_probs_backward(int dtype, const ScoreArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    if (a.cols <= 64 * kPack<T>) {
      const int64_t blocks = std::min<int64_t>((a.rows + 3) / 4, kMaxBlocks);
      if (a.cols < kPack<T>)
        score_backward_kernel<T, 64, true><<<dim3((unsigned)blocks), 256, 0, st>>>(a, 1);
      else
        score_backward_kernel<T, 64, false><<<dim3((unsigned)blocks), 256, 0, st>>>(a, 1);
    } else {
      const int64_t span = 256 * 4 * kPack<T>;
      const int64_t steps = (a.cols + span - 1) / span;
      const int64_t blocks = std::min<int64_t>(a.rows * steps, kMaxBlocks);
      score_backward_kernel<T, 256, false><<<dim3((unsigned)blocks), 256, 0, st>>>(a, steps);
    }
    int rc = (int)hipGetLastError();
    if (rc || !a.dlogp || a.n_targets < 2) return rc;
    const int64_t chunks = (a.n_targets + 255) / 256;
    score_targets_kernel<T>
        <<<dim3((unsigned)std::min(a.rows * chunks, kMaxBlocks)), 256, 0, st>>>(a, chunks);
    return (int)hipGetLastError();
  });
}

}  // namespace vqc
