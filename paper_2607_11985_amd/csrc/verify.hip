// verify.hip -- drafted outcomes verified against the target's probabilities, and the outcome drawn
// where they end.
//
//   p_i, q_i: the target's and the draft's probabilities of the i-th outcome of a sequence
//   draft d_i stands while u_i q_i(d_i) < p_i(d_i); where the first one does not, the outcome is
//   drawn from max(p_i - q_i, 0), behind the last one from p: the first j at which the sum of the
//   weights up to j passes u_K times their whole sum
//
// Everything is 64-bit, exponentials too: an outcome is a whole number, and a border of the running
// sum that is off by e turns one draw in 1 / e into its neighbour, at each of a row's borders.
//
// Two launches.  total_kernel: (m, sum e^(z - m)) of every row, in parts.  draw_kernel: each
// workgroup finds where its sequence's drafts end and sums the weights over its piece of that one
// row; the last of a sequence's to come finds the piece and the outcome in it.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layers.h"
#include "layers_device.h"

namespace vqc {
namespace {

constexpr int kMostParts = 64;  // of a row
constexpr int kThreads = 256;

// A row's weights as they add up: e^(z - m) of logits, w of weights (m is not used).
struct Total {
  double s;
  float m;
};

template <int N>
__device__ __forceinline__ double lane_xor_double(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, ((uint64_t)lane_xor<N>((uint32_t)(u >> 32)) << 32) |
                                        lane_xor<N>((uint32_t)u));
}
__device__ __forceinline__ double wave_sum(double x) {
  x += lane_xor_double<1>(x);
  x += lane_xor_double<2>(x);
  x += lane_xor_double<4>(x);
  x += lane_xor_double<8>(x);
  x += lane_xor_double<16>(x);
  return x + lane_xor_double<32>(x);
}
// NaN if any is.
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}
__device__ __forceinline__ float wave_largest(float x) {
  x = larger(x, lane_xor<1>(x));
  x = larger(x, lane_xor<2>(x));
  x = larger(x, lane_xor<4>(x));
  x = larger(x, lane_xor<8>(x));
  x = larger(x, lane_xor<16>(x));
  return larger(x, lane_xor<32>(x));
}

// 2^t for t <= 0, to 2 units in the last place; 0 from 2^-1075 down, also of -inf (and of NaN,
// which shows in m).  With n the nearest integer and f = (t - n) ln 2, |f| <= 0.347, e^f is its
// series up to f^12 / 12! (the next term is 2^-52 of it at most).
__device__ __forceinline__ double exp2_negative(double t) {
  t = fmax(t, -1100.);
  const double n = rint(t), f = (t - n) * 0x1.62e42fefa39efp-1;
  double p = 1. / 479001600.;
  p = fma(p, f, 1. / 39916800.);
  p = fma(p, f, 1. / 3628800.);
  p = fma(p, f, 1. / 362880.);
  p = fma(p, f, 1. / 40320.);
  p = fma(p, f, 1. / 5040.);
  p = fma(p, f, 1. / 720.);
  p = fma(p, f, 1. / 120.);
  p = fma(p, f, 1. / 24.);
  p = fma(p, f, 1. / 6.);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.);
  p = fma(p, f, 1.);
  return ldexp(p, (int)n);
}

// A score's weight relative to its row's largest; c = log2 e / T.  The difference is taken first,
// where it is exact: masks of the type's lowest value would lose everything else in a product.
template <bool LOGITS>
__device__ __forceinline__ double weight_of(float z, double m, double c) {
  if constexpr (LOGITS) return exp2_negative(((double)z - m) * c);
  return (double)z;
}
// (what m = -inf, a row with nothing left, is subtracted as)
__device__ __forceinline__ double reference(float m) { return m == -INFINITY ? 0. : (double)m; }

template <bool LOGITS>
__device__ __forceinline__ Total join(const Total& a, const Total& b, double c) {
  if constexpr (!LOGITS) return {a.s + b.s, 0.f};
  const float m = larger(a.m, b.m);
  const double r = reference(m);
  return {a.s * exp2_negative(((double)a.m - r) * c) + b.s * exp2_negative(((double)b.m - r) * c),
          m};
}
// The total of a row's parts, in the same order everywhere; all lanes of a wave.
template <bool LOGITS>
__device__ __forceinline__ Total total_of(const Total* parts, int n, double c) {
  const int lane = threadIdx.x & 63;  // n <= 64
  const Total t = lane < n ? parts[lane] : Total{0., -INFINITY};
  if constexpr (!LOGITS) return {wave_sum(t.s), 0.f};
  const float m = wave_largest(t.m);
  return {wave_sum(t.s * exp2_negative(((double)t.m - reference(m)) * c)), m};
}
// Whether a row has anything to draw: not if nothing is left of it or its numbers are none.
template <bool LOGITS>
__device__ __forceinline__ bool has_outcomes(const Total& t) {
  return t.s > 0. && t.s < (double)INFINITY && (!LOGITS || t.m < INFINITY);
}

struct Rows {
  int64_t per_sequence;  // target rows, then draft rows
  int parts;
  int64_t part;          // elements of a part, a multiple of 16 bytes
};

template <typename T>
__device__ __forceinline__ const T* row_of(const VerifyArgs& A, int64_t sequence, int64_t row) {
  if (row <= A.drafts)
    return static_cast<const T*>(A.target) + (sequence * (A.drafts + 1) + row) * A.ldt;
  return static_cast<const T*>(A.draft) + (sequence * A.drafts + row - A.drafts - 1) * A.ldd;
}

template <typename T, bool LOGITS, bool SHORT>
__global__ void __launch_bounds__(kThreads)
    total_kernel(const VerifyArgs A, const Rows R, Total* totals, uint32_t* counters) {
  constexpr int V = kPack<T>, U = 4;
  __shared__ Total waves[kThreads / 64];
  const int64_t id = blockIdx.x / R.parts, part = blockIdx.x % R.parts;
  const int64_t sequence = id / R.per_sequence, row = id % R.per_sequence;
  if (row == 0 && part == 0 && threadIdx.x == 0) counters[sequence] = 0;
  const T* z = row_of<T>(A, sequence, row);
  const double c = A.scale;
  const int64_t end = (part + 1) * R.part < A.cols ? (part + 1) * R.part : A.cols;
  const T none = LOGITS ? (T)-INFINITY : (T)0.f;
  Total t{0., -INFINITY};
  for (int64_t first = part * R.part + (int64_t)threadIdx.x * V; first < end;
       first += U * kThreads * V) {
    Raw raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = load_raw<T, SHORT>(z, first + u * kThreads * V, A.cols);
    Pack<T> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = first + u * kThreads * V;
      // (a part's end is that of a pack or of the row)
      p[u] = taken<T, SHORT>(raw[u], at, at < end ? A.cols : at, none);
    }
    if constexpr (LOGITS) {
      float top = (float)p[0].v[0];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) top = larger(top, (float)p[u].v[i]);
      if (!(top <= t.m)) {
        const float m = larger(top, t.m);
        t.s *= exp2_negative(((double)t.m - reference(m)) * c);
        t.m = m;
      }
    }
    const double m = reference(t.m);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < V; ++i) t.s += weight_of<LOGITS>((float)p[u].v[i], m, c);
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if constexpr (LOGITS) {
    const float m = wave_largest(t.m);
    t.s = wave_sum(t.s * exp2_negative(((double)t.m - reference(m)) * c));
    t.m = m;
  } else {
    t.s = wave_sum(t.s);
  }
  if (lane == 0) waves[wave] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    Total sum = waves[0];
    for (int w = 1; w < kThreads / 64; ++w) sum = join<LOGITS>(sum, waves[w], c);
    totals[id * R.parts + part] = sum;
  }
}

// What is drawn from, once it is known where a sequence's drafts end.
template <typename T>
struct Source {
  const T *p, *q;    // q: null where nothing is taken off
  double mp, mq;     // the rows' references
  double ip, iq;     // 1 / their totals
  int64_t without;   // an outcome that cannot come (-1: none)
};

// (weight that is drawn by, the target's own) of a pair of scores in column j.
template <typename T, bool LOGITS>
__device__ __forceinline__ void weights_at(const Source<T>& S, double c, float zp, float zq,
                                           int64_t j, double& rest, double& own) {
  own = weight_of<LOGITS>(zp, S.mp, c) * S.ip;
  rest = own;
  if (S.q) rest = fmax(own - weight_of<LOGITS>(zq, S.mq, c) * S.iq, 0.);
  if (j == S.without) rest = 0.;
}

__device__ __forceinline__ double load_shared(const double* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_shared(double* p, double v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// pieces: [sequences][R.parts][2], the sums of the two weights.
template <typename T, bool LOGITS, bool SHORT>
__global__ void __launch_bounds__(kThreads)
    draw_kernel(const VerifyArgs A, const Rows R, const Total* totals, double* pieces,
                uint32_t* counters) {
  constexpr int V = kPack<T>, W = kThreads / 64;
  __shared__ unsigned long long first_end;
  __shared__ double sums[2][W], before[kThreads];
  __shared__ int last;
  const int64_t sequence = blockIdx.x / R.parts;
  const int piece = (int)(blockIdx.x % R.parts);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double c = A.scale;
  const int64_t K = A.drafts;
  const int64_t* drafted = A.drafted + sequence * K;
  const double* u = A.uniforms + sequence * (K + 1);
  const Total* mine = totals + sequence * R.per_sequence * R.parts;

  // where the drafts end: a wave looks at every W-th draft
  if (threadIdx.x == 0) first_end = (unsigned long long)K;
  __syncthreads();
  for (int64_t i = wave; i < K; i += W) {
    const int64_t d = drafted[i];
    bool stands = d >= 0 && d < A.cols;
    if (stands) {
      const Total P = total_of<LOGITS>(mine + i * R.parts, R.parts, c);
      const double p = weight_of<LOGITS>((float)row_of<T>(A, sequence, i)[d], reference(P.m), c);
      double q = 1.;
      bool known = true;
      if (A.draft) {
        const Total Q = total_of<LOGITS>(mine + (K + 1 + i) * R.parts, R.parts, c);
        known = has_outcomes<LOGITS>(Q);
        q = weight_of<LOGITS>((float)row_of<T>(A, sequence, K + 1 + i)[d], reference(Q.m), c) *
            (1. / Q.s);
      }
      stands = known && has_outcomes<LOGITS>(P) && u[i] * q < p * (1. / P.s);
    }
    if (!stands && lane == 0) atomicMin(&first_end, (unsigned long long)i);
  }
  __syncthreads();
  const int64_t n = (int64_t)first_end;

  // the row and what is taken off it
  const Total P = total_of<LOGITS>(mine + n * R.parts, R.parts, c);
  Source<T> S{row_of<T>(A, sequence, n), nullptr, reference(P.m), 0., 1. / P.s, 0., -1};
  if (n < K && drafted[n] >= 0 && drafted[n] < A.cols) {
    if (A.draft) {
      const Total Q = total_of<LOGITS>(mine + (K + 1 + n) * R.parts, R.parts, c);
      if (has_outcomes<LOGITS>(Q)) {  // otherwise the draft's probabilities are none
        S.q = row_of<T>(A, sequence, K + 1 + n);
        S.mq = reference(Q.m);
        S.iq = 1. / Q.s;
      }
    } else {
      S.without = drafted[n];
    }
  }
  const T none = LOGITS ? (T)-INFINITY : (T)0.f;
  const int64_t begin = piece * R.part;
  const int64_t end = begin + R.part < A.cols ? begin + R.part : A.cols;
  double rest = 0., own = 0.;
  for (int64_t at = begin + (int64_t)threadIdx.x * V; at < end; at += kThreads * V) {
    const Pack<T> zp = taken<T, SHORT>(load_raw<T, SHORT>(S.p, at, A.cols), at, A.cols, none);
    Pack<T> zq = zp;
    if (S.q) zq = taken<T, SHORT>(load_raw<T, SHORT>(S.q, at, A.cols), at, A.cols, none);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      double r, o;
      weights_at<T, LOGITS>(S, c, (float)zp.v[i], (float)zq.v[i], at + i, r, o);
      rest += r;
      own += o;
    }
  }
  rest = wave_sum(rest);
  own = wave_sum(own);
  if (lane == 0) {
    sums[0][wave] = rest;
    sums[1][wave] = own;
  }
  __syncthreads();
  double* shared = pieces + sequence * R.parts * 2;
  if (threadIdx.x == 0) {
    double a = sums[0][0], b = sums[1][0];
    for (int w = 1; w < W; ++w) {
      a += sums[0][w];
      b += sums[1][w];
    }
    store_shared(shared + 2 * piece, a);
    store_shared(shared + 2 * piece + 1, b);
    const uint32_t came = __hip_atomic_fetch_add(counters + sequence, 1u, __ATOMIC_ACQ_REL,
                                                 __HIP_MEMORY_SCOPE_AGENT);
    last = came + 1 == (uint32_t)R.parts;
  }
  __syncthreads();
  if (!last) return;

  // every piece is there: the drafts that stand, then the outcome
  int64_t* outcomes = A.outcomes + sequence * (K + 1);
  for (int64_t i = threadIdx.x; i <= K; i += kThreads)
    if (i != n) outcomes[i] = i < n ? drafted[i] : -1;
  if (threadIdx.x == 0) A.accepted[sequence] = n;
  if (!has_outcomes<LOGITS>(P)) {
    if (threadIdx.x == 0) outcomes[n] = -1;
    return;
  }
  // (all threads alike) the pieces' sums, the target's own where nothing is left of the difference
  const int l = lane < R.parts ? lane : 0;
  double a = load_shared(shared + 2 * l), b = load_shared(shared + 2 * l + 1);
  if (lane >= R.parts) a = b = 0.;
  const double all_rest = wave_sum(a);
  const bool plain = !(all_rest > 0.);
  if (plain) {
    S.q = nullptr;
    S.without = -1;
    a = b;
  }
  const double x = u[K] * (plain ? wave_sum(b) : all_rest);
  // the piece at which the running sum passes x, else the last one with any weight
  double passed = 0., sum = 0.;
  int found = 0;
  bool over = false;
  for (int k = 0; k < R.parts; ++k) {
    const double v = __shfl(a, k);
    if (over || !(v > 0.)) continue;
    found = k;
    passed = sum;
    sum += v;
    over = sum > x;
  }
  // its columns, a run of them per thread
  const int64_t from = found * R.part;
  const int64_t to = from + R.part < A.cols ? from + R.part : A.cols;
  const int64_t packs = (to - from + V - 1) / V, each = (packs + kThreads - 1) / kThreads;
  const int64_t at0 = from + threadIdx.x * each * V;
  const int64_t at1 = at0 + each * V < to ? at0 + each * V : to;
  auto walk = [&](auto f) {
    for (int64_t at = at0; at < at1; at += V) {
      const Pack<T> zp = taken<T, SHORT>(load_raw<T, SHORT>(S.p, at, A.cols), at, A.cols, none);
      Pack<T> zq = zp;
      if (S.q) zq = taken<T, SHORT>(load_raw<T, SHORT>(S.q, at, A.cols), at, A.cols, none);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        double r, o;
        weights_at<T, LOGITS>(S, c, (float)zp.v[i], (float)zq.v[i], at + i, r, o);
        f(at + i, r);
      }
    }
  };
  double run = 0.;
  walk([&](int64_t, double w) { run += w; });
  before[threadIdx.x] = run;
  __syncthreads();
  // the thread in whose run the sum passes x, else the last one with any weight
  double start = passed, mine_from = passed;
  int owner = 0;
  over = false;
  for (int t = 0; t < kThreads; ++t) {
    const double v = before[t];
    if (over || !(v > 0.)) continue;
    owner = t;
    mine_from = start;
    start += v;
    over = start > x;
  }
  if ((int)threadIdx.x != owner) return;
  double at_sum = mine_from;
  int64_t best = -1;
  bool done = false;
  walk([&](int64_t j, double w) {
    if (done || !(w > 0.)) return;
    best = j;
    at_sum += w;
    done = at_sum > x;
  });
  outcomes[n] = best;
}

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// Parts of a row: as many as fill the chip, of 2048 elements at least.
Rows rows_of(int64_t sequences, int64_t drafts, int64_t cols, bool has_draft, int pack) {
  Rows R{};
  R.per_sequence = has_draft ? 2 * drafts + 1 : drafts + 1;
  const int64_t rows = sequences * R.per_sequence;
  int64_t parts = (4 * 256 + rows - 1) / std::max<int64_t>(rows, 1);
  parts = std::min({parts, (cols + 2047) / 2048, (int64_t)kMostParts});
  R.part = (cols + parts - 1) / parts;
  R.part = (R.part + pack - 1) / pack * pack;
  R.parts = (int)((cols + R.part - 1) / R.part);
  return R;
}

struct Layout {
  size_t pieces, counters, end;
};
Layout layout_of(int64_t sequences, const Rows& R) {
  Layout L;
  L.pieces = round256((size_t)sequences * (size_t)R.per_sequence * (size_t)R.parts * sizeof(Total));
  L.counters = L.pieces + round256((size_t)sequences * (size_t)R.parts * 16);
  L.end = L.counters + round256((size_t)sequences * 4);
  return L;
}

}  // namespace

size_t verify_workspace(int dtype, int64_t sequences, int64_t drafts, int64_t cols,
                        bool has_draft) {
  return layout_of(sequences,
                   rows_of(sequences, drafts, cols, has_draft, 16 / (int)element_bytes(dtype)))
      .end;
}

int launch_verify(int kind, int dtype, const VerifyArgs& args, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  VerifyArgs a = args;
  a.scale = std::fmin(a.scale * 1.4426950408889634, 1.7976931348623157e308);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    const Rows R = rows_of(a.sequences, a.drafts, a.cols, a.draft != nullptr, kPack<T>);
    const Layout L = layout_of(a.sequences, R);
    Total* totals = reinterpret_cast<Total*>(a.ws);
    double* pieces = reinterpret_cast<double*>(a.ws + L.pieces);
    uint32_t* counters = reinterpret_cast<uint32_t*>(a.ws + L.counters);
    const int64_t rows = a.sequences * R.per_sequence;
    if (rows > INT32_MAX / 256 / R.parts) return (int)hipErrorInvalidConfiguration;
    auto launch = [&](auto logits, auto is_short) {
      constexpr bool LOGITS = decltype(logits)::value, SHORT = decltype(is_short)::value;
      total_kernel<T, LOGITS, SHORT>
          <<<dim3((unsigned)(rows * R.parts)), kThreads, 0, st>>>(a, R, totals, counters);
      if (int rc = (int)hipGetLastError()) return rc;
      draw_kernel<T, LOGITS, SHORT>
          <<<dim3((unsigned)(a.sequences * R.parts)), kThreads, 0, st>>>(a, R, totals, pieces,
                                                                        counters);
      return (int)hipGetLastError();
    };
    using std::false_type;
    using std::true_type;
    if (kind == 0)
      return a.cols < kPack<T> ? launch(true_type{}, true_type{})
                               : launch(true_type{}, false_type{});
    return a.cols < kPack<T> ? launch(false_type{}, true_type{})
                             : launch(false_type{}, false_type{});
  });
}

}  // namespace vqc
