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
// Short rows: one workgroup per sequence does it all.  Otherwise total_kernel sums every row, in
// parts.  Of many scores or drafts, behind a kernel that clears the counters, the last of a draft's
// parts to come says whether the draft stands, and rows behind one that does not are passed over
// from then on; otherwise draw_kernel does, in each of its workgroups.  It sums the weights of the
// one row that a sequence's outcome is drawn from, in units of a wave; the last workgroup to come
// finds the unit and the outcome in it.
//
// Totals of logits are bound by 64-bit instructions (bf16 64 x 7 drafts of 128000: 59 us for the 144 of
// 246 MB that are read; memory would take 21), of weights by memory (32 x 4 of 65536: 14 us, 5.4
// TB/s); the draw (27 and 13 us) by both and by a chain of dependent loads.  1 x 3 of 1024: 5 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layers.h"
#include "layers_device.h"
#include "verify_plan.h"

namespace vqc {
namespace {

constexpr int kThreads = kVerifyThreads;

// ------------------------------------------------------------ 64-bit exponentials

// e^f by its series up to f^12 / 12! for |f| <= 0.347 (the next term is 2^-52 of it at most).
__device__ __forceinline__ double exp_near_zero(double f) {
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
  return fma(p, f, 1.);
}
constexpr double kLn2 = 0x1.62e42fefa39efp-1;

// 2^t for t <= 0; 0 from 2^-1075 down, also of -inf (and of NaN, which shows elsewhere).
__device__ __forceinline__ double exp2_negative(double t) {
  t = fmax(t, -1100.);
  const double n = rint(t);
  return ldexp(exp_near_zero((t - n) * kLn2), (int)n);
}

// For many of them: 2^(k / 512) from a table in LDS, and the series up to f^3 of what is left, |f|
// <= ln 2 / 1024 (the next term is 9e-15).  14 instructions a score, where the series alone takes
// 23.  The high word of an entry lacks its number's share of k << 11, so that one shift and add put
// the exponent of 2^(k / 512) in place.
constexpr int kTable = 512;
__device__ __forceinline__ void fill_table(double* table, int threads) {
  for (int i = threadIdx.x; i < kTable / 2; i += threads) {
    const double low = 2. * exp2_negative((double)(i - kTable) / kTable);
    const double of[2] = {low, low * 0x1.6a09e667f3bcdp+0};  // (the square root of 2)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      table[i + h * (kTable / 2)] = __builtin_bit_cast(
          double, __builtin_bit_cast(uint64_t, of[h]) -
                      ((uint64_t)(uint32_t)((i + h * (kTable / 2)) << 11) << 32));
  }
}

// How a row's scores become weights: e^((z - m) / T) of logits, the weights themselves.
struct Scale {
  double c;     // kTable log2 e / T
  double least; // differences z - m from which on nothing is left (2^-1020)
  const double* table;
  double k1, k2;  // coefficients of the series, in vector registers (see ready)
};

// e^(d / T) as t u, u near 1.  The difference d of a score and its row's largest is taken first,
// where it is exact: masks of the type's lowest value would lose everything else in a product.
struct Split {
  double t, u;
};
constexpr double kOne = kLn2 / kTable;
// An instruction takes one constant from the scalar registers; two of them, and the compiler moves
// one for every score.  (All threads, behind fill_table.)
__device__ __forceinline__ void ready(Scale& S, const double* table) {
  S.table = table;
  S.k1 = kOne;
  S.k2 = kOne * kOne / 2;
  asm("" : "+v"(S.k1), "+v"(S.k2));
}
__device__ __forceinline__ Split split_exp(double d, const Scale& S) {
  constexpr double kMagic = 0x1.8p52;  // the sum's last place is 1
  constexpr double k3 = kOne * kOne * kOne / 6;
  static_assert(kTable == 1 << 9, "the exponent's place is 20 bits above the word's last");
  d = fmax(d, S.least);
  const double g = fma(d, S.c, kMagic);
  const double f = fma(d, S.c, kMagic - g);
  const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, g);
  typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
  uintx2 t = *reinterpret_cast<const uintx2*>(S.table + (k & (kTable - 1)));
  uint32_t high = t.y;
  // (written out: as a sum it becomes one of 64 bits with its parts moved there and back)
  asm("v_lshl_add_u32 %0, %1, 11, %0" : "+v"(high) : "v"(k));
  t.y = high;
  return {__builtin_bit_cast(double, t), fma(fma(fma(f, k3, S.k2), f, S.k1), f, 1.)};
}

// (Where nothing is left, of -inf too, it is near 2^-1020: kNothing tells it from a weight.  What is
// less than that of its row's largest counts as nothing.)
constexpr double kNothing = 0x1p-900;
template <bool LOGITS>
__device__ __forceinline__ double weight_of(float z, double m, const Scale& S) {
  if constexpr (!LOGITS) return (double)z;
  const Split e = split_exp((double)z - m, S);
  return e.t * e.u;
}

// ------------------------------------------------------------ sums over lanes

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
// The sum of a lane's and all lower ones.
__device__ __forceinline__ double wave_running(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int n = 1; n < 64; n *= 2) {
    const double below = __shfl_up(x, n);
    if (lane >= n) x += below;
  }
  return x;
}
__device__ __forceinline__ float wave_largest(float x) {
  x = larger(x, lane_xor<1>(x));
  x = larger(x, lane_xor<2>(x));
  x = larger(x, lane_xor<4>(x));
  x = larger(x, lane_xor<8>(x));
  x = larger(x, lane_xor<16>(x));
  return larger(x, lane_xor<32>(x));
}

// ------------------------------------------------------------ totals of rows

// The sum of a row's weights; of logits relative to the largest, m.
struct Total {
  double s;
  float m;
};

// (what m = -inf, a row with nothing left, is subtracted as)
__device__ __forceinline__ double reference(float m) { return m == -INFINITY ? 0. : (double)m; }

// The sums of the lanes of a wave as one.
template <bool LOGITS>
__device__ __forceinline__ Total wave_total(const Total& t, const Scale& S) {
  if constexpr (!LOGITS) return {wave_sum(t.s), 0.f};
  const float m = wave_largest(t.m);
  return {wave_sum(t.s * weight_of<true>(t.m, reference(m), S)), m};
}
// Whether a row has anything to draw: not if nothing is left of it or its numbers are none.
template <bool LOGITS>
__device__ __forceinline__ bool has_outcomes(const Total& t) {
  if constexpr (LOGITS) return t.m > -INFINITY && t.m < INFINITY;
  return t.s > 0. && t.s < (double)INFINITY;
}

// A thread's scores of columns [begin, end), every `threads`-th pack from the first one on; begin
// and end are those of packs, or end the row's.
template <typename T, bool LOGITS, bool SHORT, int U>
__device__ __forceinline__ Total thread_total(const T* z, int64_t cols, int64_t begin, int64_t end,
                                              int thread, int threads, const Scale& S) {
  constexpr int V = kPack<T>;
  const T none = LOGITS ? (T)-INFINITY : (T)0.f;
  double s = 0.;
  float m = -INFINITY;
  for (int64_t first = begin + (int64_t)thread * V; first < end;
       first += (int64_t)U * threads * V) {
    Raw raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = load_raw<T, SHORT>(z, first + (int64_t)u * threads * V, cols);
    float v[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = first + (int64_t)u * threads * V;
      const Pack<T> p = taken<T, SHORT>(raw[u], at, at < end ? cols : at, none);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[u][i] = (float)p.v[i];
        asm("" : "+v"(v[u][i]));  // (the maximum is to be one of fp32)
      }
    }
    if constexpr (LOGITS) {
      float top = v[0][0];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; i += 2) top = larger(larger(top, v[u][i]), v[u][i + 1]);
      if (!(top <= m)) {
        const float grown = larger(top, m);
        const double e = weight_of<true>(m, reference(grown), S);
        s *= e;
        m = grown;
      }
      const double ref = reference(m);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const Split e = split_exp((double)v[u][i] - ref, S);
          s = fma(e.t, e.u, s);
        }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) s += (double)v[u][i];
    }
  }
  return {s, m};
}

// ------------------------------------------------------------ the outcome

// What is drawn from, once it is known where a sequence's drafts end.
template <typename T>
struct Source {
  const T *p, *q;    // q: null where nothing is taken off
  double mp, mq;     // the rows' references
  double ratio;      // of their totals, p's over q's
  int64_t without;   // an outcome that cannot come (-1: none)
};

template <typename T, bool LOGITS>
__device__ __forceinline__ Source<T> source_of(const VerifyArgs& A, const T* p, const Total& P,
                                               const T* q, const Total& Q, int64_t d,
                                               bool drafted) {
  Source<T> s{p, nullptr, reference(P.m), 0., 0., -1};
  if (drafted && !A.draft) s.without = d;
  if (drafted && A.draft && has_outcomes<LOGITS>(Q)) {  // else the draft's probabilities are none
    s.q = q;
    s.mq = reference(Q.m);
    s.ratio = P.s / Q.s;
  }
  return s;
}

// The probability of the score z.
template <bool LOGITS>
__device__ __forceinline__ double share_of(float z, const Total& t, const Scale& S) {
  const double w = weight_of<LOGITS>(z, reference(t.m), S);
  return w > kNothing ? w * (1. / t.s) : 0.;
}

// Whether a draft stands that the target's and the draft's scores p and q are of.
template <bool LOGITS>
__device__ __forceinline__ bool stands(bool has_draft, float p, const Total& P, float q,
                                       const Total& Q, double u, const Scale& S) {
  if (!has_outcomes<LOGITS>(P)) return false;
  const double pd = share_of<LOGITS>(p, P, S);
  if (!has_draft) return u < pd;
  if (!has_outcomes<LOGITS>(Q)) return false;
  return u * share_of<LOGITS>(q, Q, S) < pd;
}

// The pack of scores at column `at`, of both rows, and its weights.
struct RawPair {
  Raw p, q;
};
template <typename T, bool SHORT>
__device__ __forceinline__ RawPair load_pair(const Source<T>& s, int64_t cols, int64_t at) {
  RawPair r;
  r.p = load_raw<T, SHORT>(s.p, at, cols);
  r.q = s.q ? load_raw<T, SHORT>(s.q, at, cols) : r.p;
  return r;
}
template <typename T, bool LOGITS, bool SHORT>
__device__ __forceinline__ void pack_weights(const Source<T>& s, const Scale& S, int64_t cols,
                                             int64_t at, const RawPair& raw,
                                             double (&w)[kPack<T>]) {
  constexpr int V = kPack<T>;
  const T none = LOGITS ? (T)-INFINITY : (T)0.f;
  const Pack<T> zp = taken<T, SHORT>(raw.p, at, cols, none);
#pragma unroll
  for (int i = 0; i < V; ++i) w[i] = weight_of<LOGITS>((float)zp.v[i], s.mp, S);
  if (s.q) {
    const Pack<T> zq = taken<T, SHORT>(raw.q, at, cols, none);
#pragma unroll
    for (int i = 0; i < V; ++i)
      w[i] = fmax(fma(-weight_of<LOGITS>((float)zq.v[i], s.mq, S), s.ratio, w[i]), 0.);
  } else if (at <= s.without && s.without < at + V) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at + i == s.without) w[i] = 0.;
  }
}

// Consecutive packs over the lanes of a wave: a lane's run is `each` of them.
struct Span {
  int64_t begin, end, each;
};
template <int V>
__device__ __forceinline__ Span span_of(int64_t begin, int64_t end) {
  return {begin, end, ((end - begin + V - 1) / V + 63) / 64};
}

// Sums that follow each other over the lanes: the first at which their running sum, from `passed`
// on, passes x, else the last that is anything.  passed becomes the sum before it.
__device__ __forceinline__ int lane_that_passes(double a, double x, double& passed) {
  const double running = passed + wave_running(a);
  const uint64_t any = __ballot(a > kNothing), over = __ballot(a > kNothing && running > x);
  const int found = over ? __ffsll((unsigned long long)over) - 1 : any ? 63 - __clzll(any) : 0;
  const double below = __shfl(running, found ? found - 1 : 0);
  passed = found ? below : passed;
  return found;
}

// The search for an outcome: a wave goes from a span to one lane's run of it, until the runs are
// single packs.  f(a lane's sum) is called with the first span's, and says whether the wave goes
// on, with these sums or with another span.  (One loop for all of it: instructions that a wave
// runs only once come from memory, and two copies of a pack's weights made 11 us of a search.)
enum class Next { kStop, kGoOn, kAgain };
template <typename T, bool LOGITS, bool SHORT, typename F>
__device__ __forceinline__ bool descend(const Source<T>& s, const Scale& S, int64_t cols,
                                        Span span, double& x, double& passed, int64_t& outcome,
                                        F&& f) {
  constexpr int V = kPack<T>;
  const int lane = threadIdx.x & 63;
  bool top = true;
  for (;;) {
    double w[V], sum = 0.;
    const int64_t begin = span.begin + lane * span.each * V;
    const int64_t end = begin + span.each * V < span.end ? begin + span.each * V : span.end;
    RawPair next{};
    if (begin < end) next = load_pair<T, SHORT>(s, cols, begin);
#pragma unroll 1
    for (int64_t at = begin; at < end; at += V) {
      const RawPair raw = next;
      if (at + V < end) next = load_pair<T, SHORT>(s, cols, at + V);
      pack_weights<T, LOGITS, SHORT>(s, S, cols, at, raw, w);
#pragma unroll
      for (int i = 0; i < V; ++i) sum += w[i];
    }
    if (top) {
      top = false;
      const Next next = f(sum, span, x, passed);
      if (next == Next::kStop) return false;
      if (next == Next::kAgain) continue;
    }
    const int found = lane_that_passes(sum, x, passed);
    if (span.each == 1) {
      double at = passed;
      bool done = false;
      int best = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const double v = __shfl(w[i], found);
        if (done || !(v > kNothing)) continue;
        best = i;
        at += v;
        done = at > x;
      }
      outcome = span.begin + found * V + best;
      return true;
    }
    const int64_t from = span.begin + found * span.each * V;
    span = span_of<V>(from, from + span.each * V < span.end ? from + span.each * V : span.end);
  }
}

// The accepted drafts and -1 behind the drawn outcome.
__device__ __forceinline__ void write_drafts(const VerifyArgs& A, int64_t sequence, int64_t n,
                                             int threads) {
  int64_t* outcomes = A.outcomes + sequence * (A.drafts + 1);
  for (int64_t i = threadIdx.x; i <= A.drafts; i += threads)
    if (i != n) outcomes[i] = i < n ? A.drafted[sequence * A.drafts + i] : -1;
  if (threadIdx.x == 0) A.accepted[sequence] = n;
}

template <typename T>
__device__ __forceinline__ const T* target_row(const VerifyArgs& A, int64_t sequence, int64_t i) {
  return static_cast<const T*>(A.target) + (sequence * (A.drafts + 1) + i) * A.ldt;
}
template <typename T>
__device__ __forceinline__ const T* draft_row(const VerifyArgs& A, int64_t sequence, int64_t i) {
  return static_cast<const T*>(A.draft) + (sequence * A.drafts + i) * A.ldd;
}
__device__ __forceinline__ int64_t drafted_at(const VerifyArgs& A, int64_t sequence, int64_t i) {
  return A.drafted[sequence * A.drafts + i];
}
__device__ __forceinline__ bool is_outcome(const VerifyArgs& A, int64_t d) {
  return d >= 0 && d < A.cols;
}

// ------------------------------------------------------------ short rows

// One workgroup per sequence: its waves share out the rows, then all take the one row.
constexpr int kSmallThreads = 512;
template <typename T, bool LOGITS, bool SHORT>
__global__ void __launch_bounds__(kSmallThreads) small_kernel(const VerifyArgs A, Scale S) {
  constexpr int V = kPack<T>, W = kSmallThreads / 64;
  __shared__ double table[LOGITS ? kTable : 1];
  __shared__ Total parts[kSmallRows][W];
  __shared__ double sums[W];
  __shared__ int first_end;
  const int64_t sequence = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = (int)A.drafts, rows = A.draft ? 2 * K + 1 : K + 1;
  ready(S, table);
  if constexpr (LOGITS) fill_table(table, kSmallThreads);
  if (threadIdx.x == 0) first_end = K;
  __syncthreads();
  // what the drafts' tests need, on its way while the rows are summed
  const int mine = (int)threadIdx.x;
  const int64_t dm = mine < K ? drafted_at(A, sequence, mine) : -1;
  const bool tests = mine < K && is_outcome(A, dm);
  const double um = tests ? A.uniforms[sequence * (K + 1) + mine] : 0.;
  const double ulast = A.uniforms[sequence * (K + 1) + K];
  const T pm = tests ? target_row<T>(A, sequence, mine)[dm] : (T)0.f;
  const T qm = tests && A.draft ? draft_row<T>(A, sequence, mine)[dm] : (T)0.f;
  // G waves for a row: a power of two
  int G = W;
  while (G > 1 && G * rows > W) G /= 2;
  for (int row = wave / G; row < rows; row += W / G) {
    const T* z = row <= K ? target_row<T>(A, sequence, row)
                          : draft_row<T>(A, sequence, row - K - 1);
    const Total t = wave_total<LOGITS>(
        thread_total<T, LOGITS, SHORT, LOGITS ? 1 : 4>(
            z, A.cols, 0, A.cols, wave % G * 64 + lane, G * 64, S),
        S);
    if (lane == 0) parts[row][wave % G] = t;
  }
  __syncthreads();
  auto total = [&](int row) {
    Total t = parts[row][0];
    for (int g = 1; g < G; ++g) {
      const Total o = parts[row][g];
      if constexpr (LOGITS) {
        const float m = larger(t.m, o.m);
        const double r = reference(m);
        t.s = t.s * weight_of<true>(t.m, r, S) + o.s * weight_of<true>(o.m, r, S);
        t.m = m;
      } else {
        t.s += o.s;
      }
    }
    return t;
  };
  if (mine < K &&
      !(tests && stands<LOGITS>(A.draft != nullptr, (float)pm, total(mine), (float)qm,
                                A.draft ? total(K + 1 + mine) : Total{0., 0.f}, um, S)))
    atomicMin(&first_end, mine);
  __syncthreads();
  const int n = first_end;
  write_drafts(A, sequence, n, kSmallThreads);
  const Total P = total(n);
  if (!has_outcomes<LOGITS>(P)) {
    if (threadIdx.x == 0) A.outcomes[sequence * (K + 1) + n] = -1;
    return;
  }
  const int64_t d = n < K ? drafted_at(A, sequence, n) : -1;
  const bool drafted = n < K && is_outcome(A, d), pair = drafted && A.draft;
  Source<T> s = source_of<T, LOGITS>(A, target_row<T>(A, sequence, n), P,
                                     pair ? draft_row<T>(A, sequence, n) : nullptr,
                                     pair ? total(K + 1 + n) : Total{0., 0.f}, d, drafted);
  // each wave's share of the row, and the wave that has the outcome
  const int64_t packs = (A.cols + V - 1) / V, share = (packs + W - 1) / W * V;
  const int64_t begin = wave * share < A.cols ? wave * share : A.cols;
  const int64_t end = begin + share < A.cols ? begin + share : A.cols;
  double x = 0., passed = 0.;
  int64_t outcome;
  if (descend<T, LOGITS, SHORT>(s, S, A.cols, span_of<V>(begin, end), x, passed, outcome,
                                [&](double sum, Span& span, double& x, double& passed) {
        const double of_wave = wave_sum(sum);
        if (lane == 0) sums[wave] = of_wave;
        __syncthreads();
        double a = lane < W ? sums[lane] : 0.;
        const double all = wave_sum(a);
        if (!(all > kNothing)) {  // nothing is left of the difference: the target's own row
          s.q = nullptr;
          s.without = -1;
          span = span_of<V>(0, A.cols);
          x = ulast * P.s;
          return wave == 0 ? Next::kAgain : Next::kStop;
        }
        x = ulast * all;
        return lane_that_passes(a, x, passed) == wave ? Next::kGoOn : Next::kStop;
      }) && lane == 0)
    A.outcomes[sequence * (K + 1) + n] = outcome;
}

// ------------------------------------------------------------ long rows

// Counters and sums that workgroups share within a launch.
struct Counter {     // a line of its own: those of one line are counted one after the other
  uint32_t n;
  uint32_t line[31];
};
struct Shared {
  Counter* ends;     // [sequences] where the drafts end, as far as it is known
  Counter* drawn;    // [sequences] pieces that are there
  Counter* came;     // [sequences][drafts] parts that are there
  Total* totals;     // [sequences][rows][parts]
  double* units;     // [sequences][units]
};

// All of it is written and read past the XCDs' own caches (relaxed accesses of agent scope are), so
// that no cache has to be written back or emptied for it: with acquire and release of agent scope,
// which do that, weights 32 x 4 x 65536 take 165 us instead of 27.6 where later rows are passed over,
// 46 instead of 26.5 where all are read.  What a workgroup has written is there once its stores are
// acknowledged; only then is it counted.
__device__ __forceinline__ bool comes_last(uint32_t* counter, uint32_t of) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  const uint32_t before =
      __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("" ::: "memory");
  return before + 1 == of;
}
__device__ __forceinline__ double load_shared(const double* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_shared(double* p, double v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Total load_shared(const Total* p) {
  return {__hip_atomic_load(&p->s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
          __hip_atomic_load(&p->m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
}

__global__ void __launch_bounds__(kThreads)
    clear_kernel(int64_t sequences, int64_t drafts, const Shared H) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < sequences) {
    H.ends[i].n = (uint32_t)drafts;
    H.drawn[i].n = 0;
  }
  if (i < sequences * drafts) H.came[i].n = 0;
}

// The total of a row's parts, in the same order everywhere; all lanes of a wave.
template <bool LOGITS>
__device__ __forceinline__ Total total_of(const Total* parts, int n, const Scale& S) {
  const int lane = threadIdx.x & 63;  // n <= 64
  return wave_total<LOGITS>(lane < n ? load_shared(parts + lane) : Total{0., -INFINITY}, S);
}

// Workgroups go through the positions in their order, so that the rows behind the first draft that
// does not stand are mostly passed over: whether they are changes no result.
template <typename T, bool LOGITS, bool SHORT, bool EARLY>
__global__ void __launch_bounds__(kThreads)
    total_kernel(const VerifyArgs A, const VerifyPlan R, const Shared H, Scale S) {
  __shared__ double table[LOGITS ? kTable : 1];
  __shared__ Total waves[kThreads / 64];
  __shared__ int flag;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = blockIdx.x / R.parts, part = blockIdx.x % R.parts;
  const int kinds = A.draft ? 2 : 1;
  const int64_t at = id / kinds;  // (the target's rows behind the drafts come last)
  const int64_t last_ones = A.sequences * A.drafts;
  const int64_t i = at < last_ones ? at / A.sequences : A.drafts;
  const int64_t sequence = at < last_ones ? at % A.sequences : id - last_ones * kinds;
  const bool of_draft = at < last_ones && id % kinds != 0;
  const int64_t d = i < A.drafts ? drafted_at(A, sequence, i) : -1;
  const bool drafted = is_outcome(A, d);
  if constexpr (EARLY) {
    if (threadIdx.x == 0) {
      const uint32_t end =
          __hip_atomic_load(&H.ends[sequence].n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      flag = (int64_t)end < i;
      if (!drafted && i < A.drafts)
        __hip_atomic_fetch_min(&H.ends[sequence].n, (uint32_t)i, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (flag) return;
  } else if (i == A.drafts && part == 0 && threadIdx.x == 0) {
    H.drawn[sequence].n = 0;
  }
  if (of_draft && !drafted) return;
  ready(S, table);
  if constexpr (LOGITS) {
    fill_table(table, kThreads);
    __syncthreads();
  }
  const int64_t rows = kinds * A.drafts + 1;
  Total* mine = H.totals + (sequence * rows + i) * R.parts;
  Total* drafts = mine + (A.drafts + 1) * R.parts;  // (where there are any)
  const T* z = of_draft ? draft_row<T>(A, sequence, i) : target_row<T>(A, sequence, i);
  const int64_t begin = part * R.part;
  const int64_t end = begin + R.part < A.cols ? begin + R.part : A.cols;
  const Total t = wave_total<LOGITS>(
      thread_total<T, LOGITS, SHORT, 4>(z, A.cols, begin, end, threadIdx.x, kThreads, S), S);
  if (lane == 0) waves[wave] = t;
  __syncthreads();
  if (wave != 0) return;
  const Total all = wave_total<LOGITS>(
      lane < kThreads / 64 ? waves[lane] : Total{0., -INFINITY}, S);
  bool last = false;
  if (lane == 0) {
    Total* to = (of_draft ? drafts : mine) + part;
    __hip_atomic_store(&to->s, all.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&to->m, all.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (EARLY && drafted)
      last = comes_last(&H.came[sequence * A.drafts + i].n, (uint32_t)(kinds * R.parts));
  }
  if (!EARLY || !__shfl((int)last, 0)) return;
  const Total P = total_of<LOGITS>(mine, R.parts, S);
  const Total Q = A.draft ? total_of<LOGITS>(drafts, R.parts, S) : Total{0., 0.f};
  if (lane == 0 &&
      !stands<LOGITS>(A.draft != nullptr, (float)target_row<T>(A, sequence, i)[d], P,
                      A.draft ? (float)draft_row<T>(A, sequence, i)[d] : 0.f, Q,
                      A.uniforms[sequence * (A.drafts + 1) + i], S))
    __hip_atomic_fetch_min(&H.ends[sequence].n, (uint32_t)i, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}

template <typename T, bool LOGITS, bool SHORT, bool EARLY>
__global__ void __launch_bounds__(kThreads)
    draw_kernel(const VerifyArgs A, const VerifyPlan R, const Shared H, Scale S) {
  constexpr int V = kPack<T>, W = kThreads / 64;
  __shared__ double table[LOGITS ? kTable : 1];
  __shared__ unsigned long long ends;
  const int64_t sequence = blockIdx.x / R.pieces;
  const int piece = (int)(blockIdx.x % R.pieces);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  ready(S, table);
  if constexpr (LOGITS) fill_table(table, kThreads);
  const int64_t K = A.drafts;
  const double u = A.uniforms[sequence * (K + 1) + K];
  const Total* first = H.totals + sequence * (A.draft ? 2 * K + 1 : K + 1) * R.parts;
  int64_t n;
  if constexpr (EARLY) {
    n = H.ends[sequence].n;
    __syncthreads();
  } else {
    if (threadIdx.x == 0) ends = (unsigned long long)K;
    __syncthreads();
    for (int64_t i = wave; i < K; i += W) {
      const int64_t d = drafted_at(A, sequence, i);
      bool ok = is_outcome(A, d);
      if (ok) {
        const Total P = total_of<LOGITS>(first + i * R.parts, R.parts, S);
        const Total Q = A.draft ? total_of<LOGITS>(first + (K + 1 + i) * R.parts, R.parts, S)
                                : Total{0., 0.f};
        ok = stands<LOGITS>(A.draft != nullptr, (float)target_row<T>(A, sequence, i)[d], P,
                            A.draft ? (float)draft_row<T>(A, sequence, i)[d] : 0.f, Q,
                            A.uniforms[sequence * (K + 1) + i], S);
      }
      if (!ok && lane == 0) atomicMin(&ends, (unsigned long long)i);
    }
    __syncthreads();
    n = (int64_t)ends;
  }
  const int64_t d = n < K ? drafted_at(A, sequence, n) : -1;
  const bool drafted = n < K && is_outcome(A, d), pair = drafted && A.draft;
  const Total* mine = first + n * R.parts;
  const Total P = total_of<LOGITS>(mine, R.parts, S);
  const Total Q = pair ? total_of<LOGITS>(mine + (K + 1) * R.parts, R.parts, S) : Total{0., 0.f};
  Source<T> s = source_of<T, LOGITS>(A, target_row<T>(A, sequence, n), P,
                                     pair ? draft_row<T>(A, sequence, n) : nullptr, Q, d, drafted);
  // a wave's unit of the row; then, in the workgroup that comes last, the unit with the outcome
  const int64_t unit = (int64_t)piece * W + wave;
  double* shared = H.units + sequence * R.units;
  auto span_at = [&](int64_t u) {
    const int64_t begin = u * R.unit < A.cols ? u * R.unit : A.cols;
    return span_of<V>(begin, begin + R.unit < A.cols ? begin + R.unit : A.cols);
  };
  double x = 0., passed = 0.;
  int64_t outcome = -1;
  if (descend<T, LOGITS, SHORT>(s, S, A.cols, span_at(unit), x, passed, outcome,
                                [&](double sum, Span& span, double& x, double& passed) {
        sum = wave_sum(sum);
        if (lane == 0 && unit < R.units) store_shared(shared + unit, sum);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (wave != 0) return Next::kStop;
        int end = 0;
        if (lane == 0) end = comes_last(&H.drawn[sequence].n, (uint32_t)R.pieces);
        if (!__shfl(end, 0)) return Next::kStop;
        for (int64_t i = lane; i <= K; i += 64)
          if (i != n) A.outcomes[sequence * (K + 1) + i] = i < n ? drafted_at(A, sequence, i) : -1;
        if (lane == 0) A.accepted[sequence] = n;
        if (!has_outcomes<LOGITS>(P)) return Next::kGoOn;
        // a lane's run of units, then the units of the run
        const int each = (R.units + 63) / 64;
        double a = 0.;
        for (int k = 0; k < each; ++k)
          if (lane * each + k < R.units) a += load_shared(shared + lane * each + k);
        const double all = wave_sum(a);
        if (!(all > kNothing)) {  // nothing is left of the difference: the target's own row
          s.q = nullptr;
          s.without = -1;
          span = span_of<V>(0, A.cols);
          x = u * P.s;
          return Next::kAgain;
        }
        x = u * all;
        const int run = lane_that_passes(a, x, passed) * each;
        a = lane < each && run + lane < R.units ? load_shared(shared + run + lane) : 0.;
        span = span_at(run + lane_that_passes(a, x, passed));
        return Next::kAgain;
      }) && lane == 0)
    A.outcomes[sequence * (K + 1) + n] = has_outcomes<LOGITS>(P) ? outcome : -1;
}

// ------------------------------------------------------------ launches

struct Layout {
  size_t drawn, came, totals, units, end;
};
Layout layout_of(int64_t sequences, int64_t drafts, bool has_draft, const VerifyPlan& R) {
  Layout L;
  const size_t n = (size_t)sequences;
  L.drawn = round256(n * sizeof(Counter));
  L.came = L.drawn + round256(n * sizeof(Counter));
  L.totals = L.came + round256(n * (size_t)drafts * sizeof(Counter));
  L.units = L.totals + round256(n * (size_t)verify_rows(drafts, has_draft) * (size_t)R.parts *
                                sizeof(Total));
  L.end = L.units + round256(n * (size_t)R.units * 8);
  return L;
}

}  // namespace

size_t verify_workspace(int dtype, int64_t sequences, int64_t drafts, int64_t cols,
                        bool has_draft) {
  if (verify_is_small(drafts, cols, has_draft)) return 0;
  return layout_of(sequences, drafts, has_draft,
                   verify_plan_of(sequences, drafts, cols, has_draft, 16 / (int)element_bytes(dtype)))
      .end;
}

int launch_verify(int kind, int dtype, const VerifyArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  Scale S{};
  // (beyond these, differences of fp32 numbers leave nothing or all of a weight, and -inf has to
  // stay apart from them)
  S.c = std::fmax(std::fmin(a.scale * 1.4426950408889634, 0x1p1000), 0x1p-900) * kTable;
  S.least = -1020. * kTable / S.c;
  const bool has_draft = a.draft != nullptr, small = verify_is_small(a.drafts, a.cols, has_draft);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    const VerifyPlan R = verify_plan_of(a.sequences, a.drafts, a.cols, has_draft, kPack<T>);
    const Layout L = layout_of(a.sequences, a.drafts, has_draft, R);
    const Shared H{reinterpret_cast<Counter*>(a.ws),
                   reinterpret_cast<Counter*>(a.ws + L.drawn),
                   reinterpret_cast<Counter*>(a.ws + L.came),
                   reinterpret_cast<Total*>(a.ws + L.totals),
                   reinterpret_cast<double*>(a.ws + L.units)};
    // sequences of a launch: as many as a grid holds
    const int64_t rows = verify_rows(a.drafts, has_draft);
    const int64_t most = small ? INT32_MAX / kSmallThreads
                               : INT32_MAX / kThreads /
                                     std::max<int64_t>(rows * R.parts, R.pieces);
    if (most == 0) return (int)hipErrorInvalidConfiguration;
    VerifyArgs part = a;
    auto launch = [&](auto logits, auto is_short) {
      constexpr bool LOGITS = decltype(logits)::value, SHORT = decltype(is_short)::value;
      if (small) {
        small_kernel<T, LOGITS, SHORT>
            <<<dim3((unsigned)part.sequences), kSmallThreads, 0, st>>>(part, S);
        return (int)hipGetLastError();
      }
      auto both = [&](auto early) {
        constexpr bool EARLY = decltype(early)::value;
        total_kernel<T, LOGITS, SHORT, EARLY>
            <<<dim3((unsigned)(part.sequences * rows * R.parts)), kThreads, 0, st>>>(part, R, H, S);
        if (int rc = (int)hipGetLastError()) return rc;
        draw_kernel<T, LOGITS, SHORT, EARLY>
            <<<dim3((unsigned)(part.sequences * R.pieces)), kThreads, 0, st>>>(part, R, H, S);
        return (int)hipGetLastError();
      };
      if constexpr (!SHORT)  // (short rows that are not small_kernel's have more than 10 drafts)
        if (!R.early) return both(std::false_type{});
      const int64_t counters = part.sequences * std::max<int64_t>(a.drafts, 1);
      clear_kernel<<<dim3((unsigned)((counters + kThreads - 1) / kThreads)), kThreads, 0, st>>>(
          part.sequences, part.drafts, H);
      if (int rc = (int)hipGetLastError()) return rc;
      return both(std::true_type{});
    };
    using std::false_type;
    using std::true_type;
    auto launch_part = [&] {
      if (kind == 0)
        return a.cols < kPack<T> ? launch(true_type{}, true_type{})
                                 : launch(true_type{}, false_type{});
      return a.cols < kPack<T> ? launch(false_type{}, true_type{})
                               : launch(false_type{}, false_type{});
    };
    for (int64_t first = 0; first < a.sequences; first += most) {
      part.sequences = std::min(most, a.sequences - first);
      part.target = static_cast<const T*>(a.target) + first * (a.drafts + 1) * a.ldt;
      if (has_draft) part.draft = static_cast<const T*>(a.draft) + first * a.drafts * a.ldd;
      part.drafted = a.drafted + first * a.drafts;
      part.uniforms = a.uniforms + first * (a.drafts + 1);
      part.outcomes = a.outcomes + first * (a.drafts + 1);
      part.accepted = a.accepted + first;
      if (int rc = launch_part()) return rc;
    }
    return 0;
  });
}

}  // namespace vqc
