// linear_quantized.hip -- linear layers in 8-bit integers: rows quantised by their own largest
// magnitude, and y = a(s_x s_w sum_k q_x q_w + b) + r.
//
//   a_r = max_j |x_rj|,  s_r = a_r / 127 in fp32,  q_rj = 127 x_rj / a_r to the nearest integer,
//   ties to even
//
// The products of integers are summed exactly, so that a result does not depend on how the sum is
// split; it is rounded to fp32 once and multiplied by the row's and then the channel's step.
//
// Large products lose most beside their main loop: 8192 x 4096 x 4096 takes 108 us more for each 4096
// of k (2550 TOP/s) and 31 us for the ends of its tiles, 47 with gelu and residual, in which the matrix
// cores of a CU, with one workgroup on it, stand still.  Few rows are bound by W's bytes, small products
// by launches and the latency of what hangs on each other, so that those quantise x where it is
// multiplied.  bf16: 8192 x 4096 x 4096 with gelu and residual 156 us (1760 TOP/s) behind 21 us of
// quantising, 512 x 4096 x 65536 144 to 157 us (1910 to 1750 TOP/s), 5 x 4096 x 65536 47 us (5.7 TB/s),
// 1 x 4096 x 4096 6.4 us, fp32 64 x 16 x 10 3.1 us.
#include <algorithm>

#include "layers.h"
#include "linear_device.h"
#include "linear_tiles.h"

namespace vqc {
namespace {

// ------------------------------------------------------------ rows to integers

// What turns a row's elements into integers: q is near x up inv.
struct RowStep {
  float most;     // its largest magnitude
  float up, inv;  // up: 1, or what brings rows of the smallest and the largest numbers where neither
                  // 127 / most nor 127 most is an infinity
  bool finite;
};
__device__ __forceinline__ RowStep row_step(float most) {
  RowStep s;
  s.most = most;
  s.finite = most < INFINITY;  // (not of NaN)
  s.up = most < 0x1p-121f ? 0x1p64f : most > 0x1p100f ? 0x1p-64f : 1.f;
  s.inv = s.finite && most > 0.f ? 127.f / (most * s.up) : 0.f;
  return s;
}
// Rows of an infinity or a NaN have the step NaN: what is computed from them says so.
__device__ __forceinline__ float step_of(const RowStep& s) {
  return s.finite ? s.most / 127.f : __builtin_nanf("");
}

// V elements to integers in the low bytes of words.  x inv is off by 2^-16.9 at most, so that the
// integer nearest to it is the right one unless it lies that near the border between two; there
// (bf16 rows often hold exact ties) 127 x - q most decides, which is exact: in fp32 of 16-bit
// elements, whose 127 x and q most have 18 bits and a last place of most 2^-19, in 64 bits of fp32
// ones.
template <typename T, int V>
__device__ __forceinline__ void to_integers(float (&x)[V], const RowStep& s, uint32_t (&q)[V]) {
  using Exact = std::conditional_t<sizeof(T) == 2, float, double>;
  constexpr float kMagic = 12582912.f;  // 1.5 2^23: the sum's last place is 1
  if (s.up != 1.f)
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= s.up;
  float f[V];
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float g = fmaf(x[i], s.inv, kMagic);
    f[i] = g - kMagic;
    far = fmaxf(far, fabsf(fmaf(x[i], s.inv, -f[i])));
    q[i] = __builtin_bit_cast(uint32_t, g);
  }
  if (far > 0.49998f) {
    const Exact most = (Exact)s.most * (Exact)s.up;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const Exact left = fma(-(Exact)f[i], most, (Exact)127 * (Exact)x[i]);
      // more than half a step from q, or half a step and q odd: the next one on that side
      const Exact over = 2 * fabs(left) - most;
      const bool next = over > 0 || (over == 0 && (q[i] & 1));
      q[i] += next ? (left > 0 ? 1u : ~0u) : 0u;
    }
  }
  if (!s.finite)
#pragma unroll
    for (int i = 0; i < V; ++i) q[i] = 0;
}

// The low bytes of four words as one.
__device__ __forceinline__ uint32_t four_bytes(const uint32_t* q) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400),
                               __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400), 0x05040100);
}

// Columns [c, c + V) of a row of integers.
template <int V>
__device__ __forceinline__ void store_integers(int8_t* row, int64_t c, int64_t cols,
                                               const uint32_t (&q)[V]) {
  struct __attribute__((packed, aligned(1), may_alias)) Words {
    uint32_t w[V / 4];
  };
  struct __attribute__((packed, aligned(1), may_alias)) Word {
    uint32_t w;
  };
  struct __attribute__((packed, aligned(1), may_alias)) Half {
    uint16_t w;
  };
  Words o;
#pragma unroll
  for (int i = 0; i < V; i += 4) o.w[i / 4] = four_bytes(q + i);
  int8_t* to = row + c;
  const int64_t room = cols - c;
  if (room >= V) {
    *reinterpret_cast<Words*>(to) = o;
    return;
  }
  uint32_t w = o.w[0];
  if (V > 4 && (room & 4)) {
    reinterpret_cast<Word*>(to)->w = w;
    to += 4;
    w = o.w[V / 4 - 1];
  }
  if (room & 2) {
    reinterpret_cast<Half*>(to)->w = (uint16_t)w;
    to += 2;
    w >>= 16;
  }
  if (room & 1) *to = (int8_t)w;
}

// The largest magnitude, NaN if any is.
template <typename T>
__device__ __forceinline__ float magnitude(const Pack<T>& p, float most) {
  float v[kPack<T>];
#pragma unroll
  for (int i = 0; i < kPack<T>; ++i) {
    v[i] = (float)p.v[i];
    asm("" : "+v"(v[i]));  // (the maximum is to be one of fp32)
  }
#pragma unroll
  for (int i = 0; i < kPack<T>; i += 2)
    most = larger(larger(most, fabsf(v[i])), fabsf(v[i + 1]));
  return most;
}

// The largest over aligned groups of G lanes or threads (as group_sums).
template <int G>
__device__ __forceinline__ float group_most(float x, float* red) {
  x = larger(x, lane_xor<1>(x));
  x = larger(x, lane_xor<2>(x));
  x = larger(x, lane_xor<4>(x));
  x = larger(x, lane_xor<8>(x));
  if constexpr (G > 16) {
    x = larger(x, lane_xor<16>(x));
    x = larger(x, lane_xor<32>(x));
  }
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6;
    constexpr int W = G / 64;
    if ((threadIdx.x & 63) == 0) red[wave] = x;
    __syncthreads();
    const int first = wave / W * W;
#pragma unroll
    for (int w = 0; w < W; ++w) x = larger(x, red[first + w]);
  }
  return x;
}

constexpr int kMaxRegisterCols = 16384;  // 1024 threads of 16 elements, 512 of 32

// G threads per row, which stays in their registers between its maximum and its integers; WG / G
// rows at a time, C packs per thread.  SHORT: rows of less than a pack.
// Memory-bound where rows are many: bf16 8192 x 4096 18 us of a stream of calls (100 MB, 5.6 TB/s;
// 512 threads of a pack each 27), 301 x 16384 6 us.
template <typename T, int G, int WG, int C, bool SHORT>
__global__ void __launch_bounds__(WG) quantize_kernel(const QuantizeArgs A) {
  constexpr int V = kPack<T>, NG = WG / G;
  __shared__ float red[2][WG / 64];
  const int t = threadIdx.x % G, g = threadIdx.x / G;
  const int cols = (int)A.cols;
  int flip = 0;
  for (int64_t base = (int64_t)blockIdx.x * NG; base < A.rows; base += (int64_t)gridDim.x * NG) {
    const bool mine = base + g < A.rows;
    const int64_t r = mine ? base + g : A.rows - 1;
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    Raw raw[C];
    Pack<T> p[C];
#pragma unroll
    for (int c = 0; c < C; ++c) raw[c] = load_raw<T, SHORT>(x, (c * G + t) * V, cols);
    float most = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      p[c] = taken<T, SHORT>(raw[c], (c * G + t) * V, cols, (T)0.f);
      most = magnitude(p[c], most);
    }
    const RowStep s = row_step(group_most<G>(most, red[flip]));
    flip ^= 1;
    if (!mine) continue;
    if (t == 0) A.scales[r] = step_of(s);
    int8_t* q = A.q + r * A.ldq;
    for (int c = cols + t; c < A.width; c += G) q[c] = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      if (col >= cols) break;
      float v[V];
      uint32_t n[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (float)p[c].v[i];
      to_integers<T, V>(v, s, n);
      store_integers<V>(q, col, cols, n);
    }
  }
}

// Rows longer than the registers hold: one workgroup per row, read twice.
template <typename T>
__global__ void __launch_bounds__(1024) quantize_long_kernel(const QuantizeArgs A) {
  constexpr int V = kPack<T>, G = 1024;
  __shared__ float red[2][G / 64];
  int flip = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    float most = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * V; c < A.cols; c += (int64_t)G * V)
      most = magnitude(taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f), most);
    const RowStep s = row_step(group_most<G>(most, red[flip]));
    flip ^= 1;
    if (threadIdx.x == 0) A.scales[r] = step_of(s);
    int8_t* q = A.q + r * A.ldq;
    for (int64_t c = A.cols + threadIdx.x; c < A.width; c += G) q[c] = 0;
    for (int64_t c = (int64_t)threadIdx.x * V; c < A.cols; c += (int64_t)G * V) {
      const Pack<T> p = taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f);
      float v[V];
      uint32_t n[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (float)p.v[i];
      to_integers<T, V>(v, s, n);
      store_integers<V>(q, c, A.cols, n);
    }
  }
}

// Rows of integers to rows of `width` that end in zeros, a thread for every 16; rows from `first` on.
__global__ void __launch_bounds__(256) pad_kernel(const QuantizeArgs A, int64_t first) {
  const int64_t chunks = A.width / 16;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = first + id / chunks;
  const int64_t c = id % chunks * 16;
  if (r >= A.rows) return;
  *reinterpret_cast<Pack<int8_t>*>(A.q + r * A.ldq + c) =
      load_pack<int8_t>(static_cast<const int8_t*>(A.x) + r * A.ldx, c, A.cols, (int8_t)0);
}

constexpr int64_t kMaxBlocks = 1 << 20;  // grids beyond this loop over rows

template <typename T>
int quantize_rows(const QuantizeArgs& a, hipStream_t st) {
  if (a.rows == 0) return 0;
  if (a.cols > kMaxRegisterCols) {
    quantize_long_kernel<T><<<dim3((unsigned)std::min(a.rows, kMaxBlocks)), 1024, 0, st>>>(a);
    return (int)hipGetLastError();
  }
  auto launch = [&](auto g, auto c, auto is_short) {
    constexpr int G = decltype(g)::value, WG = G > 256 ? G : 256, C = decltype(c)::value;
    const int64_t blocks = std::min<int64_t>((a.rows + WG / G - 1) / (WG / G), kMaxBlocks);
    quantize_kernel<T, G, WG, C, decltype(is_short)::value>
        <<<dim3((unsigned)blocks), WG, 0, st>>>(a);
    return (int)hipGetLastError();
  };
  using std::false_type;
  using std::true_type;
  using I1 = std::integral_constant<int, 1>;
  constexpr int most = 16 / kPack<T>;  // packs of a thread's 16 elements
  auto with_packs = [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (a.cols <= G * kPack<T>) return launch(g, I1{}, false_type{});
    if constexpr (most > 2)
      if (a.cols <= 2 * G * kPack<T>)
        return launch(g, std::integral_constant<int, 2>{}, false_type{});
    return launch(g, std::integral_constant<int, most>{}, false_type{});
  };
  if (a.cols < kPack<T>) return launch(std::integral_constant<int, 16>{}, I1{}, true_type{});
  if (a.cols <= 16 * 16) return with_packs(std::integral_constant<int, 16>{});
  if (a.cols <= 64 * 16) return with_packs(std::integral_constant<int, 64>{});
  if (a.cols <= 256 * 16) return with_packs(std::integral_constant<int, 256>{});
  // Longer rows: a CU has two workgroups of 1024 threads and, of as many rows, four of 512.  us, 1024 |
  // 512 threads: f16 301 x 16384 6.9 | 5.9, 8192 x 8192 44 | 34, 4096 x 16384 42 | 35; fp32 8192 x 8192
  // 75 | 57; f16 256 x 16384 4.6 | 5.6, 1 x 16384 3.2 | 3.7.
  if (a.rows <= kCUs) return with_packs(std::integral_constant<int, 1024>{});
  using Half = std::integral_constant<int, 512>;
  if (a.cols <= 512 * 16) return launch(Half{}, std::integral_constant<int, most>{}, false_type{});
  return launch(Half{}, std::integral_constant<int, 2 * most>{}, false_type{});
}

int pad_rows(const QuantizeArgs& a, hipStream_t st) {
  if (a.rows == 0 || a.width == 0) return 0;
  // rows of a launch: as many as a grid holds
  const int64_t chunks = a.width / 16, most = (int64_t)(INT32_MAX / 256) * 256 / chunks;
  if (most == 0) return (int)hipErrorInvalidConfiguration;
  for (int64_t first = 0; first < a.rows; first += most) {
    const int64_t blocks = (std::min(most, a.rows - first) * chunks + 255) / 256;
    pad_kernel<<<dim3((unsigned)blocks), 256, 0, st>>>(a, first);
    if (int rc = (int)hipGetLastError()) return rc;
  }
  return 0;
}

// ------------------------------------------------------------ few rows

// What a thread's sum in column n of row m is finished with, read while W is on its way.
struct Ending {
  float step, bias, residual;
};
template <typename T>
__device__ __forceinline__ Ending ending_of(const ScaledProduct& P, int64_t m, int64_t n) {
  Ending e{0.f, 0.f, 0.f};
  if (n >= P.N) return e;
  e.step = P.b_scales[n];
  if (P.bias) e.bias = (float)static_cast<const T*>(P.bias)[n];
  if (P.residual) e.residual = (float)static_cast<const T*>(P.residual)[m * P.ldr + n];
  return e;
}
template <typename T>
__device__ __forceinline__ void finish(const ScaledProduct& P, int64_t m, int64_t n, float sum,
                                       float row_step, const Ending& e) {
  if (n >= P.N) return;
  const float y = activate<sizeof(T) == 2>(P.act, scaled(sum, row_step, e.step, e.bias));
  static_cast<T*>(P.out)[m * P.ldo + n] = (T)(P.residual ? plus(y, e.residual) : y);
}

// A product of which every workgroup quantises its rows of x itself: a launch less.
struct FusedProduct : ScaledProduct {
  const void* x;  // of the element type
  int64_t ldx;
  int64_t m_blocks, n_blocks;
};

// The same for four columns of a row.
struct FourEndings {
  float step[4], bias[4], residual[4];
};
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Four {
  T v[4];
};
template <typename T>
__device__ __forceinline__ FourEndings four_endings_of(const ScaledProduct& P, int64_t m,
                                                       int64_t n) {
  FourEndings e{};
  if (n + 4 <= P.N) {
    const Four<float> s = *reinterpret_cast<const Four<float>*>(P.b_scales + n);
    Four<T> b{}, r{};
    if (P.bias) b = *reinterpret_cast<const Four<T>*>(static_cast<const T*>(P.bias) + n);
    if (P.residual)
      r = *reinterpret_cast<const Four<T>*>(static_cast<const T*>(P.residual) + m * P.ldr + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e.step[i] = s.v[i];
      e.bias[i] = (float)b.v[i];
      e.residual[i] = (float)r.v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Ending one = ending_of<T>(P, m, n + i);
      e.step[i] = one.step;
      e.bias[i] = one.bias;
      e.residual[i] = one.residual;
    }
  }
  return e;
}
template <typename T>
__device__ __forceinline__ void finish(const ScaledProduct& P, int64_t m, int64_t n,
                                       const intx4& sum, float row_step, const FourEndings& e) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = scaled((float)sum[i], row_step, e.step[i], e.bias[i]);
  with_act(P.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = activate<sizeof(T) == 2>(act, y[i]);
  });
  Four<T> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = (T)(P.residual ? plus(y[i], e.residual[i]) : y[i]);
  T* to = static_cast<T*>(P.out) + m * P.ldo + n;
  if (n + 4 <= P.N) {
    *reinterpret_cast<Four<T>*>(to) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < P.N) to[i] = o.v[i];
  }
}

// One row of x: a thread takes 16 elements of k at U places, which become 16 bytes in its registers,
// and meets them with RN rows of W at a time.  bf16 1 x 4096 x 65536 42.5 us (268 MB, 6.3 TB/s).
template <typename T, int U>
__global__ void __launch_bounds__(256) one_row_kernel(const FusedProduct P) {
  constexpr int V = kPack<T>, RN = 4, E = 16 / V, W = 4;
  __shared__ float most[W];
  __shared__ int sums[2][W][RN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = (int)P.K;
  const int64_t groups = (P.N + RN - 1) / RN;
  auto load = [&](Raw (&w)[U][RN], int64_t group) {
#pragma unroll
    for (int j = 0; j < RN; ++j) {
      const int64_t n = group * RN + j;
      const int8_t* row = static_cast<const int8_t*>(P.b) + (n < P.N ? n : P.N - 1) * P.ldb;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (u * 256 + (int)threadIdx.x) * 16;
        w[u][j] = *reinterpret_cast<const Raw*>(row + (k < K ? k : 0));
      }
    }
  };
  Raw cur[U][RN], next[U][RN], raw[U][E];
  load(cur, blockIdx.x);
  const int column = (int)threadIdx.x;
  const bool ends = column < RN;
  Ending end{};
  if (ends) end = ending_of<T>(P, 0, (int64_t)blockIdx.x * RN + column);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e)
      raw[u][e] = load_raw<T>(static_cast<const T*>(P.x),
                              ((u * 256 + (int)threadIdx.x) * E + e) * V, K);
  // behind the end of k: zeros, whatever W's bytes are there
  auto pack = [&](int u, int e) {
    return taken<T>(raw[u][e], ((u * 256 + (int)threadIdx.x) * E + e) * V, K, (T)0.f);
  };
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) m = magnitude(pack(u, e), m);
  const RowStep s = row_step(group_most<256>(m, most));
  const float step = step_of(s);
  Raw x[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const Pack<T> p = pack(u, e);
      float v[V];
      uint32_t q[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = (float)p.v[k];
      to_integers<T, V>(v, s, q);
#pragma unroll
      for (int k = 0; k < V; k += 4) x[u][(e * V + k) / 4] = four_bytes(q + k);
    }
  int flip = 0;
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
    if (group + gridDim.x < groups) load(next, group + gridDim.x);
#pragma unroll
    for (int j = 0; j < RN; ++j) {
      int sum = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          sum = __builtin_amdgcn_sdot4((int)x[u][b], (int)cur[u][j][b], sum, false);
      uint32_t t = (uint32_t)sum;
      t += lane_xor<1>(t);
      t += lane_xor<2>(t);
      t += lane_xor<4>(t);
      t += lane_xor<8>(t);
      t += lane_xor<16>(t);
      t += lane_xor<32>(t);
      if (lane == 0) sums[flip][wave][j] = (int)t;
    }
    __syncthreads();
    if (ends) {
      const int sum = sums[flip][0][column] + sums[flip][1][column] + sums[flip][2][column] +
                      sums[flip][3][column];
      finish<T>(P, 0, group * RN + column, (float)sum, step, end);
      if (group + gridDim.x < groups)
        end = ending_of<T>(P, 0, (group + gridDim.x) * RN + column);
    }
    flip ^= 1;  // (the other half is not written before everyone is past the next barrier)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < RN; ++j) cur[u][j] = next[u][j];
  }
}

// 16 rows of x of up to 512 V / 16 C elements: 32 lanes quantise a row into LDS, and the 8 waves take
// 16 rows of W each, straight from memory into the registers of the matrix instruction.  For
// products whose launches, and the latency of their loads, are all of it.
template <typename T, int C>
__global__ void __launch_bounds__(512) short_rows_kernel(const FusedProduct P) {
  constexpr int V = kPack<T>, kMostK = 32 * V * C, kChunks = (kMostK + 63) / 64;
  constexpr int kRow = kChunks * 64 + 16;  // (16 bytes more, against conflicts)
  __shared__ __align__(16) char rows[16][kRow];
  __shared__ float steps[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m0 = blockIdx.x % P.m_blocks * 16, nb = blockIdx.x / P.m_blocks;
  const int K = (int)P.K;
  const int64_t tiles = (P.N + 15) / 16;
  const int k_lane = lane / 16 * 16;
  Raw w[kChunks];
  FourEndings ends;
  auto load = [&](int64_t tile) {
    const int64_t n = tile * 16 + lane % 16;
    const int8_t* row = static_cast<const int8_t*>(P.b) + (n < P.N ? n : P.N - 1) * P.ldb;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      w[c] = *reinterpret_cast<const Raw*>(row + (c * 64 + k_lane < K ? c * 64 + k_lane : 0));
    const int64_t m = m0 + lane % 16;
    ends = four_endings_of<T>(P, m < P.M ? m : P.M - 1, tile * 16 + lane / 16 * 4);
  };
  int64_t tile = nb * 8 + wave;
  if (tile < tiles) load(tile);

  const int mine = (int)threadIdx.x / 32, t = (int)threadIdx.x % 32;
  const int64_t xm = m0 + mine < P.M ? m0 + mine : P.M - 1;
  const T* x = static_cast<const T*>(P.x) + xm * P.ldx;
  Raw raw[C];
#pragma unroll
  for (int c = 0; c < C; ++c) raw[c] = load_raw<T>(x, (c * 32 + t) * V, K);
  float most = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
    most = magnitude(taken<T>(raw[c], (c * 32 + t) * V, K, (T)0.f), most);
  most = group_most<16>(most, nullptr);
  const RowStep s = row_step(larger(most, lane_xor<16>(most)));
  if (t == 0) steps[mine] = step_of(s);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int k = (c * 32 + t) * V;
    const Pack<T> p = taken<T>(raw[c], k, K, (T)0.f);
    float v[V];
    uint32_t q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)p.v[i];
    to_integers<T, V>(v, s, q);
#pragma unroll
    for (int i = 0; i < V; i += 4)
      *reinterpret_cast<uint32_t*>(&rows[mine][k + i]) = four_bytes(q + i);
  }
  __syncthreads();
  const char* row = rows[lane % 16] + k_lane;
  const float step = steps[lane % 16];
  const int64_t m = m0 + lane % 16;
  while (tile < tiles) {
    intx4 acc = {};
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
          __builtin_bit_cast(intx4, w[c]), *reinterpret_cast<const intx4*>(row + c * 64), acc, 0, 0,
          0);
    if (m < P.M) finish<T>(P, m, tile * 16 + lane / 16 * 4, acc, step, ends);
    tile += P.n_blocks * 8;
    if (tile < tiles) load(tile);
  }
}

// Up to 16 MT rows against 16 rows of W at a time, whose k the 8 waves of a workgroup share out in
// turn, 64 at a time: x stays in registers, W comes straight from memory into them as the matrix
// instruction takes it, C loads ahead.  Memory-bound in W, which is read once: bf16 5 x 4096 x 65536
// 47 us (5.7 TB/s; loads of W in this order and nothing else take 45).
// FUSED: every workgroup quantises x itself while its first rows of W are on their way, a wave 1024
// elements (with four times as much for a wave, the instructions alone arrive later than a launch
// of its own ends: 8 x 4096 x 4096 11.1 us instead of 8.7); otherwise x is integers.
template <typename T, int MT, int C, bool FUSED>
__global__ void __launch_bounds__(512) rows_kernel(const FusedProduct P) {
  constexpr int W = 8;
  static_assert(MT <= 2, "a thread has one column of a row");
  __shared__ int sums[2][W][MT][64 * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = (int)P.K, rows = (int)P.M;
  const int64_t steps = (P.N + 15) / 16;
  auto k_of = [&](int c) { return (c * W + wave) * 64 + lane / 16 * 16; };
  auto load = [&](Raw (&w)[C], int64_t step) {
    const int64_t n = step * 16 + lane % 16;
    const int8_t* row = static_cast<const int8_t*>(P.b) + (n < P.N ? n : P.N - 1) * P.ldb;
#pragma unroll
    for (int c = 0; c < C; ++c)
      w[c] = *reinterpret_cast<const Raw*>(row + (k_of(c) < K ? k_of(c) : 0));
  };
  Raw cur[C], next[C], x[MT][C];
  load(cur, blockIdx.x);
  // a thread's column of a row
  const int mine = (int)threadIdx.x / 16, column = (int)threadIdx.x % 16;
  const int at = (column / 4 * 16 + mine % 16) * 4 + column % 4;
  const bool ends = mine < rows;
  float row_step_mine = 0.f;
  Ending end{};
  if (ends) end = ending_of<T>(P, mine, (int64_t)blockIdx.x * 16 + column);
  if constexpr (FUSED) {
    constexpr int V = kPack<T>, E = 16 / V;
    static_assert(kFusedPieces == W, "a piece for each wave");
    extern __shared__ __align__(16) char integers[];  // [rows][ld], k to a multiple of 64
    __shared__ uint32_t most[16 * MT];
    const int wide = (K + 63) / 64 * 64, ld = wide + 16;  // (16 bytes more, against conflicts)
    const int per = (K + 1023) / 1024, piece = __builtin_amdgcn_readfirstlane(wave);
    const bool has = piece < rows * per;
    const int row = has ? piece / per : 0, col = piece % per * 1024 + lane * 16;
    if (threadIdx.x < 16 * MT) most[threadIdx.x] = 0;
    Raw raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      raw[e] = load_raw<T>(static_cast<const T*>(P.x) + row * P.ldx, col + e * V, K);
    __syncthreads();
    if (has) {
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
        m = magnitude(taken<T>(raw[e], col + e * V, K, (T)0.f), m);
      m = group_most<64>(m, nullptr);
      if (lane == 0) atomicMax(&most[row], __builtin_bit_cast(uint32_t, m) & 0x7FFFFFFFu);
    }
    __syncthreads();
    if (has) {
      const RowStep s = row_step(__builtin_bit_cast(float, most[row]));
      Raw q16;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const Pack<T> p = taken<T>(raw[e], col + e * V, K, (T)0.f);
        float v[V];
        uint32_t q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)p.v[i];
        to_integers<T, V>(v, s, q);
#pragma unroll
        for (int i = 0; i < V; i += 4) q16[(e * V + i) / 4] = four_bytes(q + i);
      }
      if (col < wide) *reinterpret_cast<Raw*>(integers + row * ld + col) = q16;
    }
    if (ends) row_step_mine = step_of(row_step(__builtin_bit_cast(float, most[mine])));
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int m = t * 16 + lane % 16;
#pragma unroll
      for (int c = 0; c < C; ++c)
        x[t][c] = k_of(c) < wide ? *reinterpret_cast<const Raw*>(
                                       integers + (m < rows ? m : 0) * ld + k_of(c))
                                 : Raw{0, 0, 0, 0};
    }
  } else {
    if (ends) row_step_mine = P.a_scales[mine];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int m = t * 16 + lane % 16;
      const int8_t* row = static_cast<const int8_t*>(P.a) + (m < rows ? m : 0) * P.lda;
#pragma unroll
      for (int c = 0; c < C; ++c)  // (rows of x go on with zeros to the end of their last 128)
        x[t][c] = k_of(c) < K ? *reinterpret_cast<const Raw*>(row + k_of(c)) : Raw{0, 0, 0, 0};
    }
  }
  int flip = 0;
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    if (step + gridDim.x < steps) load(next, step + gridDim.x);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      intx4 acc = {};
#pragma unroll
      for (int c = 0; c < C; ++c)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, cur[c]),
                                                    __builtin_bit_cast(intx4, x[t][c]), acc, 0, 0,
                                                    0);
      *reinterpret_cast<intx4*>(&sums[flip][wave][t][lane * 4]) = acc;
    }
    __syncthreads();
    if (ends) {
      int sum = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) sum += sums[flip][w][mine / 16][at];
      finish<T>(P, mine, step * 16 + column, (float)sum, row_step_mine, end);
      if (step + gridDim.x < steps)
        end = ending_of<T>(P, mine, (step + gridDim.x) * 16 + column);
    }
    flip ^= 1;  // (the other half is not written before everyone is past the next barrier)
#pragma unroll
    for (int c = 0; c < C; ++c) cur[c] = next[c];
  }
}

// The splits' sums, and what becomes of them.
template <typename T>
__global__ void __launch_bounds__(256)
    join_integers_kernel(const ScaledProduct P, int64_t splits) {
  const int64_t count = P.M * P.N;
  const int* partial = reinterpret_cast<const int*>(P.partial);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count;
       i += (int64_t)gridDim.x * 256) {
    // (a division of 64 bits takes a hundred instructions)
    const int64_t m = count <= INT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)P.N) : i / P.N;
    const int64_t n = i - m * P.N;
    const float row_step = P.a_scales[m];
    const Ending end = ending_of<T>(P, m, n);
    int64_t sum = 0;
    for (int64_t s = 0; s < splits; s += 12) {  // loads in flight together, the last few too
      int part[12];
#pragma unroll
      for (int u = 0; u < 12; ++u)
        part[u] = partial[(s + u < splits ? s + u : splits - 1) * count + i];
#pragma unroll
      for (int u = 0; u < 12; ++u) sum += s + u < splits ? part[u] : 0;
    }
    finish<T>(P, m, n, (float)sum, row_step, end);
  }
}

// ------------------------------------------------------------ launches

// The workspace: [rows of x for the products, with zeros to the end of a stage | their steps | the
// products' splits], the steps where x is not given as integers, the rows there and where given
// ones do not end with a stage.
struct QuantizedLayout {
  size_t scales = 0, splits = 0, end = 0;
  int64_t ld = 0;
  bool rows = false;
};
QuantizedLayout layout_of(int64_t rows, int64_t n_in, int64_t n_out, bool integers) {
  QuantizedLayout L;
  L.ld = (n_in + kIntegerStage - 1) / kIntegerStage * kIntegerStage;
  L.rows = !integers || L.ld != n_in;
  if (L.rows) L.scales = L.splits = round256((size_t)rows * (size_t)L.ld);
  if (!integers) L.splits += round256((size_t)rows * 4);
  size_t most = 0;
  for (bool direct : {false, true}) {
    if (direct && few_integer_rows(rows, n_out, n_in)) continue;
    const Plan p = integer_plan_of(direct, rows, n_out, n_in);
    if (p.splits > 1) most = std::max(most, (size_t)p.splits * (size_t)rows * (size_t)n_out * 4);
  }
  L.end = L.splits + round256(most);
  return L;
}

bool on_16(const void* p, int64_t ld, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows < 2 || ld % 16 == 0);
}

FusedProduct fused(const ScaledProduct& p, const void* x, int64_t ldx) {
  FusedProduct f{};
  static_cast<ScaledProduct&>(f) = p;
  f.x = x;
  f.ldx = ldx;
  return f;
}

template <typename T>
int one_row_product(const FusedProduct& p, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>((p.N + 3) / 4, 8 * kCUs));
  auto launch = [&](auto u) {
    one_row_kernel<T, decltype(u)::value><<<grid, 256, 0, st>>>(p);
    return (int)hipGetLastError();
  };
  if (p.K <= 4096) return launch(std::integral_constant<int, 1>{});
  if (p.K <= 8192) return launch(std::integral_constant<int, 2>{});
  return launch(std::integral_constant<int, 4>{});
}

template <typename T>
int short_rows_product(const FusedProduct& all, hipStream_t st) {
  FusedProduct p = all;
  auto launch = [&](auto c) {
    short_rows_kernel<T, decltype(c)::value>
        <<<dim3((unsigned)(p.m_blocks * p.n_blocks)), 512, 0, st>>>(p);
    return (int)hipGetLastError();
  };
  auto launch_rows = [&] {
    const int64_t lanes = 32 * kPack<T>;
    if (p.K <= lanes) return launch(std::integral_constant<int, 1>{});
    if (p.K <= 2 * lanes) return launch(std::integral_constant<int, 2>{});
    if (p.K <= 4 * lanes) return launch(std::integral_constant<int, 4>{});
    if constexpr (sizeof(T) == 4) return launch(std::integral_constant<int, 8>{});
    return (int)hipErrorInvalidValue;
  };
  constexpr int64_t most = INT32_MAX / 512 * 16;  // rows of a launch: as many as a grid holds
  for (int64_t m = 0; m < all.M; m += most) {
    p.M = std::min(most, all.M - m);
    p.x = static_cast<const T*>(all.x) + m * all.ldx;
    if (all.residual) p.residual = static_cast<const T*>(all.residual) + m * all.ldr;
    p.out = static_cast<T*>(all.out) + m * all.ldo;
    p.m_blocks = (p.M + 15) / 16;
    // two workgroups for every CU, where there are rows of W for them
    p.n_blocks = std::max<int64_t>(
        1, std::min<int64_t>((p.N + 127) / 128, 2 * kCUs / p.m_blocks));
    if (int rc = launch_rows()) return rc;
  }
  return 0;
}

template <typename T, bool FUSED>
int few_rows_product(const FusedProduct& p, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>((p.N + 15) / 16, 2 * kCUs));
  const size_t lds = FUSED ? (size_t)(p.M * ((p.K + 63) / 64 * 64 + 16)) : 0;
  auto launch = [&](auto mt, auto c) {
    rows_kernel<T, decltype(mt)::value, decltype(c)::value, FUSED><<<grid, 512, lds, st>>>(p);
    return (int)hipGetLastError();
  };
  using std::integral_constant;
  auto with_chunks = [&](auto mt) {
    if (p.K <= 512) return launch(mt, integral_constant<int, 1>{});
    if (p.K <= 1024) return launch(mt, integral_constant<int, 2>{});
    if (p.K <= 2048) return launch(mt, integral_constant<int, 4>{});
    return launch(mt, integral_constant<int, 8>{});
  };
  if constexpr (FUSED) return with_chunks(integral_constant<int, 1>{});
  return p.M <= 16 ? with_chunks(integral_constant<int, 1>{})
                   : with_chunks(integral_constant<int, 2>{});
}

template <typename T>
int integer_product(ScaledProduct p, unsigned char* ws, hipStream_t st) {
  const bool direct = on_16(p.a, p.lda, p.M) && on_16(p.b, p.ldb, p.N) && p.K > 0;
  if (direct && few_integer_rows(p.M, p.N, p.K))
    return few_rows_product<T, false>(fused(p, nullptr, 0), st);
  const Plan plan = integer_plan_of(direct, p.M, p.N, p.K);
  const int64_t tiles = tiles_of(p.M, p.N, plan.tile);
  p.k_step = plan.k_step;
  p.partial = plan.splits > 1 ? reinterpret_cast<float*>(ws) : nullptr;
  if (tiles > INT32_MAX / 256 || plan.splits > 65535) return (int)hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)tiles, (unsigned)plan.splits);
  if (plan.tile == 256)
    tile_kernel<T, false, false, 4, 2, 2, 4, 128, 2, int8_t><<<grid, 512, 0, st>>>(p);
  else if (plan.tile == 128)
    tile_kernel<T, false, false, 2, 2, 2, 2, 64, 3, int8_t><<<grid, 256, 0, st>>>(p);
  else if (plan.tile == 64 && direct)
    tile_kernel<T, false, false, 1, 1, 2, 2, 128, 3, int8_t><<<grid, 256, 0, st>>>(p);
  else if (plan.tile == 64)
    staged_kernel<T, int8_t, int8_t, false, false, 2, 2, 1><<<grid, 256, 0, st>>>(p);
  else
    staged_kernel<T, int8_t, int8_t, false, false, 1, 1, 4><<<grid, 256, 0, st>>>(p);
  int rc = (int)hipGetLastError();
  if (rc || plan.splits == 1) return rc;
  const int64_t blocks = std::min<int64_t>((p.M * p.N + 255) / 256, 1 << 16);
  join_integers_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(p, plan.splits);
  return (int)hipGetLastError();
}

}  // namespace

int launch_quantize(int dtype, const QuantizeArgs& a, void* stream) {
  return by_dtype(dtype, [&](auto type) {
    return quantize_rows<decltype(type)>(a, static_cast<hipStream_t>(stream));
  });
}

size_t linear_quantized_workspace(int64_t rows, int64_t n_in, int64_t n_out, bool integers) {
  return layout_of(rows, n_in, n_out, integers).end;
}

int launch_linear_quantized(int dtype, const QuantizedArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const QuantizedLayout L = layout_of(a.rows, a.n_in, a.n_out, a.x_scales != nullptr);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    ScaledProduct p{};
    p.M = a.rows;
    p.N = a.n_out;
    p.K = a.n_in;
    p.a = a.x;
    p.lda = a.ldx;
    p.a_scales = a.x_scales;
    p.b = a.weight;
    p.ldb = a.ldw;
    p.b_scales = a.w_scales;
    p.bias = a.bias;
    p.residual = a.residual;
    p.ldr = a.ldr;
    p.act = a.act;
    p.out = a.y;
    p.ldo = a.ldy;
    const bool aligned = on_16(p.b, p.ldb, p.N);
    if (!a.x_scales && aligned) {
      if (short_integer_rows(sizeof(T), p.M, p.N, p.K))
        return short_rows_product<T>(fused(p, a.x, a.ldx), st);
      if (one_integer_row(p.M, p.N, p.K))
        return one_row_product<T>(fused(p, a.x, a.ldx), st);
      if (fused_integer_rows(p.M, p.N, p.K))
        return few_rows_product<T, true>(fused(p, a.x, a.ldx), st);
    }
    if (L.rows) {
      QuantizeArgs q{};
      q.rows = a.rows;
      q.cols = a.n_in;
      q.x = a.x;
      q.ldx = a.ldx;
      q.q = reinterpret_cast<int8_t*>(a.ws);
      q.ldq = q.width = L.ld;
      q.scales = reinterpret_cast<float*>(a.ws + L.scales);
      if (int rc = a.x_scales ? pad_rows(q, st) : quantize_rows<T>(q, st)) return rc;
      p.a = q.q;
      p.lda = q.ldq;
      if (!a.x_scales) p.a_scales = q.scales;
    }
    return integer_product<T>(p, a.ws + L.splits, st);
  });
}

}  // namespace vqc
