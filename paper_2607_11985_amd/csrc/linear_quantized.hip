// linear_quantized.hip -- linear layers in 8-bit integers: rows quantised by their own largest
// magnitude, and y = a(s_x s_w sum_k q_x q_w + b) + r.
//
//   a_r = max_j |x_rj|,  s_r = a_r / 127 in fp32,  q_rj = 127 x_rj / a_r to the nearest integer,
//   ties to even
//
// The products of integers are summed exactly, so that a result does not depend on how the sum is
// split; it is rounded to fp32 once and multiplied by the row's and then the channel's step.
#include <algorithm>

#include "layers.h"
#include "linear_device.h"
#include "linear_tiles.h"

namespace vqc {
namespace {

// ------------------------------------------------------------ rows to integers

// What turns a row's elements into integers.
struct RowStep {
  float most;     // its largest magnitude
  float up, inv;  // q is near x up inv
  bool finite;
};

// The magnitude's bits (NaN above infinity above all numbers).
__device__ __forceinline__ RowStep row_step(uint32_t most_bits) {
  RowStep s;
  s.most = __builtin_bit_cast(float, most_bits);
  s.finite = most_bits < 0x7F800000u;
  // in units in which 127 / most is no infinity
  s.up = s.most < 0x1p-60f ? 0x1p64f : 1.f;
  s.inv = s.finite && most_bits ? 127.f / (s.most * s.up) : 0.f;
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
__device__ __forceinline__ void to_integers(const float (&x)[V], const RowStep& s,
                                            uint32_t (&q)[V]) {
  using Exact = std::conditional_t<sizeof(T) == 2, float, double>;
  constexpr float kMagic = 12582912.f;  // 1.5 2^23: the sum's last place is 1
  float f[V];
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float v = x[i] * s.up, g = fmaf(v, s.inv, kMagic);
    f[i] = g - kMagic;
    far = fmaxf(far, fabsf(fmaf(v, s.inv, -f[i])));
    q[i] = __builtin_bit_cast(uint32_t, g);
  }
  if (far > 0.49998f) {
    const Exact up = (Exact)s.up, most = (Exact)s.most * up;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const Exact left = fma(-(Exact)f[i], most, (Exact)127 * ((Exact)x[i] * up));
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
  for (int i = 0; i < V; i += 4)
    o.w[i / 4] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[i + 3], q[i + 2], 0x0c0c0400),
                                       __builtin_amdgcn_perm(q[i + 1], q[i], 0x0c0c0400),
                                       0x05040100);
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
template <typename T>
__device__ __forceinline__ uint32_t magnitude_bits(const Pack<T>& p, uint32_t most) {
#pragma unroll
  for (int i = 0; i < kPack<T>; ++i) {
    const uint32_t u = __builtin_bit_cast(uint32_t, (float)p.v[i]) & 0x7FFFFFFFu;
    most = most > u ? most : u;
  }
  return most;
}

// The largest over aligned groups of G lanes or threads (as group_sums).
template <int N>
__device__ __forceinline__ uint32_t lanes_most(uint32_t x) {
  const uint32_t o = lane_xor<N>(x);
  return x > o ? x : o;
}
template <int G>
__device__ __forceinline__ uint32_t group_most(uint32_t x, uint32_t* red) {
  x = lanes_most<1>(x);
  x = lanes_most<2>(x);
  x = lanes_most<4>(x);
  x = lanes_most<8>(x);
  if constexpr (G > 16) {
    x = lanes_most<16>(x);
    x = lanes_most<32>(x);
  }
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6;
    constexpr int W = G / 64;
    if ((threadIdx.x & 63) == 0) red[wave] = x;
    __syncthreads();
    const int first = wave / W * W;
#pragma unroll
    for (int w = 0; w < W; ++w) x = x > red[first + w] ? x : red[first + w];
  }
  return x;
}

constexpr int kMaxRegisterCols = 16384;  // 1024 threads of 16 elements

// G threads per row, which stays in their registers between its maximum and its integers; WG / G
// rows at a time, C packs per thread.  SHORT: rows of less than a pack.
template <typename T, int G, int WG, int C, bool SHORT>
__global__ void __launch_bounds__(WG) quantize_kernel(const QuantizeArgs A) {
  constexpr int V = kPack<T>, NG = WG / G;
  __shared__ uint32_t red[2][WG / 64];
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
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      p[c] = taken<T, SHORT>(raw[c], (c * G + t) * V, cols, (T)0.f);
      most = magnitude_bits(p[c], most);
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
      Pack<T> now = p[0];
#pragma unroll
      for (int k = 1; k < C; ++k)
        if (c == k) now = p[k];
      float v[V];
      uint32_t n[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (float)now.v[i];
      to_integers<T, V>(v, s, n);
      store_integers<V>(q, col, cols, n);
    }
  }
}

// Rows longer than the registers hold: one workgroup per row, read twice.
template <typename T>
__global__ void __launch_bounds__(1024) quantize_long_kernel(const QuantizeArgs A) {
  constexpr int V = kPack<T>, G = 1024;
  __shared__ uint32_t red[2][G / 64];
  int flip = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    uint32_t most = 0;
    for (int64_t c = (int64_t)threadIdx.x * V; c < A.cols; c += (int64_t)G * V)
      most = magnitude_bits(taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f), most);
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

// Rows of integers to rows of `width` that end in zeros, a thread for every 16.
__global__ void __launch_bounds__(256) pad_kernel(const QuantizeArgs A) {
  const int64_t chunks = A.width / 16;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = id / chunks;
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
  auto of = [](auto n) { return n; };
  using std::false_type;
  using std::true_type;
  using I1 = std::integral_constant<int, 1>;
  constexpr int most = 16 / kPack<T>;  // packs of a thread's 16 elements
  auto with_packs = [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (a.cols <= G * kPack<T>) return launch(g, I1{}, false_type{});
    if constexpr (most > 2)
      if (a.cols <= 2 * G * kPack<T>)
        return launch(g, of(std::integral_constant<int, 2>{}), false_type{});
    return launch(g, of(std::integral_constant<int, most>{}), false_type{});
  };
  if (a.cols < kPack<T>) return launch(std::integral_constant<int, 16>{}, I1{}, true_type{});
  if (a.cols <= 16 * 16) return with_packs(std::integral_constant<int, 16>{});
  if (a.cols <= 64 * 16) return with_packs(std::integral_constant<int, 64>{});
  if (a.cols <= 256 * 16) return with_packs(std::integral_constant<int, 256>{});
  return with_packs(std::integral_constant<int, 1024>{});
}

int pad_rows(const QuantizeArgs& a, hipStream_t st) {
  if (a.rows == 0 || a.width == 0) return 0;
  const int64_t blocks = (a.rows * (a.width / 16) + 255) / 256;
  if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
  pad_kernel<<<dim3((unsigned)blocks), 256, 0, st>>>(a);
  return (int)hipGetLastError();
}

// ------------------------------------------------------------ few rows

// One to MR rows of x against RN rows of W per workgroup, whose threads take 16 bytes of k in
// turn and add up at the end.  Memory-bound: W is read once.
template <typename T, int MR, int RN>
__global__ void __launch_bounds__(256) few_rows_i8_kernel(const ScaledProduct P) {
  constexpr int U = MR > 4 ? 1 : 2;
  __shared__ int sums[4][MR * RN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * RN;
  const int8_t *x[MR], *w[RN];
#pragma unroll
  for (int i = 0; i < MR; ++i) x[i] = static_cast<const int8_t*>(P.a) + (i < P.M ? i : 0) * P.lda;
#pragma unroll
  for (int j = 0; j < RN; ++j)
    w[j] = static_cast<const int8_t*>(P.b) + (n0 + j < P.N ? n0 + j : n0) * P.ldb;
  int acc[MR][RN] = {};
  for (int64_t k0 = (int64_t)threadIdx.x * 16; k0 - lane * 16 < P.K; k0 += U * 256 * 16) {
    Raw xr[U][MR], wr[U][RN];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + u * 256 * 16;
#pragma unroll
      for (int j = 0; j < RN; ++j) wr[u][j] = load_raw<int8_t>(w[j], k, P.K);
#pragma unroll
      for (int i = 0; i < MR; ++i) xr[u][i] = load_raw<int8_t>(x[i], k, P.K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + u * 256 * 16, over = k + 16 - P.K;
      // W's last 16 bytes are read whole: x's part of what was read before is 0
#pragma unroll
      for (int i = 0; i < MR; ++i)
        if (over > 0) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int64_t off = over - 4 * b;  // bytes of this word that were read before
            xr[u][i][b] &= off <= 0 ? 0xFFFFFFFFu : off >= 4 ? 0u : 0xFFFFFFFFu << (8 * off);
          }
        }
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            acc[i][j] =
                __builtin_amdgcn_sdot4((int)xr[u][i][b], (int)wr[u][j][b], acc[i][j], false);
    }
  }
#pragma unroll
  for (int i = 0; i < MR; ++i)
#pragma unroll
    for (int j = 0; j < RN; ++j) {
      uint32_t s = (uint32_t)acc[i][j];
      s += lane_xor<1>(s);
      s += lane_xor<2>(s);
      s += lane_xor<4>(s);
      s += lane_xor<8>(s);
      s += lane_xor<16>(s);
      s += lane_xor<32>(s);
      if (lane == 0) sums[wave][i * RN + j] = (int)s;
    }
  __syncthreads();
  const int i = threadIdx.x / RN, j = threadIdx.x % RN;
  if (i < MR && i < P.M && n0 + j < P.N)
    finish<T>(P, i, n0 + j,
              sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] +
                  sums[3][threadIdx.x]);
}

// The splits' sums, and what becomes of them.
template <typename T>
__global__ void __launch_bounds__(256)
    join_integers_kernel(const ScaledProduct P, int64_t splits) {
  const int64_t count = P.M * P.N;
  const int* partial = reinterpret_cast<const int*>(P.partial);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count;
       i += (int64_t)gridDim.x * 256) {
    int64_t z = 0;
#pragma unroll 4
    for (int64_t s = 0; s < splits; ++s) z += partial[s * count + i];
    const int64_t m = i / P.N, n = i - m * P.N;
    finish<T>(static_cast<const Product&>(P), m, n, (float)z * P.a_scales[m] * P.b_scales[n]);
  }
}

// ------------------------------------------------------------ launches

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

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
    const Plan p = integer_plan_of(direct, rows, n_out, n_in);
    if (p.splits > 1) most = std::max(most, (size_t)p.splits * (size_t)rows * (size_t)n_out * 4);
  }
  L.end = L.splits + round256(most);
  return L;
}

bool on_16(const void* p, int64_t ld, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows < 2 || ld % 16 == 0);
}

template <typename T>
int integer_product(ScaledProduct p, unsigned char* ws, hipStream_t st) {
  if (few_integer_rows(p.M, p.N, p.K)) {
    const int64_t blocks = (p.N + 3) / 4;
    if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
    if (p.M == 1)
      few_rows_i8_kernel<T, 1, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
    else if (p.M == 2)
      few_rows_i8_kernel<T, 2, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
    else if (p.M <= 4)
      few_rows_i8_kernel<T, 4, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
    else
      few_rows_i8_kernel<T, 8, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
    return (int)hipGetLastError();
  }
  const bool direct = on_16(p.a, p.lda, p.M) && on_16(p.b, p.ldb, p.N) && p.K > 0;
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
    if (!a.x_scales || (L.rows && !few_integer_rows(p.M, p.N, p.K))) {
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
