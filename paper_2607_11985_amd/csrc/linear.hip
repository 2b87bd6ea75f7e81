// linear.hip -- linear layers: y = a(x W^T + b) + r and its gradients.
//
//   z = x W^T + b, y = a(z) + r
//   dz = dy a'(z), dx = dz W, dW = dz^T x, db = sum_rows dz
//
// Three products C[m, n] = sum_k A(m, k) B(n, k) that differ in which operand's k runs along
// its rows: forward x and W by rows; dx takes W by columns; dW takes both by columns.
//
// bf16 8192 x 4096 x 4096: forward with bias, gelu, residual and z saved 290 us (950 TFLOP/s), dx
// 242 (1140), dW 229 (1200), dz and db 57; matrix cores busy 66 to 73 % in the gradients, at the
// clock that this load leaves.  fp32 likewise 1920 to 1990 us each (138 to 143 TFLOP/s).  One row,
// bf16 4096 x 4096: 7.3 us (4.6 TB/s).  fp32 1024 x 768 x 384: 16, 13 and 16 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layers.h"
#include "layers_device.h"
#include "linear_tiles.h"

namespace vqc {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------ activations

// Two forms: fp32 elements take the math library's functions; 16-bit ones shorter forms whose
// relative errors (some 2^-22) vanish in the rounding to 11 or 8 bits.  The short gelu is less
// exact where its result is small: by 5e-4 of it at z = -4 (half an ulp of fp16), 2e-3 at -5 (of
// bf16), 1e-2 at -8, where the result is -5e-15.

__device__ __forceinline__ float fast_exp(float x) {
  return __builtin_amdgcn_exp2f(x * 1.44269504f);
}
__device__ __forceinline__ float fast_logistic(float z) {
  return __builtin_amdgcn_rcpf(1.f + fast_exp(-z));
}
__device__ __forceinline__ float fast_tanh(float z) {
  const float q = z * z;
  // near 0 the difference would cancel: the first terms of the series
  return fabsf(z) < 0.0625f ? z * (1.f + q * (-0.333333333f + q * 0.133333333f))
                            : 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + fast_exp(2.f * z));
}
// 1 - tanh^2 z without the difference, which has no digits left beyond |z| = 9.
template <bool FAST>
__device__ __forceinline__ float tanh_slope(float z) {
  const float q = FAST ? fast_exp(-2.f * fabsf(z)) : expf(-2.f * fabsf(z)), d = 1.f + q;
  if constexpr (FAST) {
    const float r = __builtin_amdgcn_rcpf(d);
    return 4.f * q * r * r;
  }
  return 4.f * q / (d * d);
}
// Phi(z) and e = exp(-z^2 / 2): Abramowitz and Stegun 7.1.26, |error of erf| <= 1.5e-7.
__device__ __forceinline__ float fast_normal(float z, float& e) {
  const float x = fabsf(z) * 0.70710678f;
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * x);
  e = fast_exp(-0.5f * z * z);
  const float tail =
      0.5f * e * t *
      (0.254829592f +
       t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  return z < 0.f ? tail : 1.f - tail;
}

template <bool FAST>
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case 1: return z > 0.f ? z : (z != z ? z : 0.f);
    case 2: {
      if constexpr (FAST) {
        float e;
        return z * fast_normal(z, e);
      }
      return 0.5f * z * erfcf(z * -0.70710678f);
    }
    case 3: return FAST ? z * fast_logistic(z) : z / (1.f + expf(-z));
    case 4: return FAST ? fast_tanh(z) : tanhf(z);
    default: return z;
  }
}

template <bool FAST>
__device__ __forceinline__ float activation_slope(int act, float z) {
  switch (act) {
    case 1: return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case 2: {
      if constexpr (FAST) {
        float e;
        const float p = fast_normal(z, e);
        return p + z * e * 0.39894228f;
      }
      return 0.5f * erfcf(z * -0.70710678f) + z * expf(-0.5f * z * z) * 0.39894228f;
    }
    case 3: {
      const float p = FAST ? fast_logistic(z) : 1.f / (1.f + expf(-z));
      return p * (1.f + z * (1.f - p));
    }
    case 4: return tanh_slope<FAST>(z);
    default: return 1.f;
  }
}

// f(activation code as a constant): one branch around a loop instead of one per element.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    default: f(std::integral_constant<int, 0>{});
  }
}

// ------------------------------------------------------------ products

struct Product {
  int64_t M, N, K;
  const void *a, *b;
  int64_t lda, ldb;
  // what becomes of a sum
  const void *bias, *residual;
  int64_t ldr;
  int act;
  void* out;
  int64_t ldo;
  float* pre;
  // split over k: partial sums [splits][M][N]
  int64_t k_step;  // multiple of the tile's k
  float* partial;
};

template <typename T>
__device__ __forceinline__ void finish(const Product& P, int64_t m, int64_t n, float z) {
  if (P.bias) z += (float)static_cast<const T*>(P.bias)[n];
  if (P.pre) P.pre[m * P.N + n] = z;
  float y = activate<sizeof(T) == 2>(P.act, z);
  if (P.residual) y += (float)static_cast<const T*>(P.residual)[m * P.ldr + n];
  static_cast<T*>(P.out)[m * P.ldo + n] = (T)y;
}

// Tiles of WM x WN waves of (32 MT) x (32 NT) each.  A stage is KB bytes of k per row (64: 32
// elements, 16 in fp32), brought from memory straight into LDS, NB stages deep: while one is
// multiplied the others have arrived or are arriving, with one barrier per stage.  A stage is
// multiplied in steps of 32 bytes of k, and the LDS reads of the next step, at the end those of
// the next stage, are on their way while the matrix instructions of a step run.
//
// An operand by rows lies in LDS as [row][KB bytes of k], its 16-byte chunks swapped by bits of
// the row, so that 16 rows at the same chunk fall on all 64 banks.  One by columns lies as
// [k][rows], as in memory; 16-bit elements are transposed by the LDS read itself (16 lanes read
// 4 k by 16 rows), with groups of chunks swapped by the low bits of k to the same end; fp32
// elements are read one by one.  The loads write LDS in lane order, so the swap is made by
// which chunk a lane asks memory for.

// 16 bytes per lane to lds + 16 * lane.  Written out because the compiler, which cannot tell
// the stages apart, would otherwise wait for every load before the transposing LDS reads; it
// counts none of these, so the waits are wait_loads'.  (m0 is a reserved register: the compiler
// writes it right before a use of its own and keeps no value in it.)
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(p), "s"(lds)
               : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  // vmcnt <= N, and this wave's LDS reads are through (they are: its products used them)
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

__device__ __forceinline__ void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// R rows of an operand's tile, brought by THREADS threads.
template <typename T, int R, bool BYCOL, int KB, int THREADS>
struct Operand {
  static constexpr int E = kPack<T>;            // elements of a chunk
  static constexpr int K = KB / (int)sizeof(T);
  static constexpr int kBytes = R * KB;
  static constexpr int N = kBytes / 16 / THREADS;           // chunks per thread
  static constexpr int kChunks = BYCOL ? R / E : KB / 16;   // chunks of a line of LDS
  const char* p[N];
  int64_t step;

  // What is added (mod 2) to the number of the chunk at row (by rows) or k (by columns).
  __device__ static int swap(int at) {
    if constexpr (!BYCOL) return KB == 64 ? (at >> 2) & 3 : KB == 128 ? (at >> 1) & 7 : at & 15;
    if constexpr (sizeof(T) == 4 || R == 32) return 0;
    return R >= 128 ? (at & 3) << 2 : ((at >> 1) & 1) << 2;
  }
  // Row and first k of a thread's i-th chunk within the tile (by columns: k and first row).
  __device__ static void place(int i, int& row, int& k) {
    const int q = i * THREADS + threadIdx.x;
    const int line = q / kChunks, chunk = ((q % kChunks) ^ swap(line)) * E;
    row = BYCOL ? chunk : line;
    k = BYCOL ? line : chunk;
  }
  // Rows beyond the end read row 0: their sums are not stored.
  __device__ void init(const T* base, int64_t ld, int64_t m0, int64_t M, int64_t k0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int row, k;
      place(i, row, k);
      const int64_t m = m0 + row < M ? m0 + row : 0;
      p[i] = reinterpret_cast<const char*>(BYCOL ? base + (k0 + k) * ld + m
                                                 : base + m * ld + k0 + k);
    }
    step = BYCOL ? (int64_t)K * ld * (int64_t)sizeof(T) : KB;
  }
  // own: the LDS address of this wave's first 64 chunks; on: whether the next load is of the
  // next stage (otherwise of the same one again)
  __device__ void load_one(uint32_t own, int i, bool on) {
    load_to_lds(p[i], own + i * THREADS * 16);
    p[i] += on ? step : 0;
  }
  __device__ void load(uint32_t own, bool on) {
#pragma unroll
    for (int i = 0; i < N; ++i) load_one(own, i, on);
  }
  // The stage at k through registers, at any alignment and of any element type; zeros behind
  // row M and k1.  whole: the tile lies within them.
  template <typename S>
  __device__ static void fetch(Pack<T> (&v)[N], const S* base, int64_t ld, int64_t m0, int64_t M,
                               int64_t k0, int64_t k1, bool whole) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int row, k;
      place(i, row, k);
      const int64_t m = m0 + row, kk = k0 + k;
      const S* at = base + (BYCOL ? kk * ld + m : m * ld + kk);
      const int64_t room = BYCOL ? M - m : k1 - kk;  // elements up to the row's end
      const bool inside = m < M && kk < k1;
      if (std::is_same_v<S, T> && (whole || (inside && room >= E))) {
        v[i] = *reinterpret_cast<const Pack<T>*>(at);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i].v[e] = inside && e < room ? (T)at[e] : (T)0.f;
      }
    }
  }
  __device__ static void put(char* lds, const Pack<T> (&v)[N]) {
    typedef T vec __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int i = 0; i < N; ++i)
      *reinterpret_cast<vec*>(lds + (i * THREADS + threadIdx.x) * 16) =
          __builtin_bit_cast(vec, v[i]);
  }
  // The 32 rows from r0 at step s: 16 bytes of k per lane, lane % 32 the row.
  __device__ static floatx4 fragment(const char* lds, int r0, int s) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (!BYCOL) {
      const int row = r0 + (lane & 31);
      return *reinterpret_cast<const floatx4*>(lds + row * KB + (((2 * s + h) ^ swap(row)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef short shortx4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
      const int j = lane & 15, g = lane >> 4;
      const int k = s * 16 + (g >> 1) * 8 + (j >> 2), row = r0 + (g & 1) * 16 + (j & 3) * 4;
      const char* at = lds + k * (R * 2) + (((row >> 3) ^ swap(k)) << 4) + (row & 7) * 2;
      struct {
        shortx4 lo, hi;
      } v;
      v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)at);
      v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(at + 4 * R * 2));
      return __builtin_bit_cast(floatx4, v);
    } else {
      const float* at = reinterpret_cast<const float*>(lds) + (2 * s + h) * 4 * R + r0 +
                        (lane & 31);
      return floatx4{at[0], at[R], at[2 * R], at[3 * R]};
    }
  }
};

__device__ __forceinline__ void multiply(floatx16& acc, floatx4 a, floatx4 b, f16) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                               __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void multiply(floatx16& acc, floatx4 a, floatx4 b, bf16) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void multiply(floatx16& acc, floatx4 a, floatx4 b, float) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
}

// Columns [n, n + V) of row m.
template <typename T, int V>
__device__ __forceinline__ void finish_pack(const Product& P, int64_t m, int64_t n,
                                            float (&z)[V]) {
  if (P.bias) {
    const Pack<T> b = load_pack<T>(static_cast<const T*>(P.bias), n, P.N, (T)0.f);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] += (float)b.v[i];
  }
  if (P.pre) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const Pack<float> o = {{z[4 * q], z[4 * q + 1], z[4 * q + 2], z[4 * q + 3]}};
      store_pack<float>(P.pre + m * P.N, n + 4 * q, P.N, o);
    }
  }
  with_act(P.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = activate<sizeof(T) == 2>(act, z[i]);
  });
  if (P.residual) {
    const Pack<T> r =
        load_pack<T>(static_cast<const T*>(P.residual) + m * P.ldr, n, P.N, (T)0.f);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] += (float)r.v[i];
  }
  Pack<T> o;
#pragma unroll
  for (int i = 0; i < V; ++i) o.v[i] = (T)z[i];
  store_pack<T>(static_cast<T*>(P.out) + m * P.ldo, n, P.N, o);
}

// Tile of a workgroup: workgroups go round the 8 XCDs, so each XCD gets a run of tiles of its
// own, and within it tiles go in bands of 8 tile rows: neighbours in time share operands in
// the XCD's L2.
__device__ __forceinline__ void tile_of(int64_t tiles_m, int64_t tiles_n, int64_t& tm,
                                        int64_t& tn) {
  const int64_t total = tiles_m * tiles_n, x = blockIdx.x % 8, q = total / 8, rest = total % 8;
  const int64_t id = x * q + (x < rest ? x : rest) + blockIdx.x / 8;
  const int64_t band = id / (8 * tiles_n), first = band * 8;
  const int64_t height = tiles_m - first < 8 ? tiles_m - first : 8;
  const int64_t in = id - band * 8 * tiles_n;
  tm = first + in % height;
  tn = in / height;
}

// 32 rows of a wave's sums in LDS, padded against bank conflicts: floats of a row, bytes.
template <int NT>
constexpr int strip_row() {
  return 32 * NT + 4;
}
template <int NT>
constexpr int strip_bytes() {
  return 32 * strip_row<NT>() * 4;
}

// 32 x 32 sums of a wave into its strip.
__device__ __forceinline__ void write_strip(float* strip, int row, int col,
                                            const floatx16& acc) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    strip[(r / 4 * 8 + lane / 32 * 4 + r % 4) * row + col + lane % 32] = acc[r];
}

// A wave's sums through LDS, 32 rows at a time, so that memory is read and written in 16-byte
// packs.
template <typename T, int MT, int NT>
__device__ __forceinline__ void store_tile(const Product& P, float* strip,
                                           const floatx16 (&acc)[MT][NT], int64_t m0,
                                           int64_t n0) {
  constexpr int V = kPack<T>, kRowPacks = 32 * NT / V, kRow = strip_row<NT>();
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int j = 0; j < NT; ++j) write_strip(strip, kRow, 32 * j, acc[i][j]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 2
    for (int q = lane; q < 32 * kRowPacks; q += 64) {
      const int row = q / kRowPacks, col = q % kRowPacks * V;
      const int64_t m = m0 + 32 * i + row, n = n0 + col;
      if (m >= P.M || n >= P.N) continue;
      float z[V];
#pragma unroll
      for (int v = 0; v < V; v += 4)
        *reinterpret_cast<floatx4*>(z + v) =
            *reinterpret_cast<const floatx4*>(strip + row * kRow + col + v);
      if (P.partial) {
        float* out = P.partial + ((int64_t)blockIdx.y * P.M + m) * P.N;
#pragma unroll
        for (int v = 0; v < V / 4; ++v) {
          const Pack<float> o = {{z[4 * v], z[4 * v + 1], z[4 * v + 2], z[4 * v + 3]}};
          store_pack<float>(out, n + 4 * v, P.N, o);
        }
      } else {
        finish_pack<T, V>(P, m, n, z);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, bool ACOL, bool BCOL, int MT, int NT, int WM, int WN, int KB, int NB>
__global__ void __launch_bounds__(64 * WM * WN, 2) tile_kernel(const Product P) {
  constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, kThreads = 64 * WM * WN, S = KB / 32;
  using A = Operand<T, BM, ACOL, KB, kThreads>;
  using B = Operand<T, BN, BCOL, KB, kThreads>;
  constexpr int kStage = A::kBytes + B::kBytes, K = A::K, kLoads = A::N + B::N;
  constexpr int kStrip = strip_bytes<NT>();
  __shared__ __align__(16) char lds[NB * kStage > WM * WN * kStrip ? NB * kStage
                                                                    : WM * WN * kStrip];
  const int wave = threadIdx.x >> 6;
  const int wm = wave / WN * 32 * MT, wn = wave % WN * 32 * NT;
  int64_t tm, tn;
  tile_of((P.M + BM - 1) / BM, (P.N + BN - 1) / BN, tm, tn);
  const int64_t m0 = tm * BM, n0 = tn * BN;
  const int64_t k0 = P.partial ? blockIdx.y * P.k_step : 0;
  const int64_t k1 = P.partial && k0 + P.k_step < P.K ? k0 + P.k_step : P.K;
  const T* pa = static_cast<const T*>(P.a);
  const T* pb = static_cast<const T*>(P.b);
  const int stages = (int)((k1 - k0) / K);
  floatx16 acc[MT][NT] = {};
  floatx4 fa[2][MT], fb[2][NT];

  // The q-th fragment of a step, in the order the products need them.
  auto read_one = [&](const char* st, int s, int set, int q) {
    if (q == 0)
      fa[set][0] = A::fragment(st, wm, s);
    else if (q <= NT)
      fb[set][q - 1] = B::fragment(st + A::kBytes, wn + 32 * (q - 1), s);
    else
      fa[set][q - NT] = A::fragment(st, wm + 32 * (q - NT), s);
  };
  auto read = [&](const char* st, int s, int set) {
#pragma unroll
    for (int q = 0; q < MT + NT; ++q) read_one(st, s, set, q);
  };
  // The products of a step, with beside(q) between them: a matrix instruction takes 32 cycles,
  // in which the wave can issue 7 others.
  auto products = [&](int set, auto beside) {
#pragma unroll
    for (int q = 0; q < MT * NT; ++q) {
      beside(q);
      multiply(acc[q / NT][q % NT], fa[set][q / NT], fb[set][q % NT], T{});
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto nothing = [](int) {};
  // i-th of n things at the q-th of the products
  auto due = [](int i, int n, int q) { return i * MT * NT / n == q; };

  A la;
  B lb;
  la.init(pa, P.lda, m0, P.M, k0);
  lb.init(pb, P.ldb, n0, P.N, k0);
  const uint32_t own = __builtin_amdgcn_readfirstlane(lds_address(lds) + wave * 1024);
  // Behind the last stage it is loaded again, into buffers that are not read any more: the
  // loop has no branch and its waits are always for the same number of loads.
  if (stages > 0) {
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      la.load(own + t * kStage, t + 1 < stages);
      lb.load(own + t * kStage + A::kBytes, t + 1 < stages);
    }
    wait_loads<(NB - 1) * kLoads>();
    barrier_only();
    read(lds, 0, 0);
  }
  int cur = 0;
  for (int t = 0; t < stages; ++t) {
#pragma unroll
    for (int s = 0; s + 1 < S; ++s)
      products(s & 1, [&](int q) {
#pragma unroll
        for (int i = 0; i < MT + NT; ++i)
          if (due(i, MT + NT, q)) read_one(lds + cur, s + 1, (s + 1) & 1, i);
      });
    // this wave's part of stage t + 1 is there and it has read all of stage t, then everyone
    const int next = cur == (NB - 1) * kStage ? 0 : cur + kStage;
    wait_loads<(NB - 2) * kLoads>();
    barrier_only();
    const bool on = t + NB + 1 < stages;
    products((S - 1) & 1, [&](int q) {
#pragma unroll
      for (int i = 0; i < MT + NT; ++i)
        if (due(i, MT + NT, q)) read_one(lds + next, 0, 0, i);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (due(i, kLoads, q)) {
          if (i < A::N)
            la.load_one(own + cur, i, on);
          else
            lb.load_one(own + cur + A::kBytes, i - A::N, on);
        }
    });
    cur = next;
  }
  wait_loads<0>();
  if (k0 + (int64_t)stages * K < k1) {
    const int64_t k = k0 + (int64_t)stages * K;
    Pack<T> ra[A::N], rb[B::N];
    A::fetch(ra, pa, P.lda, m0, P.M, k, k1, false);
    B::fetch(rb, pb, P.ldb, n0, P.N, k, k1, false);
    __syncthreads();
    A::put(lds, ra);
    B::put(lds + A::kBytes, rb);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < S; ++s) {
      read(lds, s, 0);
      products(0, nothing);
    }
  }
  __syncthreads();
  store_tile<T, MT, NT>(P, reinterpret_cast<float*>(lds + wave * kStrip), acc, m0 + wm, n0 + wn);
}

// Tiles through registers, for operands at any alignment.  A stage is 128 bytes of k, 256 where
// waves share k; stage i + 3 is fetched while stage i is multiplied, and stage i + 1 written to the
// other of two buffers of LDS.  (Two stages' time to arrive is not what the loads get: fetch
// branches by chunk, so that the compiler cannot count them and waits for all that are in flight
// before it writes a stage.)
//
// BM x BN per workgroup, its four waves as WM x WN x WK: waves along k take parts of a stage, and
// their sums are added up at the end.  32 x 32 x (4 along k) is the tile of products too small
// to fill the chip otherwise.  A's and B's elements are multiplied as TC; the products' outputs
// are T.
template <typename T, typename TA, typename TB, bool ACOL, bool BCOL, int WM, int WN, int WK>
__global__ void __launch_bounds__(256, 2) staged_kernel(const Product P) {
  using TC = std::conditional_t<sizeof(TA) == 4, TA, TB>;
  constexpr int KB = WK > 1 ? 256 : 128, BM = 32 * WM, BN = 32 * WN;
  using A = Operand<TC, BM, ACOL, KB, 256>;
  using B = Operand<TC, BN, BCOL, KB, 256>;
  constexpr int kStage = A::kBytes + B::kBytes, K = A::K, kStrip = strip_bytes<1>();
  constexpr int kSteps = KB / 32 / WK;  // of a stage, a wave's
  __shared__ __align__(16) char lds[2 * kStage > 4 * kStrip ? 2 * kStage : 4 * kStrip];
  const int wave = threadIdx.x >> 6;
  const int wm = wave / (WN * WK) * 32, wn = wave / WK % WN * 32, wk = wave % WK;
  int64_t tm, tn;
  tile_of((P.M + BM - 1) / BM, (P.N + BN - 1) / BN, tm, tn);
  const int64_t m0 = tm * BM, n0 = tn * BN;
  const int64_t k0 = P.partial ? blockIdx.y * P.k_step : 0;
  const int64_t k1 = P.partial && k0 + P.k_step < P.K ? k0 + P.k_step : P.K;
  const TA* pa = static_cast<const TA*>(P.a);
  const TB* pb = static_cast<const TB*>(P.b);
  const int stages = (int)((k1 - k0 + K - 1) / K);
  floatx16 acc[1][1] = {};
  Pack<TC> ra[2][A::N], rb[2][B::N];  // stage i in set i % 2
  auto fetch = [&](int set, int stage) {
    if (stage >= stages) return;
    const int64_t k = k0 + (int64_t)stage * K;
    A::fetch(ra[set], pa, P.lda, m0, P.M, k, k1, m0 + BM <= P.M && k + K <= k1);
    B::fetch(rb[set], pb, P.ldb, n0, P.N, k, k1, n0 + BN <= P.N && k + K <= k1);
  };
  auto put = [&](char* st, int set) {
    A::put(st, ra[set]);
    B::put(st + A::kBytes, rb[set]);
  };
  // stage i, in buffer and set SET
  auto step = [&](auto SET, int i) {
    constexpr int set = decltype(SET)::value;
    __syncthreads();  // stage i is there, and everyone is done with stage i - 1
    if (i + 1 < stages) put(lds + (1 - set) * kStage, 1 - set);
    fetch(1 - set, i + 3);
    const char* st = lds + set * kStage;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      multiply(acc[0][0], A::fragment(st, wm, wk * kSteps + s),
               B::fragment(st + A::kBytes, wn, wk * kSteps + s), TC{});
  };
  if (stages > 0) {
    fetch(0, 0);
    fetch(1, 1);
    put(lds, 0);
    fetch(0, 2);
  }
  for (int i = 0; i < stages; i += 2) {
    step(std::integral_constant<int, 0>{}, i);
    if (i + 1 < stages) step(std::integral_constant<int, 1>{}, i + 1);
  }
  __syncthreads();
  if constexpr (WK == 1) {
    store_tile<T, 1, 1>(P, reinterpret_cast<float*>(lds + wave * kStrip), acc, m0 + wm, n0 + wn);
  } else {
    static_assert(WM == 1 && WN == 1, "all waves share one 32 x 32 of sums");
    constexpr int kRow = strip_row<1>();
    float* strips = reinterpret_cast<float*>(lds);
    write_strip(strips + wave * (kStrip / 4), kRow, 0, acc[0][0]);
    __syncthreads();
    const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4;
    floatx4 z = *reinterpret_cast<const floatx4*>(strips + row * kRow + col);
#pragma unroll
    for (int w = 1; w < WK; ++w)
      z += *reinterpret_cast<const floatx4*>(strips + w * (kStrip / 4) + row * kRow + col);
    const int64_t m = m0 + row, n = n0 + col;
    if (m >= P.M) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i >= P.N) continue;
      if (P.partial)
        P.partial[((int64_t)blockIdx.y * P.M + m) * P.N + n + i] = z[i];
      else
        finish<T>(P, m, n + i, z[i]);
    }
  }
}

// The first half of N lanes' values in lanes without bit B, the second in those with it, each with
// the partner's added; the values left are the first ones of the array.
template <int B, int N>
__device__ __forceinline__ void halve(float (&z)[N], int lane) {
  constexpr int H = N * B / 64;  // values that stay
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const bool up = lane & B;
    const float keep = up ? z[i + H] : z[i], give = up ? z[i] : z[i + H];
    z[i] = keep + lane_xor<B>(give);
  }
}

// Few rows of x: one to MR of them against RN rows of W per workgroup, whose threads take the
// packs of k in turn and add up at the end.  Memory-bound (W is read once; bf16 4096 x 4096 7.0
// us, 4.8 TB/s, fp32 13.3 us), any alignment; a tile of 32 rows would be empty but for MR.  Two
// steps of k are in flight, one where 8 rows of x take the registers.
template <typename T, int MR, int RN>
__global__ void __launch_bounds__(256) few_rows_kernel(const Product P) {
  constexpr int V = kPack<T>, U = MR > 4 ? 1 : 2;
  __shared__ float sums[4][MR * RN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * RN;
  const T *x[MR], *w[RN];
#pragma unroll
  for (int i = 0; i < MR; ++i) x[i] = static_cast<const T*>(P.a) + (i < P.M ? i : 0) * P.lda;
#pragma unroll
  for (int j = 0; j < RN; ++j)
    w[j] = static_cast<const T*>(P.b) + (n0 + j < P.N ? n0 + j : n0) * P.ldb;
  float acc[MR][RN] = {};
  for (int64_t k0 = (int64_t)threadIdx.x * V; k0 - lane * V < P.K; k0 += U * 256 * V) {
    Raw xr[U][MR], wr[U][RN];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + u * 256 * V;
#pragma unroll
      for (int j = 0; j < RN; ++j) wr[u][j] = load_raw<T>(w[j], k, P.K);
#pragma unroll
      for (int i = 0; i < MR; ++i) xr[u][i] = load_raw<T>(x[i], k, P.K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + u * 256 * V;
      Pack<T> xp[MR];
#pragma unroll
      for (int i = 0; i < MR; ++i) xp[i] = taken<T>(xr[u][i], k, P.K, (T)0.f);
#pragma unroll
      for (int j = 0; j < RN; ++j) {
        const Pack<T> wp = taken<T>(wr[u][j], k, P.K, (T)0.f);
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
          for (int v = 0; v < V; ++v) acc[i][j] += (float)xp[i].v[v] * (float)wp.v[v];
      }
    }
  }
  // each lane's MR * RN sums over the wave: a step adds one half of them in each of two lanes,
  // until a lane has one, its own
  constexpr int N = MR * RN, G = 64 / N;
  float z[N];
#pragma unroll
  for (int q = 0; q < N; ++q) z[q] = acc[q / RN][q % RN];
  halve<32>(z, lane);
  if constexpr (N > 2) halve<16>(z, lane);
  if constexpr (N > 4) halve<8>(z, lane);
  if constexpr (N > 8) halve<4>(z, lane);
  if constexpr (N > 16) halve<2>(z, lane);
  z[0] = lanes_sum<G>(z[0]);
  if (lane % G == 0) sums[wave][lane / G] = z[0];
  __syncthreads();
  const int i = threadIdx.x / RN, j = threadIdx.x % RN;
  if (i < MR && i < P.M && n0 + j < P.N)
    finish<T>(P, i, n0 + j,
              sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] +
                  sums[3][threadIdx.x]);
}

// The splits' sums, in their order, and what becomes of them.
template <typename T>
__global__ void __launch_bounds__(256) join_splits_kernel(const Product P, int64_t splits) {
  const int64_t count = P.M * P.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count;
       i += (int64_t)gridDim.x * 256) {
    float z = 0.f;
#pragma unroll 4
    for (int64_t s = 0; s < splits; ++s) z += P.partial[s * count + i];
    const int64_t m = i / P.N;
    finish<T>(P, m, i - m * P.N, z);
  }
}

// ------------------------------------------------------------ dz and db

// Rows per partial column sum: up to 64, fewer where that leaves CUs idle; up to 32 rows need
// no second launch.
int64_t sum_rows(int64_t rows, int64_t n_out) {
  if (rows <= 32) return 32;
  const int64_t blocks_n = (n_out + 511) / 512;
  const int64_t per = (rows * blocks_n + 511) / 512;
  return per < 8 ? 8 : per > 64 ? 64 : (per + 7) / 8 * 8;
}

// dz = dy a'(z), rounded to TZ, and the partial column sums of dz before it is rounded.
// Memory-bound (bf16 8192 x 4096: 268 MB in 53 us, 5.1 TB/s).  A workgroup takes TC packs of
// columns of sum_rows rows; its 256 / TC rows of threads add up through LDS in their order.
template <typename T, typename TZ, int TC, bool SHORT>
__global__ void __launch_bounds__(256) slope_kernel(const LinearArgs A, TZ* dz, int64_t ldz,
                                                    float* partial, int64_t per) {
  constexpr int V = kPack<T>, TR = 256 / TC;
  __shared__ float sums[V][256];
  const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
  const int64_t blocks_n = (A.n_out + TC * V - 1) / (TC * V);
  const int64_t n = (blockIdx.x % blocks_n * TC + tc) * V;
  const int64_t m0 = blockIdx.x / blocks_n * per;
  const int64_t m1 = m0 + per < A.rows ? m0 + per : A.rows;
  float s[V] = {};
  with_act(A.act, [&](auto act) {
    if (n >= A.n_out) return;
    // two rows' loads in flight together
    for (int64_t first = m0 + tr; first < m1; first += 2 * TR) {
      Raw graw[2], zraw[2][V / 4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t m = first + j * TR < m1 ? first + j * TR : first;
        graw[j] = load_raw<T, SHORT>(static_cast<const T*>(A.dy) + m * A.lddy, n, A.n_out);
        if constexpr (act != 0)
#pragma unroll
          for (int q = 0; q < V / 4; ++q)
            zraw[j][q] = load_raw<float, SHORT>(A.pre_in + m * A.n_out, n + 4 * q, A.n_out);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t m = first + j * TR;
        if (m >= m1) break;
        const Pack<T> g = taken<T, SHORT>(graw[j], n, A.n_out, (T)0.f);
        float v[V];
        if constexpr (act != 0) {
#pragma unroll
          for (int q = 0; q < V / 4; ++q) {
            const Pack<float> z = taken<float, SHORT>(zraw[j][q], n + 4 * q, A.n_out, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              v[4 * q + i] = (float)g.v[4 * q + i] *
                             activation_slope<sizeof(T) == 2>(act, z.v[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = (float)g.v[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += v[i];
        if (!dz) continue;
#pragma unroll
        for (int q = 0; q < V; q += kPack<TZ>) {
          Pack<TZ> o;
#pragma unroll
          for (int i = 0; i < kPack<TZ>; ++i) o.v[i] = (TZ)v[q + i];
          store_pack<TZ>(dz + m * ldz, n + q, A.n_out, o);
        }
      }
    }
  });
  if (!partial && !A.dbias) return;
#pragma unroll
  for (int i = 0; i < V; ++i) sums[i][threadIdx.x] = s[i];
  __syncthreads();
  for (int q = threadIdx.x; q < TC * V; q += 256) {
    const int64_t col = blockIdx.x % blocks_n * TC * V + q;
    if (col >= A.n_out) continue;
    float v = 0.f;
#pragma unroll
    for (int r = 0; r < TR; ++r) v += sums[q % V][r * TC + q / V];
    if (partial)
      partial[blockIdx.x / blocks_n * A.n_out + col] = v;
    else
      static_cast<T*>(A.dbias)[col] = (T)v;  // all rows were this workgroup's
  }
}

template <typename T>
__global__ void __launch_bounds__(256) join_sums_kernel(int64_t n_out, int64_t parts,
                                                        const float* partial, T* db) {
  __shared__ float sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (n < n_out)
#pragma unroll 8  // loads in flight together; the sum keeps its order
    for (int64_t p = wave; p < parts; p += 4) s += partial[p * n_out + n];
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && n < n_out)
    db[n] = (T)(sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]);
}

// ------------------------------------------------------------ alignment

// Rows to a stride that keeps them on 16-byte chunks; what lies behind a row's end is not
// written and reaches no result (a product's rows and columns behind the end are not stored).
// A wave takes 63 chunks of a row: its lanes read the 64 aligned chunks that hold them, each
// once, and shift them by the row's offset, the higher bytes coming from the next lane (reads
// at the elements' own alignment took 1.5 times as long).  A chunk that holds an element lies
// in the same page, whatever else it holds.
template <typename T>
__global__ void __launch_bounds__(256) align_kernel(int64_t rows, int64_t cols, const T* src,
                                                    int64_t ld, T* dst, int64_t ldd) {
  constexpr int V = kPack<T>, kRowsPerWave = 4;
  typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
  const int64_t blocks_n = (cols + 63 * V - 1) / (63 * V);
  const int64_t c = (blockIdx.x % blocks_n * 63 + lane) * V;  // this lane's chunk of dst
  const int64_t r0 = blockIdx.x / blocks_n * (4 * kRowsPerWave) + (threadIdx.x >> 6);
  uintx4 v[kRowsPerWave];
  uint32_t off[kRowsPerWave];
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    v[i] = uintx4{0, 0, 0, 0};
    const int64_t r = r0 + 4 * i;
    if (r >= rows) continue;
    const uintptr_t row = reinterpret_cast<uintptr_t>(src + r * ld);
    off[i] = (uint32_t)(row & 15);
    const uintptr_t chunk = (row & ~(uintptr_t)15) + (uintptr_t)(c * (int64_t)sizeof(T));
    if (chunk < row + (uintptr_t)(cols * (int64_t)sizeof(T)))
      v[i] = *reinterpret_cast<const uintx4*>(chunk);
  }
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    const int64_t r = r0 + 4 * i;
    if (r >= rows) continue;  // the same for the whole wave
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = v[i][j];
      w[4 + j] = (uint32_t)__shfl_down((int)v[i][j], 1);
    }
    const uint32_t words = off[i] >> 2, bits = (off[i] & 3) * 8;
    uintx4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t lo = w[j], hi = w[j + 1];
#pragma unroll
      for (int q = 1; q < 4; ++q)
        if (words == (uint32_t)q) {
          lo = w[j + q];
          hi = w[j + q + 1 < 8 ? j + q + 1 : 7];
        }
      o[j] = __builtin_amdgcn_alignbit(hi, lo, bits);
    }
    if (lane < 63 && c < cols)
      store_pack<T>(dst + r * ldd, c, cols, __builtin_bit_cast(Pack<T>, o));
  }
}

// ------------------------------------------------------------ launches

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

size_t product_workspace(int dtype, bool acol, int64_t M, int64_t N, int64_t K) {
  size_t most = 0;
  for (bool direct : {false, true}) {
    const Plan p = plan_of(dtype, direct, acol, M, N, K);
    if (p.splits > 1) most = std::max(most, (size_t)p.splits * (size_t)M * (size_t)N * 4);
  }
  return round256(most);
}

// Rows as the products read them.  padded: there is room behind the last row's end.
struct Rows {
  const void* p;
  int64_t ld;
  bool aligned, padded;
};

Rows rows_of(const void* p, int64_t ld, int64_t rows, size_t bytes) {
  return {p, ld,
          reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows < 2 || ld * (int64_t)bytes % 16 == 0),
          false};
}

template <typename T>
int align_rows(Rows& r, int64_t rows, int64_t cols, unsigned char* to, hipStream_t st) {
  if (r.aligned || !to) return 0;
  const int64_t ldd = aligned_stride(cols, sizeof(T));
  const int64_t blocks = (rows + 15) / 16 * ((cols + 63 * kPack<T> - 1) / (63 * kPack<T>));
  if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
  align_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(
      rows, cols, static_cast<const T*>(r.p), r.ld, reinterpret_cast<T*>(to), ldd);
  r = {to, ldd, true, true};
  return (int)hipGetLastError();
}

// T: the outputs' type and B's; TA: A's, T or fp32.
template <typename T, typename TA, bool ACOL, bool BCOL>
int launch_product(Product p, const Rows& a, const Rows& b, unsigned char* ws, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return 0;
  p.a = a.p;
  p.lda = a.ld;
  p.b = b.p;
  p.ldb = b.ld;
  if constexpr (std::is_same_v<T, TA> && !ACOL && !BCOL)
    if (few_rows((int64_t)sizeof(T), p.M, p.N, p.K)) {
      const int64_t blocks = (p.N + 3) / 4;
      if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
      if (p.M == 1)
        few_rows_kernel<T, 1, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
      else if (p.M == 2)
        few_rows_kernel<T, 2, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
      else if (p.M <= 4)
        few_rows_kernel<T, 4, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
      else
        few_rows_kernel<T, 8, 4><<<dim3((unsigned)blocks), 256, 0, st>>>(p);
      return (int)hipGetLastError();
    }
  const bool direct = std::is_same_v<T, TA> &&
                      on_chunks(kPack<T>, ACOL, p.M, a.aligned, a.padded) &&
                      on_chunks(kPack<T>, BCOL, p.N, b.aligned, b.padded);
  const Plan plan = plan_of(sizeof(TA) == 4 ? 0 : 1, direct, ACOL, p.M, p.N, p.K);
  const int64_t tiles = tiles_of(p.M, p.N, plan.tile);
  p.k_step = plan.k_step;
  p.partial = plan.splits > 1 ? reinterpret_cast<float*>(ws) : nullptr;
  if (tiles > INT32_MAX / 256 || p.K / 16 > INT32_MAX) return (int)hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)tiles, (unsigned)plan.splits);
  // Bytes of k of a 64 tile's stages.  Such products wait for memory rather than multiply, and
  // twice the bytes in flight serve 16-bit rows; fp32 multiplies longer than that, and with both
  // operands by columns a stage has whole lines anyway.  us at M x N x K, 64 | 128 bytes, bf16: x
  // W^T 1024^3 9.9 | 8.2, 768 x 384 x 8192 24.0 | 18.4, 6736 x 624 x 1536 34 | 26; W by columns
  // 3816 x 320 x 3352 32.9 | 29.8, 8192 x 512 x 512 10.7 | 11.4; both 1536 x 6736 x 624 28.5 |
  // 31.9; fp32 the same.
  constexpr int kSmallStage = sizeof(T) == 2 && !ACOL ? 128 : 64;
  if constexpr (std::is_same_v<T, TA>) {
    if (plan.tile == 256)
      tile_kernel<T, ACOL, BCOL, 4, 2, 2, 4, 128, 2><<<grid, 512, 0, st>>>(p);
    else if (plan.tile == 128)
      tile_kernel<T, ACOL, BCOL, 2, 2, 2, 2, 64, 3><<<grid, 256, 0, st>>>(p);
    else if (plan.tile == 64 && direct)
      tile_kernel<T, ACOL, BCOL, 1, 1, 2, 2, kSmallStage, 3><<<grid, 256, 0, st>>>(p);
  }
  if (plan.tile == 64 && !direct)
    staged_kernel<T, TA, T, ACOL, BCOL, 2, 2, 1><<<grid, 256, 0, st>>>(p);
  else if (plan.tile == 32)
    staged_kernel<T, TA, T, ACOL, BCOL, 1, 1, 4><<<grid, 256, 0, st>>>(p);
  int rc = (int)hipGetLastError();
  if (rc || plan.splits == 1) return rc;
  const int64_t blocks = std::min<int64_t>((p.M * p.N + 255) / 256, 1 << 16);
  join_splits_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(p, plan.splits);
  return (int)hipGetLastError();
}

// The workspace: [dz | partial sums of db | x and the weight in aligned rows | the products'
// splits].  dz and the sums in the backward only, the aligned rows by copies_rows.
struct Layout {
  size_t sums = 0, x = 0, w = 0, splits = 0, end = 0;
  bool aligns = false;
};
Layout layout_of(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool training) {
  Layout L;
  const size_t b = element_bytes(dtype);
  if (training) {
    const int64_t per = sum_rows(rows, n_out);
    const size_t z = exact_dz(dtype, rows, n_out) ? 4 : b;
    L.sums = round256((size_t)rows * (size_t)aligned_stride(n_out, z) * z);
    L.x = L.sums + round256((size_t)((rows + per - 1) / per) * (size_t)n_out * 4);
  }
  L.aligns = copies_rows(dtype, rows, n_in, n_out);
  const size_t row = (size_t)aligned_stride(n_in, b) * b;
  L.w = L.x + (L.aligns ? round256((size_t)rows * row) : 0);
  L.splits = L.w + (L.aligns ? round256((size_t)n_out * row) : 0);
  const int tz = training && exact_dz(dtype, rows, n_out) ? 0 : dtype;
  L.end = L.splits + (training ? std::max({product_workspace(dtype, false, rows, n_in, n_out),
                                           product_workspace(dtype, true, n_out, n_in, rows),
                                           product_workspace(tz, false, rows, n_in, n_out),
                                           product_workspace(tz, true, n_out, n_in, rows)})
                               : product_workspace(dtype, false, rows, n_out, n_in));
  return L;
}

}  // namespace

size_t linear_workspace(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool training) {
  return layout_of(dtype, rows, n_in, n_out, training).end;
}

int launch_linear(int dtype, const LinearArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Layout L = layout_of(dtype, a.rows, a.n_in, a.n_out, false);
  const size_t b = element_bytes(dtype);
  Product p{};
  p.M = a.rows;
  p.N = a.n_out;
  p.K = a.n_in;
  p.bias = a.bias;
  p.residual = a.residual;
  p.ldr = a.ldr;
  p.act = a.act;
  p.out = a.y;
  p.ldo = a.ldy;
  p.pre = a.pre;
  Rows x = rows_of(a.x, a.ldx, a.rows, b), w = rows_of(a.weight, a.ldw, a.n_out, b);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    int rc;
    if ((rc = align_rows<T>(x, a.rows, a.n_in, L.aligns ? a.ws + L.x : nullptr, st)) ||
        (rc = align_rows<T>(w, a.n_out, a.n_in, L.aligns ? a.ws + L.w : nullptr, st)))
      return rc;
    return launch_product<T, T, false, false>(p, x, w, a.ws + L.splits, st);
  });
}

int launch_linear_backward(int dtype, const LinearArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Layout L = layout_of(dtype, a.rows, a.n_in, a.n_out, true);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    Rows x = rows_of(a.x, a.ldx, a.rows, sizeof(T));
    Rows w = rows_of(a.weight, a.ldw, a.n_out, sizeof(T));
    Rows dz = rows_of(a.dy, a.lddy, a.rows, sizeof(T));
    // without an activation dz is dy, unless its rows are worth aligning
    const bool own = (a.dx || a.dweight) &&
                     (a.act != 0 || (!dz.aligned && worth_aligning(a.rows, a.n_in, a.n_out)));
    const bool exact = own && a.act != 0 && exact_dz(dtype, a.rows, a.n_out);
    if (own) dz = {a.ws, aligned_stride(a.n_out, exact ? 4 : sizeof(T)), true, true};
    const int64_t per = sum_rows(a.rows, a.n_out), parts = (a.rows + per - 1) / per;
    float* sums = a.dbias && parts != 1 ? reinterpret_cast<float*>(a.ws + L.sums) : nullptr;
    int rc = 0;
    if ((own || a.dbias) && parts > 0 && a.n_out > 0) {
      const int64_t packs = (a.n_out + kPack<T> - 1) / kPack<T>;
      auto slope = [&](auto tc, auto is_short, auto tz) {
        constexpr int TC = decltype(tc)::value;
        constexpr bool SHORT = decltype(is_short)::value;
        using TZ = decltype(tz);
        const int64_t blocks = parts * ((packs + TC - 1) / TC);
        if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
        slope_kernel<T, TZ, TC, SHORT><<<dim3((unsigned)blocks), 256, 0, st>>>(
            a, own ? reinterpret_cast<TZ*>(a.ws) : nullptr, dz.ld, sums, per);
        return (int)hipGetLastError();
      };
      auto by_width = [&](auto tz) {
        if (a.n_out < kPack<T>)
          return slope(std::integral_constant<int, 8>{}, std::true_type{}, tz);
        return packs <= 8 ? slope(std::integral_constant<int, 8>{}, std::false_type{}, tz)
                          : slope(std::integral_constant<int, 64>{}, std::false_type{}, tz);
      };
      rc = exact ? by_width(float{}) : by_width(T{});
      if (rc) return rc;
    }
    if (a.dbias && parts != 1 && a.n_out > 0) {
      const int64_t blocks = (a.n_out + 63) / 64;
      if (blocks > INT32_MAX / 256) return (int)hipErrorInvalidConfiguration;
      join_sums_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(a.n_out, parts, sums,
                                                                 static_cast<T*>(a.dbias));
      if ((rc = (int)hipGetLastError())) return rc;
    }
    Product p{};
    if (a.dx) {
      if ((rc = align_rows<T>(w, a.n_out, a.n_in, L.aligns ? a.ws + L.w : nullptr, st)))
        return rc;
      p.M = a.rows;
      p.N = a.n_in;
      p.K = a.n_out;
      p.out = a.dx;
      p.ldo = a.lddx;
      rc = exact ? launch_product<T, float, false, true>(p, dz, w, a.ws + L.splits, st)
                 : launch_product<T, T, false, true>(p, dz, w, a.ws + L.splits, st);
      if (rc) return rc;
    }
    if (a.dweight) {
      if ((rc = align_rows<T>(x, a.rows, a.n_in, L.aligns ? a.ws + L.x : nullptr, st)))
        return rc;
      p.M = a.n_out;
      p.N = a.n_in;
      p.K = a.rows;
      p.out = a.dweight;
      p.ldo = a.lddw;
      rc = exact ? launch_product<T, float, true, true>(p, dz, x, a.ws + L.splits, st)
                 : launch_product<T, T, true, true>(p, dz, x, a.ws + L.splits, st);
    }
    return rc;
  });
}

}  // namespace vqc
