// linear_device.h -- what the linear layers' kernels share: activations, what becomes of a
// product's sums, tiles of the matrix instructions fed through LDS (linear.hip holds floating
// elements, linear_quantized.hip 8-bit integers).
#pragma once

#include <cmath>
#include <type_traits>

#include "layers_device.h"

namespace vqc {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
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

// One of integers: a sum stands for itself times its row's and its column's step.  Its partial
// sums are integers in the places of the floats.
struct ScaledProduct : Product {
  const float *a_scales, *b_scales;
};

// By the type of the elements multiplied: the arguments, and 32 x 32 sums of a wave.
template <typename E>
using ProductOf = std::conditional_t<std::is_same_v<E, int8_t>, ScaledProduct, Product>;
template <typename E>
using SumsOf = std::conditional_t<std::is_same_v<E, int8_t>, intx16, floatx16>;

template <typename T>
__device__ __forceinline__ void finish(const Product& P, int64_t m, int64_t n, float z) {
  if (P.bias) z += (float)static_cast<const T*>(P.bias)[n];
  if (P.pre) P.pre[m * P.N + n] = z;
  float y = activate<sizeof(T) == 2>(P.act, z);
  if (P.residual) y += (float)static_cast<const T*>(P.residual)[m * P.ldr + n];
  static_cast<T*>(P.out)[m * P.ldo + n] = (T)y;
}
// The sum is rounded to fp32 once, and nothing behind it is contracted: it does not matter how a
// sum was put together, nor which kernel does.
__device__ __forceinline__ float scaled(float sum, float row_step, float step, float bias) {
#pragma clang fp contract(off)
  const float z = sum * row_step * step;
  return z + bias;
}
__device__ __forceinline__ float plus(float y, float residual) {
#pragma clang fp contract(off)
  return y + residual;
}
template <typename T>
__device__ __forceinline__ void finish(const ScaledProduct& P, int64_t m, int64_t n, int sum) {
  const float bias = P.bias ? (float)static_cast<const T*>(P.bias)[n] : 0.f;
  float y = activate<sizeof(T) == 2>(P.act,
                                     scaled((float)sum, P.a_scales[m], P.b_scales[n], bias));
  if (P.residual) y = plus(y, (float)static_cast<const T*>(P.residual)[m * P.ldr + n]);
  static_cast<T*>(P.out)[m * P.ldo + n] = (T)y;
}
template <typename T>
__device__ __forceinline__ void finish_raw(const Product& P, int64_t m, int64_t n, float raw) {
  finish<T>(P, m, n, raw);
}
template <typename T>
__device__ __forceinline__ void finish_raw(const ScaledProduct& P, int64_t m, int64_t n,
                                           float raw) {
  finish<T>(P, m, n, __builtin_bit_cast(int, raw));
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

// R rows of an operand's tile, brought by THREADS threads.  LIMIT: chunks behind `limit` are read
// there instead (they are multiplied by zeros).
template <typename T, int R, bool BYCOL, int KB, int THREADS, bool LIMIT = false>
struct Operand {
  static constexpr int E = kPack<T>;            // elements of a chunk
  static constexpr int K = KB / (int)sizeof(T);
  static constexpr int kBytes = R * KB;
  static constexpr int N = kBytes / 16 / THREADS;           // chunks per thread
  static constexpr int kChunks = BYCOL ? R / E : KB / 16;   // chunks of a line of LDS
  const char* p[N];
  const char* limit = nullptr;
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
    load_to_lds(LIMIT && p[i] > limit ? limit : p[i], own + i * THREADS * 16);
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

__device__ __forceinline__ void multiply(intx16& acc, floatx4 a, floatx4 b, int8_t) {
  acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(intx4, a),
                                              __builtin_bit_cast(intx4, b), acc, 0, 0, 0);
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

template <typename T, int V>
__device__ __forceinline__ void finish_pack(const ScaledProduct& P, int64_t m, int64_t n,
                                            float (&z)[V]) {
  const float s = P.a_scales[m];
  Pack<T> b{}, r{}, o;
  if (P.bias) b = load_pack<T>(static_cast<const T*>(P.bias), n, P.N, (T)0.f);
  if (P.residual)
    r = load_pack<T>(static_cast<const T*>(P.residual) + m * P.ldr, n, P.N, (T)0.f);
#pragma unroll
  for (int q = 0; q < V; q += 4) {
    const Pack<float> w = load_pack<float>(P.b_scales, n + q, P.N, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      z[q + i] = scaled((float)__builtin_bit_cast(int, z[q + i]), s, w.v[i], (float)b.v[q + i]);
  }
  with_act(P.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = activate<sizeof(T) == 2>(act, z[i]);
  });
#pragma unroll
  for (int i = 0; i < V; ++i) o.v[i] = (T)(P.residual ? plus(z[i], (float)r.v[i]) : z[i]);
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

// 32 x 32 sums of a wave into its strip (integers as they are).
template <typename ACC>
__device__ __forceinline__ void write_strip(float* strip, int row, int col, const ACC& acc) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const auto sum = acc[r];  // (the bits of a vector's element itself would be the first one's)
    strip[(r / 4 * 8 + lane / 32 * 4 + r % 4) * row + col + lane % 32] =
        __builtin_bit_cast(float, sum);
  }
}

// A wave's sums through LDS, 32 rows at a time, so that memory is read and written in 16-byte
// packs.
template <typename T, int MT, int NT, typename ARGS, typename ACC>
__device__ __forceinline__ void store_any(const ARGS& P, float* strip, const ACC (&acc)[MT][NT],
                                           int64_t m0, int64_t n0) {
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

template <typename T, int MT, int NT, typename ACC>
__device__ __forceinline__ void store_tile(const Product& P, float* strip, const ACC (&acc)[MT][NT],
                                           int64_t m0, int64_t n0) {
  store_any<T, MT, NT>(P, strip, acc, m0, n0);
}

// Sums of integers, where all columns are there: a lane's columns are the same in every row, so that
// the channels' steps and the bias are read once, and the rows' steps and the residual two rows
// ahead.  Neither loop is unrolled (the sums move up instead): the code runs once for a tile, and
// instructions that have not run yet come from memory.
template <typename T, int MT, int NT, typename ACC>
__device__ __forceinline__ void store_tile(const ScaledProduct& P, float* strip,
                                           const ACC (&sums)[MT][NT], int64_t m0, int64_t n0) {
  if (P.partial || n0 + 32 * NT > P.N) {
    store_any<T, MT, NT>(P, strip, sums, m0, n0);
    return;
  }
  constexpr int V = kPack<T>, kRowPacks = 32 * NT / V, kRow = strip_row<NT>();
  constexpr int R = 64 / kRowPacks, kPasses = MT * 32 / R;  // rows at a time
  const int lane = threadIdx.x & 63, col = lane % kRowPacks * V, r = lane / kRowPacks;
  const int64_t n = n0 + col;
  float step[V], bias[V];
  Pack<T> b{};
  if (P.bias) b = *reinterpret_cast<const Pack<T>*>(static_cast<const T*>(P.bias) + n);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    step[v] = P.b_scales[n + v];
    bias[v] = P.bias ? (float)b.v[v] : 0.f;
  }
  struct Ahead {
    float step;
    Pack<T> residual;
  };
  auto row = [&](int pass) { return m0 + pass * R + r; };
  auto load = [&](int pass) {
    Ahead a{};
    const int64_t m = row(pass < kPasses ? pass : 0), in = m < P.M ? m : P.M - 1;
    a.step = P.a_scales[in];
    if (P.residual)
      a.residual =
          *reinterpret_cast<const Pack<T>*>(static_cast<const T*>(P.residual) + in * P.ldr + n);
    return a;
  };
  ACC acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = sums[i][j];
  Ahead now = load(0), next = load(1);
  int pass = 0;
#pragma unroll 1
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int j = 0; j < NT; ++j) write_strip(strip, kRow, 32 * j, acc[0][j]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int it = 0; it < 32 / R; ++it, ++pass) {
      const Ahead last = load(pass + 2);
      float z[V];
#pragma unroll
      for (int v = 0; v < V; v += 4)
        *reinterpret_cast<floatx4*>(z + v) =
            *reinterpret_cast<const floatx4*>(strip + (it * R + r) * kRow + col + v);
#pragma unroll
      for (int v = 0; v < V; ++v)
        z[v] = scaled((float)__builtin_bit_cast(int, z[v]), now.step, step[v], bias[v]);
      with_act(P.act, [&](auto act) {
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = activate<sizeof(T) == 2>(act, z[v]);
      });
      Pack<T> o;
#pragma unroll
      for (int v = 0; v < V; ++v)
        o.v[v] = (T)(P.residual ? plus(z[v], (float)now.residual.v[v]) : z[v]);
      const int64_t m = row(pass);
      if (m < P.M)
        *reinterpret_cast<Pack<T>*>(static_cast<T*>(P.out) + m * P.ldo + n) = o;
      now = next;
      next = last;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k + 1 < MT; ++k)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[k][j] = acc[k + 1][j];
  }
}

// The products' outputs are T, the elements multiplied E.
template <typename T, bool ACOL, bool BCOL, int MT, int NT, int WM, int WN, int KB, int NB,
          typename E = T>
__global__ void __launch_bounds__(64 * WM * WN, 2) tile_kernel(const ProductOf<E> P) {
  constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, kThreads = 64 * WM * WN, S = KB / 32;
  // a last stage that k ends in: integers in full (A's rows go on with zeros), others on their own
  constexpr bool kFull = std::is_same_v<E, int8_t>;
  using A = Operand<E, BM, ACOL, KB, kThreads>;
  using B = Operand<E, BN, BCOL, KB, kThreads, kFull>;
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
  const E* pa = static_cast<const E*>(P.a);
  const E* pb = static_cast<const E*>(P.b);
  const int stages = (int)((k1 - k0 + (kFull ? K - 1 : 0)) / K);
  SumsOf<E> acc[MT][NT] = {};
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
      multiply(acc[q / NT][q % NT], fa[set][q / NT], fb[set][q % NT], E{});
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
  if constexpr (kFull)
    lb.limit = reinterpret_cast<const char*>(pb + (P.N - 1) * P.ldb + (P.K - 1) / B::E * B::E);
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
  if (!kFull && k0 + (int64_t)stages * K < k1) {
    const int64_t k = k0 + (int64_t)stages * K;
    Pack<E> ra[A::N], rb[B::N];
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
__global__ void __launch_bounds__(256, 2) staged_kernel(const ProductOf<TA> P) {
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
  SumsOf<TC> acc[1][1] = {};
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
    using Sum4 = std::conditional_t<std::is_same_v<TC, int8_t>, intx4, floatx4>;
    auto part = [&](int w) {
      return __builtin_bit_cast(
          Sum4, *reinterpret_cast<const floatx4*>(strips + w * (kStrip / 4) + row * kRow + col));
    };
    Sum4 sum = part(0);
#pragma unroll
    for (int w = 1; w < WK; ++w) sum += part(w);
    const floatx4 z = __builtin_bit_cast(floatx4, sum);
    const int64_t m = m0 + row, n = n0 + col;
    if (m >= P.M) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i >= P.N) continue;
      if (P.partial)
        P.partial[((int64_t)blockIdx.y * P.M + m) * P.N + n + i] = z[i];
      else
        finish_raw<T>(P, m, n + i, z[i]);
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

}  // namespace
}  // namespace vqc
