// linear.hip -- linear layers: y = a(x W^T + b) + r and its gradients.
//
//   z = x W^T + b, y = a(z) + r
//   dz = dy a'(z), dx = dz W, dW = dz^T x, db = sum_rows dz
//
// Three products C[m, n] = sum_k A(m, k) B(n, k) that differ in which operand's k runs along
// its rows: forward x and W by rows; dx takes W by columns; dW takes both by columns.
#include <algorithm>
#include <type_traits>

#include "layers.h"
#include "layers_device.h"

namespace vqc {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------ activations

__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case 1: return z > 0.f ? z : (z != z ? z : 0.f);
    case 2: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    case 3: return z / (1.f + expf(-z));
    case 4: return tanhf(z);
    default: return z;
  }
}

__device__ __forceinline__ float activation_slope(int act, float z) {
  switch (act) {
    case 1: return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case 2:
      return 0.5f * (1.f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
    case 3: {
      const float p = 1.f / (1.f + expf(-z));
      return p * (1.f + z * (1.f - p));
    }
    case 4: {
      const float t = tanhf(z);
      return 1.f - t * t;
    }
    default: return 1.f;
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
  float y = activate(P.act, z);
  if (P.residual) y += (float)static_cast<const T*>(P.residual)[m * P.ldr + n];
  static_cast<T*>(P.out)[m * P.ldo + n] = (T)y;
}

// acc += A B^T over 16 k of 32 x 32: a lane holds 8 adjacent k of row lane % 32, the lower
// half-wave the first 8.  In fp32 instruction j takes the j-th of both halves.
__device__ __forceinline__ void mma32(floatx16& acc, const f16* a, const f16* b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const f16x8*)a, *(const f16x8*)b, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma32(floatx16& acc, const bf16* a, const bf16* b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)a, *(const bf16x8*)b, acc, 0, 0,
                                                0);
}
__device__ __forceinline__ void mma32(floatx16& acc, const float* a, const float* b) {
  const floatx4 a0 = *(const floatx4*)a, a1 = *(const floatx4*)(a + 4);
  const floatx4 b0 = *(const floatx4*)b, b1 = *(const floatx4*)(b + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a0[j], b0[j], acc, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a1[j], b1[j], acc, 0, 0, 0);
}

constexpr int kTile = 64, kTileK = 32;

// A 64 x 32 tile of one operand: from memory into registers, and from there into LDS as
// rows of k.  BYCOL: k runs along the columns (element (m, k) at p[k * ld + m]).
template <typename T, bool BYCOL>
struct TileLoad {
  static constexpr int V = kPack<T>, N = kTile * kTileK / 256 / V;
  static constexpr int kRow = kTileK + V;  // padded: 16-byte aligned, rows spread over the banks
  Pack<T> r[N];

  __device__ void load(const T* p, int64_t ld, int64_t m0, int64_t M, int64_t k0, int64_t k1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = i * 256 + threadIdx.x;
      if constexpr (!BYCOL) {
        const int64_t m = m0 + s / (kTileK / V), k = k0 + s % (kTileK / V) * V;
        if (m < M && k < k1) {
          r[i] = load_pack<T>(p + m * ld, k, k1, (T)0.f);
        } else {
          r[i] = Pack<T>{};
        }
      } else {
        const int64_t k = k0 + s / (kTile / V), m = m0 + s % (kTile / V) * V;
        if (k < k1 && m < M) {
          r[i] = load_pack<T>(p + k * ld, m, M, (T)0.f);
        } else {
          r[i] = Pack<T>{};
        }
      }
    }
  }
  __device__ void store(T* lds) const {
    typedef T vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = i * 256 + threadIdx.x;
      if constexpr (!BYCOL) {
        *reinterpret_cast<vec*>(lds + s / (kTileK / V) * kRow + s % (kTileK / V) * V) =
            __builtin_bit_cast(vec, r[i]);
      } else {
        const int k = s / (kTile / V), m = s % (kTile / V) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) lds[(m + j) * kRow + k] = r[i].v[j];
      }
    }
  }
};

// Any sizes, strides and alignment: 64 x 64 of C per workgroup, four waves of 32 x 32.
template <typename T, bool ACOL, bool BCOL>
__global__ void __launch_bounds__(256) product_kernel(const Product P) {
  constexpr int kRow = TileLoad<T, ACOL>::kRow;
  __shared__ __align__(16) T la[kTile * kRow], lb[kTile * kRow];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tiles_n = (P.N + kTile - 1) / kTile;
  const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * kTile;
  const int64_t n0 = (int64_t)(blockIdx.x % tiles_n) * kTile;
  const int64_t k0 = P.partial ? blockIdx.y * P.k_step : 0;
  const int64_t k1 = P.partial && k0 + P.k_step < P.K ? k0 + P.k_step : P.K;
  const T* a = static_cast<const T*>(P.a);
  const T* b = static_cast<const T*>(P.b);
  const int wm = wave / 2 * 32, wn = wave % 2 * 32;
  floatx16 acc = {};
  TileLoad<T, ACOL> ta;
  TileLoad<T, BCOL> tb;
  if (k0 < k1) {
    ta.load(a, P.lda, m0, P.M, k0, k1);
    tb.load(b, P.ldb, n0, P.N, k0, k1);
  }
  for (int64_t k = k0; k < k1; k += kTileK) {
    __syncthreads();
    ta.store(la);
    tb.store(lb);
    __syncthreads();
    if (k + kTileK < k1) {
      ta.load(a, P.lda, m0, P.M, k + kTileK, k1);
      tb.load(b, P.ldb, n0, P.N, k + kTileK, k1);
    }
#pragma unroll
    for (int s = 0; s < kTileK; s += 16)
      mma32(acc, la + (wm + lane % 32) * kRow + s + lane / 32 * 8,
            lb + (wn + lane % 32) * kRow + s + lane / 32 * 8);
  }
  const int64_t n = n0 + wn + lane % 32;
  if (n >= P.N) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t m = m0 + wm + i / 4 * 8 + lane / 32 * 4 + i % 4;
    if (m >= P.M) continue;
    if (P.partial)
      P.partial[((int64_t)blockIdx.y * P.M + m) * P.N + n] = acc[i];
    else
      finish<T>(P, m, n, acc[i]);
  }
}

// ------------------------------------------------------------ large products

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
// counts none of these, so the waits are wait_loads'.  (m0 is no register the compiler keeps
// values in.)
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
    if constexpr (!BYCOL) return KB == 64 ? (at >> 2) & 3 : (at >> 1) & 7;
    if constexpr (sizeof(T) == 4) return 0;
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
  // The last k < K of them, zeros behind.
  __device__ void load_rest(const T* base, int64_t ld, int64_t m0, int64_t M, int64_t k0,
                            int64_t k1, char* lds) {
    typedef T vec __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int row, k;
      place(i, row, k);
      Pack<T> v{};
      if (m0 + row < M && k0 + k < k1)
        v = BYCOL ? load_pack<T>(base + (k0 + k) * ld, m0 + row, M, (T)0.f)
                  : load_pack<T>(base + (m0 + row) * ld, k0 + k, k1, (T)0.f);
      *reinterpret_cast<vec*>(lds + (i * THREADS + threadIdx.x) * 16) =
          __builtin_bit_cast(vec, v);
    }
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

template <int V>
__device__ __forceinline__ void activate_all(int act, float (&z)[V]) {
  switch (act) {
    case 1:
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = activate(1, z[i]);
      break;
    case 2:
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = activate(2, z[i]);
      break;
    case 3:
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = activate(3, z[i]);
      break;
    case 4:
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = activate(4, z[i]);
      break;
  }
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
  activate_all(P.act, z);
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

template <typename T, bool ACOL, bool BCOL, int MT, int NT, int WM, int WN, int KB, int NB>
__global__ void __launch_bounds__(64 * WM * WN, 2) tile_kernel(const Product P) {
  constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, kThreads = 64 * WM * WN, S = KB / 32;
  using A = Operand<T, BM, ACOL, KB, kThreads>;
  using B = Operand<T, BN, BCOL, KB, kThreads>;
  constexpr int kStage = A::kBytes + B::kBytes, K = A::K, kLoads = A::N + B::N;
  constexpr int kStripRow = 32 * NT + 4;  // floats of a row of the outputs' strip
  constexpr int kStrip = 32 * kStripRow * 4;
  __shared__ __align__(16) char lds[NB * kStage > WM * WN * kStrip ? NB * kStage
                                                                    : WM * WN * kStrip];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
    __syncthreads();
    const int64_t k = k0 + (int64_t)stages * K;
    la.load_rest(pa, P.lda, m0, P.M, k, k1, lds);
    lb.load_rest(pb, P.ldb, n0, P.N, k, k1, lds + A::kBytes);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < S; ++s) {
      read(lds, s, 0);
      products(0, nothing);
    }
  }
  // The sums through LDS, 32 rows of a wave at a time, so that memory is read and written in
  // 16-byte packs.
  __syncthreads();
  constexpr int V = kPack<T>, kRowPacks = 32 * NT / V;
  float* strip = reinterpret_cast<float*>(lds + wave * kStrip);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(r / 4 * 8 + lane / 32 * 4 + r % 4) * kStripRow + 32 * j + lane % 32] = acc[i][j][r];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 2
    for (int q = lane; q < 32 * kRowPacks; q += 64) {
      const int row = q / kRowPacks, col = q % kRowPacks * V;
      const int64_t m = m0 + wm + 32 * i + row, n = n0 + wn + col;
      if (m >= P.M || n >= P.N) continue;
      float z[V];
#pragma unroll
      for (int v = 0; v < V; v += 4)
        *reinterpret_cast<floatx4*>(z + v) =
            *reinterpret_cast<const floatx4*>(strip + row * kStripRow + col + v);
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

constexpr int64_t kSumRows = 64;  // rows per partial column sum

// dz = dy a'(z), rounded to T, and the partial column sums of dz before it is rounded: a
// workgroup takes 64 columns of kSumRows rows, its four waves every fourth row.
template <typename T>
__global__ void __launch_bounds__(256) slope_kernel(const LinearArgs A, T* dz, float* partial) {
  __shared__ float sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t blocks_n = (A.n_out + 63) / 64;
  const int64_t n = blockIdx.x % blocks_n * 64 + lane;
  const int64_t m0 = blockIdx.x / blocks_n * kSumRows;
  const int64_t m1 = m0 + kSumRows < A.rows ? m0 + kSumRows : A.rows;
  float s = 0.f;
  if (n < A.n_out)
    for (int64_t m = m0 + wave; m < m1; m += 4) {
      float v = (float)static_cast<const T*>(A.dy)[m * A.lddy + n];
      if (A.act) v *= activation_slope(A.act, A.pre_in[m * A.n_out + n]);
      s += v;
      if (dz) dz[m * A.n_out + n] = (T)v;
    }
  if (!partial) return;
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && n < A.n_out)
    partial[m0 / kSumRows * A.n_out + n] =
        sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
}

template <typename T>
__global__ void __launch_bounds__(256) join_sums_kernel(int64_t n_out, int64_t parts,
                                                        const float* partial, T* db) {
  __shared__ float sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (n < n_out)
    for (int64_t p = wave; p < parts; p += 4) s += partial[p * n_out + n];
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && n < n_out)
    db[n] = (T)(sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]);
}

// ------------------------------------------------------------ launches

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

constexpr int kCUs = 256;

// The kernel of a product and its splits of k.
struct Plan {
  int kind;  // 0: any; 1: 128 x 256; 2: 128 x 128; 3: 64 x 64
  int64_t bm, bn, splits, k_step;
};

bool aligned16(const void* p, int64_t ld, int64_t rows, size_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows < 2 || ld * (int64_t)bytes % 16 == 0);
}

// Splits of k so that a product of few tiles fills the chip, as long as a split keeps 256.
int64_t splits_of(int64_t tiles, int64_t K, int64_t fill) {
  if (tiles == 0) return 1;
  return std::max<int64_t>(1, std::min<int64_t>(fill / tiles, K / 256));
}

// The most partial sums that any plan of these sizes keeps.
Plan plan_of(int kind, int64_t M, int64_t N, int64_t K) {
  static const int64_t bm[] = {64, 128, 128, 64}, bn[] = {64, 256, 128, 64};
  Plan p;
  p.kind = kind;
  p.bm = bm[kind];
  p.bn = bn[kind];
  const int64_t tiles = ((M + p.bm - 1) / p.bm) * ((N + p.bn - 1) / p.bn);
  const int64_t fill = kind == 1 ? 2 * kCUs : kind == 2 ? 3 * kCUs : 2 * kCUs;
  int64_t splits = splits_of(tiles, K, fill);
  const int64_t per = (K + splits - 1) / splits;
  p.k_step = (per + 63) / 64 * 64;
  p.splits = splits > 1 ? (K + p.k_step - 1) / p.k_step : 1;
  return p;
}

int kind_of(int64_t M, int64_t N, int64_t K, bool fast) {
  if (!fast) return 0;
  const int64_t large = ((M + 127) / 128) * ((N + 255) / 256);
  const int64_t middle = ((M + 127) / 128) * ((N + 127) / 128);
  if (large >= kCUs) return 1;
  if (middle >= kCUs / 2) return 2;
  return 3;
}

size_t product_workspace(int64_t M, int64_t N, int64_t K) {
  size_t most = 0;
  for (bool fast : {false, true}) {
    const Plan p = plan_of(kind_of(M, N, K, fast), M, N, K);
    if (p.splits > 1) most = std::max(most, (size_t)p.splits * (size_t)M * (size_t)N * 4);
  }
  return round256(most);
}

template <typename T, bool ACOL, bool BCOL>
int launch_product(Product p, unsigned char* ws, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return 0;
  // 16-byte chunks: every row of an operand starts on one, and by columns they do not straddle
  // the last row's end
  constexpr int V = kPack<T>;
  const bool fast = aligned16(p.a, p.lda, ACOL ? p.K : p.M, sizeof(T)) &&
                    aligned16(p.b, p.ldb, BCOL ? p.K : p.N, sizeof(T)) &&
                    (!ACOL || p.M % V == 0) && (!BCOL || p.N % V == 0);
  const Plan plan = plan_of(kind_of(p.M, p.N, p.K, fast), p.M, p.N, p.K);
  const int64_t tiles = ((p.M + plan.bm - 1) / plan.bm) * ((p.N + plan.bn - 1) / plan.bn);
  p.k_step = plan.k_step;
  p.partial = plan.splits > 1 ? reinterpret_cast<float*>(ws) : nullptr;
  if (tiles > INT32_MAX / 256 || p.K / 16 > INT32_MAX) return (int)hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)tiles, (unsigned)plan.splits);
  switch (plan.kind) {
    case 1: tile_kernel<T, ACOL, BCOL, 2, 4, 2, 2, 64, 3><<<grid, 256, 0, st>>>(p); break;
    case 2: tile_kernel<T, ACOL, BCOL, 2, 2, 2, 2, 64, 3><<<grid, 256, 0, st>>>(p); break;
    case 3: tile_kernel<T, ACOL, BCOL, 1, 1, 2, 2, 64, 3><<<grid, 256, 0, st>>>(p); break;
    default: product_kernel<T, ACOL, BCOL><<<grid, 256, 0, st>>>(p);
  }
  int rc = (int)hipGetLastError();
  if (rc || plan.splits == 1) return rc;
  const int64_t blocks = std::min<int64_t>((p.M * p.N + 255) / 256, 1 << 16);
  join_splits_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(p, plan.splits);
  return (int)hipGetLastError();
}

// The backward's workspace: [dz | partial sums of db | the products' splits]
struct BackwardLayout {
  size_t sums = 0, splits = 0, end = 0;
};
BackwardLayout backward_layout(int dtype, int64_t rows, int64_t n_in, int64_t n_out) {
  BackwardLayout L;
  L.sums = round256((size_t)rows * (size_t)n_out * element_bytes(dtype));
  L.splits = L.sums + round256((size_t)((rows + kSumRows - 1) / kSumRows) * (size_t)n_out * 4);
  L.end = L.splits + std::max(product_workspace(rows, n_in, n_out),
                              product_workspace(n_out, n_in, rows));
  return L;
}

}  // namespace

size_t linear_workspace(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool training) {
  return training ? backward_layout(dtype, rows, n_in, n_out).end
                  : product_workspace(rows, n_out, n_in);
}

int launch_linear(int dtype, const LinearArgs& a, void* stream) {
  Product p{};
  p.M = a.rows;
  p.N = a.n_out;
  p.K = a.n_in;
  p.a = a.x;
  p.lda = a.ldx;
  p.b = a.weight;
  p.ldb = a.ldw;
  p.bias = a.bias;
  p.residual = a.residual;
  p.ldr = a.ldr;
  p.act = a.act;
  p.out = a.y;
  p.ldo = a.ldy;
  p.pre = a.pre;
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    return launch_product<T, false, false>(p, a.ws, static_cast<hipStream_t>(stream));
  });
}

int launch_linear_backward(int dtype, const LinearArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const BackwardLayout L = backward_layout(dtype, a.rows, a.n_in, a.n_out);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    // without an activation dz is dy
    const bool own = a.act != 0 && (a.dx || a.dweight);
    T* dz = own ? reinterpret_cast<T*>(a.ws) : nullptr;
    float* sums = a.dbias ? reinterpret_cast<float*>(a.ws + L.sums) : nullptr;
    const int64_t parts = (a.rows + kSumRows - 1) / kSumRows, blocks_n = (a.n_out + 63) / 64;
    if (parts * blocks_n > INT32_MAX) return (int)hipErrorInvalidConfiguration;
    int rc = 0;
    if ((dz || sums) && parts * blocks_n > 0) {
      slope_kernel<T><<<dim3((unsigned)(parts * blocks_n)), 256, 0, st>>>(a, dz, sums);
      if ((rc = (int)hipGetLastError())) return rc;
    }
    if (a.dbias && blocks_n > 0) {
      join_sums_kernel<T><<<dim3((unsigned)blocks_n), 256, 0, st>>>(a.n_out, parts, sums,
                                                                   static_cast<T*>(a.dbias));
      if ((rc = (int)hipGetLastError())) return rc;
    }
    Product p{};
    p.a = own ? static_cast<const void*>(dz) : a.dy;
    p.lda = own ? a.n_out : a.lddy;
    if (a.dx) {
      p.M = a.rows;
      p.N = a.n_in;
      p.K = a.n_out;
      p.b = a.weight;
      p.ldb = a.ldw;
      p.out = a.dx;
      p.ldo = a.lddx;
      if ((rc = launch_product<T, false, true>(p, a.ws + L.splits, st))) return rc;
    }
    if (a.dweight) {
      p.M = a.n_out;
      p.N = a.n_in;
      p.K = a.rows;
      p.b = a.x;
      p.ldb = a.ldx;
      p.out = a.dweight;
      p.ldo = a.lddw;
      rc = launch_product<T, true, true>(p, a.ws + L.splits, st);
    }
    return rc;
  });
}

}  // namespace vqc
