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

// Splits of k so that a product of few tiles fills the chip, as long as a split keeps 256.
int64_t splits_of(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ((M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  if (tiles == 0) return 1;
  return std::max<int64_t>(1, std::min<int64_t>(512 / tiles, K / 256));
}
int64_t split_step(int64_t K, int64_t splits) {
  const int64_t per = (K + splits - 1) / splits;
  return (per + kTileK - 1) / kTileK * kTileK;
}
size_t product_workspace(int64_t M, int64_t N, int64_t K) {
  const int64_t s = splits_of(M, N, K);
  return s > 1 ? round256((size_t)s * (size_t)M * (size_t)N * 4) : 0;
}

template <typename T, bool ACOL, bool BCOL>
int launch_product(Product p, unsigned char* ws, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return 0;
  const int64_t tiles = ((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile);
  int64_t splits = splits_of(p.M, p.N, p.K);
  p.k_step = split_step(p.K, splits);
  if (splits > 1) splits = (p.K + p.k_step - 1) / p.k_step;
  p.partial = splits > 1 ? reinterpret_cast<float*>(ws) : nullptr;
  if (tiles > INT32_MAX) return (int)hipErrorInvalidConfiguration;
  product_kernel<T, ACOL, BCOL><<<dim3((unsigned)tiles, (unsigned)splits), 256, 0, st>>>(p);
  int rc = (int)hipGetLastError();
  if (rc || splits == 1) return rc;
  const int64_t blocks = std::min<int64_t>((p.M * p.N + 255) / 256, 1 << 16);
  join_splits_kernel<T><<<dim3((unsigned)blocks), 256, 0, st>>>(p, splits);
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
