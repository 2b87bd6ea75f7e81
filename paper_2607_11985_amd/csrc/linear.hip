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
#include <type_traits>

#include "layers.h"
#include "linear_device.h"
#include "linear_tiles.h"

namespace vqc {
namespace {

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
