// layer_norm.hip -- layer norm over rows, forward and backward.
//
//   mean = sum x / n, r = (sum (x - mean)^2 / n + eps)^(-1/2), h = (x - mean) r
//   y = h w + b
//   g = dy w, dx = r (g - sum g / n - h sum(g h) / n), dw = sum_rows dy h, db = sum_rows dy
//
// Memory-bound: x is read and y written once; the backward reads x and dy and writes dx.
// A row stays in the registers of a group of threads between its sums and its outputs, so
// the variance is the sum of squares about the mean (no cancellation) at no extra read.
//
// bf16 8192 x 4096: forward 33.6 us (134 MB, 4.0 TB/s), backward 41 us (201 MB, 4.9 TB/s) and 4 us
// for dw and db; copies of that size run at 5.2 TB/s.  fp32 1000 x 769: 5, 7 and 6 us, where
// launches and the chain of sums are all of it.
#include <algorithm>

#include "layers.h"
#include "layers_device.h"

namespace vqc {
namespace {

constexpr int kMaxRegisterCols = 16384;  // 1024 threads of 16 elements

// G threads per row, WG / G rows at a time, C packs per thread.  One workgroup per 256 / G rows and
// no loop in practice: many short workgroups overlap one's loads with another's sums.  (A wave per
// row of 4096 or 128 threads per row hold more registers each: 63 us instead of 34.)
// SHORT: rows of less than a pack.
template <typename T, int G, int WG, int C, bool SHORT>
__global__ void __launch_bounds__(WG) norm_kernel(const NormArgs A) {
  constexpr int V = kPack<T>, NG = WG / G;
  __shared__ float red[2][WG / 64];
  const int t = threadIdx.x % G, g = threadIdx.x / G;
  const T* w = static_cast<const T*>(A.weight);
  const T* b = static_cast<const T*>(A.bias);
  const int cols = (int)A.cols;
  const float n = (float)cols;
  for (int64_t base = (int64_t)blockIdx.x * NG; base < A.rows; base += (int64_t)gridDim.x * NG) {
    const int64_t r = base + g < A.rows ? base + g : A.rows - 1;
    const bool mine = base + g < A.rows;
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    Raw raw[C];
    Pack<T> p[C];
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) raw[c] = load_raw<T, SHORT>(x, (c * G + t) * V, cols);
#pragma unroll
    for (int c = 0; c < C; ++c)
      p[c] = taken<T, SHORT>(raw[c], (c * G + t) * V, cols, (T)0.f);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += (float)p[c].v[i];
    group_sums<G>(s, red[0]);
    const float mean = s[0] / n;
    float q[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int col = (c * G + t) * V + i;
        const float d = (float)p[c].v[i] - mean;
        if (col < cols) q[0] += d * d;
      }
    group_sums<G>(q, red[1]);
    const float rstd = 1.f / sqrtf(q[0] / n + A.eps);
    if (!mine) continue;
    if (A.mean && t == 0) {
      A.mean[r] = mean;
      A.rstd[r] = rstd;
    }
    T* y = static_cast<T*>(A.y) + r * A.ldy;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      if (col >= cols) continue;
      Raw wr, br;
      if (w) wr = load_raw<T, SHORT>(w, col, cols);
      if (b) br = load_raw<T, SHORT>(b, col, cols);
      Pack<T> wp, bp, o;
      if (w) wp = taken<T, SHORT>(wr, col, cols, (T)0.f);
      if (b) bp = taken<T, SHORT>(br, col, cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float h = ((float)p[c].v[i] - mean) * rstd;
        if (w) h *= (float)wp.v[i];
        if (b) h += (float)bp.v[i];
        o.v[i] = (T)h;
      }
      store_pack<T>(y, col, cols, o);
    }
  }
}

// Rows longer than the registers hold: one workgroup per row, read once for each sum and
// once for y.
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs A) {
  constexpr int V = kPack<T>, G = 1024;
  __shared__ float red[2][G / 64];
  const int t = threadIdx.x;
  const T* w = static_cast<const T*>(A.weight);
  const T* b = static_cast<const T*>(A.bias);
  const float n = (float)A.cols;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    float s[1] = {0.f}, q[1] = {0.f};
    for (int64_t c = (int64_t)t * V; c < A.cols; c += (int64_t)G * V) {
      const Pack<T> p = taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += (float)p.v[i];
    }
    group_sums<G>(s, red[0]);
    const float mean = s[0] / n;
    for (int64_t c = (int64_t)t * V; c < A.cols; c += (int64_t)G * V) {
      const Pack<T> p = taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = (float)p.v[i] - mean;
        if (c + i < A.cols) q[0] += d * d;
      }
    }
    group_sums<G>(q, red[1]);
    const float rstd = 1.f / sqrtf(q[0] / n + A.eps);
    if (A.mean && t == 0) {
      A.mean[r] = mean;
      A.rstd[r] = rstd;
    }
    T* y = static_cast<T*>(A.y) + r * A.ldy;
    for (int64_t c = (int64_t)t * V; c < A.cols; c += (int64_t)G * V) {
      const Pack<T> p = taken<T>(load_raw<T>(x, c, A.cols), c, A.cols, (T)0.f);
      Pack<T> wp, bp, o;
      if (w) wp = taken<T>(load_raw<T>(w, c, A.cols), c, A.cols, (T)0.f);
      if (b) bp = taken<T>(load_raw<T>(b, c, A.cols), c, A.cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float h = ((float)p.v[i] - mean) * rstd;
        if (w) h *= (float)wp.v[i];
        if (b) h += (float)bp.v[i];
        o.v[i] = (T)h;
      }
      store_pack<T>(y, c, A.cols, o);
    }
  }
}

// The backward of rows in registers.  A thread keeps its columns for all its rows, so the
// sums over rows stay in registers too; at the end the workgroup's groups add up through
// LDS in a fixed order and write one partial row of dw and db.  256 workgroups at most, so that
// the partial rows (8 MB at 4096 columns) cost a tenth of the rows' own traffic.
template <typename T, int G, int WG, int C, bool SHORT>
__global__ void __launch_bounds__(WG) norm_backward_kernel(const NormArgs A) {
  constexpr int V = kPack<T>, NG = WG / G, E = C * V;
  __shared__ float red[2][2 * (WG / 64)];
  __shared__ float acc[NG > 1 ? 2 * G * E : 1];
  const int t = threadIdx.x % G, g = threadIdx.x / G;
  const T* w = static_cast<const T*>(A.weight);
  const int cols = (int)A.cols;
  const float inv = 1.f / (float)cols;
  Raw wr[C];  // as in memory: in 16 bits they take half the registers
  float dw[E], db[E];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * G + t) * V;
    Pack<T> wp;
#pragma unroll
    for (int i = 0; i < V; ++i) wp.v[i] = (T)1.f;
    if (w) wp = taken<T, SHORT>(load_raw<T, SHORT>(w, col, cols), col, cols, (T)0.f);
    wr[c] = __builtin_bit_cast(Raw, wp);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[c * V + i] = db[c * V + i] = 0.f;
  }
  int flip = 0;
  for (int64_t base = (int64_t)blockIdx.x * NG; base < A.rows; base += (int64_t)gridDim.x * NG) {
    const bool mine = base + g < A.rows;
    const int64_t r = mine ? base + g : A.rows - 1;
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    const T* dy = static_cast<const T*>(A.dy) + r * A.lddy;
    Raw xr[C], dr[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      xr[c] = load_raw<T, SHORT>(x, col, cols);
      dr[c] = load_raw<T, SHORT>(dy, col, cols);
    }
    const float mean = A.mean_in[r], rstd = A.rstd_in[r];
    Pack<T> xp[C], dp[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      // Behind the end: x the row's last element (which a clamped load has last), dy 0, so that
      // 0 times an h of the row joins the sums.  (With x = 0, h = -mean rstd may be infinite where
      // no h of the row is, and 0 times that NaN.)
      xp[c] = taken<T, SHORT>(xr[c], col, cols, __builtin_bit_cast(Pack<T>, xr[c]).v[V - 1]);
      dp[c] = taken<T, SHORT>(dr[c], col, cols, (T)0.f);
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      const Pack<T> wp = __builtin_bit_cast(Pack<T>, opaque(wr[c]));
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = c * V + i;
        const float d = (float)dp[c].v[i], g = d * (float)wp.v[i];
        float h = ((float)xp[c].v[i] - mean) * rstd;
        if (SHORT && col + i >= cols) h = 0.f;  // these loads are not clamped
        s[0] += g;
        s[1] += g * h;
        if (mine) {
          dw[e] += d * h;
          db[e] += d;
        }
      }
    }
    group_sums<G>(s, red[flip]);
    flip ^= 1;
    if (!mine || !A.dx) continue;
    const float c1 = s[0] * inv, c2 = s[1] * inv;
    T* dx = static_cast<T*>(A.dx) + r * A.lddx;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * G + t) * V;
      if (col >= cols) continue;
      const Pack<T> wp = __builtin_bit_cast(Pack<T>, opaque(wr[c]));
      Pack<T> o;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float h = ((float)xp[c].v[i] - mean) * rstd;
        o.v[i] = (T)(rstd * ((float)dp[c].v[i] * (float)wp.v[i] - c1 - h * c2));
      }
      store_pack<T>(dx, col, cols, o);
    }
  }
  if (!A.partial) return;
  if constexpr (NG > 1) {
    for (int k = 0; k < NG; ++k) {
      if (g == k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (k == 0) {
            acc[e * G + t] = dw[e];
            acc[(E + e) * G + t] = db[e];
          } else {
            acc[e * G + t] += dw[e];
            acc[(E + e) * G + t] += db[e];
          }
        }
      __syncthreads();
    }
  }
  if (g != 0) return;
  float* out = A.partial + (int64_t)blockIdx.x * 2 * A.cols;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = c * V + i;
      const int col = (c * G + t) * V + i;
      if (col >= cols) continue;
      out[col] = NG > 1 ? acc[e * G + t] : dw[e];
      out[cols + col] = NG > 1 ? acc[(E + e) * G + t] : db[e];
    }
}

// Long rows: dx row by row ...
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_backward_kernel(const NormArgs A) {
  constexpr int V = kPack<T>, G = 1024;
  __shared__ float red[2][2 * (G / 64)];
  const int t = threadIdx.x;
  const T* w = static_cast<const T*>(A.weight);
  const float inv = 1.f / (float)A.cols;
  int flip = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + r * A.ldx;
    const T* dy = static_cast<const T*>(A.dy) + r * A.lddy;
    const float mean = A.mean_in[r], rstd = A.rstd_in[r];
    float s[2] = {0.f, 0.f};
    for (int64_t c = (int64_t)t * V; c < A.cols; c += (int64_t)G * V) {
      const Raw xr = load_raw<T>(x, c, A.cols), dr = load_raw<T>(dy, c, A.cols);
      const Pack<T> xp = taken<T>(xr, c, A.cols, (T)0.f), dp = taken<T>(dr, c, A.cols, (T)0.f);
      Pack<T> wp;
      if (w) wp = taken<T>(load_raw<T>(w, c, A.cols), c, A.cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float gy = (float)dp.v[i] * (w ? (float)wp.v[i] : 1.f);
        s[0] += gy;
        s[1] += gy * ((float)xp.v[i] - mean) * rstd;
      }
    }
    group_sums<G>(s, red[flip]);
    flip ^= 1;
    const float c1 = s[0] * inv, c2 = s[1] * inv;
    T* dx = static_cast<T*>(A.dx) + r * A.lddx;
    for (int64_t c = (int64_t)t * V; c < A.cols; c += (int64_t)G * V) {
      const Raw xr = load_raw<T>(x, c, A.cols), dr = load_raw<T>(dy, c, A.cols);
      const Pack<T> xp = taken<T>(xr, c, A.cols, (T)0.f), dp = taken<T>(dr, c, A.cols, (T)0.f);
      Pack<T> wp, o;
      if (w) wp = taken<T>(load_raw<T>(w, c, A.cols), c, A.cols, (T)0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float gy = (float)dp.v[i] * (w ? (float)wp.v[i] : 1.f);
        o.v[i] = (T)(rstd * (gy - c1 - ((float)xp.v[i] - mean) * rstd * c2));
      }
      store_pack<T>(dx, c, A.cols, o);
    }
  }
}

// ... and the sums over rows column by column: a workgroup takes 256 packs of columns and
// every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormArgs A) {
  constexpr int V = kPack<T>;
  const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
  if (col >= A.cols) return;
  float dw[V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
  for (int64_t r = blockIdx.y; r < A.rows; r += gridDim.y) {
    const Raw xr = load_raw<T>(static_cast<const T*>(A.x) + r * A.ldx, col, A.cols);
    const Raw dr = load_raw<T>(static_cast<const T*>(A.dy) + r * A.lddy, col, A.cols);
    const Pack<T> xp = taken<T>(xr, col, A.cols, (T)0.f), dp = taken<T>(dr, col, A.cols, (T)0.f);
    const float mean = A.mean_in[r], rstd = A.rstd_in[r];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dw[i] += (float)dp.v[i] * ((float)xp.v[i] - mean) * rstd;
      db[i] += (float)dp.v[i];
    }
  }
  float* out = A.partial + (int64_t)blockIdx.y * 2 * A.cols;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (col + i < A.cols) {
      out[col + i] = dw[i];
      out[A.cols + col + i] = db[i];
    }
}

// dw and db from the partial rows: 64 columns per workgroup, its four waves share the
// parts, added up in a fixed order.
template <typename T>
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs A, int64_t parts) {
  __shared__ float sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane;  // over [dw | db]
  float s = 0.f;
  if (i < 2 * A.cols)
#pragma unroll 8  // loads in flight together; the sum keeps its order
    for (int64_t p = wave; p < parts; p += 4) s += A.partial[p * 2 * A.cols + i];
  sums[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || i >= 2 * A.cols) return;
  s = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
  if (i < A.cols) {
    if (A.dweight) static_cast<T*>(A.dweight)[i] = (T)s;
  } else if (A.dbias) {
    static_cast<T*>(A.dbias)[i - A.cols] = (T)s;
  }
}

// Threads per row, for rows up to kMaxRegisterCols: the fewest that hold the row in 16
// elements each.
int group_of(int64_t cols) {
  return cols <= 16 * 16 ? 16 : cols <= 64 * 16 ? 64 : cols <= 256 * 16 ? 256 : 1024;
}

template <int N>
using IC = std::integral_constant<int, N>;

// f(G, packs per thread, whether rows are shorter than a pack)
template <typename T, typename F>
int by_row(int64_t cols, F&& f) {
  const int G = group_of(cols);
  const int64_t packs = (cols + kPack<T> - 1) / kPack<T>;
  const int c = (int)((packs + G - 1) / G);
  auto with_c = [&](auto g) {
    if (c <= 1) return f(g, IC<1>{}, IC<0>{});
    if (c <= 2 || sizeof(T) == 2) return f(g, IC<2>{}, IC<0>{});
    if constexpr (sizeof(T) == 4) return f(g, IC<4>{}, IC<0>{});
    return (int)hipErrorInvalidValue;
  };
  if (cols < kPack<T>) return f(IC<16>{}, IC<1>{}, IC<1>{});
  switch (G) {
    case 16: return with_c(IC<16>{});
    case 64: return with_c(IC<64>{});
    case 256: return with_c(IC<256>{});
    default: return with_c(IC<1024>{});
  }
}

constexpr int64_t kMaxBlocks = 1 << 20;  // grids beyond this loop over rows
constexpr int64_t kParts = 256;          // partial rows: one workgroup of 1024 threads per CU
// Threads of a backward workgroup: more rows at a time where there are rows for every CU (fp32
// 1000 x 769: 1024 threads 12 us, 256 7 us).
int backward_threads(int64_t rows, int64_t cols) {
  const int g = group_of(cols);
  return g == 1024 || (rows + 1024 / g - 1) / (1024 / g) >= kParts ? 1024 : 256;
}

}  // namespace

int64_t norm_parts(int64_t rows, int64_t cols) {
  if (rows == 0) return 0;
  const int ng =
      cols > kMaxRegisterCols ? 1 : backward_threads(rows, cols) / group_of(cols);
  return std::min<int64_t>((rows + ng - 1) / ng, kParts);
}

int launch_layer_norm(int dtype, const NormArgs& a, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    if (a.cols > kMaxRegisterCols) {
      norm_long_kernel<T><<<dim3((unsigned)std::min(a.rows, kMaxBlocks)), 1024, 0, st>>>(a);
      return (int)hipGetLastError();
    }
    return by_row<T>(a.cols, [&](auto g, auto c, auto is_short) {
      constexpr int G = decltype(g)::value, WG = G > 256 ? G : 256, C = decltype(c)::value;
      constexpr bool SHORT = decltype(is_short)::value;
      const int64_t blocks = std::min<int64_t>((a.rows + WG / G - 1) / (WG / G), kMaxBlocks);
      norm_kernel<T, G, WG, C, SHORT><<<dim3((unsigned)blocks), WG, 0, st>>>(a);
      return (int)hipGetLastError();
    });
  });
}

int launch_layer_norm_backward(int dtype, const NormArgs& args, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NormArgs a = args;
  const bool sums = a.dweight || a.dbias;
  if (!sums) a.partial = nullptr;
  const int64_t parts = norm_parts(a.rows, a.cols);
  return by_dtype(dtype, [&](auto type) {
    using T = decltype(type);
    int rc = 0;
    if (a.rows > 0 && a.cols > kMaxRegisterCols) {
      if (a.dx)
        norm_long_backward_kernel<T>
            <<<dim3((unsigned)std::min(a.rows, kMaxBlocks)), 1024, 0, st>>>(a);
      if (a.partial) {
        const int64_t blocks = (a.cols + 256 * kPack<T> - 1) / (256 * kPack<T>);
        norm_columns_kernel<T>
            <<<dim3((unsigned)blocks, (unsigned)parts), 256, 0, st>>>(a);
      }
      rc = (int)hipGetLastError();
    } else if (a.rows > 0) {
      rc = by_row<T>(a.cols, [&](auto g, auto c, auto is_short) {
        constexpr int G = decltype(g)::value, C = decltype(c)::value;
        constexpr bool SHORT = decltype(is_short)::value;
        if constexpr (G < 1024) {
          if (backward_threads(a.rows, a.cols) == 256) {
            norm_backward_kernel<T, G, 256, C, SHORT><<<dim3((unsigned)parts), 256, 0, st>>>(a);
            return (int)hipGetLastError();
          }
        }
        norm_backward_kernel<T, G, 1024, C, SHORT><<<dim3((unsigned)parts), 1024, 0, st>>>(a);
        return (int)hipGetLastError();
      });
    }
    if (rc || !sums) return rc;
    norm_join_kernel<T><<<dim3((unsigned)((2 * a.cols + 63) / 64)), 256, 0, st>>>(a, parts);
    return (int)hipGetLastError();
  });
}

}  // namespace vqc
