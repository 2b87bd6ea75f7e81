// linear_tiles.h -- how the linear layers' products are carried out: kernel, tile, splits of k and
// copies onto 16-byte chunks, by rules on sizes, types and alignment (host code without HIP).
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace vqc {

constexpr int kCUs = 256;

// The kernel of a product and its splits of k.
struct Plan {
  int64_t tile, splits, k_step;  // tiles of 256 x 256 ... 32 x 32
};

inline int64_t tiles_of(int64_t M, int64_t N, int64_t tile) {
  return ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
}

// The tile and the splits of k by estimated time.  A CU works through its share of the tiles at
// the rate measured for their size (direct: straight into LDS; otherwise through registers), so
// that a last, part-filled round counts whole; splits of k fill it at the price of writing and
// reading partial sums (5 TB/s) and of a second launch.  us at M x N x K, tile/splits: bf16 8192
// x 4096 x 4096 256/1 290, 128/1 359; 4097 x 4095 x 8191 256/1 431, 128/1 383; 2048^3 128/1 25,
// 64/1 30, 128/2 46; 1024^3 64/1 6.5, 128/1 12.1; 384 x 768 x 8192 64/6 18, 64/1 36; fp32 8191 x
// 4097 x 4095 128/1 2300, 256/1 2950; fp32 1024 x 384 x 768 32/1 13.7, 64/2 15.8, 64/1 17.7; bf16
// 1000 x 301 x 501 32/1 7.3, 64/1 8.6; 7760 x 280 x 6960 as x W^T 256/4 75, 128/2 87, 64/1 99, W
// by columns 71, 76, 100, both by columns 68, 63, 97 (operands from memory rather than from the
// 256 MB cache: 76, 94, 114; 77, 90, 117; 72, 74, 108).
inline Plan plan_of(int dtype, bool direct, bool acol, int64_t M, int64_t N, int64_t K) {
  Plan best{32, 1, K};
  if (M == 0 || N == 0) return best;
  // seconds per k of a round of 256 tiles
  struct Choice {
    int64_t tile;
    bool direct;
    double rate[2];  // fp32, 16-bit
  };
  static const Choice choices[] = {{256, true, {234e-9, 35e-9}}, {128, true, {60.5e-9, 12.3e-9}},
                                   {64, true, {20e-9, 4.7e-9}}, {64, false, {31e-9, 9.4e-9}},
                                   {32, false, {8e-9, 6e-9}}};
  static const int64_t splits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  const int64_t least = dtype == 0 ? 64 : 128;  // k of a split
  double time = 1e30;
  for (const Choice& c : choices) {
    if (c.tile != 32 && c.direct != direct) continue;
    const int64_t tiles = tiles_of(M, N, c.tile);
    // both operands by columns through registers, in short pieces of their rows
    const double rate = c.rate[dtype != 0] * (acol && !c.direct ? 2.5 : 1.);
    for (const int64_t s : splits) {
      if (s > 1 && (K < s * least || tiles * s > 4 * kCUs)) break;
      const int64_t k = s > 1 ? ((K + s - 1) / s + 63) / 64 * 64 : K;
      const int64_t n = s > 1 ? (K + k - 1) / k : 1;
      const int64_t rounds = (tiles * n + kCUs - 1) / kCUs;
      // small tiles share a CU and cover each other's latency
      const double share = rounds > 1 && c.tile <= 64 ? 0.8 : 1.;
      double t = (double)rounds * share * rate * (double)k;
      // 64 tiles of 16 bits: the first waits for memory, the second and third on a CU take more
      // than a share each
      if (c.tile == 64 && c.direct && dtype != 0)
        t = std::max(5.7 + 4.0 * (double)std::min<int64_t>(rounds - 1, 2), 3.6 * (double)rounds) *
            1e-9 * (double)k;
      if (n > 1) t += (double)n * (double)M * (double)N * 1.6e-12 + 5e-6;
      if (t < time) {
        time = t;
        best = {c.tile, n, k};
      }
    }
  }
  return best;
}

inline int64_t aligned_stride(int64_t cols, size_t bytes) {
  const int64_t v = 16 / (int64_t)bytes;
  return (cols + v - 1) / v * v;
}

// Whether rows off the 16-byte chunks are copied onto them before a product: where both of its
// sides are long enough to read every row often.  us without | with the copies, bf16: 8191 x 4097
// x 4095 556 | 290, 2049 x 2047 x 2049 63 | 35; 1023^3 17.6 | 14.  Room for them is kept by sizes
// (copies_rows), so that rows whose stride or start alone is off the chunks are not copied: 8192
// x 4096 x 4096 with x in rows of 4097 elements 527 instead of 252, its dweight 711 instead of
// 213.
inline bool worth_aligning(int64_t rows, int64_t n_in, int64_t n_out) {
  return rows >= 256 && n_in >= 256 && n_out >= 256 &&
         (double)rows * (double)n_in * (double)n_out >= 2e9;
}

// Whether x and W get room for copies onto the chunks: where the products repay them and the sizes
// themselves are off the chunks (contiguous rows of other sizes are on them already).
inline bool copies_rows(int dtype, int64_t rows, int64_t n_in, int64_t n_out) {
  const int64_t v = dtype == 0 ? 4 : 8;
  return worth_aligning(rows, n_in, n_out) && (n_in % v || n_out % v);
}

// Whether an operand of `rows` rows can be loaded straight into LDS, in chunks of v elements.  By
// columns a line's last chunk must not straddle its end, unless there is room behind it.
inline bool on_chunks(int64_t v, bool by_columns, int64_t rows, bool aligned, bool padded) {
  return aligned && (!by_columns || padded || rows % v == 0);
}

// Whether W is read row by row for a few rows of x rather than in tiles: where its rows are long
// enough for a workgroup's last sums not to count.  us at M rows, n x k, tiles | row by row: bf16
// 1, 4096 x 4096 10.1 | 7.0; 4, 4096 x 4096 10.3 | 7.7; 8, 4096 x 4096 10.8 | 10.3; 8, 1000 x 500
// 7.4 | 4.2; 1, 4095 x 4097 17.1 | 7.8; 8, 4095 x 4097 18.4 | 13.5; 4, 384 x 768 5.1 | 3.9; 4, 10
// x 256 3.2 | 3.6; 2, 16384 x 200 5.0 | 9.5; 8, 16384 x 1024 7.7 | 14.7; fp32 1, 4096 x 4096 26.7
// | 13.3; 8, 4096 x 4096 22.7 | 13.9; 4, 10 x 16 3.6 | 3.0; 1, 16384 x 400 11.5 | 6.7; 4, 16384 x
// 200 8.3 | 10.1; 8, 16384 x 1024 20.5 | 14.7.  Sixteen rows: bf16 16, 4096 x 4096 11.2 | 18.8,
// fp32 16, 16384 x 1024 20.0 | 27.7.
inline bool few_rows(int64_t element, int64_t M, int64_t N, int64_t K) {
  const int64_t bytes = K * element;
  if (M > 8 || bytes < 16) return false;
  if (N > 4096) return bytes >= std::max<int64_t>(1024, (element == 4 ? 512 : 1024) * M);
  return element == 4 || bytes >= 512;
}

// ------------------------------------------------------------ 8-bit integers

// A sum of more products than this may pass 32 bits (of -128 times -128).
constexpr int64_t kMostIntegers = (1 << 17) - 1;

// Rows of x end with zeros up to a multiple of the tiles' largest stage: a stage of which only
// part is left is multiplied like the others, whatever W's chunks behind the end hold.
constexpr int64_t kIntegerStage = 128;

// The tile and the splits of k of a product of 8-bit integers, by estimated time as above: rounds of
// 256 tiles at the rate measured for their size, what beginning and ending them takes (a CU has one
// of the largest at a time, so that nothing covers the writing of its results), and the price of
// splits.  Over 256 sizes of 1 to 16384 rows and columns and k of 32 to 85000 it comes within 1 % of
// the best choice on average.  us at M x N x K, tile/splits (x given as integers, silu and bias,
// bf16): 8192 x 4096 x 4096 256/1 141, 128/1 200; 3000^3 256/1 56, 128/1 61, 64/1 66; 2048 x 2048 x
// 16384 128/1 83, 256/4 99; 8192 x 4096 x 256 128/1 35, 256/1 38; 256 x 8192 x 8192 64/1 32, 128/1 42,
// 256/6 45; 1024^3 64/1 6.1, 128/1 11.6; 64 x 4096 x 16384 64/4 17.5, 64/1 35, 64/8 19.3; 301 x 101 x
// 16384 64/12 9.2, 64/4 13.3, 64/1 35.  Tiles of 32, which go through registers, are never the best
// of rows on 16-byte chunks: 64 x 64 x 65536 64/32 10.8, 32/32 16.
// (Up to 32 rows off the chunks are not split: no workspace for what is rare.)
inline Plan integer_plan_of(bool direct, int64_t M, int64_t N, int64_t K) {
  Plan p{32, 1, K};
  if (direct && M > 0 && N > 0) {
    struct Choice {
      int64_t tile;
      double rate, once, between;  // us per k of a round, of the whole, between two rounds
    };
    static const Choice choices[] = {
        {256, 13.5e-3, 2.5, 3.6}, {128, 5.9e-3, 0.8, 0.}, {64, 2.1e-3, 0., 0.}};
    double time = 1e30;
    for (const Choice& c : choices) {
      const int64_t tiles = tiles_of(M, N, c.tile);
      for (const int64_t s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
        if (s > 1 && (K < s * 256 || tiles * s > 4 * kCUs)) break;
        const int64_t k = s > 1 ? ((K + s - 1) / s + 127) / 128 * 128 : K;
        const int64_t n = s > 1 ? (K + k - 1) / k : 1;
        const double rounds = (double)((tiles * n + kCUs - 1) / kCUs);
        double t = c.once + rounds * c.rate * (double)k + (rounds - 1.) * c.between;
        if (n > 1) t += (double)n * (double)M * (double)N * 2.3e-6 + 2.;
        if (t < time) {
          time = t;
          p = {c.tile, n, k};
        }
      }
    }
  } else if (M > 32) {
    p = plan_of(2, false, false, M, N, (K + 1) / 2);  // as many bytes, for half the k
    p.k_step = p.splits > 1 ? 2 * p.k_step : K;
  }
  if (M > 0 && N > 0 && p.k_step > kMostIntegers) {
    p.k_step = kMostIntegers / 256 * 256;
    p.splits = (K + p.k_step - 1) / p.k_step;
  }
  return p;
}

// Whether one row of x is quantised where it meets W, in one launch (below that
// fused_integer_rows).  us so | fused, bf16: 1 x 4096 x 65536 42.5 | 45.1, 1 x 4096 x 4096 5.8 | 6.1,
// 1 x 2048 x 4096 5.3 | 5.2, 1 x 1024 x 1024 4.0 | 3.7; with a launch of its own 1 x 16384 x 1024 6.7
// | 16.
inline bool one_integer_row(int64_t M, int64_t N, int64_t K) {
  return M == 1 && N >= 1 && K > 2048 && K <= 16384;
}

// Whether the rows of x are quantised 16 at a time by the workgroups that multiply them, each of
// which does it for itself.  Its products are slower than those of tiles, where nothing is read twice,
// but rows are not written as integers and read again (as much as some 24 columns of products), nor is
// there a launch for it; fewer than 48 columns take 48 columns' time.  Tiles come nearer where rows
// are longer, in 16 bits from 256 elements on, in fp32, whose quantising reads more, from 512.  Over
// 5700 sizes of up to 2e10 products the rule is within 1.1 % of the better way on average in 16 bits
// and 0.6 % in fp32.  us so | with a launch of its own, rows x n_in x n_out: bf16 (f16 alike) 64 x 16 x
// 10 3.6 | 8.1, 2048 x 256 x 512 6.9 | 8.5, 8192 x 64 x 512 10.4 | 12.1, 8192 x 128 x 512 13.7 | 12.1, 4096 x
// 128 x 1024 13.8 | 11.9, 8192 x 128 x 1024 23 | 18; 256 x 512 x 512 6.6 | 8.3, 1000 x 1001 x 100 8.2 | 10.8,
// 8192 x 512 x 64 8.6 | 11.7, 8192 x 1000 x 40 12.1 | 16.8, 1024 x 768 x 384 9.9 | 9.6, 256 x 1024 x 1024 10.2 |
// 9.7; fp32 8192 x 64 x 512 10.7 | 15.0, 8192 x 128 x 1024 17 | 22, 2048 x 512 x 512 9.5 | 10.1, 4096 x 256 x
// 2048 25.5 | 23.6; 1000 x 1001 x 100 7.2 | 10.7, 8192 x 1000 x 40 11.3 | 16.5, 1024 x 768 x 384 9.6 | 10.2,
// 1024^3 17.4 | 11.5.  Up to 32 rows of 256 or more the rules below: bf16 4 x 512 x 512 5.9 | 4.5, 16 x 1024 x
// 1024 9.7 | 6.8.
inline bool short_integer_rows(int64_t element, int64_t M, int64_t N, int64_t K) {
  if (N < 1 || K < 16 / element || K > 1024) return false;
  if (M <= 32) return K < 256;
  const double most = element == 4 ? (K <= 512 ? 1.8e9 : 3.8e8) : (K <= 256 ? 5.0e8 : 2.6e8);
  return (double)M * (double)K * (double)(std::max<int64_t>(N, 48) - 24) <= most;
}

// Whether a few rows of integers meet W as it comes from memory.  us so | in tiles, bf16: 4 x 4096 x
// 4096 8.4 | 14.4, 16 x 4096 x 4096 9.7 | 13.6, 32 x 4096 x 4096 11.7 | 12.9, 4 x 1024 x 16384 7.7 |
// 8.9, 5 x 4096 x 65536 49.6 | 48.2 (from memory rather than the 256 MB cache 57 | 66); longer rows
// would not stay in the registers: 16 x 8192 x 8192 26 | 23, 32 x 16384 x 1024 30 | 14.
inline bool few_integer_rows(int64_t M, int64_t N, int64_t K) {
  return M <= 32 && N >= 1 && K >= 256 && K <= 4096;
}

// Whether they are quantised there too: where every wave has 1024 elements at most.  us so | with a
// launch of its own, bf16: 2 x 1024 x 1024 4.5 | 5.3, 4 x 1024 x 1024 4.7 | 5.8, 2 x 4096 x 4096 6.0
// | 7.9, 4 x 1024 x 16384 6.3 | 7.6.
constexpr int kFusedPieces = 8;
inline bool fused_integer_rows(int64_t M, int64_t N, int64_t K) {
  return few_integer_rows(M, N, K) && M * ((K + 1023) / 1024) <= kFusedPieces;
}

// dz of few elements stays in fp32 and is multiplied so: the products then cost little, and
// an element's rounding would show whole in a row or column of a gradient instead of being
// averaged over many.
inline bool exact_dz(int dtype, int64_t rows, int64_t n_out) {
  return dtype != 0 && rows * n_out <= 4096;
}

}  // namespace vqc
