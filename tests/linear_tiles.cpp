// linear_tiles.cpp -- prints how the three products of a linear layer on contiguous tensors are
// carried out (test_linear_tiles_cpu.py):
//   linear_tiles < sizes, a line each: dtype act rows n_in n_out
//   x W^T, dz W and dz^T x, each as: few (row by row) or tile, splits, direct; whether x or W is
//   copied onto 16-byte chunks
#include <cstdio>
#include <cstring>

#include "linear_tiles.h"

namespace {

struct Operand {
  bool aligned, padded;
};

Operand contiguous(int64_t v, int64_t rows, int64_t cols, bool copied) {
  const bool on = rows < 2 || cols % v == 0;
  return {on || copied, !on && copied};
}

void print(int dtype, bool same_types, bool acol, bool bcol, int64_t M, int64_t N, int64_t K,
           Operand a, Operand b) {
  const int64_t v = dtype == 0 ? 4 : 8;
  if (same_types && !acol && !bcol && vqc::few_rows(16 / v, M, N, K)) {
    std::printf("few 1 1 ");
    return;
  }
  const bool direct = same_types && vqc::on_chunks(v, acol, M, a.aligned, a.padded) &&
                      vqc::on_chunks(v, bcol, N, b.aligned, b.padded);
  const vqc::Plan p = vqc::plan_of(same_types ? dtype : 0, direct, acol, M, N, K);
  std::printf("%lld %lld %d ", (long long)p.tile, (long long)p.splits, (int)direct);
}

}  // namespace

int main() {
  long long act, rows, n_in, n_out;
  int dtype;
  while (std::scanf("%d %lld %lld %lld %lld", &dtype, &act, &rows, &n_in, &n_out) == 5) {
    const int64_t v = dtype == 0 ? 4 : 8;
    const bool copies = vqc::copies_rows(dtype, rows, n_in, n_out);
    const Operand x = contiguous(v, rows, n_in, copies), w = contiguous(v, n_out, n_in, copies);
    Operand dz = contiguous(v, rows, n_out, false);
    const bool own = act != 0 || (!dz.aligned && vqc::worth_aligning(rows, n_in, n_out));
    const bool exact = own && act != 0 && vqc::exact_dz(dtype, rows, n_out);
    if (own) dz = {true, true};
    print(dtype, true, false, false, rows, n_out, n_in, x, w);
    print(dtype, !exact, false, true, rows, n_in, n_out, dz, w);
    print(dtype, !exact, true, true, n_out, n_in, rows, dz, x);
    std::printf("%d\n", (int)(copies && (x.padded || w.padded)));
  }
}
