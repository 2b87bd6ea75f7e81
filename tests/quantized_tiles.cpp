// quantized_tiles.cpp -- prints how linear layers in 8-bit integers are carried out on rows that start
// on 16 bytes (test_serving_cpu.py):
//   quantized_tiles < sizes, a line each: element rows n_in n_out (element: bytes of one of x, 1
//   where x is given as integers)
//   one, short, fused, few, or a tile and its splits of k
#include <cstdio>

#include "linear_tiles.h"

int main() {
  long long element, M, K, N;
  while (std::scanf("%lld %lld %lld %lld", &element, &M, &K, &N) == 4) {
    if (element > 1 && vqc::short_integer_rows(element, M, N, K)) {
      std::printf("short 1\n");
    } else if (element > 1 && vqc::one_integer_row(M, N, K)) {
      std::printf("one 1\n");
    } else if (element > 1 && vqc::fused_integer_rows(M, N, K)) {
      std::printf("fused 1\n");
    } else if (vqc::few_integer_rows(M, N, K)) {
      std::printf("few 1\n");
    } else {
      const vqc::Plan p = vqc::integer_plan_of(true, M, N, K);
      const bool full = p.splits == 1 ? p.k_step == K : p.k_step % vqc::kIntegerStage == 0;
      const bool fits = p.k_step <= vqc::kMostIntegers && p.k_step * p.splits >= K;
      std::printf("%lld %lld%s\n", (long long)p.tile, (long long)p.splits,
                  full && fits ? "" : " wrong");
    }
  }
}
