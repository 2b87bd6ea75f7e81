// verify_ways.cpp -- prints how drafts are verified (test_verify_ways_cpu.py):
//   verify_ways < sizes, a line each: bytes of an element, sequences, drafts, outcomes, 1 where the
//   draft's scores are given
//   small (a workgroup per sequence), read (all rows are) or passed (rows behind a refused draft are
//   passed over), whether a row is shorter than 16 bytes, parts of a row, units and workgroups of the
//   drawn one, packs of a lane
#include <cstdio>

#include "verify_plan.h"

int main() {
  long long element, n, k, cols, draft;
  while (std::scanf("%lld %lld %lld %lld %lld", &element, &n, &k, &cols, &draft) == 5) {
    const int pack = 16 / (int)element;
    const bool has_draft = draft && k > 0, is_short = cols < pack;
    if (vqc::verify_is_small(k, cols, has_draft)) {
      std::printf("small %d 0 0 0 0\n", is_short);
      continue;
    }
    const vqc::VerifyPlan R = vqc::verify_plan_of(n, k, cols, has_draft, pack);
    const bool parts = R.parts >= 1 && R.parts <= vqc::kMostParts && R.part % pack == 0 &&
                       R.part * R.parts >= cols && R.part * (R.parts - 1) < cols;
    const bool units = R.units >= 1 && R.units <= 4096 && R.unit % (64 * pack) == 0 &&
                       R.unit * R.units >= cols && R.unit * (R.units - 1) < cols &&
                       R.pieces * (vqc::kVerifyThreads / 64) >= R.units;
    std::printf("%s %d %d %d %d %lld\n", !parts || !units ? "wrong" : R.early ? "passed" : "read",
                is_short, R.parts, R.units, R.pieces, (long long)(R.unit / (64 * pack)));
  }
}
