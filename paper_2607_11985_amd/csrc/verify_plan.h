// verify_plan.h -- how the verification of drafts is carried out: kernels, parts of rows and units of
// the drawn row, by rules on sizes (host code without HIP).
#pragma once

#include <algorithm>
#include <cstdint>

#include "linear_tiles.h"  // kCUs

namespace vqc {

constexpr int kVerifyThreads = 256;  // of a workgroup of total_kernel and draw_kernel
constexpr int kMostParts = 64;       // of a row
constexpr int kSmallRows = 64;       // of a sequence in small_kernel

struct VerifyPlan {
  int parts;        // of a row in total_kernel
  int64_t part;     // its elements, a multiple of 16 bytes
  int units;        // of the drawn row in draw_kernel, a wave's each
  int64_t unit;     // their elements
  int pieces;       // workgroups with them
  bool early;       // where drafts end is found on the way, and later rows are passed over
};

// Rows of scores of a sequence.
inline int64_t verify_rows(int64_t drafts, bool has_draft) {
  return has_draft ? 2 * drafts + 1 : drafts + 1;
}

// Whether a workgroup takes a whole sequence: few enough scores.
inline bool verify_is_small(int64_t drafts, int64_t cols, bool has_draft) {
  const int64_t rows = verify_rows(drafts, has_draft);
  return rows <= kSmallRows && rows * cols <= 32768;
}

// Equal cuts of a row, at packs: `wanted` of them where each has `least` elements.
inline void cut_row(int64_t cols, int64_t wanted, int64_t least, int pack, int& parts,
                    int64_t& part) {
  wanted = std::min({wanted, (cols + least - 1) / least, (int64_t)kMostParts});
  wanted = std::max<int64_t>(wanted, 1);
  part = ((cols + wanted - 1) / wanted + pack - 1) / pack * pack;
  parts = (int)((cols + part - 1) / part);
}

inline VerifyPlan verify_plan_of(int64_t sequences, int64_t drafts, int64_t cols, bool has_draft,
                                 int pack) {
  VerifyPlan R{};
  const int64_t rows = std::max<int64_t>(1, sequences * verify_rows(drafts, has_draft));
  const int64_t step = 4 * kVerifyThreads * pack;  // a thread's four packs
  cut_row(cols, std::max((4 * kCUs + rows - 1) / rows, (cols + step - 1) / step), step / 4,
          pack, R.parts, R.part);
  // packs for each lane: as many as leave every CU four workgroups, and no more than 64 times 64
  // units
  const int64_t lanes = 64 * pack, all = (cols + lanes - 1) / lanes;
  const int64_t each = std::max(sequences * all / (4 * 4 * kCUs), (all + 4095) / 4096);
  R.unit = std::max<int64_t>(each, 1) * lanes;
  R.units = (int)((cols + R.unit - 1) / R.unit);
  R.pieces = (R.units + kVerifyThreads / 64 - 1) / (kVerifyThreads / 64);
  // us, later rows passed over | all of them read, without the launch that clears the counters (medians
  // of 7 blocks of passes in turn, which lie within 0.3 us of each other but for the largest, and for
  // logits 32 x 4 x 65536, where they reach 32.3 | 31.5): fp32 weights 32 x 4 x 65536 (19 M scores) 27.6 |
  // 26.5, 24 x 7 x 65536 (24 M) 29.0 | 31.0, 64 x 7 x 128000 125 | 155, 256 x 0 x 65536 49.0 | 46.9; bf16
  // logits 32 x 4 x 65536 30.1 | 29.7, 24 x 7 x 65536 32.0 | 33.4, 16 x 7 x 128000 (31 M) 36.5 | 38.7, 64 x
  // 7 x 128000 85 | 122.  (All read, draw_kernel tests all drafts in every workgroup:) bf16 logits 4 x 8 x
  // 8000 18.2 | 17.2, 4 x 12 x 8000 18.1 | 18.9, 4 x 64 x 8000 22 | 45, 1 x 200 x 3000 20 | 88.
  R.early = drafts > 10 || (drafts > 0 && rows * cols > 20000000);
  return R;
}

}  // namespace vqc
