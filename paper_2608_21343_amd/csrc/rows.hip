// How the row operators cut their rows (rows.hpp).
#include "rows.hpp"

namespace tbias {
namespace rows {

Plan plan(int32_t dtype, int64_t n_rows, int32_t C) {
  const int pv = dtype == TB_F32 ? 4 : 8;
  // One wave per row where it holds the row: no barriers, little work beside the
  // values, and results that do not depend on the number of rows. Longer rows
  // take the fewest waves that give the card's 1024 SIMDs two each.
  int best = -1;
  for (int i = 0; i < kShapes; ++i) {
    const Shape s = kShape[i];
    if (C > capacity(s, pv)) continue;
    if (best >= 0 && s.nwr == kShape[best].nwr) continue;  // more pieces than needed
    best = i;
    if (s.nwr == 1 || n_rows * s.nwr >= 2048) break;
  }
  // A few of the longest bfloat16 rows are cut across the card nevertheless: one
  // row of 131,073 with 8 alternatives 17.9 -> 13.6 us, 64 of them 20.1 -> 15.0,
  // 128 23.6 -> 20.6, but distillation gradients of 128 24.0 -> 23.7 (one of
  // 40,001 9.5 -> 14.9: a second launch).
  const bool few = best == kShapes - 1 && pv == 8 && n_rows <= 64;
  if (best >= 0 && !few) return {best, 1, C};
  // segments as short as one lane each allows
  for (int i = 0; i < kShapes; ++i) {
    const Shape s = kShape[i];
    const int32_t cap = capacity(s, pv), n_seg = (C + cap - 1) / cap;
    if (cuts(s) && n_seg <= kMaxSeg) return {i, n_seg, (C + n_seg - 1) / n_seg};
  }
  return {-1, 0, 0};
}

}  // namespace rows
}  // namespace tbias
