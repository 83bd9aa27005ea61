// How the row operators cut their rows (rows.hpp).
#include "rows.hpp"

namespace tbias {
namespace rows {

namespace {

// Segments of the shape (4, np); false where that takes too many.
bool cut(int np, int pv, int32_t C, Plan* p) {
  for (int i = 0; i < kShapes; ++i) {
    const Shape s = kShape[i];
    if (!cuts(s) || s.np != np) continue;
    const int32_t cap = capacity(s, pv), n_seg = (C + cap - 1) / cap;
    *p = {i, n_seg, (C + n_seg - 1) / n_seg};
    return n_seg <= kMaxSeg;
  }
  return false;
}

}  // namespace

Plan plan(int32_t dtype, int64_t n_rows, int32_t C, bool grad) {
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
  if (best >= 0) {
    // Rows of sixteen waves are better cut where nothing is written back and the
    // rows do not fit the card at once: 4096 rows of 33,000 bfloat16 with 8
    // alternatives 96 us whole, 64 cut; 256 rows 12 and 15. Those that fill the
    // registers of a CU are cut at any number of rows (bfloat16: 64 of 131,073
    // 20 us and 15, 256 29 and 27, 2048 171 and 100), but for a gradient only
    // where they are few, for it reads cut rows twice (one row of 131,073 17 us
    // whole, 15 cut, 128 24 and 24, 2048 227 and more than 300).
    const Shape s = kShape[best];
    const bool all = fills(s, pv);
    const bool whole = s.nwr < 16 || (grad ? !all || n_rows > 64 : !all && n_rows <= 512);
    if (whole) return {best, 1, C};
  }
  // few rows: short segments on many CUs; many: fewer lists and sums to join
  // (2048 rows of 131,073 bfloat16 with 8 alternatives 107 us in segments of
  // (4, 8), 100 in those of (4, 16); 64 rows 12.7 and 14.2)
  Plan p;
  if ((n_rows <= 512 && cut(8, pv, C, &p)) || cut(16, pv, C, &p)) return p;
  return {-1, 0, 0};
}

int64_t most_workspace(int32_t dtype, int64_t n_rows, int32_t C, int32_t n_alt) {
  // Fewer rows may be cut into more segments: the last counts before plan() decides
  // otherwise.
  int64_t most = 0;
  for (int64_t n : {n_rows, (int64_t)64, (int64_t)127, (int64_t)511, (int64_t)512, (int64_t)1023}) {
    n = n < n_rows ? n : n_rows;
    for (bool grad : {false, true}) {
      const int64_t b = workspace_bytes(plan(dtype, n, C, grad), n, grad ? 0 : n_alt);
      most = b > most ? b : most;
    }
  }
  return most;
}

}  // namespace rows
}  // namespace tbias
