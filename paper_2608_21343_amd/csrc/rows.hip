// How the row operators cut their rows (rows.hpp).
#include "rows.hpp"

namespace tbias {
namespace rows {

Plan plan(int32_t dtype, int64_t n_rows, int32_t C) {
  const int pv = dtype == TB_F32 ? 4 : 8;
  for (int i = 0; i < kShapes; ++i)
    if (C <= capacity(shape(pv, i), pv)) return {i, 1, C};
  // longer rows: segments as short as one lane each allows
  for (int i = 0; i < kShapes; ++i) {
    const Shape s = shape(pv, i);
    const int32_t cap = capacity(s, pv), n_seg = (C + cap - 1) / cap;
    if (cuts(s) && n_seg <= kMaxSeg) return {i, n_seg, (C + n_seg - 1) / n_seg};
  }
  return {-1, 0, 0};
}

}  // namespace rows
}  // namespace tbias
