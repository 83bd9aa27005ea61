// Log probabilities, entropy and alternatives of float32 rows (rows_score.hpp).
#include "rows_score.hpp"

namespace tbias {
namespace rows {

hipError_t score_f32(const Rows& a, const ScoreIO& io, const Plan& p, hipStream_t st) {
  return score_t<float>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
