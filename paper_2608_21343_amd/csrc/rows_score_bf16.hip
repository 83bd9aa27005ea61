// Log probabilities, entropy and alternatives of bfloat16 rows (rows_score.hpp).
#include "rows_score.hpp"

namespace tbias {
namespace rows {

hipError_t score_bf16(const Rows& a, const ScoreIO& io, const Plan& p, hipStream_t st) {
  return score_t<uint16_t>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
