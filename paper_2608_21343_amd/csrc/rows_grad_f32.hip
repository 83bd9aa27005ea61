// Gradient of log probabilities, log-sum-exp and entropy of float32 rows (rows_grad.hpp).
#include "rows_grad.hpp"

namespace tbias {
namespace rows {

hipError_t grad_f32(const Rows& a, const GradIO& io, const Plan& p, hipStream_t st) {
  return grad_t<float>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
