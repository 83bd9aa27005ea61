// Gradient of log probabilities, log-sum-exp and entropy of bfloat16 rows (rows_grad.hpp).
#include "rows_grad.hpp"

namespace tbias {
namespace rows {

hipError_t grad_bf16(const Rows& a, const GradIO& io, const Plan& p, hipStream_t st) {
  return grad_t<uint16_t>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
