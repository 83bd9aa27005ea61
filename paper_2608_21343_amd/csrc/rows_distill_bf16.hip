// Distillation loss and gradient of bfloat16 rows (rows_grad.hpp).
#include "rows_grad.hpp"

namespace tbias {
namespace rows {

hipError_t distill_bf16(const Rows& a, const DistillIO& io, const Plan& p, hipStream_t st) {
  return distill_t<uint16_t>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
