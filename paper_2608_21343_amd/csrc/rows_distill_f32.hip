// Distillation loss and gradient of float32 rows (rows_grad.hpp).
#include "rows_grad.hpp"

namespace tbias {
namespace rows {

hipError_t distill_f32(const Rows& a, const DistillIO& io, const Plan& p, hipStream_t st) {
  return distill_t<float>(a, io, p, st);
}

}  // namespace rows
}  // namespace tbias
