// Logits' statistics and gradients of float32 layers (linear_gemm.hpp).
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

hipError_t stats_f32(const Gemm& g, hipStream_t st) { return launch<kStats, float>(g, st); }
hipError_t logit_grad_f32(const Gemm& g, hipStream_t st) { return launch<kLogitGrad, float>(g, st); }

}  // namespace linear
}  // namespace tbias
