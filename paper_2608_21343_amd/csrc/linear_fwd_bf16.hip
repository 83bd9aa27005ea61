// Logits' statistics and gradients of bfloat16 layers (linear_gemm.hpp).
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

hipError_t stats_bf16(const Gemm& g, hipStream_t st) { return launch<kStats, uint16_t>(g, st); }
hipError_t logit_grad_bf16(const Gemm& g, hipStream_t st) { return launch<kLogitGrad, uint16_t>(g, st); }

}  // namespace linear
}  // namespace tbias
