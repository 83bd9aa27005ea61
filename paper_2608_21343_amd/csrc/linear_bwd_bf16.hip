// Products with the logits' gradients of bfloat16 layers (linear_gemm.hpp).
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

hipError_t dx_bf16(const Gemm& g, hipStream_t st) { return launch<kDx, uint16_t>(g, st); }
hipError_t dw_bf16(const Gemm& g, hipStream_t st) { return launch<kDw, uint16_t>(g, st); }

}  // namespace linear
}  // namespace tbias
