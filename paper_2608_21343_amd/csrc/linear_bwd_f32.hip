// Products with the logits' gradients of float32 layers (linear_gemm.hpp).
#include "linear_gemm.hpp"

namespace tbias {
namespace linear {

hipError_t dx_f32(const Gemm& g, hipStream_t st) { return launch<kDx, float>(g, st); }
hipError_t dw_f32(const Gemm& g, hipStream_t st) { return launch<kDw, float>(g, st); }

}  // namespace linear
}  // namespace tbias
