// An AdamW step over many tensors, and the values of its 8-bit moments.
#pragma once

#include <cstdint>

#include "device.hpp"
#include "launch.hpp"

namespace tbias {
namespace adamw {

constexpr int32_t kBlock = 256;   // values that share a unit
constexpr int32_t kMost = 52;     // tensors of a launch: their records fit the kernel's arguments

struct Step {
  int32_t dtype, bits;
  bool master;
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* grad_scale;
  uint32_t seed;
};

hipError_t step(const tb_adamw_tensor* t, int32_t n, const Step& s, hipStream_t st);
hipError_t moments(const tb_adamw_tensor* t, int32_t n, float* const* out_m, float* const* out_v,
                   hipStream_t st);

}  // namespace adamw
}  // namespace tbias
