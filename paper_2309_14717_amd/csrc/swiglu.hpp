// The elementwise part of a SwiGLU block and its slopes, in fp32.
#pragma once
#include "common.hpp"

namespace qalora {

__device__ __forceinline__ float sigmoidf_(float v) { return 1.0f / (1.0f + __expf(-v)); }
__device__ __forceinline__ float swiglu_value(float g, float u) { return g * sigmoidf_(g) * u; }
// dgate = dh * up * d/dg[g sigmoid(g)] = dh * up * sig * (1 + g (1 - sig));  dup = dh * g * sig
__device__ __forceinline__ void swiglu_slopes(float d, float g, float u, float& dg, float& du) {
  const float s = sigmoidf_(g);
  dg = d * u * (s * (1.0f + g * (1.0f - s)));
  du = d * g * s;
}

}  // namespace qalora
