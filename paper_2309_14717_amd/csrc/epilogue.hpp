// What follows a linear, applied before its result leaves the kernel that has it:
//   z = (x W~' ) + bias;   y = act(z) * mul + residual        (z may be stored too, in bf16, for the backward)
// All in fp32 on the fp32 result; y is rounded once.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace qalora {

enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_GELU = 3, ACT_GELU_TANH = 4 };

struct Epilogue {
  const float* bias;     // [N], or null
  const uint16_t* mul;   // bf16 [M, N], or null
  const void* residual;  // [M, N] of y's type, or null
  uint16_t* z;           // bf16 [M, N], or null
  int act;
  int on;                // whether there is anything to do
};

// 1 / (1 + exp(-v)); zero and one where that is what fp32 holds.  The hardware's exponential takes v log2(e) rounded to fp32, so the
// relative error grows by |v| 2^-24 (measured: 1.2 |v| + 2 half steps of fp32 at v = -85); for bf16 results, and for fp32 ones that a
// sum follows, that is less than what follows.  erfc below grows by v^2 2^-24 likewise (1.3 v^2 measured).
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }
constexpr float kTanhSlope = 1.5957691216057308f;  // 2 sqrt(2 / pi): 0.5 (1 + tanh(u)) = logistic(2 u)
__device__ __forceinline__ float gelu_tanh_arg(float v) { return kTanhSlope * v * __builtin_fmaf(0.044715f * v, v, 1.0f); }

// (relu keeps a NaN.  The normal distribution function by erfc, which keeps its relative precision for negative v.)
template <int ACT>
__device__ __forceinline__ float act_value(float v) {
  if constexpr (ACT == ACT_RELU) return v < 0.0f ? 0.0f : v;
  if constexpr (ACT == ACT_SILU) return v * logistic(v);
  if constexpr (ACT == ACT_GELU) return 0.5f * v * erfcf(-0.70710678f * v);
  if constexpr (ACT == ACT_GELU_TANH) return v * logistic(gelu_tanh_arg(v));
  return v;
}
// f(integral_constant<the activation>): the choice is made once for many elements
template <typename Fn>
__device__ __forceinline__ void with_act(int act, Fn&& f) {
  switch (act) {
    case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>{});
    case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>{});
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>{});
    case ACT_GELU_TANH: return f(std::integral_constant<int, ACT_GELU_TANH>{});
    default: return f(std::integral_constant<int, ACT_NONE>{});
  }
}
template <int N, typename V>
__device__ __forceinline__ void act_values(int act, V& v) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = act_value<decltype(a)::value>(v[k]);
  });
}

// act(v) and its slope.  Beyond +-16 (silu: +-100) every slope is zero or one in fp32: the argument is held there, so that
// no product of an overflow and a zero arises.  (Comparisons, not fmin and fmax, which would lose a NaN.)
__device__ __forceinline__ float held(float v, float at) { return v > at ? at : (v < -at ? -at : v); }
template <int ACT>
__device__ __forceinline__ void act_slope(float v, float& value, float& slope) {
  if constexpr (ACT == ACT_RELU) {
    value = v < 0.0f ? 0.0f : v;
    slope = v > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == ACT_SILU) {
    const float c = held(v, 100.0f), s = logistic(c);
    value = v * s;
    slope = s * __builtin_fmaf(c, 1.0f - s, 1.0f);
  } else if constexpr (ACT == ACT_GELU) {
    const float c = held(v, 16.0f), cdf = 0.5f * erfcf(-0.70710678f * c);
    value = v * cdf;
    slope = __builtin_fmaf(0.39894228f * c, __expf(-0.5f * c * c), cdf);
  } else if constexpr (ACT == ACT_GELU_TANH) {
    const float c = held(v, 16.0f), s = logistic(gelu_tanh_arg(c));
    value = v * s;
    slope = __builtin_fmaf(c * s * (1.0f - s), kTanhSlope * __builtin_fmaf(3.0f * 0.044715f * c, c, 1.0f), s);
  } else {
    value = v;
    slope = 1.0f;
  }
}

typedef uint32_t epi_vec4 __attribute__((ext_vector_type(4)));

// The operands of eight neighbouring elements, requested before they are needed (for a tile that waits in LDS).
struct EpilogueOperands {
  epi_vec4 mul, residual[2];
};
__device__ __forceinline__ void request_operands(const Epilogue& e, size_t at, int out_bf16, EpilogueOperands& o) {
  if (e.mul) o.mul = *reinterpret_cast<const epi_vec4*>(e.mul + at);
  if (e.residual) {
    if (out_bf16) {
      o.residual[0] = *reinterpret_cast<const epi_vec4*>(static_cast<const uint16_t*>(e.residual) + at);
    } else {
      const epi_vec4* r = reinterpret_cast<const epi_vec4*>(static_cast<const float*>(e.residual) + at);
      o.residual[0] = r[0];
      o.residual[1] = r[1];
    }
  }
}
// ... and y of them from z, which is stored where that is asked for
__device__ __forceinline__ void apply_epilogue8(const Epilogue& e, const EpilogueOperands& o, float (&v)[8], size_t at, int out_bf16) {
  auto half = [](const epi_vec4& w, int k) { return __uint_as_float((k & 1) ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16); };
  if (e.z)
    *reinterpret_cast<epi_vec4*>(e.z + at) =
        epi_vec4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  act_values<8>(e.act, v);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (e.mul) v[k] *= half(o.mul, k);
    if (e.residual) v[k] += out_bf16 ? half(o.residual[0], k) : __uint_as_float(o.residual[k >> 2][k & 3]);
  }
}

// Four neighbouring elements (the first at element `at`, column `col`; both multiples of four): y from the linear's sums.
// Where residual is y itself, each is read here before the caller stores it.
__device__ __forceinline__ f32x4 apply_epilogue(const Epilogue& e, f32x4 v, size_t at, int col, int out_bf16) {
  typedef uint32_t pair __attribute__((ext_vector_type(2)));
  if (e.bias) v += *reinterpret_cast<const f32x4*>(e.bias + col);
  if (e.z) *reinterpret_cast<pair*>(e.z + at) = pair{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  act_values<4>(e.act, v);
  if (e.mul) {
    const pair m = *reinterpret_cast<const pair*>(e.mul + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= __uint_as_float((k & 1) ? m[k >> 1] & 0xffff0000u : m[k >> 1] << 16);
  }
  if (e.residual) {
    if (out_bf16) {
      const pair r = *reinterpret_cast<const pair*>(static_cast<const uint16_t*>(e.residual) + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += __uint_as_float((k & 1) ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
    } else {
      v += *reinterpret_cast<const f32x4*>(static_cast<const float*>(e.residual) + at);
    }
  }
  return v;
}

}  // namespace qalora
