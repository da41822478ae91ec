// Values in 8 bits, device side: codes of rows with one scale each (tokens, weight channels), and of groups of 32 columns
// that share an exponent (kept activations).
#pragma once
#include <type_traits>

#include "common.hpp"
#include "epilogue.hpp"

namespace qalora {

typedef uint32_t u8x8 __attribute__((ext_vector_type(2)));  // eight codes
typedef uint32_t u16x8 __attribute__((ext_vector_type(4)));  // eight bf16

// 1.5 * 2^23: adding it rounds to a whole number (ties to even), which then is the low byte of the sum, in two's complement
constexpr float kWhole = 12582912.0f;

// The low bytes of four words
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return ab | (cd << 16);
}
__device__ __forceinline__ float code_value(uint32_t word, int byte) { return (float)(int8_t)(word >> (8 * byte)); }
__device__ __forceinline__ float bf16_of(const u16x8& w, int k) {
  return __uint_as_float((k & 1) ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
}

// silu(gate) * up of eight columns.  (The hardware's reciprocal: with a division rows of hidden activations to 8 bits are bound by their
// arithmetic.)
__device__ __forceinline__ u16x8 swiglu8(const u16x8& g, const u16x8& u) {
  u16x8 h;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float g0 = bf16_of(g, 2 * k), g1 = bf16_of(g, 2 * k + 1);
    h[k] = pack_bf16x2(g0 * logistic(g0) * bf16_of(u, 2 * k), g1 * logistic(g1) * bf16_of(u, 2 * k + 1));
  }
  return h;
}

// ---- one scale a row: s = fl32(top fl32(1 / 127)), code = rne(v / s) of the exact quotient -----------------------------------

struct RowScale {
  float s;    // as stored: NaN for a row with an infinity or a NaN, then all codes are 0
  float up;   // v and s times this power of two are ordinary numbers whatever the row's magnitude
  float by;   // s * up
  float inv;  // 1 / by (to 2^-24 (1 + 2^-20) of it), 0 for a row without a scale
};
// `top`: the bits of the row's largest magnitude (as integers those of finite values, infinities and NaNs come in that order)
__device__ __forceinline__ RowScale row_scale_of(uint32_t top) {
  RowScale r;
  const bool finite = top < 0x7f800000u;
  // The largest magnitude times 1 / 127 (which fp32 has to 2^-28), a last place from the quotient at most: what an elementwise division by 127
  // is on this GPU's tensors, so that scales and codes that a program makes of them are these.
  const float s = __uint_as_float(top) * (1.0f / 127.0f);
  r.s = finite ? s : __uint_as_float(0x7fc00000u);
  r.up = top < 0x20000000u ? 0x1p64f : 1.0f;  // below 2^-63
  r.by = finite ? s * r.up : 0.0f;
  const float guess = __builtin_amdgcn_rcpf(r.by), inv = __builtin_fmaf(__builtin_fmaf(-r.by, guess, 1.0f), guess, guess);
  r.inv = r.by > 0.0f ? inv : 0.0f;
  return r;
}
// The largest of a wavefront's words, the same in every lane.
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  auto with = [&](auto control) { v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(control)::value, 0xf, 0xf, true)); };
  with(std::integral_constant<int, 0xb1>{});   // the neighbour
  with(std::integral_constant<int, 0x4e>{});   // the other pair of four
  with(std::integral_constant<int, 0x141>{});  // half a row of sixteen, mirrored
  with(std::integral_constant<int, 0x140>{});  // the row, mirrored
  uint32_t rows[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) rows[k] = (uint32_t)__builtin_amdgcn_readlane((int)v, 16 * k);
  return max(max(rows[0], rows[1]), max(rows[2], rows[3]));
}
// The codes of eight v.  inv is a last place from 1 / by at most, so v inv is off by at most 127 2^-24 (1 + 2^-20) = 7.6e-6 from the quotient, and
// rounding it can go wrong only that close to the middle between two codes; there the remainder v - code s, which fp32 holds exactly (it
// is a multiple of the smaller of the last places of v and s, and at most about s / 2), says which side v is on.  (A quotient is past
// 127 only where s is subnormal.)
__device__ __forceinline__ float exact_code(float v, float t, const RowScale& r) {
  const float q = __builtin_rintf(t), left = __builtin_fmaf(-q, r.by, v), twice = __builtin_fabsf(left) + __builtin_fabsf(left);
  const bool past = (twice > r.by) | ((twice == r.by) & (((int)q & 1) != 0));
  return __builtin_amdgcn_fmed3f(q + (past ? __builtin_copysignf(1.0f, left) : 0.0f), -127.0f, 127.0f) + kWhole;
}
__device__ __forceinline__ u8x8 row_codes(const float (&v)[8], const RowScale& r) {
  float f[8], worst = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    f[k] = __builtin_fmaf(v[k], r.inv, kWhole);  // the code in its low byte
    worst = fmaxf(worst, __builtin_fabsf(__builtin_fmaf(v[k], r.inv, kWhole - f[k])));
  }
  if (worst > 0.49999f || r.up != 1.0f) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w = v[k] * r.up;
      f[k] = exact_code(w, w * r.inv, r);
    }
  }
  uint32_t c[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) c[k] = __float_as_uint(f[k]);
  const uint32_t mask = r.inv > 0.0f ? 0xffffffffu : 0u;  // (no scale: codes 0)
  return u8x8{low_bytes(c[0], c[1], c[2], c[3]) & mask, low_bytes(c[4], c[5], c[6], c[7]) & mask};
}

// (acc s) by of four columns, each product rounded: not joined with a bias or a residual that is added next, so that a token's results do not
// depend on the kernel that the number of tokens chooses.
template <typename Sums>
__device__ __forceinline__ f32x4 scaled_sums(const Sums& acc, float s, const f32x4& by) {
#pragma clang fp contract(off)
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = (float)acc[r] * s * by[r];
  return v;
}

// ---- 32 neighbouring columns share an exponent ---------------------------------------------------------------------------

constexpr int kKeepGroup = 32;  // columns: four lanes of eight
// Bytes of [rows, cols] kept in 8 bits: the codes, row by row, then a biased exponent for each group of a row.
__host__ __device__ constexpr size_t keep8_groups(size_t cols) { return (cols + kKeepGroup - 1) / kKeepGroup; }
__host__ __device__ constexpr size_t keep8_exponents_at(size_t rows, size_t cols) { return (rows * cols + 15) / 16 * 16; }
__host__ __device__ constexpr size_t keep8_bytes(size_t rows, size_t cols) {
  return (keep8_exponents_at(rows, cols) + rows * keep8_groups(cols) + 15) / 16 * 16;
}

// The biased exponent E of the largest magnitude of four lanes' eight bf16 (1 for subnormal ones, 255 where there is an infinity or a NaN)
__device__ __forceinline__ uint32_t group_exponent(const u16x8& w) {
  typedef uint16_t pair __attribute__((ext_vector_type(2)));
  pair m = {0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(pair, w[k] & 0x7fff7fffu));
  uint32_t top = m.x > m.y ? m.x : m.y;
  top = max(top, (uint32_t)__shfl_xor((int)top, 1, 4));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2, 4));
  return max(top >> 7, 1u);
}
// The step between codes is 2^(E - 133): the largest magnitude, in [2^(E - 127), 2^(E - 126)), gets a code from 64 to 127.5, and that
// last one is held at 127, half a step off like any other.
__device__ __forceinline__ u8x8 group_codes(const u16x8& w, uint32_t E) {
  uint32_t c[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float t = __builtin_amdgcn_ldexpf(bf16_of(w, k), 133 - (int)E);
    c[k] = E < 255u ? __float_as_uint(__builtin_amdgcn_fmed3f(t, -127.0f, 127.0f) + kWhole) : 0u;
  }
  return u8x8{low_bytes(c[0], c[1], c[2], c[3]), low_bytes(c[4], c[5], c[6], c[7])};
}
// ... and back: bf16 numbers, exactly (seven bits and a power of two); all NaN for E = 255.
__device__ __forceinline__ float group_step(uint32_t E) {
  return E < 255u ? __builtin_amdgcn_ldexpf(1.0f, (int)E - 133) : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ void restore8(const u8x8& c, uint32_t E, float (&v)[8]) {
  const float step = group_step(E);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = code_value(c[k >> 2], k & 3) * step;
}

}  // namespace qalora
