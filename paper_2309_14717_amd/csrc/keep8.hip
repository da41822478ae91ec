// Activations kept in 8 bits for the backward: 32 neighbouring columns of a row share the exponent of their largest magnitude, codes
// are whole multiples of 2^(E - 133).  What comes back are bf16 numbers.
// Elementwise passes bound by their bytes: a lane has eight columns, four lanes a group.  4096 x 11008: SwiGLU 68 us each way (5.3 TB/s);
// 1531 x 13824 kept alone 12.6 us (5.1 TB/s), restored 12.1.
#include "int8.hpp"
#include "kernels.hpp"
#include "swiglu.hpp"

namespace qalora {

namespace {
// The places of a thread, one after the other, in rows of `per_row` (a multiple of four, the last of them past the row where its
// columns are not a multiple of 32).
struct Places {
  size_t row;
  int at;
  size_t row_step;
  int at_step;
  __device__ Places(int per_row) {
    const size_t first = blockIdx.x * (size_t)blockDim.x + threadIdx.x, stride = (size_t)gridDim.x * blockDim.x;
    row = first / per_row;
    at = (int)(first % per_row);
    row_step = stride / per_row;
    at_step = (int)(stride % per_row);
  }
  __device__ void next(int per_row) {
    row += row_step;
    at += at_step;
    if (at >= per_row) {
      at -= per_row;
      ++row;
    }
  }
};
}  // namespace

__global__ __launch_bounds__(256) void keep8_kernel(const Keep8Args p) {
  const int eights = p.cols / 8, per_row = round_up(eights, 4);
  const size_t groups = keep8_groups(p.cols);
  uint8_t* exponents = p.kept + keep8_exponents_at(p.rows, p.cols);
  for (Places i(per_row); i.row < p.rows; i.next(per_row)) {  // (a group's four lanes leave together)
    u16x8 w{0, 0, 0, 0};
    if (i.at < eights) w = reinterpret_cast<const u16x8*>(p.x)[i.row * eights + i.at];
    const uint32_t E = group_exponent(w);
    if (i.at >= eights) continue;
    reinterpret_cast<u8x8*>(p.kept)[i.row * eights + i.at] = group_codes(w, E);
    if (i.at % 4 == 0) exponents[i.row * groups + i.at / 4] = (uint8_t)E;
  }
}

__global__ __launch_bounds__(256) void restore8_kernel(const Keep8Args p) {
  const int eights = p.cols / 8, per_row = round_up(eights, 4);
  const size_t groups = keep8_groups(p.cols);
  const uint8_t* exponents = p.kept + keep8_exponents_at(p.rows, p.cols);
  for (Places i(per_row); i.row < p.rows; i.next(per_row)) {
    if (i.at >= eights) continue;
    float v[8];
    restore8(reinterpret_cast<const u8x8*>(p.kept)[i.row * eights + i.at], exponents[i.row * groups + i.at / 4], v);
    reinterpret_cast<u16x8*>(p.x)[i.row * eights + i.at] =
        u16x8{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
}

// (h or what is kept may be left out.)  gu = [gate | up] is [2 rows, cols] to what keeps it: a token's gate is row 2t, its up row 2t + 1.
__global__ __launch_bounds__(256) void swiglu_keep8_kernel(const Swiglu8Args p) {
  const int eights = p.cols / 8, per_row = round_up(eights, 4);
  const size_t groups = keep8_groups(p.cols);
  uint8_t* exponents = p.kept + keep8_exponents_at(2 * p.rows, p.cols);
  for (Places i(per_row); i.row < p.rows; i.next(per_row)) {
    u16x8 g{0, 0, 0, 0}, u{0, 0, 0, 0};
    const size_t at = i.row * 2 * eights + i.at;
    if (i.at < eights) {
      g = reinterpret_cast<const u16x8*>(p.gu)[at];
      u = reinterpret_cast<const u16x8*>(p.gu)[at + eights];
    }
    const uint32_t eg = group_exponent(g), eu = group_exponent(u);
    if (i.at >= eights) continue;
    if (p.h) reinterpret_cast<u16x8*>(p.h)[i.row * eights + i.at] = swiglu8(g, u);
    if (!p.kept) continue;
    reinterpret_cast<u8x8*>(p.kept)[at] = group_codes(g, eg);
    reinterpret_cast<u8x8*>(p.kept)[at + eights] = group_codes(u, eu);
    if (i.at % 4 == 0) {
      exponents[i.row * 2 * groups + i.at / 4] = (uint8_t)eg;
      exponents[(i.row * 2 + 1) * groups + i.at / 4] = (uint8_t)eu;
    }
  }
}

__global__ __launch_bounds__(256) void swiglu_kept8_back_kernel(const Swiglu8Args p) {
  const int eights = p.cols / 8, per_row = round_up(eights, 4);
  const size_t groups = keep8_groups(p.cols);
  const uint8_t* exponents = p.kept + keep8_exponents_at(2 * p.rows, p.cols);
  for (Places i(per_row); i.row < p.rows; i.next(per_row)) {
    if (i.at >= eights) continue;
    const size_t at = i.row * 2 * eights + i.at, e = i.row * 2 * groups + i.at / 4;
    const u16x8 d = reinterpret_cast<const u16x8*>(p.h)[i.row * eights + i.at];
    float g[8], u[8], dg[8], du[8];
    restore8(reinterpret_cast<const u8x8*>(p.kept)[at], exponents[e], g);
    restore8(reinterpret_cast<const u8x8*>(p.kept)[at + eights], exponents[e + groups], u);
#pragma unroll
    for (int k = 0; k < 8; ++k) swiglu_slopes(bf16_of(d, k), g[k], u[k], dg[k], du[k]);
    u16x8* out = reinterpret_cast<u16x8*>(p.gu) + at;
    out[0] = u16x8{pack_bf16x2(dg[0], dg[1]), pack_bf16x2(dg[2], dg[3]), pack_bf16x2(dg[4], dg[5]), pack_bf16x2(dg[6], dg[7])};
    out[eights] = u16x8{pack_bf16x2(du[0], du[1]), pack_bf16x2(du[2], du[3]), pack_bf16x2(du[4], du[5]), pack_bf16x2(du[6], du[7])};
  }
}

namespace {
unsigned places_blocks(size_t rows, size_t cols) {
  const size_t n = (rows * (size_t)round_up((int)(cols / 8), 4) + 255) / 256;
  return (unsigned)(n < 4096 ? n : 4096);
}
}  // namespace

hipError_t launch_keep8(const Keep8Args& a, hipStream_t st) {
  keep8_kernel<<<places_blocks(a.rows, a.cols), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_restore8(const Keep8Args& a, hipStream_t st) {
  restore8_kernel<<<places_blocks(a.rows, a.cols), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_swiglu_keep8(const Swiglu8Args& a, hipStream_t st) {
  swiglu_keep8_kernel<<<places_blocks(a.rows, a.cols), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_swiglu_kept8_backward(const Swiglu8Args& a, hipStream_t st) {
  swiglu_kept8_back_kernel<<<places_blocks(a.rows, a.cols), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qalora
