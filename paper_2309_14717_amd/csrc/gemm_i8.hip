// Products of 8-bit integers, exact in 32 bits, with a scale for each token and (forward) each output channel:
//   forward   z[t, j]  = s[t] sw[j] sum_i q[t, i] w8[j, i]      K = d_in
//   backward  dx[t, i] = s[t] sum_j q[t, j] w8[j, i]            K = d_out (the channels' scales are in q)
// and the epilogue on that.  One copy of the weight's codes, [d_out, d_in], serves both directions: the forward's operands lie along K in
// it, the backward's are turned by transposing LDS reads.
#include "int8.hpp"
#include "epilogue.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
}  // namespace

// A block: 64 tokens by 64 columns, a wavefront has sixteen of the columns.
template <bool BWD>
__global__ __launch_bounds__(256) void gemm_i8_kernel(const Int8GemmArgs p) {
  constexpr int ROW = 64 + 16;
  __shared__ __align__(16) int8_t xs[64 * ROW], ws[64 * ROW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_n = ceil_div(p.N, 64);
  const int n0 = (int)(blockIdx.x % tiles_n) * 64, m0 = (int)(blockIdx.x / tiles_n) * 64;
  const int lr = tid / 4, lc = (tid % 4) * 16;  // what this thread loads: sixteen bytes of a row of either tile
  i32x4 acc[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) acc[f] = i32x4{0, 0, 0, 0};
  for (int k0 = 0; k0 < p.K; k0 += 64) {
    i32x4 a{0, 0, 0, 0}, w{0, 0, 0, 0};
    if (m0 + lr < p.M && k0 + lc < p.lda) a = *reinterpret_cast<const i32x4*>(p.tokens + (size_t)(m0 + lr) * p.lda + k0 + lc);
    if (BWD) {
      if (k0 + lr < p.K && n0 + lc < p.N) w = *reinterpret_cast<const i32x4*>(p.codes + (size_t)(k0 + lr) * p.N + n0 + lc);
    } else {
      if (n0 + lr < p.N && k0 + lc < p.K) w = *reinterpret_cast<const i32x4*>(p.codes + (size_t)(n0 + lr) * p.K + k0 + lc);
    }
    __syncthreads();
    *reinterpret_cast<i32x4*>(xs + lr * ROW + lc) = a;
    *reinterpret_cast<i32x4*>(ws + lr * ROW + lc) = w;
    __syncthreads();
    i32x4 wf;
    if (BWD) {
      // sixteen lanes: eight rows (of K) by sixteen columns, a lane gives half a row's address and takes a column
      const int r = 16 * (lane >> 4) + ((lane & 15) >> 1), c = 16 * wave + 8 * (lane & 1);
      const i32x2 lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(ws + r * ROW + c));
      const i32x2 hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(ws + (r + 8) * ROW + c));
      wf = i32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      wf = *reinterpret_cast<const i32x4*>(ws + (16 * wave + (lane & 15)) * ROW + 16 * (lane >> 4));
    }
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const i32x4 xf = *reinterpret_cast<const i32x4*>(xs + (16 * f + (lane & 15)) * ROW + 16 * (lane >> 4));
      acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, xf, acc[f], 0, 0, 0);
    }
  }
  const int n = n0 + 16 * wave + 4 * (lane >> 4);
  if (n >= p.N) return;  // (N is a multiple of eight)
  f32x4 by = {1.0f, 1.0f, 1.0f, 1.0f};
  if (!BWD) by = *reinterpret_cast<const f32x4*>(p.col_scale + n);
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int m = m0 + 16 * f + (lane & 15);
    if (m >= p.M) continue;
    const float s = p.row_scale[m];
    f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (float)acc[f][r] * s * by[r];
    const size_t at = (size_t)m * p.N + n;
    v = apply_epilogue(p.epi, v, at, n, p.out_bf16);
    if (p.out_bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    else
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = v;
  }
}

hipError_t launch_gemm_i8(const Int8GemmArgs& a, hipStream_t st) {
  const unsigned blocks = (unsigned)((size_t)ceil_div(a.M, 64) * ceil_div(a.N, 64));
  if (a.back) gemm_i8_kernel<true><<<blocks, 256, 0, st>>>(a);
  else gemm_i8_kernel<false><<<blocks, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qalora
