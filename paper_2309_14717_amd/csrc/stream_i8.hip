// The product of 8-bit integers for few tokens (decode) in one launch: every block brings the tokens to 8 bits for itself, in LDS, while
// its first weights are on their way, and the weight is read once, straight into registers.
//   z[t, j] = s[t] sw[j] sum_i q[t, i] w8[j, i]
// A block has sixteen output channels and all tokens; its wavefronts share K, every eighth 128 bytes of the rows each, so that a
// channel's sum needs no other block.  Bound by the weight's bytes: 1 x 22016 x 8192 33 us, 5.4 TB/s (more loads ahead, or fewer registers for
// another block a compute unit: no faster); 16 x 1024 x 1024 6 us, of which the tokens' codes are 2.5.
#include "int8.hpp"
#include "epilogue.hpp"
#include "kernels.hpp"
#include "stream_i8_plan.hpp"

namespace qalora {

namespace {
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t kPastRows = 0xffff0000u;  // a byte offset past any sixteen rows: reads zero
constexpr int kReadOnce = 2;                 // cache policy: nontemporal
}  // namespace

__global__ __launch_bounds__(S8_WAVES * 64, 4) void stream_i8_kernel(const StreamI8Args p) {
  extern __shared__ __align__(16) int8_t xq[];  // [tokens][K + 16]: sixteen rows' reads of one chunk fall on different banks
  __shared__ __align__(16) int sums[S8_WAVES][64][4];
  __shared__ float scales[S8_TOKENS];
  __shared__ uint32_t tops[S8_WAVES][S8_TOKENS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 15, fc = lane >> 4, n0 = blockIdx.x * S8_COLS;
  const uint32_t rows = min((uint32_t)S8_COLS, (uint32_t)(p.N - n0)), K = (uint32_t)p.K;
  const __amdgpu_buffer_rsrc_t rs_w =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.codes + (size_t)n0 * p.K), 0, (int)(rows * K), 0x00020000);
  // A load takes eight channels' 128 bytes, whole cache lines: lane l sixteen of channel l % 8 (and 8 more in a piece's second load).
  // (Sixteen channels' 64 bytes, the matrix instruction's operand as it stands, took 35.4 instead of 28.9 us for 180 MB of loads alone.)
  const uint32_t w_at[2] = {(lane & 7) * K + 16 * (lane >> 3), ((lane & 7) + 8) * K + 16 * (lane >> 3)};
  const bool w_in[2] = {(uint32_t)(lane & 7) < rows, (uint32_t)(lane & 7) + 8 < rows};
  i32x4 wf[2][2], acc{0, 0, 0, 0};
  auto ask = [&](int set, int piece) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t k = (uint32_t)(piece * S8_WAVES + wave) * 128;
      const bool in = w_in[h] && k + 16 * (lane >> 3) < K;
      wf[set][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, (int)(in ? w_at[h] + k : kPastRows), 0, kReadOnce));
    }
  };
  ask(0, 0);

  // What the sums are finished with, on its way meanwhile: loads behind the sums would be waited for at the block's end.
  const int n = n0 + 4 * fc;
  const size_t at = (size_t)fr * p.N + n;
  const bool mine = wave == 0 && n < p.N && fr < p.M;
  f32x4 by = {0.0f, 0.0f, 0.0f, 0.0f};
  EpilogueFour operands{};
  if (mine) {
    by = *reinterpret_cast<const f32x4*>(p.col_scale + n);
    request_four(p.epi, at, n, p.out_bf16, operands);
  }

  // The tokens, each to as many wavefronts as there are for it
  const u16x8* x = reinterpret_cast<const u16x8*>(p.x);
  const int eights = p.K / 8, share = p.M == 1 ? 8 : p.M == 2 ? 4 : p.M <= 4 ? 2 : 1, first = (wave % share) * 64 + lane;
  for (int t = wave / share; t < p.M; t += S8_WAVES / share) {
    uint32_t top = 0;
    for (int e = first; e < eights; e += 64 * share) {
      const u16x8 w = x[(size_t)t * eights + e];
#pragma unroll
      for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(bf16_of(w, k)) & 0x7fffffffu);
    }
    top = wave_top(top);
    if (lane == 0) tops[wave % share][t] = top;
  }
  __syncthreads();
  for (int t = wave / share; t < p.M; t += S8_WAVES / share) {
    uint32_t top = 0;
    for (int w = 0; w < share; ++w) top = max(top, tops[w][t]);
    const RowScale r = row_scale_of(top);
    if (lane == 0) scales[t] = r.s;  // (the same from each of its wavefronts)
    for (int e = first; e < eights; e += 64 * share) {
      const u16x8 w = x[(size_t)t * eights + e];
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = bf16_of(w, k);
      *reinterpret_cast<u8x8*>(xq + t * (p.K + 16) + 8 * e) = row_codes(v, r);
    }
  }
  __syncthreads();

  auto multiply = [&](int set, int piece) {
    const uint32_t k = (uint32_t)(piece * S8_WAVES + wave) * 128 + 32 * fc;
    i32x4 x0{0, 0, 0, 0}, x1{0, 0, 0, 0};
    if (fr < p.M && k < K) x0 = *reinterpret_cast<const i32x4*>(xq + fr * (p.K + 16) + k);
    if (fr < p.M && k + 16 < K) x1 = *reinterpret_cast<const i32x4*>(xq + fr * (p.K + 16) + k + 16);
    // The matrix instruction's operand is sixteen channels by four chunks: lanes 8 to 15 of each sixteen and the two loads change places,
    // after which the first holds chunks 0, 2, 4, 6 of all channels and the second the others.
    i32x4 even, odd;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      even[r] = __builtin_amdgcn_update_dpp(wf[set][0][r], wf[set][1][r], 0x128, 0xf, 0xc, false);  // row_ror:8
      odd[r] = __builtin_amdgcn_update_dpp(wf[set][1][r], wf[set][0][r], 0x128, 0xf, 0x3, false);
    }
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, x0, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, x1, acc, 0, 0, 0);
  };
  const int pieces = ceil_div(p.K, 128 * S8_WAVES);
#pragma nounroll
  for (int k = 0;; k += 2) {  // the next piece is on its way while this one is multiplied (past the last: zeros)
    ask(1, k + 1);
    multiply(0, k);
    if (k + 1 >= pieces) break;
    ask(0, k + 2);
    multiply(1, k + 1);
    if (k + 2 >= pieces) break;
  }

  *reinterpret_cast<i32x4*>(sums[wave][lane]) = acc;
  __syncthreads();
  if (!mine) return;
#pragma unroll
  for (int w = 1; w < S8_WAVES; ++w) acc += *reinterpret_cast<const i32x4*>(sums[w][lane]);
  const float s = scales[fr];
  const f32x4 v = apply_four(p.epi, operands, scaled_sums(acc, s, by), at);
  if (p.out_bf16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = v;
}

hipError_t launch_stream_i8(const StreamI8Args& a, hipStream_t st) {
  stream_i8_kernel<<<ceil_div(a.N, S8_COLS), S8_WAVES * 64, (size_t)a.M * (a.K + 16), st>>>(a);
  return hipGetLastError();
}

}  // namespace qalora
