// The forward product with an epilogue (gemm_dq_impl.hpp's kernel, which applies it as the tile leaves), and the sum over
// the slices of a split K range with one.
#include "gemm_dq_impl.hpp"
#include "split_sum.hpp"

namespace qalora {

template <int NBITS>
static hipError_t launch_fwd(const GemmEpiArgs& a, hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  if (a.a_main_padded_rows >= round_up(a.M, 256) && gemm_fast_shape(a.K_main, a.group)) {
    if (a.tile_rows == 256) return launch_cfg<NBITS, false, 256, 256, 2, 4, true>(a, 1, st, e0, e1);
    if (a.tile_rows == 192) return launch_cfg<NBITS, false, 192, 256, 2, 4, true>(a, 1, st, e0, e1);
    if (a.tile_rows == 128) return launch_cfg<NBITS, false, 128, 256, 2, 4, true>(a, 1, st, e0, e1);
    return launch_cfg<NBITS, false, 64, 256, 1, 8, true>(a, 1, st, e0, e1);
  }
  if (a.tile_rows > 64) return launch_cfg<NBITS, false, 128, 256, 2, 4, false>(a, 1, st, e0, e1);
  return launch_cfg<NBITS, false, 64, 256, 1, 8, false>(a, 1, st, e0, e1);
}

hipError_t launch_gemm_dq_epi(int bits, const GemmEpiArgs& a, hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  if (bits == 4) return launch_fwd<4>(a, st, e0, e1);
  return bits == 3 ? launch_fwd<3>(a, st, e0, e1) : launch_fwd<2>(a, st, e0, e1);
}

__global__ __launch_bounds__(256) void split_epilogue_kernel(const SplitSum s, const Epilogue epi, int cols) {
  const size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x;  // group of 4 elements
  if (i >= s.n4) return;
  const f32x4 v = apply_epilogue(epi, split_sum_value(s, i), 4 * i, (int)(4 * i % (size_t)cols), s.out_bf16);
  split_sum_store(s, i, v);
}

hipError_t launch_split_epilogue(const SplitSum& s, const Epilogue& epi, int cols, hipStream_t st) {
  split_epilogue_kernel<<<(unsigned)((s.n4 + 255) / 256), 256, 0, st>>>(s, epi, cols);
  return hipGetLastError();
}

}  // namespace qalora
