// Backward of a linear's epilogue y = act(z) * mul + residual, z = x W~' + bias:
//   dz = dy * mul * act'(z),   dmul = dy * act(z),   dbias = sum over the tokens of dz   (d residual = dy)
// One pass over dy, z and mul, bound by their bytes: sixteen bytes a thread of each operand, a wavefront along a row.  dz is
// what the linear's backward takes as its dy, in bf16 as there; dbias is the sum of the unrounded fp32 values, each
// block's rows first, then the blocks in order (a second small launch): no atomics, reruns are bit-identical.
#include "epilogue.hpp"
#include "int8.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void unpack8(const u32x4& w, float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = __uint_as_float((k & 1) ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
}  // namespace

// KEPT8: z and mul as they were kept in 8 bits (int8.hpp): one byte a column of each, and one more for 32
template <bool DY_BF16, bool KEPT8>
__global__ __launch_bounds__(EB_THREADS) void epilogue_back_kernel(const EpilogueBackArgs p) {
  __shared__ float share[EB_THREADS][8 + 1];
  const int lane = threadIdx.x & (p.plan.lanes - 1), row_in = threadIdx.x / p.plan.lanes;
  const int at_once = EB_THREADS / p.plan.lanes;
  const int col = (blockIdx.x * p.plan.lanes + lane) * 8;
  const bool live = col < p.cols;
  const long r0 = (long)blockIdx.y * p.plan.rows_per, r1 = min((long)p.rows, r0 + p.plan.rows_per);
  float sum[8] = {};
  struct Row {
    u32x4 dy[2], z, mul;
  };
  auto load = [&](long r) {
    const size_t at = (size_t)r * p.cols + col;
    Row w{};
    if (DY_BF16) {
      w.dy[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.dy) + at);
    } else {
      const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const float*>(p.dy) + at);
      w.dy[0] = src[0];
      w.dy[1] = src[1];
    }
    if constexpr (KEPT8) {
      const size_t e = keep8_exponents_at(p.rows, p.cols) + (size_t)r * keep8_groups(p.cols) + col / kKeepGroup;
      auto load8 = [&](const uint8_t* kept) {
        const u8x8 c = *reinterpret_cast<const u8x8*>(kept + at);
        return u32x4{c[0], c[1], kept[e], 0};
      };
      if (p.z8) w.z = load8(p.z8);
      if (p.mul8) w.mul = load8(p.mul8);
    } else {
      if (p.z) w.z = *reinterpret_cast<const u32x4*>(p.z + at);
      if (p.mul) w.mul = *reinterpret_cast<const u32x4*>(p.mul + at);
    }
    return w;
  };
  if (live && r0 + row_in < r1) {
    Row next = load(r0 + row_in);
    for (long r = r0 + row_in; r < r1; r += at_once) {
      const Row w = next;
      if (r + at_once < r1) next = load(r + at_once);  // while this row is worked on
      const size_t at = (size_t)r * p.cols + col;
      float dy[8], z[8], mul[8];
      if (DY_BF16) {
        unpack8(w.dy[0], dy);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) dy[k] = __uint_as_float(w.dy[k >> 2][k & 3]);
      }
      if constexpr (KEPT8) {
        restore8(u8x8{w.z[0], w.z[1]}, w.z[2], z);
        restore8(u8x8{w.mul[0], w.mul[1]}, w.mul[2], mul);
      } else {
        unpack8(w.z, z);
        unpack8(w.mul, mul);
      }
      float dz[8], dmul[8];
      with_act(p.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float value, slope;
          act_slope<decltype(act)::value>(z[k], value, slope);
          dmul[k] = dy[k] * value;
          dz[k] = dy[k] * slope;
        }
      });
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (KEPT8 ? p.mul8 != nullptr : p.mul != nullptr) dz[k] *= mul[k];
        sum[k] += dz[k];
      }
      if (p.dz) *reinterpret_cast<u32x4*>(p.dz + at) = pack8(dz);
      if (p.dmul) *reinterpret_cast<u32x4*>(p.dmul + at) = pack8(dmul);
    }
  }
  if (!p.dbias) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) share[threadIdx.x][k] = sum[k];
  __syncthreads();
  // A column's rows are added up in order, by a thread for each column (64 x 1024, gelu: 6.2 us, and 7.1 by a thread for eight).
  for (int v = threadIdx.x; v < p.plan.lanes * 8; v += EB_THREADS) {
    const int c = blockIdx.x * p.plan.lanes * 8 + v;
    if (c >= p.cols) break;
    float total = share[v / 8][v % 8];
#pragma unroll 8
    for (int r = 1; r < at_once; ++r) total += share[r * p.plan.lanes + v / 8][v % 8];
    const bool whole = gridDim.y == 1;  // the block has all rows
    float* o = whole ? p.dbias + c : p.partial + (size_t)blockIdx.y * p.cols + c;
    *o = whole && p.accumulate ? *o + total : total;
  }
}

// dbias = (accumulate ? dbias : 0) + the row blocks' shares, in order: 32 columns a block, their shares dealt to eight
// groups of threads (a thread that adds 94 of them by itself: 7 us)
__global__ __launch_bounds__(256) void epilogue_bias_kernel(const float* __restrict__ partial, int blocks, int cols, int accumulate,
                                                            float* __restrict__ dbias) {
  __shared__ float part[8][32];
  const int e = threadIdx.x & 31, group = threadIdx.x >> 5, c = blockIdx.x * 32 + e;
  const int per = (blocks + 7) / 8, b0 = min(blocks, group * per), b1 = min(blocks, b0 + per);
  float v = 0.0f;
  if (c < cols)
#pragma unroll 16
    for (int b = b0; b < b1; ++b) v += partial[(size_t)b * cols + c];
  part[group][e] = v;
  __syncthreads();
  if (group > 0 || c >= cols) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) v += part[k][e];
  dbias[c] = accumulate ? dbias[c] + v : v;
}

hipError_t launch_epilogue_backward(const EpilogueBackArgs& args, hipStream_t st) {
  EpilogueBackArgs a = args;
  a.plan = epilogue_back_plan(a.rows, a.cols);
  const dim3 grid(a.plan.col_blocks, a.plan.row_blocks);
  const bool kept8 = a.z8 || a.mul8;
  auto kernel = a.dy_bf16 ? (kept8 ? epilogue_back_kernel<true, true> : epilogue_back_kernel<true, false>)
                          : (kept8 ? epilogue_back_kernel<false, true> : epilogue_back_kernel<false, false>);
  kernel<<<grid, EB_THREADS, 0, st>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.dbias || a.plan.row_blocks == 1) return e;
  epilogue_bias_kernel<<<a.cols / 32 + (a.cols % 32 ? 1 : 0), 256, 0, st>>>(a.partial, a.plan.row_blocks, a.cols, a.accumulate, a.dbias);
  return hipGetLastError();
}

}  // namespace qalora
