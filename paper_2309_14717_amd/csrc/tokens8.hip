// Rows in 8 bits with one scale each: tokens (bf16, as they are, times a factor for each column, or as a SwiGLU's hidden activations)
// and the channels of a weight.
//   s = fl32(max |v| fl32(1 / 127)),   code = rne(v / s)
// The tokens' kernel reads a row once, up to 65536 columns (hidden activations: 32768; longer rows twice): a block (or a wavefront, for rows
// up to 1024 columns) has it whole in registers as bf16 when the largest magnitude is known.  Bound by its bytes, 3 a column (SwiGLU: 5,
// and 2 more with the kept halves), and a good part of them by its arithmetic, eleven operations a column: 4096 rows of 11008 with
// factors 26.6 us, 5.1 TB/s, 4096 plain ones of 4096 12.5 us, 1531 rows of 13824 hidden activations 22 us (kept too: 33.5); without the
// codes' arithmetic 24.6, 10.0 and 20.
#include "int8.hpp"
#include "kernels.hpp"
#include "tokens8_plan.hpp"

namespace qalora {

namespace {
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
}  // namespace

template <int LANES, int PIECES, int FROM>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void tokens8_kernel(const Tokens8Args p) {
  constexpr int WAVES = LANES / 64;
  constexpr bool HOLD = LANES < 1024 || PIECES <= (FROM == TOKENS8_SWIGLU ? 4 : 8);  // (else a row is read twice)
  const int lane = threadIdx.x % LANES, eights = p.cols / 8;
  // The factors of a thread's columns, for all rows it comes to: read for each row they would be more bytes than the row.
  // (Where they are too many for the registers, of rows beyond 16384 columns, they are.)
  constexpr bool KEEP = FROM == TOKENS8_SCALED && PIECES * 8 <= 64 && LANES < 1024;
  f32x4 factor[KEEP ? PIECES : 1][2];
  if constexpr (KEEP)
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
      const int at = lane + q * LANES;
      factor[q][0] = factor[q][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (at < eights) {
        factor[q][0] = reinterpret_cast<const f32x4*>(p.factor)[2 * at];
        factor[q][1] = reinterpret_cast<const f32x4*>(p.factor)[2 * at + 1];
      }
    }
  auto values = [&](const u16x8& w, int q, float (&v)[8]) {
    f32x4 f[2];
    if constexpr (KEEP && HOLD) {
      f[0] = factor[q][0];
      f[1] = factor[q][1];
    } else if (FROM == TOKENS8_SCALED && lane + q * LANES < eights) {
      f[0] = reinterpret_cast<const f32x4*>(p.factor)[2 * (lane + q * LANES)];
      f[1] = reinterpret_cast<const f32x4*>(p.factor)[2 * (lane + q * LANES) + 1];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = FROM == TOKENS8_SCALED ? bf16_of(w, k) * f[k >> 2][k & 3] : bf16_of(w, k);
  };

  struct Columns {  // eight of a row: as they are, or gate and up
    u16x8 x, up;
  };
  auto load = [&](size_t row, int q) {
    const int at = lane + q * LANES;
    Columns c{u16x8{0, 0, 0, 0}, u16x8{0, 0, 0, 0}};
    if (at < eights && row < (size_t)p.row_end) {
      const u16x8* src = reinterpret_cast<const u16x8*>(p.x) + row * eights * (FROM == TOKENS8_SWIGLU ? 2 : 1) + at;
      c.x = src[0];
      if (FROM == TOKENS8_SWIGLU) c.up = src[eights];
    }
    return c;
  };
  // What is brought to 8 bits of them; what else is asked for of a SwiGLU is stored.
  auto finish = [&](size_t row, const Columns& c, int q) {
    if (FROM != TOKENS8_SWIGLU) return c.x;
    const int at = lane + q * LANES;
    const u16x8 h = swiglu8(c.x, c.up);
    if (p.kept) {  // (a group's four lanes go together: lanes past the row have zeros)
      const uint32_t eg = group_exponent(c.x), eu = group_exponent(c.up);
      if (at < eights) {
        u8x8* codes = reinterpret_cast<u8x8*>(p.kept) + row * 2 * eights + at;
        codes[0] = group_codes(c.x, eg);
        codes[eights] = group_codes(c.up, eu);
        if (at % 4 == 0) {
          const size_t groups = keep8_groups(p.cols);
          uint8_t* e = p.kept + keep8_exponents_at(2 * (size_t)p.rows, p.cols) + row * 2 * groups + at / 4;
          e[0] = (uint8_t)eg;
          e[groups] = (uint8_t)eu;
        }
      }
    }
    if (p.h && at < eights) reinterpret_cast<u16x8*>(p.h)[row * eights + at] = h;
    return h;
  };
  uint32_t top = 0;
  auto largest = [&](const u16x8& w, int q) {
    if (lane + q * LANES >= eights) return;
    float v[8];
    values(w, q, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, magnitude(v[k]));
  };

  // A row's columns stay in registers, and the next row's are on their way while this one's codes are made.
  [[maybe_unused]] int turn = 0;
  const size_t step = (size_t)gridDim.x * (LANES == 64 ? 4 : 1);
  size_t row = (size_t)p.row_begin + (LANES == 64 ? blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x);
  Columns next[HOLD ? PIECES : 1];
  u16x8 held[HOLD ? PIECES : 1];
  if constexpr (HOLD)
#pragma unroll
    for (int q = 0; q < PIECES; ++q) next[q] = load(row, q);
  for (; row < (size_t)p.row_end; row += step) {
    top = 0;
    if constexpr (HOLD) {
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        held[q] = finish(row, next[q], q);
        largest(held[q], q);
      }
#pragma unroll
      for (int q = 0; q < PIECES; ++q) next[q] = load(row + step, q);
    } else {
#pragma nounroll
      for (int q = 0; q < PIECES; ++q) largest(finish(row, load(row, q), q), q);
    }
    top = wave_top(top);
    if constexpr (WAVES > 1) {
      __shared__ uint32_t tops[2][WAVES];  // alternating: a wavefront may be a row ahead
      uint32_t(&now)[WAVES] = tops[turn];
      turn ^= 1;
      if (threadIdx.x % 64 == 0) now[threadIdx.x / 64] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = max(top, now[w]);
    }
    const RowScale r = row_scale_of(top);
    if (lane == 0) p.scale[row] = r.s;
    auto store = [&](const u16x8& w, int q) {
      const int at = lane + q * LANES;
      if (at >= p.ld / 8) return;  // (the columns up to a longer row's end are zeros)
      float v[8] = {};
      if (at < eights) values(w, q, v);
      reinterpret_cast<u8x8*>(p.codes)[row * (p.ld / 8) + at] = row_codes(v, r);
    };
    if constexpr (HOLD) {
#pragma unroll
      for (int q = 0; q < PIECES; ++q) store(held[q], q);
    } else {
#pragma nounroll
      for (int q = 0; q < PIECES; ++q) {
        const Columns c = load(row, q);
        store(FROM == TOKENS8_SWIGLU ? swiglu8(c.x, c.up) : c.x, q);
      }
    }
  }
}

hipError_t launch_tokens8(const Tokens8Args& args, hipStream_t st) {
  const Tokens8Plan plan = tokens8_plan(args.rows, args.ld);
  Tokens8Args a = args;
  auto go = [&](auto from_c) {
    constexpr int FROM = decltype(from_c)::value;
    const size_t want = ((size_t)a.row_end - a.row_begin + plan.rows - 1) / plan.rows;
    const size_t most = tokens8_blocks(plan, a.rows, FROM == TOKENS8_PLAIN, FROM == TOKENS8_SWIGLU);
    const unsigned blocks = (unsigned)(want < most ? want : most);
    switch (plan.lanes * 100 + plan.pieces) {
      case 6401: tokens8_kernel<64, 1, FROM><<<blocks, 256, 0, st>>>(a); break;
      case 6402: tokens8_kernel<64, 2, FROM><<<blocks, 256, 0, st>>>(a); break;
      case 25601: tokens8_kernel<256, 1, FROM><<<blocks, 256, 0, st>>>(a); break;
      case 25602: tokens8_kernel<256, 2, FROM><<<blocks, 256, 0, st>>>(a); break;
      case 51202: tokens8_kernel<512, 2, FROM><<<blocks, 512, 0, st>>>(a); break;
      case 51203: tokens8_kernel<512, 3, FROM><<<blocks, 512, 0, st>>>(a); break;
      case 51204: tokens8_kernel<512, 4, FROM><<<blocks, 512, 0, st>>>(a); break;
      case 102401: tokens8_kernel<1024, 1, FROM><<<blocks, 1024, 0, st>>>(a); break;
      case 102402: tokens8_kernel<1024, 2, FROM><<<blocks, 1024, 0, st>>>(a); break;
      case 102404: tokens8_kernel<1024, 4, FROM><<<blocks, 1024, 0, st>>>(a); break;
      case 102408: tokens8_kernel<1024, 8, FROM><<<blocks, 1024, 0, st>>>(a); break;
      case 102416: tokens8_kernel<1024, 16, FROM><<<blocks, 1024, 0, st>>>(a); break;
      default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
  };
  hipError_t e = hipSuccess;
  for (int r = 0; r < a.rows && e == hipSuccess; r = a.row_end) {  // (a launch has at most 2^32 threads)
    a.row_begin = r;
    a.row_end = a.rows - r > T8_MOST_ROWS ? r + T8_MOST_ROWS : a.rows;
    switch (a.from) {
      case TOKENS8_PLAIN: e = go(std::integral_constant<int, TOKENS8_PLAIN>{}); break;
      case TOKENS8_SCALED: e = go(std::integral_constant<int, TOKENS8_SCALED>{}); break;
      default: e = go(std::integral_constant<int, TOKENS8_SWIGLU>{}); break;
    }
  }
  return e;
}

// ---- a weight's channels -------------------------------------------------------------------------------------------------
// W [d_in, d_out] fp32, or alpha code + beta (one rounding) of a quantized layer, to codes [d_out, d_in].  Done once for a model (4096 x 11008 115 us, 8192 x
// 22016 440; of INT4 layers 130 and 420: W, or the packed codes, are read twice, by a lane a channel): the
// channels' largest magnitudes (by atomic maxima of their bits, whose order does not matter), then the codes, then the scales.

template <int NBITS>  // 0: W
__device__ __forceinline__ float weight_at(const Weight8Args& p, int i, int j) {
  if constexpr (NBITS == 0) {
    return p.W[(size_t)i * p.d_out + j];
  } else {
    constexpr int RB = PackFmt<NBITS>::kRowsPerWord0, LB = NBITS == 3 ? 2 : NBITS;
    const int r = i % RB;
    uint32_t code = (p.plane0[(size_t)(i / RB) * p.d_out + j] >> (LB * (r >> 1) + 16 * (r & 1))) & ((1u << LB) - 1);
    if constexpr (NBITS == 3) {
      const int r1 = i % 32;
      code |= ((p.plane1[(size_t)(i / 32) * p.d_out + j] >> ((r1 >> 1) + 16 * (r1 & 1))) & 1u) << 2;
    }
    const size_t at = (size_t)(i / p.group) * p.d_out + j;
    return __builtin_fmaf(p.alpha[at], (float)code, p.beta[at]);
  }
}

__global__ __launch_bounds__(256) void weight8_clear_kernel(const Weight8Args p) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j < p.d_out) p.scale[j] = 0.0f;
}
constexpr int W8_ROWS = 256;  // of W, a block's share of a channel's magnitudes
template <int NBITS>
__global__ __launch_bounds__(256) void weight8_top_kernel(const Weight8Args p) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= p.d_out) return;
  const int i0 = blockIdx.y * W8_ROWS, i1 = min(p.d_in, i0 + W8_ROWS);
  uint32_t top = 0;
#pragma unroll 8
  for (int i = i0; i < i1; ++i) top = max(top, magnitude(weight_at<NBITS>(p, i, j)));
  atomicMax(reinterpret_cast<uint32_t*>(p.scale) + j, top);
}
// 64 rows of W by 64 channels, transposed through LDS
template <int NBITS>
__global__ __launch_bounds__(256) void weight8_codes_kernel(const Weight8Args p) {
  __shared__ uint8_t tile[64][64 + 4];
  const int c = threadIdx.x % 64, j = blockIdx.x * 64 + c, i0 = blockIdx.y * 64;
  if (j < p.d_out) {
    const RowScale r = row_scale_of(reinterpret_cast<const uint32_t*>(p.scale)[j]);
    for (int k = threadIdx.x / 64; k < 64 && i0 + k < p.d_in; k += 4) {
      const float w = weight_at<NBITS>(p, i0 + k, j) * r.up;
      tile[c][k] = r.inv > 0.0f ? (uint8_t)__float_as_uint(exact_code(w, w * r.inv, r)) : (uint8_t)0;
    }
  }
  __syncthreads();
  const int t = threadIdx.x / 16, q = threadIdx.x % 16;  // sixteen lanes a channel, four rows each
  if (i0 + 4 * q >= p.d_in) return;                      // (d_in is a multiple of 16)
  for (int k = t; k < 64; k += 16)
    if (blockIdx.x * 64 + k < (unsigned)p.d_out)
      *reinterpret_cast<uint32_t*>(p.codes + (size_t)(blockIdx.x * 64 + k) * p.d_in + i0 + 4 * q) =
          *reinterpret_cast<const uint32_t*>(&tile[k][4 * q]);
}
__global__ __launch_bounds__(256) void weight8_scale_kernel(const Weight8Args p) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j < p.d_out) p.scale[j] = row_scale_of(reinterpret_cast<const uint32_t*>(p.scale)[j]).s;
}

hipError_t launch_weight8(const Weight8Args& a, hipStream_t st) {
  const unsigned by256 = ceil_div(a.d_out, 256);
  auto go = [&](auto bits_c) {
    constexpr int NBITS = decltype(bits_c)::value;
    weight8_clear_kernel<<<by256, 256, 0, st>>>(a);
    weight8_top_kernel<NBITS><<<dim3(by256, ceil_div(a.d_in, W8_ROWS)), 256, 0, st>>>(a);
    weight8_codes_kernel<NBITS><<<dim3(ceil_div(a.d_out, 64), ceil_div(a.d_in, 64)), 256, 0, st>>>(a);
    weight8_scale_kernel<<<by256, 256, 0, st>>>(a);
    return hipGetLastError();
  };
  switch (a.bits) {
    case 0: return go(std::integral_constant<int, 0>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    default: return go(std::integral_constant<int, 4>{});
  }
}

}  // namespace qalora
