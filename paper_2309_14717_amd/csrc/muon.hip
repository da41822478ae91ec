// The orthogonalised update (Muon): momentum, Newton-Schulz products on each matrix of a list, and the step.  It stands
// beside the AdamW step: only the adapters' A [L, r] and B [r, d_out] are trained (Sec. 3.1), so one side of every
// matrix is the rank, at most 128.
//
//   m  = mu m + g;   u = g + mu m (Nesterov) or m
//   X0 = u / (|u|_F + eps), seen as [shorter side r x longer side n]
//   X <- (a I + b G + c G^2) X with G = X X^T, `steps` times: the singular values go through the odd polynomial
//        a t + b t^3 + c t^5 and its iterates bring them all near one, while the singular vectors stay
//   p  = p (1 - lr wd) - lr scale X
//
// G is r x r: it fits a compute unit, X does not.  So a step of the iteration is one pass over X: a block takes G, forms
// P = a I + b G + c G^2 in LDS (r^3 operations, repeated by every block, against r^2 per column of X), replaces its
// columns of X by P X and adds the new columns' products to its own share of the next G; a small launch adds the shares in
// block order (no atomics: a step is bit-reproducible).  X0's norm is the root of the first G's trace and goes into the first
// pass, so the norm takes no pass of its own.
//
// (G alone could carry the whole iteration: P is a polynomial in the first G.  But an error of 2^-24 in that G then meets
// the smallest singular values with the full gain a^steps, 1.5 % of the result for the coefficients in use.  G made
// anew from X in every pass keeps it at 2^-24 times the gain.)
//
// Everything is fp32: products by v_mfma_f32_16x16x4_f32, operands read from LDS 16 bytes a lane where the contraction
// index is contiguous (G, P by their symmetry, and X in X X^T), the four values then being those of four instructions.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {

constexpr int XLD = MUON_CHUNK + 4;  // floats between rows of a chunk in LDS: 16-byte reads of 16 rows meet all banks

// Upper tiles of a symmetric matrix in the order (0,0), (0,1), (1,1), (0,2), ...: tile `id` is (i, j), i <= j.
__device__ __forceinline__ void tile_of(int id, int& i, int& j) {
  j = 0;
  while ((j + 1) * (j + 2) / 2 <= id) ++j;
  i = id - j * (j + 1) / 2;
}

// acc += rows of tile i times rows of tile j over 16 `groups` columns of a matrix in LDS with rows `ld` apart
__device__ __forceinline__ f32x4 rows_product(const float* rows_i, const float* rows_j, int groups, f32x4 acc) {
  for (int s = 0; s < groups; ++s) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(rows_i + 16 * s), b = *reinterpret_cast<const f32x4*>(rows_j + 16 * s);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc, 0, 0, 0);
  }
  return acc;
}

// The tensor whose blocks the launch's block lies in.  (All starts are compared at once: a search that reads one after
// the other waits for each, 0.15 us a tensor.)
__device__ __forceinline__ int muon_find(const int (&first)[MUON_MAX_TENSORS]) {
  int ti = 0;
#pragma unroll
  for (int i = 1; i < MUON_MAX_TENSORS; ++i) ti += (int)blockIdx.x >= first[i] ? 1 : 0;
  return ti;
}
struct Where {
  const MuonTensor* t;
  int c0, c1;  // chunks
  int slice;
};
__device__ __forceinline__ Where muon_where(const MuonTable& table) {
  const int ti = muon_find(table.block0);
  const MuonTensor& t = table.t[ti];
  Where w{&t, 0, 0, (int)blockIdx.x - table.block0[ti]};
  w.c0 = w.slice * table.per_block;
  w.c1 = min(t.chunks, w.c0 + table.per_block);
  return w;
}

// A thread's share of a chunk of a [rows, cols] matrix: W neighbours in memory (4 where rows of it are whole 16-byte pieces,
// else 1) at a time, f(k, element, place in the chunk's LDS tile, distance of the neighbours there) for the k-th of them.  The
// count is a constant, so that all loads of a share are in flight together.
template <int MAXT, int NT, int W, typename Fn>
__device__ __forceinline__ void each_piece(const MuonTensor& t, int chunk, Fn&& f) {
  const int n0 = chunk * MUON_CHUNK;
  const bool wide = t.rows <= t.cols;
  const int per_row = wide ? MUON_CHUNK / W : t.cols / W, rows = wide ? t.rows : min(MUON_CHUNK, t.rows - n0);
#pragma unroll
  for (int k = 0; k < 16 * MAXT * MUON_CHUNK / (NT * W); ++k) {
    const int e = threadIdx.x + NT * k;
    const int r = wide ? e / (MUON_CHUNK / W) : e / per_row, c = W * (e - r * per_row);
    if (r >= rows || (wide && n0 + c >= t.cols)) continue;
    f(k, wide ? (size_t)r * t.cols + n0 + c : (size_t)(n0 + r) * t.cols + c, wide ? r * XLD + c : c * XLD + r, wide ? 1 : XLD);
  }
}
template <int W>
struct Piece {
  float v[W];
};
template <int W>
__device__ __forceinline__ Piece<W> load_piece(const float* p) {
  Piece<W> r;
  if constexpr (W == 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p);
    for (int e = 0; e < 4; ++e) r.v[e] = v[e];
  } else {
    r.v[0] = *p;
  }
  return r;
}
template <int W>
__device__ __forceinline__ void store_piece(float* p, const Piece<W>& r) {
  if constexpr (W == 4) *reinterpret_cast<f32x4*>(p) = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
  else *p = r.v[0];
}

// A block's share of G from the chunks it has in LDS one after the other: tile wave + NW q of the upper tiles in acc[q].
template <int MAXT, int NW>
struct Gram {
  static constexpr int Q = (muon_gram_tiles(MAXT) + NW - 1) / NW;
  f32x4 acc[Q];
  int at_i[Q], at_j[Q];
  __device__ __forceinline__ Gram(int tiles, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      int i = 0, j = 0;
      if (wave + NW * q < muon_gram_tiles(tiles)) tile_of(wave + NW * q, i, j);
      at_i[q] = (16 * i + (lane & 15)) * XLD + 4 * (lane >> 4);
      at_j[q] = (16 * j + (lane & 15)) * XLD + 4 * (lane >> 4);
    }
  }
  __device__ __forceinline__ void add(const float* xs, int tiles, int wave) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (wave + NW * q < muon_gram_tiles(tiles)) acc[q] = rows_product(xs + at_i[q], xs + at_j[q], MUON_CHUNK / 16, acc[q]);
  }
  __device__ __forceinline__ void store(float* partial, int tiles, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (wave + NW * q < muon_gram_tiles(tiles)) reinterpret_cast<f32x4*>(partial)[(wave + NW * q) * 64 + lane] = acc[q];
  }
};

constexpr int muon_waves(int maxt) { return maxt > 4 ? 8 : 4; }
constexpr int muon_pld(int maxt) { return 16 * maxt + 4; }  // floats between rows of G and P in LDS
constexpr size_t muon_start_lds(int maxt) { return (size_t)16 * maxt * XLD * 4; }
constexpr size_t muon_pass_lds(int maxt) { return muon_start_lds(maxt) + (size_t)16 * maxt * muon_pld(maxt) * 4; }

}  // namespace

// Momentum, u into X, and the blocks' shares of u u^T.
template <int MAXT>
__global__ __launch_bounds__(64 * muon_waves(MAXT)) void muon_start_kernel(const MuonTable table, const MuonHyper h, float* ws) {
  constexpr int NW = muon_waves(MAXT), NT = 64 * NW;
  extern __shared__ __align__(16) float xs[];
  const Where w = muon_where(table);
  const MuonTensor& t = *w.t;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Gram<MAXT, NW> gram(t.tiles, wave, lane);
  // rows beyond the shorter side stay zero for the whole kernel, columns beyond the longer one are in the last chunk only
  for (int e = threadIdx.x; e < 16 * t.tiles * XLD; e += NT) xs[e] = 0.0f;
  __syncthreads();
  for (int c = w.c0; c < w.c1; ++c) {
    if (c > w.c0 && c + 1 == t.chunks) {
      for (int e = threadIdx.x; e < 16 * t.tiles * XLD; e += NT) xs[e] = 0.0f;
      __syncthreads();
    }
    auto momentum = [&](auto width) {
      constexpr int W = decltype(width)::value, K = 16 * MAXT * MUON_CHUNK / (NT * W);
      Piece<W> g[K], m[K];
      each_piece<MAXT, NT, W>(t, c, [&](int k, size_t at, int, int) {
        g[k] = load_piece<W>(t.g + at);
        m[k] = load_piece<W>(t.m + at);
      });
      each_piece<MAXT, NT, W>(t, c, [&](int k, size_t at, int in_lds, int step) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          m[k].v[e] = __builtin_fmaf(h.momentum, m[k].v[e], g[k].v[e]);
          xs[in_lds + e * step] = h.nesterov ? __builtin_fmaf(h.momentum, m[k].v[e], g[k].v[e]) : m[k].v[e];
        }
        store_piece<W>(t.m + at, m[k]);
        if (h.zero_grads) store_piece<W>(t.g + at, Piece<W>{});
      });
    };
    if (t.cols % 4 == 0) momentum(std::integral_constant<int, 4>{});
    else momentum(std::integral_constant<int, 1>{});
    __syncthreads();
    f32x4* x = reinterpret_cast<f32x4*>(ws + t.x) + (size_t)c * t.tiles * 16 * (MUON_CHUNK / 4);
    for (int e = threadIdx.x; e < t.tiles * 16 * (MUON_CHUNK / 4); e += NT)
      x[e] = *reinterpret_cast<const f32x4*>(xs + (e >> 4) * XLD + 4 * (e & 15));
    gram.add(xs, t.tiles, wave);
    __syncthreads();
  }
  gram.store(ws + t.partial + (size_t)w.slice * muon_gram_tiles(t.tiles) * 256, t.tiles, wave, lane);
}

// G = sum of the blocks' shares: 32 pieces of 16 bytes a block, their shares dealt to eight groups of threads.
__global__ __launch_bounds__(256) void muon_reduce_kernel(const MuonTable table, float* ws) {
  __shared__ f32x4 part[8][32];
  const int ti = muon_find(table.reduce0);
  const MuonTensor& t = table.t[ti];
  const int slices = (t.chunks + table.per_block - 1) / table.per_block;
  const int e = threadIdx.x & 31, group = threadIdx.x >> 5;
  const size_t pieces = (size_t)muon_gram_tiles(t.tiles) * 64, at = (size_t)(blockIdx.x - table.reduce0[ti]) * 32 + e;
  const f32x4* src = reinterpret_cast<const f32x4*>(ws + t.partial) + at;
  const int per = (slices + 7) / 8, z0 = min(slices, group * per), z1 = min(slices, z0 + per);
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
  for (int z = z0; z < z1; ++z) v += src[(size_t)z * pieces];
  part[group][e] = v;
  __syncthreads();
  if (group == 0) {
#pragma unroll
    for (int k = 1; k < 8; ++k) v += part[k][e];
    reinterpret_cast<f32x4*>(ws + t.gram)[at] = v;
  }
}

// One step of the iteration on the block's chunks.  FIRST: X holds u, whose norm comes off here.  LAST: the result goes into the
// parameters, else back to X with the shares of the next G.
template <int MAXT, bool FIRST, bool LAST>
__global__ __launch_bounds__(64 * muon_waves(MAXT)) void muon_pass_kernel(const MuonTable table, const MuonHyper h, float* ws) {
  constexpr int NW = muon_waves(MAXT), NT = 64 * NW, PLD = muon_pld(MAXT);
  extern __shared__ __align__(16) float xs[];  // [16 tiles][XLD]
  float* ps = xs + 16 * MAXT * XLD;            // [16 tiles][PLD]: G, then P
  const Where w = muon_where(table);
  const MuonTensor& t = *w.t;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lo = lane & 15, hi = lane >> 4;
  const int upper = muon_gram_tiles(t.tiles);

  // The chunk that comes next, on its way: the first one while P is made, each later one while the one before is worked on.
  constexpr int XK = 16 * MAXT * (MUON_CHUNK / 4) / NT;
  f32x4 coming[XK];
  const int pieces = t.tiles * 16 * (MUON_CHUNK / 4);
  auto chunk_at = [&](int c) { return reinterpret_cast<f32x4*>(ws + t.x) + (size_t)c * pieces; };
  auto request = [&](int c) {
#pragma unroll
    for (int k = 0; k < XK; ++k)
      if (threadIdx.x + NT * k < (unsigned)pieces) coming[k] = chunk_at(c)[threadIdx.x + NT * k];
  };

  // ---- P = a I + b G + c G^2 -------------------------------------------------------------
  constexpr int Q = (muon_gram_tiles(MAXT) + NW - 1) / NW;
  f32x4 g[Q];  // upper tiles wave + NW q: element (16 i + 4 hi + v, 16 j + lo)
  auto put = [&](int id, const f32x4& v) {  // a tile and its mirror image
    int i, j;
    tile_of(id, i, j);
#pragma unroll
    for (int e = 0; e < 4; ++e) ps[(16 * i + 4 * hi + e) * PLD + 16 * j + lo] = v[e];
    if (i != j) *reinterpret_cast<f32x4*>(ps + (16 * j + lo) * PLD + 16 * i + 4 * hi) = v;
  };
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (wave + NW * q < upper) g[q] = reinterpret_cast<const f32x4*>(ws + t.gram)[(wave + NW * q) * 64 + lane];
  request(w.c0);
  float x_scale = 1.0f;
  if constexpr (FIRST) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (wave + NW * q < upper) put(wave + NW * q, g[q]);
    __syncthreads();
    float trace = 0.0f;
    for (int d = lane; d < 16 * t.tiles; d += 64) trace += ps[d * PLD + d];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) trace += __shfl_xor(trace, off, 64);
    x_scale = 1.0f / (__fsqrt_rn(trace) + h.eps);
    __syncthreads();  // every wave has read the diagonal
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (wave + NW * q < upper) g[q] *= x_scale * x_scale;
  }
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (wave + NW * q < upper) put(wave + NW * q, g[q]);
  __syncthreads();
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (wave + NW * q >= upper) continue;
    int i, j;
    tile_of(wave + NW * q, i, j);
    const f32x4 square = rows_product(ps + (16 * i + lo) * PLD + 4 * hi, ps + (16 * j + lo) * PLD + 4 * hi, t.tiles,
                                      f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float one = (i == j && 4 * hi + e == lo) ? h.a : 0.0f;
      g[q][e] = x_scale * __builtin_fmaf(h.c, square[e], __builtin_fmaf(h.b, g[q][e], one));
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (wave + NW * q < upper) put(wave + NW * q, g[q]);

  // ---- the block's columns: X <- P X -----------------------------------------------------
  Gram<MAXT, NW> gram(t.tiles, wave, lane);
  const int col = 16 * (wave & 3) + lo, tile0 = 4 * (wave >> 2);  // four row tiles of sixteen columns a wavefront
  for (int c = w.c0; c < w.c1; ++c) {
#pragma unroll
    for (int k = 0; k < XK; ++k) {
      const int e = threadIdx.x + NT * k;
      if (e < pieces) *reinterpret_cast<f32x4*>(xs + (e >> 4) * XLD + 4 * (e & 15)) = coming[k];
    }
    __syncthreads();
    if (c + 1 < w.c1) request(c + 1);
    f32x4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < t.tiles; ++s) {
      float b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = xs[(16 * s + 4 * hi + e) * XLD + col];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (tile0 + k >= t.tiles) continue;
        const f32x4 a = *reinterpret_cast<const f32x4*>(ps + (16 * (tile0 + k) + lo) * PLD + 16 * s + 4 * hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc[k], 0, 0, 0);
      }
    }
    __syncthreads();  // every wave has read the old columns
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (tile0 + k < t.tiles)
#pragma unroll
        for (int e = 0; e < 4; ++e) xs[(16 * (tile0 + k) + 4 * hi + e) * XLD + col] = acc[k][e];
    __syncthreads();
    if constexpr (LAST) {
      auto update = [&](auto width) {
        constexpr int W = decltype(width)::value, K = 16 * MAXT * MUON_CHUNK / (NT * W);
        Piece<W> p[K];
        each_piece<MAXT, NT, W>(t, c, [&](int k, size_t at, int, int) { p[k] = load_piece<W>(t.p + at); });
        each_piece<MAXT, NT, W>(t, c, [&](int k, size_t at, int in_lds, int step) {
#pragma unroll
          for (int e = 0; e < W; ++e) p[k].v[e] = __builtin_fmaf(p[k].v[e], h.decay, -t.step_size * xs[in_lds + e * step]);
          store_piece<W>(t.p + at, p[k]);
        });
      };
      if (t.cols % 4 == 0) update(std::integral_constant<int, 4>{});
      else update(std::integral_constant<int, 1>{});
    } else {
      for (int e = threadIdx.x; e < pieces; e += NT) chunk_at(c)[e] = *reinterpret_cast<const f32x4*>(xs + (e >> 4) * XLD + 4 * (e & 15));
      gram.add(xs, t.tiles, wave);
    }
    __syncthreads();  // the next chunk overwrites these columns
  }
  if constexpr (!LAST)
    gram.store(ws + t.partial + (size_t)w.slice * muon_gram_tiles(t.tiles) * 256, t.tiles, wave, lane);
}

namespace {

template <int MAXT, bool FIRST, bool LAST>
hipError_t launch_pass(const MuonTable& t, const MuonHyper& h, float* ws, hipStream_t st) {
  static std::atomic<uint64_t> granted{0};  // per instantiation
  auto kern = muon_pass_kernel<MAXT, FIRST, LAST>;
  constexpr size_t lds = muon_pass_lds(MAXT);
  if (hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kern), (int)lds, granted); e != hipSuccess) return e;
  kern<<<t.blocks, 64 * muon_waves(MAXT), lds, st>>>(t, h, ws);
  return hipGetLastError();
}

template <int MAXT>
hipError_t launch_steps(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  muon_start_kernel<MAXT><<<t.blocks, 64 * muon_waves(MAXT), muon_start_lds(MAXT), st>>>(t, h, ws);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  for (int k = 0; k < steps; ++k) {
    muon_reduce_kernel<<<t.reduce_blocks, 256, 0, st>>>(t, ws);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const bool first = k == 0, last = k + 1 == steps;
    const hipError_t e = first ? (last ? launch_pass<MAXT, true, true>(t, h, ws, st) : launch_pass<MAXT, true, false>(t, h, ws, st))
                               : (last ? launch_pass<MAXT, false, true>(t, h, ws, st) : launch_pass<MAXT, false, false>(t, h, ws, st));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_muon(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  return t.max_tiles > 4 ? launch_steps<8>(t, h, steps, ws, st) : launch_steps<4>(t, h, steps, ws, st);
}

}  // namespace qalora
