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
// Products.  X, G and P are fp32; for the matrix cores a value is split in two fp16, hi = fp16(S v) and lo = fp16(2^12 (S v - hi)),
// S a power of two that keeps S v below 2^15.  Three products, hi hi + 2^-12 (hi lo + lo hi), miss 2^-24 of the operands, as
// rounding them to fp32 does, and take a fifth of the time of the fp32 instruction (which has a sixteenth of the fp16 rate).
// (The scale of lo keeps it away from fp16's subnormals, and makes up for hi where that is one: S may be far from tight.  It
// comes from bounds: |G_ij| <= trace G, |X_ij| <= |X|_F = sqrt(trace G), |P_ij| <= |a| + |b| trace G + |c| (trace G)^2, and of
// P X their product.)
//
// Layout.  v_mfma_f32_32x32x16_f16: X in LDS as [rows i][64 columns n] planes of hi and lo.  P X is computed transposed (A operand: X
// read transposed, ds_read_b64_tr_b16; B operand: rows of P, by its symmetry), so a lane holds four neighbouring n of a
// row i and writes them back 8 bytes at a time; X X^T reads rows of the same planes.  In memory X is kept as the lanes hold
// it ([32 x 32 tile][register quad][lane] of 16 bytes), so a pass reads and writes it in whole kilobytes.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int XLD = MUON_CHUNK + 8;  // halves between rows of a chunk's plane: 16-byte reads of 32 rows meet all banks
constexpr float kLoScale = 4096.0f;

// A power of two that brings magnitudes up to `bound` below 2^15.
__device__ __forceinline__ float scale_below(float bound) {
  const int e = (int)((__float_as_uint(bound) >> 23) & 255u) - 127;
  return __uint_as_float((uint32_t)(127 + 14 - max(-100, min(100, e))) << 23);
}
__device__ __forceinline__ float inverse_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }
// What sqrt(trace) may miss: squares below the smallest fp32 that were lost in the sums.
constexpr float kLostNorm = 0x1p-47f;

// hi and lo of a value.  (The value is pinned to its fp32 rounding: where it is a product, the compiler rounds that once
// more, to fp16, for the hi that is stored and otherwise for the hi that lo is taken from, and near a tie the two differ.)
__device__ __forceinline__ void split(float v, _Float16& h, _Float16& l) {
  asm volatile("" : "+v"(v));
  h = (_Float16)v;
  l = (_Float16)((v - (float)h) * kLoScale);
}
// Four neighbouring values into the planes (lo `lo_at` halves behind hi).
__device__ __forceinline__ void put4(_Float16* hi, int lo_at, const f32x4& v) {
  f16x4 h, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 a, b;
    split(v[e], a, b);
    h[e] = a;
    l[e] = b;
  }
  *reinterpret_cast<f16x4*>(hi) = h;
  *reinterpret_cast<f16x4*>(hi + lo_at) = l;
}
__device__ __forceinline__ void put1(_Float16* hi, int lo_at, float v) {
  _Float16 h, l;
  split(v, h, l);
  *hi = h;
  hi[lo_at] = l;
}
__device__ __forceinline__ f16x8 read8(const _Float16* p) { return *reinterpret_cast<const f16x8*>(p); }
// Eight rows of one column per lane: the operand whose 32 columns and 16 rows start at `tile`
__device__ __forceinline__ f16x8 read_columns(const _Float16* tile, int lane) {
  const int i = lane & 15, row = 8 * (lane >> 5) + (i >> 2), col = 16 * ((lane >> 4) & 1) + 4 * (i & 3);
  const _Float16* p = tile + row * XLD + col;
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * XLD));
  return __builtin_bit_cast(f16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A 32 x 32 tile of a product: `main` of the hi pieces, `cross` of hi and lo.  Register r of a lane is element
// (8 (r / 4) + 4 (lane / 32) + r % 4, lane % 32).
struct Tile {
  f32x16 main, cross;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < 16; ++r) main[r] = cross[r] = 0.0f;
  }
  __device__ __forceinline__ void add(const f16x8& a, const f16x8& a_lo, const f16x8& b, const f16x8& b_lo) {
    main = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, main, 0, 0, 0);
    cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b_lo, cross, 0, 0, 0);
    cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(a_lo, b, cross, 0, 0, 0);
  }
  __device__ __forceinline__ f32x4 quad(int g, float scale) const {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(cross[4 * g + e], 1.0f / kLoScale, main[4 * g + e]) * scale;
    return v;
  }
};
// += rows of tile i times rows of tile j over 16 `groups` columns; both at the lane's first operand
__device__ __forceinline__ void add_rows(Tile& t, const _Float16* rows_i, const _Float16* rows_j, int lo_at, int groups) {
#pragma unroll 2
  for (int s = 0; s < groups; ++s)
    t.add(read8(rows_i + 16 * s), read8(rows_i + 16 * s + lo_at), read8(rows_j + 16 * s), read8(rows_j + 16 * s + lo_at));
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
// else 1) at a time, f(k, element, i, n) for the k-th of them, (i, n) the first one's place in X's chunk; the others follow
// along n where the matrix is wide, along i where it is tall.  The count is a constant, so that all loads of a share are in
// flight together.
template <int RT, int NT, int W, typename Fn>
__device__ __forceinline__ void each_piece(const MuonTensor& t, int chunk, Fn&& f) {
  const int n0 = chunk * MUON_CHUNK;
  const bool wide = t.rows <= t.cols;
  const int per_row = wide ? MUON_CHUNK / W : t.cols / W, rows = wide ? t.rows : min(MUON_CHUNK, t.rows - n0);
#pragma unroll
  for (int k = 0; k < 32 * RT * MUON_CHUNK / (NT * W); ++k) {
    const int e = threadIdx.x + NT * k;
    const int r = wide ? e / (MUON_CHUNK / W) : e / per_row, c = W * (e - r * per_row);
    if (r >= rows || (wide && n0 + c >= t.cols)) continue;
    f(k, wide ? (size_t)r * t.cols + n0 + c : (size_t)(n0 + r) * t.cols + c, wide ? r : c, wide ? c : r);
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

// Where element (i, n) of a chunk is kept in memory (floats; n's neighbours in a run of four follow).
__device__ __forceinline__ int kept_at(int i, int n) {
  return (((i >> 5) * 2 + (n >> 5)) * 4 + ((n & 31) >> 3)) * 256 + ((i & 31) + 32 * ((n >> 2) & 1)) * 4 + (n & 3);
}

constexpr int muon_waves(int rt) { return 2 * rt; }  // a wavefront per 32 x 32 tile of a chunk
constexpr int muon_pld(int rt) { return 32 * rt + 8; }  // halves between rows of a plane of G and P
constexpr int muon_x_halves(int rt) { return 32 * rt * XLD; }  // of a plane
constexpr int muon_p_halves(int rt) { return 32 * rt * muon_pld(rt); }
constexpr size_t muon_pass_lds(int rt) { return 2 * (size_t)(2 * muon_x_halves(rt) + muon_p_halves(rt)) * 2; }

// A block's share of G: its wavefronts' tiles (a, b), `wave + NW q` of a tiles x tiles grid.
template <int RT>
struct Gram {
  static constexpr int NW = muon_waves(RT), Q = RT * RT / NW;
  int at_a[Q], at_b[Q], tiles, wave;
  __device__ __forceinline__ Gram(int tiles_, int wave_, int lane, int ld) : tiles(tiles_), wave(wave_) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int id = wave + NW * q, a = id / tiles, b = id - a * tiles;
      at_a[q] = (32 * a + (lane & 31)) * ld + 8 * (lane >> 5);
      at_b[q] = (32 * b + (lane & 31)) * ld + 8 * (lane >> 5);
    }
  }
  __device__ __forceinline__ bool live(int q) const { return wave + NW * q < tiles * tiles; }
};

}  // namespace

// Momentum, u into X, and the blocks' shares of u u^T.
template <int RT>
__global__ __launch_bounds__(64 * muon_waves(RT)) void muon_start_kernel(const MuonTable table, const MuonHyper h, float* ws) {
  constexpr int NW = muon_waves(RT), NT = 64 * NW, LO = muon_x_halves(RT), Q = Gram<RT>::Q;
  __shared__ __align__(16) _Float16 xs[2 * LO];
  __shared__ float wave_max[NW];
  const Where w = muon_where(table);
  const MuonTensor& t = *w.t;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool wide = t.rows <= t.cols;
  const Gram<RT> gram(t.tiles, wave, lane, XLD);
  f32x4 sum[Q][4];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int g = 0; g < 4; ++g) sum[q][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int c = w.c0; c < w.c1; ++c) {
    float* x = ws + t.x + (size_t)c * t.tiles * 32 * MUON_CHUNK;
    const bool part = c == w.c0 || c + 1 == t.chunks;  // rows or columns outside the matrix are not zero yet
    if (part) {
      for (int e = threadIdx.x; e < 2 * LO / 8; e += NT) reinterpret_cast<f32x4*>(xs)[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // (memory outside the matrix: the few elements that the pieces below do not write)
    const int rows_in = wide ? t.rows : t.cols, cols_in = min(MUON_CHUNK, (wide ? t.cols : t.rows) - c * MUON_CHUNK);
    if (rows_in < 32 * t.tiles || cols_in < MUON_CHUNK)
      for (int e = threadIdx.x; e < 32 * t.tiles * MUON_CHUNK; e += NT) {
        const int i = e / MUON_CHUNK, n = e % MUON_CHUNK;
        if (i >= rows_in || n >= cols_in) x[kept_at(i, n)] = 0.0f;
      }
    auto momentum = [&](auto width) {
      constexpr int W = decltype(width)::value, K = 32 * RT * MUON_CHUNK / (NT * W);
      Piece<W> g[K], m[K];
      float most = 0.0f;
      each_piece<RT, NT, W>(t, c, [&](int k, size_t at, int, int) {
        g[k] = load_piece<W>(t.g + at);
        m[k] = load_piece<W>(t.m + at);
      });
      each_piece<RT, NT, W>(t, c, [&](int k, size_t at, int, int) {
#pragma unroll
        for (int e = 0; e < W; ++e) m[k].v[e] = __builtin_fmaf(h.momentum, m[k].v[e], g[k].v[e]);
        store_piece<W>(t.m + at, m[k]);
        if (h.zero_grads) store_piece<W>(t.g + at, Piece<W>{});
#pragma unroll
        for (int e = 0; e < W; ++e) {
          if (h.nesterov) m[k].v[e] = __builtin_fmaf(h.momentum, m[k].v[e], g[k].v[e]);
          most = fmaxf(most, fabsf(m[k].v[e]));
        }
      });
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
      if (lane == 0) wave_max[wave] = most;
      __syncthreads();  // (the planes are cleared, and those of the chunk before have been read)
#pragma unroll
      for (int k = 0; k < NW; ++k) most = fmaxf(most, wave_max[k]);
      const float s = scale_below(most);
      each_piece<RT, NT, W>(t, c, [&](int k, size_t, int i, int n) {
        if (W == 4 && wide) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = m[k].v[e % W];
          *reinterpret_cast<f32x4*>(x + kept_at(i, n)) = v;
          put4(xs + i * XLD + n, LO, v * s);
        } else {
#pragma unroll
          for (int e = 0; e < W; ++e) {
            x[kept_at(i + e, n)] = m[k].v[e];
            put1(xs + (i + e) * XLD + n, LO, m[k].v[e] * s);
          }
        }
      });
      return s;
    };
    const float s = t.cols % 4 == 0 ? momentum(std::integral_constant<int, 4>{}) : momentum(std::integral_constant<int, 1>{});
    __syncthreads();
    const float back = inverse_power(s);  // (twice: its square may be below the smallest fp32)
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (gram.live(q)) {
        Tile p;
        p.clear();
        add_rows(p, xs + gram.at_a[q], xs + gram.at_b[q], LO, MUON_CHUNK / 16);
#pragma unroll
        for (int g = 0; g < 4; ++g) sum[q][g] += p.quad(g, back) * back;
      }
    __syncthreads();  // the next chunk's wave_max and planes
  }
  f32x4* out = reinterpret_cast<f32x4*>(ws + t.partial) + (size_t)w.slice * t.tiles * t.tiles * 256;
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (gram.live(q))
#pragma unroll
      for (int g = 0; g < 4; ++g) out[((wave + NW * q) * 4 + g) * 64 + lane] = sum[q][g];
}

// G = sum of the blocks' shares: 32 pieces of 16 bytes a block, their shares dealt to eight groups of threads.
__global__ __launch_bounds__(256) void muon_reduce_kernel(const MuonTable table, float* ws) {
  __shared__ f32x4 part[8][32];
  const int ti = muon_find(table.reduce0);
  const MuonTensor& t = table.t[ti];
  const int slices = (t.chunks + table.per_block - 1) / table.per_block;
  const int e = threadIdx.x & 31, group = threadIdx.x >> 5;
  const size_t pieces = (size_t)t.tiles * t.tiles * 256, at = (size_t)(blockIdx.x - table.reduce0[ti]) * 32 + e;
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
template <int RT, bool FIRST, bool LAST>
__global__ __launch_bounds__(64 * muon_waves(RT)) void muon_pass_kernel(const MuonTable table, const MuonHyper h, float* ws) {
  constexpr int NW = muon_waves(RT), NT = 64 * NW, PLD = muon_pld(RT), Q = Gram<RT>::Q;
  constexpr int XLO = muon_x_halves(RT), PLO = muon_p_halves(RT);
  extern __shared__ __align__(16) _Float16 lds[];
  _Float16* xs = lds;           // [hi, lo][32 RT][XLD]: X
  _Float16* ys = xs + 2 * XLO;  // P X
  _Float16* ps = ys + 2 * XLO;  // [hi, lo][32 RT][PLD]: G, then P
  const Where w = muon_where(table);
  const MuonTensor& t = *w.t;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lo5 = lane & 31, hi1 = lane >> 5;
  const int it = wave >> 1, nt = wave & 1;  // the wavefront's tile of a chunk
  const bool mine = it < t.tiles;

  // ---- requests: G's diagonal and tiles, the first chunk --------------------------------------
  const float* gram_at = ws + t.gram;
  float diagonal = 0.0f;
#pragma unroll
  for (int k = 0; k < (32 * RT + 63) / 64; ++k) {
    const int d = lane + 64 * k, a = d >> 5, dd = d & 31;
    if (d < 32 * t.tiles)
      diagonal += gram_at[(((a * t.tiles + a) * 4 + (dd >> 3)) * 64 + dd + 32 * ((dd >> 2) & 1)) * 4 + (dd & 3)];
  }
  const Gram<RT> square(t.tiles, wave, lane, PLD);
  f32x4 g[Q][4];
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (square.live(q))
#pragma unroll
      for (int k = 0; k < 4; ++k) g[q][k] = reinterpret_cast<const f32x4*>(gram_at)[((wave + NW * q) * 4 + k) * 64 + lane];
  // The chunk that comes next, on its way: the first one while P is made, each later one while the one before is worked on.
  f32x4 coming[4];
  auto chunk_at = [&](int c) {
    return reinterpret_cast<f32x4*>(ws + t.x) + ((size_t)c * t.tiles * 2 + wave) * 256 + lane;
  };
  auto request = [&](int c) {
    if (mine)
#pragma unroll
      for (int k = 0; k < 4; ++k) coming[k] = chunk_at(c)[64 * k];
  };
  request(w.c0);

  // ---- scales ---------------------------------------------------------------------------------
  float trace = diagonal;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) trace += __shfl_xor(trace, off, 64);
  float x_norm = 1.0f;  // times X as it is kept
  if constexpr (FIRST) {
    x_norm = 1.0f / (__fsqrt_rn(trace) + h.eps);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int k = 0; k < 4; ++k) g[q][k] *= x_norm * x_norm;
  }
  const float x_bound = (__fsqrt_rn(trace) + kLostNorm) * x_norm;
  trace *= x_norm * x_norm;
  const float p_bound = fabsf(h.a) + fabsf(h.b) * trace + fabsf(h.c) * trace * trace;
  const float s_g = scale_below(trace), s_p = scale_below(p_bound), s_x = scale_below(x_bound),
              s_y = scale_below(1.001f * p_bound * x_bound);

  // ---- P = a I + b G + c G^2 ------------------------------------------------------------------
  // A lane's quads of tile (a, b) go to rows 32 b + lane % 32: the transposed place, where a symmetric matrix has the same
  auto put_tile = [&](int q, int k, const f32x4& v) {
    const int id = wave + NW * q, a = id / t.tiles, b = id - a * t.tiles;
    put4(ps + (32 * b + lo5) * PLD + 32 * a + 8 * k + 4 * hi1, PLO, v);
  };
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (square.live(q))
#pragma unroll
      for (int k = 0; k < 4; ++k) put_tile(q, k, g[q][k] * s_g);
  __syncthreads();
  const float g_back = inverse_power(s_g) * inverse_power(s_g);
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (square.live(q)) {
      const int id = wave + NW * q, a = id / t.tiles, b = id - a * t.tiles;
      Tile p;
      p.clear();
      add_rows(p, ps + square.at_a[q], ps + square.at_b[q], PLO, 2 * t.tiles);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 g2 = p.quad(k, g_back);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float one = (a == b && 8 * k + 4 * hi1 + e == lo5) ? h.a : 0.0f;
          g[q][k][e] = __builtin_fmaf(h.c, g2[e], __builtin_fmaf(h.b, g[q][k][e], one));
        }
      }
    }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (square.live(q))
#pragma unroll
      for (int k = 0; k < 4; ++k) put_tile(q, k, g[q][k] * s_p);

  // ---- the block's columns: X <- P X ----------------------------------------------------------
  const Gram<RT> gram(t.tiles, wave, lane, XLD);
  Tile next_g[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) next_g[q].clear();
  const int place = (32 * it + lo5) * XLD + 32 * nt + 4 * hi1;  // + 8 k: the lane's quads in a plane
  const float in_scale = x_norm * s_x, y_back = inverse_power(s_x) * inverse_power(s_p);
  for (int c = w.c0; c < w.c1; ++c) {
    if (mine)
#pragma unroll
      for (int k = 0; k < 4; ++k) put4(xs + place + 8 * k, XLO, coming[k] * in_scale);
    __syncthreads();  // (also: everybody is done with the columns before)
    if (c + 1 < w.c1) request(c + 1);
    f32x4 y[4];
    if (mine) {
      Tile p;
      p.clear();
      const _Float16* rows = ps + (32 * it + lo5) * PLD + 8 * hi1;
#pragma unroll 2
      for (int s = 0; s < 2 * t.tiles; ++s) {
        const _Float16* cols = xs + 16 * s * XLD + 32 * nt;
        p.add(read_columns(cols, lane), read_columns(cols + XLO, lane), read8(rows + 16 * s), read8(rows + 16 * s + PLO));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = p.quad(k, y_back);
    }
    if constexpr (LAST) {
      // through LDS as fp32 (in the room of P X), so that the parameters are read and written in whole rows
      float* out = reinterpret_cast<float*>(ys);
      constexpr int OLD = MUON_CHUNK + 4;
      static_assert(32 * RT * OLD * 4 <= 2 * XLO * 2, "the tile fits");
      if (mine)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          *reinterpret_cast<f32x4*>(out + (32 * it + lo5) * OLD + 32 * nt + 8 * k + 4 * hi1) = y[k];
      auto update = [&](auto width) {
        constexpr int W = decltype(width)::value, K = 32 * RT * MUON_CHUNK / (NT * W);
        Piece<W> p[K];
        each_piece<RT, NT, W>(t, c, [&](int k, size_t at, int, int) { p[k] = load_piece<W>(t.p + at); });
        __syncthreads();
        each_piece<RT, NT, W>(t, c, [&](int k, size_t at, int i, int n) {
          const int step = t.rows <= t.cols ? 1 : OLD;
#pragma unroll
          for (int e = 0; e < W; ++e) p[k].v[e] = __builtin_fmaf(p[k].v[e], h.decay, -t.step_size * out[i * OLD + n + e * step]);
          store_piece<W>(t.p + at, p[k]);
        });
      };
      if (t.cols % 4 == 0) update(std::integral_constant<int, 4>{});
      else update(std::integral_constant<int, 1>{});
    } else {
      if (mine)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          chunk_at(c)[64 * k] = y[k];
          put4(ys + place + 8 * k, XLO, y[k] * s_y);
        }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (gram.live(q)) add_rows(next_g[q], ys + gram.at_a[q], ys + gram.at_b[q], XLO, MUON_CHUNK / 16);
    }
  }
  if constexpr (!LAST) {
    const float back = inverse_power(s_y) * inverse_power(s_y);
    f32x4* out = reinterpret_cast<f32x4*>(ws + t.partial) + (size_t)w.slice * t.tiles * t.tiles * 256;
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (gram.live(q))
#pragma unroll
        for (int k = 0; k < 4; ++k) out[((wave + NW * q) * 4 + k) * 64 + lane] = next_g[q].quad(k, back);
  }
}

namespace {

template <int RT, bool FIRST, bool LAST>
hipError_t launch_pass(const MuonTable& t, const MuonHyper& h, float* ws, hipStream_t st) {
  static std::atomic<uint64_t> granted{0};  // per instantiation
  auto kern = muon_pass_kernel<RT, FIRST, LAST>;
  constexpr size_t lds = muon_pass_lds(RT);
  if (hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kern), (int)lds, granted); e != hipSuccess) return e;
  kern<<<t.blocks, 64 * muon_waves(RT), lds, st>>>(t, h, ws);
  return hipGetLastError();
}

template <int RT>
hipError_t launch_steps(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  muon_start_kernel<RT><<<t.blocks, 64 * muon_waves(RT), 0, st>>>(t, h, ws);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  for (int k = 0; k < steps; ++k) {
    muon_reduce_kernel<<<t.reduce_blocks, 256, 0, st>>>(t, ws);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const bool first = k == 0, last = k + 1 == steps;
    const hipError_t e = first ? (last ? launch_pass<RT, true, true>(t, h, ws, st) : launch_pass<RT, true, false>(t, h, ws, st))
                               : (last ? launch_pass<RT, false, true>(t, h, ws, st) : launch_pass<RT, false, false>(t, h, ws, st));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_muon(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  return t.max_tiles > 2 ? launch_steps<4>(t, h, steps, ws, st) : launch_steps<2>(t, h, steps, ws, st);
}

}  // namespace qalora
