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
// G is r x r: it fits a compute unit, X mostly does not.  So a step of the iteration is one pass over X: a block takes G, forms
// P = a I + b G + c G^2 (r^3 operations, repeated by every block, against r^2 per column of X), replaces its
// columns of X by P X and adds the new columns' products to its own share of the next G; a small launch adds the shares in
// block order (no atomics: a step is bit-reproducible).  X0's norm is the root of the first G's trace and goes into the first
// pass, so the norm takes no pass of its own.  Where the shares are few, every block of a pass adds them by itself instead of a launch
// between passes; small matrices take one launch for all, a block each.  Otherwise five passes are eleven launches.
//
// (G alone could carry the whole iteration: P is a polynomial in the first G.  But an error of 2^-24 in that G then meets
// the smallest singular values with the full gain a^steps, 1.5 % of the result for the coefficients in use.  G made
// anew from X in every pass keeps it at its own products' and sums' error times the gain.)
//
// Products.  X, G and P are fp32; for the matrix cores a value v is split in two fp16, hi = fp16(S v) and lo = fp16(S v - hi), S a
// power of two that keeps S v below 2^15.  hi has 11 bits and lo 11 with a sign, where v has 24: a value in four loses its last bit,
// 2^-23 of it, while S v is above 1/4 (below, lo is an fp16 subnormal and 2^-25 / S is lost, however small v).  Three products,
// hi hi + hi lo + lo hi, leave out lo lo, up to 2^-22: a product is off by 2^-21 of itself at worst and 2^-23.7 in the root mean square,
// where fp32 operands are exact and only the sums round.  That is a choice for speed: three such products take a fifth of the time of
// the fp32 instruction (which has a sixteenth of the fp16 rate), and five passes of the recipe with exact sums are off by 8e-7 of the result, with sums in
// fp32 alone by 4e-7; a fourth product for lo lo would leave the root mean square at 2^-23.9.  S comes from bounds: |G_ij| <= trace G,
// |X_ij| <= |X|_F = sqrt(trace G), |P_ij| <= |P|_F, and of P X their product; the values of most weight are then 2^3 and more,
// P X's 2^-2.
//
// Layout.  A wavefront owns 32 columns of X at a time and needs neither LDS nor other wavefronts for them.  The 32 x 32 result of
// v_mfma_f32_32x32x16_f16 leaves in lane l the column l % 32 and, of quad q (registers 4 q ..), the rows 8 q + 4 (l / 32) + 0..3.  As an
// operand a lane supplies eight values of the contraction index for its row (or column) l % 32, and which index is which is
// free as long as both operands agree: with quads 2 s and 2 s + 1 as the eight values of slice s, a result IS an operand
// whose row is its column.  So X is kept (in memory too: [32 columns][32-row tile][quad][lane], 16 bytes a lane) as P X leaves the
// matrix cores, and goes back into them as it is; P, symmetric, likewise; and for X X^T, whose contraction runs over the columns,
// the tile is turned by a product with the unit matrix, exact for hi and lo each.
//
// Measured, five passes: the seven adapters of a 4096 / 11008 layer at rank 64, 44 MB of p, g, m and X: 81 us (the bytes that cannot be
// spared 11 us, three fp16 products for each of the recipe's 6): 15 us of momentum and first G, 5 x 4.2 us adding shares, 5 x 10.3 us
// passes, each a launch, its waits for its matrix's entry, for G and for X, and one chunk of most wavefronts.
// Rank 128 at 8192 / 22016, 178 MB: 255 us, of 64, 5 x 5.0 and 4 x 32 + 49 us: X, 45 MB, comes from behind the L2 in every pass and goes
// back there (counters: 49 MB read and 54 written a pass, 3.3 TB/s; 2.8 in the last, 3.0 in the first launch), beside 170 matrix instructions and 600 others
// a chunk of one wavefront a SIMD (its sums and operands take more than half of the registers).  Two adapters of 1024 at rank 16: 33 us, six
// launches of 5 us, most of each waits for memory one after the other (one launch: 38).
// Tried: operands of P and X through LDS, 64 columns a block, with the searches and barriers of the time: 57, 107 and 266 us.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {

// A power of two that brings magnitudes up to `bound` below 2^15.
__device__ __forceinline__ float scale_below(float bound) {
  const int e = (int)((__float_as_uint(bound) >> 23) & 255u) - 127;
  return __uint_as_float((uint32_t)(127 + 14 - max(-100, min(100, e))) << 23);
}
__device__ __forceinline__ float inverse_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }
// What sqrt(trace) may miss: squares below the smallest fp32 that were lost in the sums.
constexpr float kLostNorm = 0x1p-47f;

// hi and lo of the operand of one slice: two quads.
struct Operand {
  f16x8 hi, lo;
};
// Four instructions for two values: two at a time to fp16, and the rest by v_fma_mix_f32, which takes hi as it is (with a minus
// one that the compiler does not see through; with a constant it makes a conversion and a difference of it).  The values are
// pinned to their fp32 rounding: where one is a product, the compiler rounds that once more, to fp16, for the hi that is
// kept and otherwise for the hi that lo is taken from, and near a tie the two differ.
__device__ __forceinline__ Operand split(const f32x4& q0, const f32x4& q1) {
  float minus_one = -1.0f;
  asm("" : "+s"(minus_one));
  f16x2 hi[4], lo[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f32x2 v = k < 2 ? f32x2{q0[2 * k], q0[2 * k + 1]} : f32x2{q1[2 * k - 4], q1[2 * k - 3]};
    asm volatile("" : "+v"(v));
    hi[k] = __builtin_convertvector(v, f16x2);
    const f32x2 rest = {__builtin_fmaf((float)hi[k][0], minus_one, v[0]), __builtin_fmaf((float)hi[k][1], minus_one, v[1])};
    lo[k] = __builtin_convertvector(rest, f16x2);
  }
  return Operand{__builtin_shufflevector(__builtin_shufflevector(hi[0], hi[1], 0, 1, 2, 3), __builtin_shufflevector(hi[2], hi[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7),
                 __builtin_shufflevector(__builtin_shufflevector(lo[0], lo[1], 0, 1, 2, 3), __builtin_shufflevector(lo[2], lo[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7)};
}
__device__ __forceinline__ f16x8 to_half(const f32x16& v, int first) {
  f16x2 p[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = __builtin_convertvector((f32x2{v[first + 2 * k], v[first + 2 * k + 1]}), f16x2);
  return __builtin_shufflevector(__builtin_shufflevector(p[0], p[1], 0, 1, 2, 3), __builtin_shufflevector(p[2], p[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ void add(f32x16& acc, const Operand& a, const Operand& b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.hi, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.lo, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.lo, b.hi, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}
__device__ __forceinline__ f32x4 quad_of(const f32x16& v, int q) { return f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}; }

// The unit matrix as an operand: slice s of a tile.
__device__ __forceinline__ f16x8 unit_slice(int s, int lane) {
  f16x8 u;
#pragma unroll
  for (int k = 0; k < 8; ++k) u[k] = (_Float16)(16 * s + (k >> 2) * 8 + 4 * (lane >> 5) + (k & 3) == (lane & 31) ? 1.0f : 0.0f);
  return u;
}
// The operand tile `in` (its two slices) with rows and contraction index exchanged.
__device__ __forceinline__ void turn(const Operand (&in)[2], const f16x8 (&unit)[2], Operand (&out)[2]) {
  f32x16 hi = zero16(), lo = zero16();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    hi = __builtin_amdgcn_mfma_f32_32x32x16_f16(in[s].hi, unit[s], hi, 0, 0, 0);
    lo = __builtin_amdgcn_mfma_f32_32x32x16_f16(in[s].lo, unit[s], lo, 0, 0, 0);
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) out[s] = Operand{to_half(hi, 8 * s), to_half(lo, 8 * s)};
}

// A barrier for what goes through LDS: loads of coming columns stay in flight, and stores of X (which its own wavefront reads again)
// are not waited for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// op over the wavefront, in every lane, between neighbours, quads, eights, rows of 16 and halves.  (Lane by lane through LDS, as
// __shfl_xor goes, six steps are 0.4 us, and each pass waits for two sums.)
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <typename Op>
__device__ __forceinline__ float over_wave(float v, Op&& op) {
  v = op(v, moved<0xb1>(v));   // lane ^ 1
  v = op(v, moved<0x4e>(v));   // lane ^ 2
  v = op(v, moved<0x141>(v));  // 7 - lane of eight
  v = op(v, moved<0x140>(v));  // 15 - lane of sixteen
  uint32_t w = __float_as_uint(v);
  const auto row = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  w = __float_as_uint(op(__uint_as_float(row[0]), __uint_as_float(row[1])));
  const auto half = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return op(__uint_as_float(half[0]), __uint_as_float(half[1]));
}
__device__ __forceinline__ float wave_sum(float v) {
  return over_wave(v, [](float x, float y) { return x + y; });
}

// The upper tiles of a symmetric RT x RT matrix of tiles in the order (0,0), (0,1), (1,1), (0,2), ...
constexpr int muon_upper(int tiles) { return muon_upper_tiles(tiles); }
constexpr int upper_at(int a, int b) { return b * (b + 1) / 2 + a; }

// The tensor whose blocks the launch's block lies in, and the block's number in it.  A lane reads each tensor's first block and entry, and
// the right one's words are handed round: one wait for memory, where a search and then its entry are two (0.5 us, in every
// launch).
__device__ __forceinline__ MuonTensor muon_find(const MuonTable& table, const int (&first)[MUON_MAX_TENSORS], int& number) {
  constexpr int WORDS = sizeof(MuonTensor) / 4;
  static_assert(MUON_MAX_TENSORS == 32 && sizeof(MuonTensor) % 4 == 0, "a lane for each");
  struct Words {
    int w[WORDS];
  };
  const int mine = threadIdx.x & 31;
  const int begin = first[mine];
  Words e = __builtin_bit_cast(Words, table.t[mine]);
  const int ti = __builtin_popcount((uint32_t)__ballot((int)blockIdx.x >= begin)) - 1;
  number = (int)blockIdx.x - __builtin_amdgcn_readlane(begin, ti);
#pragma unroll
  for (int k = 0; k < WORDS; ++k) e.w[k] = __builtin_amdgcn_readlane(e.w[k], ti);
  return __builtin_bit_cast(MuonTensor, e);
}

// Reads or writes the lane's elements of 32 columns of X, from column n0 on, in a [rows, cols] matrix.
// Wide (rows <= cols): 32 lanes take 128 bytes of a row.  A buffer per row (its start is the same for the wavefront) and no
// branches: what lies outside the matrix is aimed past the buffer, where loads give zero and stores nothing.  (With a branch around
// each load the compiler waits for them a few at a time.)
// Tall (an adapter's A): the 32 columns of X are one run of memory; it goes through the wavefront's room in LDS, as
// [n][MUON_TURN_LD].  (Lanes reading their elements from as many rows took 21 us of the first launch over muon_layer's matrices.)
constexpr int muon_turn_ld(int rt) { return 32 * rt + 4; }
constexpr size_t muon_turn_floats(int rt) { return (size_t)32 * muon_turn_ld(rt); }
template <int RT>
struct Elements {
  static constexpr int LD = muon_turn_ld(RT);
  bool wide, column;
  int rows, cols, hi4, lane, run;
  size_t base;
  uint32_t away, reciprocal;
  float* room;
  __device__ __forceinline__ Elements(const MuonTensor& t, int n0, int lane_, float* room_)
      : wide(t.rows <= t.cols), rows(t.rows), cols(t.cols), hi4(4 * (lane_ >> 5)), lane(lane_), room(room_) {
    column = n0 + (lane & 31) < max(rows, cols);
    base = wide ? (size_t)n0 : (size_t)n0 * cols;
    away = column ? 4u * ((uint32_t)hi4 * (uint32_t)cols + (lane & 31)) : 0xfffffffcu;
    run = wide ? 0 : min(32, rows - n0) * cols;                       // of a tall matrix
    reciprocal = wide ? 0 : ((1u << 20) + cols - 1) / (uint32_t)cols;  // e / cols = e * this >> 20 for e < 4096, cols <= 128
  }
  // The buffers of rows, for one use.  (Opaque: the compiler would work out all rows' starts and sizes ahead of the loop over
  // chunks and for the next use, and keep them in the lanes of vector registers: 1500 moves a chunk at 128 rows.)
  struct Rows {
    float* start;
    int rows, cols;
    __device__ __forceinline__ Rows(const Elements& e, const float* p) : start(const_cast<float*>(p) + e.base), rows(e.rows), cols(e.cols) {
      asm volatile("" : "+s"(start), "+s"(rows), "+s"(cols));
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t operator[](int k) const {
      const uint32_t bytes = k + 4 < rows ? 0xfffffffcu : (k < rows ? 16u * cols : 0u);  // (row k + 4 is the upper lanes')
      return __builtin_amdgcn_make_buffer_rsrc(start + (size_t)k * cols, 0, (int)bytes, 0x00020000);
    }
  };
  // element lane + 64 k of the run, in LDS
  __device__ __forceinline__ float* turned(int k) const {
    int at = lane;
    asm volatile("" : "+v"(at));  // (else all of them are worked out once, and their registers held throughout)
    const uint32_t e = at + 64 * k, n = e * reciprocal >> 20;
    return room + n * LD + (e - n * cols);
  }
  __device__ __forceinline__ int mine() const {  // what of the run lies from the lane on
    int left = run - lane;
    asm volatile("" : "+v"(left));
    return left;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t run_buffer(const float* p) const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p) + base, 0, 4 * run, 0x00020000);
  }
  static __device__ __forceinline__ void handed_over() {  // between the lanes of the wavefront, through LDS
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // In two parts, so that other work can lie between: the loads, and (of a tall matrix) each element to its lane.
  __device__ __forceinline__ void request(const float* p, f32x4 (&v)[4 * RT]) const {
    if (wide) {
      const Rows row(*this, p);
#pragma unroll
      for (int q = 0; q < 4 * RT; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row[8 * q + e], (int)away, 0, 0));
        __builtin_amdgcn_sched_barrier(0);  // (else the buffers of all rows are made first, and scalar registers run out)
      }
      return;
    }
    const __amdgpu_buffer_rsrc_t rs = run_buffer(p);
#pragma unroll
    for (int k = 0; k < 16 * RT; ++k) v[k >> 2][k & 3] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, 4 * (lane + 64 * k), 0, 0));
  }
  __device__ __forceinline__ void settle(f32x4 (&v)[4 * RT]) const {
    if (wide) return;
    handed_over();
    const int left = mine();
#pragma unroll
    for (int k = 0; k < 16 * RT; ++k)
      if (64 * k < left) *turned(k) = v[k >> 2][k & 3];
    handed_over();
    int limit = column ? cols - hi4 : 0;
    asm volatile("" : "+v"(limit));
#pragma unroll
    for (int q = 0; q < 4 * RT; ++q) {
      const f32x4 r = *reinterpret_cast<const f32x4*>(room + (lane & 31) * LD + 8 * q + hi4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q][e] = 8 * q + e < limit ? r[e] : 0.0f;
    }
  }
  __device__ __forceinline__ void store(float* p, const f32x4 (&v)[4 * RT]) const {
    if (wide) {
      const Rows row(*this, p);
#pragma unroll
      for (int q = 0; q < 4 * RT; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[q][e]), row[8 * q + e], (int)away, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      return;
    }
    handed_over();
#pragma unroll
    for (int q = 0; q < 4 * RT; ++q) *reinterpret_cast<f32x4*>(room + (lane & 31) * LD + 8 * q + hi4) = v[q];
    handed_over();
    const __amdgpu_buffer_rsrc_t rs = run_buffer(p);
    const int left = mine();
    float r[16 * RT];
#pragma unroll
    for (int k = 0; k < 16 * RT; ++k) r[k] = 64 * k < left ? *turned(k) : 0.0f;
#pragma unroll
    for (int k = 0; k < 16 * RT; ++k) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(r[k]), rs, 4 * (lane + 64 * k), 0, 0);
  }
};

constexpr int muon_waves(int rt) { return muon_waves_of(rt); }  // of a block: 512 registers each, or 256

// The wavefronts' G tiles (upper ones, in results' layout) added in order through LDS, some tiles at a time:
// sink(tile, quad, lane, sum), from the whole block.
constexpr int muon_tiles_at_once(int rt) { return rt > 2 ? muon_upper(rt) / 2 : muon_upper(rt); }
template <int RT, typename Sink>
__device__ __forceinline__ void add_shares(const f32x16 (&g)[muon_upper(RT)], f32x4* lds, int wave, int lane, Sink&& sink) {
  constexpr int NW = muon_waves(RT), U = muon_upper(RT), AT_ONCE = muon_tiles_at_once(RT);
  static_assert(U % AT_ONCE == 0, "whole batches");
#pragma unroll
  for (int u0 = 0; u0 < U; u0 += AT_ONCE) {
    lds_barrier();
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) lds[((wave * AT_ONCE + u) * 4 + q) * 64 + lane] = quad_of(g[u0 + u], q);
    lds_barrier();
#pragma unroll
    for (int k = 0; k < (AT_ONCE * 4 + NW - 1) / NW; ++k) {
      const int piece = wave + NW * k;  // tile and quad: 64 pieces of 16 bytes
      if (piece >= AT_ONCE * 4) break;
      f32x4 v = lds[piece * 64 + lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += lds[(w * AT_ONCE * 4 + piece) * 64 + lane];
      sink(u0 + (piece >> 2), piece & 3, lane, v);
    }
  }
}
template <int RT>
__device__ __forceinline__ void store_share(const f32x16 (&g)[muon_upper(RT)], f32x4* lds, f32x4* out, int wave, int lane) {
  add_shares<RT>(g, lds, wave, lane, [&](int u, int q, int l, const f32x4& v) { out[(u * 4 + q) * 64 + l] = v; });
}
// Row and column of the upper tile u.
__device__ __forceinline__ void upper_tile(int u, int& a, int& b) {
  b = 0;
  while ((b + 1) * (b + 2) / 2 <= u) ++b;
  a = u - b * (b + 1) / 2;
}
// Quad q of G's tile (a, b) and, off the diagonal, its mirror image: element (8 q + 4 (lane / 32) + k, lane % 32) at its place.
template <int RT>
__device__ __forceinline__ void put_gram(float* gram, int a, int b, int q, int lane, const f32x4& v) {
  *reinterpret_cast<f32x4*>(gram + (a * RT + b) * 1024 + (q * 64 + lane) * 4) = v;
  if (a == b) return;
  const int col = lane & 31;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int row = 8 * q + 4 * (lane >> 5) + k;
    gram[(b * RT + a) * 1024 + ((col >> 3) * 64 + row + 32 * ((col >> 2) & 1)) * 4 + (col & 3)] = v[k];
  }
}
constexpr size_t muon_share_lds(int rt) { return (size_t)muon_waves(rt) * muon_tiles_at_once(rt) * 4096; }
constexpr size_t muon_p_lds(int rt) { return (size_t)rt * rt * 4096; }
constexpr size_t muon_turn_lds(int rt) { return muon_waves(rt) * muon_turn_floats(rt) * 4; }
constexpr size_t muon_start_lds(int rt) { return std::max(muon_share_lds(rt), muon_turn_lds(rt)); }
constexpr size_t muon_alone_lds(int rt) { return 2 * muon_p_lds(rt) + muon_start_lds(rt); }
constexpr size_t muon_pass_lds(int rt, bool last, bool direct) {  // (the shares lie where P and G have been)
  const size_t p = muon_p_lds(rt) * (direct ? 2 : 1);
  return last ? p + muon_turn_lds(rt) : std::max(muon_share_lds(rt), p);
}

// G's tiles from 32 columns of X as operands, rows of X as rows: g[(a, b)] += x_a x_b^T.
template <int RT>
__device__ __forceinline__ void add_gram(f32x16 (&g)[muon_upper(RT)], const Operand (&x)[RT][2]) {
#pragma unroll
  for (int b = 0; b < RT; ++b)
#pragma unroll
    for (int a = 0; a <= b; ++a)
#pragma unroll
      for (int s = 0; s < 2; ++s) add(g[upper_at(a, b)], x[a][s], x[b][s]);
}

// u = the momentum's step on 32 columns, in results' layout; returns the largest magnitude in the wavefront.
template <int RT>
__device__ __forceinline__ float momentum_step(const MuonTensor& t, const MuonHyper& h, int n0, int lane, float* room, f32x4 (&u)[4 * RT]) {
  const Elements<RT> at(t, n0, lane, room);
  f32x4 m[4 * RT];
  at.request(t.g, u);
  at.request(t.m, m);
  at.settle(u);
  at.settle(m);
  float most = 0.0f;
#pragma unroll
  for (int q = 0; q < 4 * RT; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m[q][e] = __builtin_fmaf(h.momentum, m[q][e], u[q][e]);
      u[q][e] = h.nesterov ? __builtin_fmaf(h.momentum, m[q][e], u[q][e]) : m[q][e];
      most = fmaxf(most, fabsf(u[q][e]));
    }
  __builtin_amdgcn_sched_barrier(0);  // (stores between the waits for loads would be waited for, too)
  at.store(t.m, m);
  if (h.zero_grads) {
    f32x4 zero[4 * RT];
#pragma unroll
    for (int q = 0; q < 4 * RT; ++q) zero[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    at.store(t.g, zero);
  }
  return over_wave(most, [](float x, float y) { return fmaxf(x, y); });
}

// The scales of a pass and the norm that comes off X in the first one.
struct Scales {
  float x_norm, g, x;  // x: of X once its norm is off
  float p, y;          // of P and of P X (once P is there)
  float trace, x_bound;
  __device__ __forceinline__ Scales(float trace_, float eps, bool first) {
    // (A norm that squares lost below the smallest fp32 may miss counts as that much: with a small eps, X0 could be of any size.
    // A comparison, which keeps a NaN.)
    const float norm = __fsqrt_rn(trace_);
    x_norm = first ? 1.0f / ((norm < kLostNorm ? kLostNorm : norm) + eps) : 1.0f;
    x_bound = (norm + kLostNorm) * x_norm;
    trace = trace_ * x_norm * x_norm;
    g = scale_below(trace);
    x = scale_below(x_bound);
  }
};

// Operands in LDS: [tile][slice][hi, lo][lane] of 16 bytes.
__device__ __forceinline__ void put_operands(f32x4* lds, int tile, int lane, const f32x4 (&q)[4], float scale) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const Operand o = split(q[2 * s] * scale, q[2 * s + 1] * scale);
    lds[(2 * tile + s) * 128 + lane] = __builtin_bit_cast(f32x4, o.hi);
    lds[(2 * tile + s) * 128 + 64 + lane] = __builtin_bit_cast(f32x4, o.lo);
  }
}
__device__ __forceinline__ Operand operand_at(const f32x4* lds, int tile, int s, int lane) {
  const f32x4* at = lds + (2 * tile + s) * 128 + lane;
  return Operand{__builtin_bit_cast(f16x8, at[0]), __builtin_bit_cast(f16x8, at[64])};
}

// The chunks of a wavefront: every muon_waves-th of its block's.
template <int RT>
struct Columns {
  const MuonTensor& t;
  f32x4* x;     // X
  int first, end;
  int wave, lane;
  float* room;  // the wavefront's, for tall matrices
  __device__ __forceinline__ Columns(const MuonTensor& t_, float* ws, int begin, int end_, float* rooms)
      : t(t_), end(end_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {
    first = begin + wave;
    x = reinterpret_cast<f32x4*>(ws + t.x);
    room = rooms + wave * muon_turn_floats(RT);
  }
  __device__ __forceinline__ f32x4* at(int c) const { return x + (size_t)c * RT * 256 + lane; }
  // (No branch for a chunk beyond the last: behind one, a wait for what was requested before takes these loads for absent and
  // waits for them too.  The buffer is empty instead.)
  __device__ __forceinline__ void request(int c, f32x4 (&coming)[4 * RT]) const {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(x + (size_t)c * RT * 256, 0, c < end ? RT * 4096 : 0, 0x00020000);
#pragma unroll
    for (int q = 0; q < 4 * RT; ++q)
      coming[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * lane + 1024 * q, 0, 0));
  }
};

// Momentum, u into X, and the wavefront's share of u u^T.
template <int RT>
__device__ __forceinline__ void start_columns(const Columns<RT>& w, const MuonHyper& h, f32x16 (&g)[muon_upper(RT)]) {
  const f16x8 unit[2] = {unit_slice(0, w.lane), unit_slice(1, w.lane)};
#pragma unroll
  for (int u = 0; u < muon_upper(RT); ++u) g[u] = zero16();
  for (int c = w.first; c < w.end; c += muon_waves(RT)) {
    f32x4 u[4 * RT];
    const float s = scale_below(momentum_step<RT>(w.t, h, c * MUON_CHUNK, w.lane, w.room, u));
    f32x4* x = w.at(c);
#pragma unroll
    for (int q = 0; q < 4 * RT; ++q) x[64 * q] = u[q];
    Operand rows[RT][2];
#pragma unroll
    for (int a = 0; a < RT; ++a) {
      const Operand in[2] = {split(u[4 * a] * s, u[4 * a + 1] * s), split(u[4 * a + 2] * s, u[4 * a + 3] * s)};
      turn(in, unit, rows[a]);
    }
    const float back = inverse_power(s);  // (twice: its square may be below the smallest fp32)
#pragma unroll
    for (int b = 0; b < RT; ++b)
#pragma unroll
      for (int a = 0; a <= b; ++a) {
        f32x16 part = zero16();
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) add(part, rows[a][sl], rows[b][sl]);
#pragma unroll
        for (int r = 0; r < 16; ++r) g[upper_at(a, b)][r] += part[r] * back * back;
      }
  }
}

// P = a I + b G + c G^2 as operands in LDS, its tile (t, a) at a RT + t (G's were there before).  meanwhile() requests what is
// needed after it: behind G's loads, whose wait would otherwise include it.
template <int RT, typename Fn>
__device__ __forceinline__ Scales make_p(const float* gram, const MuonHyper& h, bool first, f32x4* lds, float* squares, int wave, int lane, Fn&& meanwhile) {
  constexpr int NW = muon_waves(RT);
  // A wavefront has tiles (t, a) of G and of P, in results' layout: the operand for rows of tile a and slices of tile t.
  constexpr int PT = (RT * RT + NW - 1) / NW;
  f32x4 p[PT][4];
#pragma unroll
  for (int k = 0; k < PT; ++k)  // (some wavefronts for nothing: no branch, see Columns::request)
#pragma unroll
    for (int q = 0; q < 4; ++q) p[k][q] = reinterpret_cast<const f32x4*>(gram)[min(wave + NW * k, RT * RT - 1) * 256 + q * 64 + lane];
  float ds[(32 * RT + 63) / 64];
#pragma unroll
  for (int k = 0; k < (32 * RT + 63) / 64; ++k) {
    const int d = lane + 64 * k, a = min(d >> 5, RT - 1), dd = d & 31;
    const float on = gram[(a * RT + a) * 1024 + ((dd >> 3) * 64 + dd + 32 * ((dd >> 2) & 1)) * 4 + (dd & 3)];
    ds[k] = d < 32 * RT ? on : 0.0f;
  }
  __builtin_amdgcn_sched_barrier(0);
  meanwhile();
  __builtin_amdgcn_sched_barrier(0);
  float diagonal = 0.0f;
#pragma unroll
  for (int k = 0; k < (32 * RT + 63) / 64; ++k) diagonal += ds[k];
  Scales s(wave_sum(diagonal), h.eps, first);
#pragma unroll
  for (int k = 0; k < PT; ++k)
    if (wave + NW * k < RT * RT) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        p[k][q] *= s.x_norm * s.x_norm;
      put_operands(lds, wave + NW * k, lane, p[k], s.g);
    }
  lds_barrier();
  float square = 0.0f;
  const float g_back = inverse_power(s.g) * inverse_power(s.g);
#pragma unroll
  for (int k = 0; k < PT; ++k)
    if (wave + NW * k < RT * RT) {
      const int tt = (wave + NW * k) / RT, a = (wave + NW * k) % RT;
      f32x16 g2 = zero16();
#pragma unroll
      for (int u = 0; u < RT; ++u)
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) add(g2, operand_at(lds, u * RT + tt, sl, lane), operand_at(lds, u * RT + a, sl, lane));
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float one = (tt == a && 8 * q + 4 * (lane >> 5) + e == (lane & 31)) ? h.a : 0.0f;
          p[k][q][e] = __builtin_fmaf(h.c, g2[4 * q + e] * g_back, __builtin_fmaf(h.b, p[k][q][e], one));
          square = __builtin_fmaf(p[k][q][e], p[k][q][e], square);
        }
    }
  square = wave_sum(square);
  if (lane == 0) squares[wave] = square;
  lds_barrier();  // (also: G has been read, and its place is free)
  float p_bound = 0.0f;
#pragma unroll
  for (int k = 0; k < NW; ++k) p_bound += squares[k];
  p_bound = __fsqrt_rn(p_bound) * 1.001f;
  s.p = scale_below(p_bound);
  s.y = scale_below(p_bound * s.x_bound);
#pragma unroll
  for (int k = 0; k < PT; ++k)
    if (wave + NW * k < RT * RT) put_operands(lds, (wave + NW * k) % RT * RT + (wave + NW * k) / RT, lane, p[k], s.p);
  lds_barrier();
  return s;
}

// X <- P X on the wavefront's columns.  LAST: the result goes into the parameters, else back to X with its share of the next G.
template <int RT, bool LAST>
__device__ __forceinline__ void pass_columns(const Columns<RT>& w, const MuonHyper& h, const Scales& s, const f32x4* p, f32x4 (&coming)[4 * RT],
                                             f32x16 (&g)[muon_upper(RT)]) {
  constexpr int NW = muon_waves(RT);
  const f16x8 unit[2] = {unit_slice(0, w.lane), unit_slice(1, w.lane)};
#pragma unroll
  for (int u = 0; u < muon_upper(RT); ++u) g[u] = zero16();
  const float in_scale = s.x_norm * s.x, y_back = inverse_power(s.x) * inverse_power(s.p);
  for (int c = w.first; c < w.end; c += NW) {
    Operand x[RT][2];
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) x[a][sl] = split(coming[4 * a + 2 * sl] * in_scale, coming[4 * a + 2 * sl + 1] * in_scale);
    w.request(c + NW, coming);
    const Elements<RT> at(w.t, c * MUON_CHUNK, w.lane, w.room);
    f32x4 param[4 * RT];
    if constexpr (LAST) at.request(w.t.p, param);
    Operand rows[RT][2];
    // two row tiles at a time: their products alternate, and the operands of the next slice are read meanwhile
    constexpr int PAIR = RT > 1 ? 2 : 1;
    auto p_at = [&](int a, int k) { return operand_at(p, a * RT + (k >> 1), k & 1, w.lane); };  // rows of tile a, slice k
#pragma unroll
    for (int a0 = 0; a0 < RT; a0 += PAIR) {
      f32x16 acc[PAIR];
      Operand now[PAIR], next[PAIR];
#pragma unroll
      for (int j = 0; j < PAIR; ++j) {
        acc[j] = zero16();
        next[j] = p_at(a0 + j, 0);
      }
#pragma unroll
      for (int k = 0; k < 2 * RT; ++k) {
#pragma unroll
        for (int j = 0; j < PAIR; ++j) {
          now[j] = next[j];
          if (k + 1 < 2 * RT) next[j] = p_at(a0 + j, k + 1);
        }
        const Operand& xk = x[k >> 1][k & 1];
#pragma unroll
        for (int j = 0; j < PAIR; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[j].hi, xk.hi, acc[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < PAIR; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[j].hi, xk.lo, acc[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < PAIR; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[j].lo, xk.hi, acc[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (LAST && a0 == 0) at.settle(param);
#pragma unroll
      for (int j = 0; j < PAIR; ++j) {
        const int a = a0 + j;
        f32x4 y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = quad_of(acc[j], q) * y_back;
        if constexpr (LAST) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) param[4 * a + q][e] = __builtin_fmaf(param[4 * a + q][e], h.decay, -w.t.step_size * y[q][e]);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) w.at(c)[64 * (4 * a + q)] = y[q];
          const Operand in[2] = {split(y[0] * s.y, y[1] * s.y), split(y[2] * s.y, y[3] * s.y)};
          turn(in, unit, rows[a]);
        }
      }
    }
    if constexpr (LAST) {
      __builtin_amdgcn_sched_barrier(0);
      at.store(w.t.p, param);
    } else {
      add_gram<RT>(g, rows);
    }
  }
  if constexpr (!LAST) {
    const float back = inverse_power(s.y) * inverse_power(s.y);
#pragma unroll
    for (int u = 0; u < muon_upper(RT); ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) g[u][r] *= back;
  }
}

}  // namespace

template <int RT>
__global__ __launch_bounds__(64 * muon_waves(RT), 1) void muon_start_kernel(const MuonTable table, const MuonHyper h, float* ws) {
  extern __shared__ __align__(16) f32x4 lds[];
  int slice;
  const MuonTensor t = muon_find(table, table.block0, slice);
  const Columns<RT> w(t, ws, slice * table.per_block, min(t.chunks, (slice + 1) * table.per_block), reinterpret_cast<float*>(lds));
  f32x16 g[muon_upper(RT)];
  start_columns<RT>(w, h, g);
  store_share<RT>(g, lds, reinterpret_cast<f32x4*>(ws + t.partial) + (size_t)slice * muon_upper(RT) * 256, w.wave, w.lane);
}

// G = sum of the blocks' shares, upper tiles, and their mirror images: 32 pieces of 16 bytes a block, their shares dealt to
// eight groups of threads.
template <int RT>
__global__ __launch_bounds__(256) void muon_reduce_kernel(const MuonTable table, float* ws) {
  __shared__ f32x4 part[8][32];
  int number;
  const MuonTensor t = muon_find(table, table.reduce0, number);
  const int slices = (t.chunks + table.per_block - 1) / table.per_block;
  const int e = threadIdx.x & 31, group = threadIdx.x >> 5;
  constexpr int pieces = muon_upper(RT) * 256;
  const int at = number * 32 + e;
  const f32x4* src = reinterpret_cast<const f32x4*>(ws + t.partial) + at;
  const int per = (slices + 7) / 8, z0 = min(slices, group * per), z1 = min(slices, z0 + per);
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
  for (int z = z0; z < z1; ++z) v += src[(size_t)z * pieces];
  part[group][e] = v;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) v += part[k][e];
  int a, b;
  upper_tile(at >> 8, a, b);
  put_gram<RT>(ws + t.gram, a, b, (at >> 6) & 3, at & 63, v);
}

// One step of the iteration (in the first one X holds u, whose norm comes off).  DIRECT: each block adds its matrix's shares of G by
// itself, and leaves its share of the next one in the other of two places.
template <int RT, bool LAST, bool DIRECT>
__global__ __launch_bounds__(64 * muon_waves(RT), 1) void muon_pass_kernel(const MuonTable table, const MuonHyper h, int step, float* ws) {
  extern __shared__ __align__(16) f32x4 lds[];
  __shared__ float squares[muon_waves(RT)];
  int slice;
  const MuonTensor t = muon_find(table, table.block0, slice);
  const Columns<RT> w(t, ws, slice * table.per_block, min(t.chunks, (slice + 1) * table.per_block),
                      reinterpret_cast<float*>(lds) + muon_p_lds(RT) / 4 * (DIRECT ? 2 : 1));
  f32x4* partial = reinterpret_cast<f32x4*>(ws + t.partial);
  const float* gram = ws + t.gram;
  if constexpr (DIRECT) {
    constexpr int NW = muon_waves(RT), PIECES = muon_upper(RT) * 4;  // of 64 times 16 bytes
    const int slices = (t.chunks + table.per_block - 1) / table.per_block;
    const size_t place = (size_t)slices * PIECES * 64;
    const f32x4* src = partial + (step & 1 ? place : 0) + w.lane;
    if (!(step & 1)) partial += place;
    float* sum = reinterpret_cast<float*>(lds) + muon_p_lds(RT) / 4;
#pragma unroll
    for (int k = 0; k < (PIECES + NW - 1) / NW; ++k) {
      const int piece = w.wave + NW * k;
      if (piece >= PIECES) break;
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
      for (int z = 0; z < slices; ++z) v += src[((size_t)z * PIECES + piece) * 64];
      int a, b;
      upper_tile(piece >> 2, a, b);
      put_gram<RT>(sum, a, b, piece & 3, w.lane, v);
    }
    lds_barrier();
    gram = sum;
  }
  // The columns that come next are on their way: the first ones while P is made, later ones while those before are worked on.
  f32x4 coming[4 * RT];
  const Scales s = make_p<RT>(gram, h, step == 0, lds, squares, w.wave, w.lane, [&] { w.request(w.first, coming); });
  f32x16 g[muon_upper(RT)];
  pass_columns<RT, LAST>(w, h, s, lds, coming, g);
  if constexpr (!LAST) store_share<RT>(g, lds, partial + (size_t)slice * muon_upper(RT) * 256, w.wave, w.lane);
}

// All steps of a matrix in one block, G in its LDS: the launches above take 5 to 7 us each however little there is to do.
template <int RT>
__global__ __launch_bounds__(64 * muon_waves(RT), 1) void muon_alone_kernel(const MuonTable table, const MuonHyper h, int steps, float* ws) {
  extern __shared__ __align__(16) f32x4 lds[];  // operands of G and P, then G, then the shares or the rooms for tall matrices
  __shared__ float squares[muon_waves(RT)];
  const MuonTensor& t = table.t[blockIdx.x];
  f32x4* shares = lds + 2 * muon_p_lds(RT) / 16;
  float* gram = reinterpret_cast<float*>(lds) + muon_p_lds(RT) / 4;
  const Columns<RT> w(t, ws, 0, t.chunks, reinterpret_cast<float*>(shares));
  f32x16 g[muon_upper(RT)];
  start_columns<RT>(w, h, g);
  f32x4 coming[4 * RT];
  auto next_p = [&](bool first) {
    int lane = w.lane;
    asm volatile("" : "+v"(lane));  // (else the places in LDS that depend on it are held in registers throughout)
    add_shares<RT>(g, shares, w.wave, lane, [&](int u, int q, int l, const f32x4& v) {
      int a, b;
      upper_tile(u, a, b);
      put_gram<RT>(gram, a, b, q, l, v);
    });
    lds_barrier();
    return make_p<RT>(gram, h, first, lds, squares, w.wave, lane, [&] { w.request(w.first, coming); });
  };
  for (int k = 0; k + 1 < steps; ++k) {
    const Scales s = next_p(k == 0);
    pass_columns<RT, false>(w, h, s, lds, coming, g);
  }
  const Scales s = next_p(steps == 1);
  pass_columns<RT, true>(w, h, s, lds, coming, g);
}

namespace {

template <typename Kernel, typename... Args>
hipError_t launch(Kernel kern, int blocks, int rt, size_t lds, std::atomic<uint64_t>& granted, hipStream_t st, const Args&... args) {
  if (hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kern), (int)lds, granted); e != hipSuccess) return e;
  kern<<<blocks, 64 * muon_waves(rt), lds, st>>>(args...);
  return hipGetLastError();
}

template <int RT, bool DIRECT>
hipError_t launch_steps(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  static std::atomic<uint64_t> granted[3];
  if (hipError_t e = launch(muon_start_kernel<RT>, t.blocks, RT, muon_start_lds(RT), granted[0], st, t, h, ws); e != hipSuccess) return e;
  for (int k = 0; k < steps; ++k) {
    if constexpr (!DIRECT) {
      muon_reduce_kernel<RT><<<t.reduce_blocks, 256, 0, st>>>(t, ws);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const hipError_t e = k + 1 < steps ? launch(muon_pass_kernel<RT, false, DIRECT>, t.blocks, RT, muon_pass_lds(RT, false, DIRECT), granted[1], st, t, h, k, ws)
                                       : launch(muon_pass_kernel<RT, true, DIRECT>, t.blocks, RT, muon_pass_lds(RT, true, DIRECT), granted[2], st, t, h, k, ws);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int RT>
hipError_t launch_alone(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  static std::atomic<uint64_t> granted{0};
  return launch(muon_alone_kernel<RT>, t.n, RT, muon_alone_lds(RT), granted, st, t, h, steps, ws);
}

}  // namespace

hipError_t launch_muon(const MuonTable& t, const MuonHyper& h, int steps, float* ws, hipStream_t st) {
  if (t.alone) return t.tiles == 2 ? launch_alone<2>(t, h, steps, ws, st) : launch_alone<1>(t, h, steps, ws, st);
  if (t.tiles > 2) return launch_steps<4, false>(t, h, steps, ws, st);
  if (t.direct) return t.tiles == 2 ? launch_steps<2, true>(t, h, steps, ws, st) : launch_steps<1, true>(t, h, steps, ws, st);
  return t.tiles == 2 ? launch_steps<2, false>(t, h, steps, ws, st) : launch_steps<1, false>(t, h, steps, ws, st);
}

}  // namespace qalora
