// Products of 8-bit integers, exact in 32 bits, with a scale for each token and (forward) each output channel:
//   forward   z[t, j]  = s[t] sw[j] sum_i q[t, i] w8[j, i]      K = d_in
//   backward  dx[t, i] = s[t] sum_j q[t, j] w8[j, i]            K = d_out (the channels' scales are in q)
// and the epilogue on that.  One copy of the weight's codes, [d_out, d_in], serves both directions: the forward's operands lie along K in
// it, the backward's are turned by transposing LDS reads.
// Large products are bound by the matrix instructions and the chip's power: 4096 tokens, K = 11008, 4096 columns, either direction 152 us
// behind a pause, 2430 TOP/s, and 164 one after the other.  A step of K is 128, whole cache lines of every row (64: 216 us for 4096 x 11008 x 4096 that take 180); the backward's reads
// wait in a block of their own (by the builtin, before which all loads on their way are waited for: 183 us).
#include <atomic>
#include <type_traits>

#include "int8.hpp"
#include "epilogue.hpp"
#include "gemm_i8_plan.hpp"
#include "kernels.hpp"

namespace qalora {

namespace {
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) const int8_t lds_i8;
constexpr uint32_t kPast = 0xffff0000u;  // a byte offset past any tile: reads zero

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// Each XCD gets a contiguous run of tiles (consecutive blocks are dealt to the eight in turn).
__device__ __forceinline__ int xcd_run(int b, int n) { return n % 8 ? b : (b % 8) * (n / 8) + b / 8; }
// Codes in LDS, turned: sixteen lanes at 8-byte addresses get the columns of eight rows, from OFF on and from DOWN bytes further (the
// lower and upper half of a matrix instruction's sixteen of K).  In one block with its wait: the compiler, which cannot tell which LDS the
// builtin reads, would have it wait for all loads on their way to other stages.
template <int OFF, int DOWN>
__device__ __forceinline__ void read_turned(const uint32_t (&at)[4], i32x4 (&out)[4]) {
  i32x2 l[4], h[4];
  asm volatile(
      "ds_read_b64_tr_b8 %0, %8 offset:%12\n\tds_read_b64_tr_b8 %1, %8 offset:%13\n\t"
      "ds_read_b64_tr_b8 %2, %9 offset:%12\n\tds_read_b64_tr_b8 %3, %9 offset:%13\n\t"
      "ds_read_b64_tr_b8 %4, %10 offset:%12\n\tds_read_b64_tr_b8 %5, %10 offset:%13\n\t"
      "ds_read_b64_tr_b8 %6, %11 offset:%12\n\tds_read_b64_tr_b8 %7, %11 offset:%13\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(l[0]), "=&v"(h[0]), "=&v"(l[1]), "=&v"(h[1]), "=&v"(l[2]), "=&v"(h[2]), "=&v"(l[3]), "=&v"(h[3])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(OFF), "n"(OFF + DOWN)
      : "memory");
#pragma unroll
  for (int a = 0; a < 4; ++a) out[a] = i32x4{l[a][0], l[a][1], h[a][0], h[a][1]};
}
template <int OFF, int DOWN>
__device__ __forceinline__ void read_turned(const uint32_t (&at)[2], i32x4 (&out)[2]) {
  i32x2 l[2], h[2];
  asm volatile(
      "ds_read_b64_tr_b8 %0, %4 offset:%6\n\tds_read_b64_tr_b8 %1, %4 offset:%7\n\t"
      "ds_read_b64_tr_b8 %2, %5 offset:%6\n\tds_read_b64_tr_b8 %3, %5 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(l[0]), "=&v"(h[0]), "=&v"(l[1]), "=&v"(h[1])
      : "v"(at[0]), "v"(at[1]), "n"(OFF), "n"(OFF + DOWN)
      : "memory");
#pragma unroll
  for (int a = 0; a < 2; ++a) out[a] = i32x4{l[a][0], l[a][1], h[a][0], h[a][1]};
}

// Calls f with the stages of the pipeline as pointers that the compiler may tell apart: else it would wait for the loads that are on
// their way to one of them before every read of another.
template <typename F>
__device__ __forceinline__ void each_stage(int8_t* __restrict__ a, int8_t* __restrict__ b, F&& f) { f(a, b); }
template <typename F>
__device__ __forceinline__ void each_stage(int8_t* __restrict__ a, int8_t* __restrict__ b, int8_t* __restrict__ c, F&& f) { f(a, b, c); }
template <typename F>
__device__ __forceinline__ void each_stage(int8_t* __restrict__ a, int8_t* __restrict__ b, int8_t* __restrict__ c, int8_t* __restrict__ d, F&& f) {
  f(a, b, c, d);
}
template <int STAGES, typename F>
__device__ __forceinline__ void with_stages(int8_t* lds, int bytes, F&& f) {
  static_assert(STAGES >= 2 && STAGES <= 4, "as many as there are forms of each_stage");
  if constexpr (STAGES == 2) each_stage(lds, lds + bytes, f);
  else if constexpr (STAGES == 3) each_stage(lds, lds + bytes, lds + 2 * bytes, f);
  else each_stage(lds, lds + bytes, lds + 2 * bytes, lds + 3 * bytes, f);
}
}  // namespace

// BM tokens from m0 on by BN columns from n0 on, of WM x WN wavefronts; a wavefront has TM x TN tiles of 16 x 16, and the operand that runs
// down a result's registers is the weight's, so that a lane has four neighbouring columns of a token.
// ONCE: the weight is read by one row of tiles only, past the caches.
template <bool BWD, int BM, int BN, int WM, int WN, int STAGES, bool ONCE>
__device__ __forceinline__ void gemm_i8_tile(const Int8GemmArgs& p, int8_t* lds, int m0, int n0) {
  constexpr int NT = WM * WN * 64, WAVES = WM * WN, POLICY = ONCE ? 2 : 0;  // 2: nontemporal
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int X_TILE = BM * I8_STEP, W_TILE = BN * I8_STEP, STAGE = X_TILE + W_TILE;
  constexpr int X_LOADS = X_TILE / 16 / NT, W_LOADS = W_TILE / 16 / NT;  // sixteen bytes each, of a thread
  static_assert(X_LOADS * NT * 16 == X_TILE && W_LOADS * NT * 16 == W_TILE, "whole loads");
  static_assert(!BWD || (BN / 16 & (BN / 16 - 1)) == 0, "places by exclusive or");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  // blockIdx.y: which slice of K (its sums are added up by a later launch)
  const int all = ceil_div(p.K, I8_STEP), per = ceil_div(all, (int)gridDim.y);
  const int begin = blockIdx.y * per, steps = min(all, begin + per) - begin;
  const int k_end = min(p.K, (begin + steps) * I8_STEP);

  // ---- loads: global to LDS, each wavefront 1 KB at a time, lane i to byte 16 i of it.
  // Tokens, and the forward's weights: eight rows of 128 bytes.  Two rows share 256 bytes; the place of a row's chunk c among its eight is
  // c ^ (row / 2 % 8), so that sixteen rows' reads of one chunk fall on sixteen places.
  // The backward's weights: rows (of K) of BN columns; the place of chunk c of row r is c ^ (r % 8 + 8 (r / 16 % 2)): what 32 lanes of
  // a transposing read ask for, two times eight rows of one chunk, falls on sixteen places.
  static_assert(WAVES % 2 == 0, "a lane's chunk is the same for all its loads");
  const int row8 = 2 * (lane >> 4) + ((lane >> 3) & 1), chunk8 = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
  const uint32_t x_rows = min((uint32_t)BM, (uint32_t)(p.M - m0));
  const __amdgpu_buffer_rsrc_t rs_x = tile_rsrc(p.tokens + (size_t)m0 * p.lda, x_rows * (uint32_t)p.lda);
  uint32_t x_off[X_LOADS], w_off[W_LOADS];
#pragma unroll
  for (int q = 0; q < X_LOADS; ++q) x_off[q] = (uint32_t)((q * WAVES + wave) * 8 + row8) * (uint32_t)p.lda + 16 * chunk8;
  const int8_t* w_base = BWD ? p.codes + n0 : p.codes + (size_t)n0 * p.K;
  const uint32_t w_rows = min((uint32_t)BN, (uint32_t)(p.N - n0));
#pragma unroll
  for (int q = 0; q < W_LOADS; ++q) {
    if (BWD) {
      constexpr int RW = BN / 16;  // chunks of a row
      const int at = (q * WAVES + wave) * 64 + lane, r = at / RW;
      const int c = (at % RW) ^ (((r & 7) | ((r >> 1) & 8)) % RW);
      w_off[q] = (uint32_t)r * (uint32_t)p.N + 16 * c;
    } else {
      w_off[q] = (uint32_t)((q * WAVES + wave) * 8 + row8) * (uint32_t)p.K + 16 * chunk8;
    }
  }
  auto request = [&](int it, int8_t* to) {
    const int k0 = (begin + it) * I8_STEP;
    const uint32_t dead = k0 + 16 * chunk8 < k_end ? 0u : kPast;  // (past the last step too: as many loads whatever the step)
    const int from = k0 < k_end ? k0 : 0;                         // (a scalar offset past the operand's end has no meaning)
#pragma unroll
    for (int q = 0; q < X_LOADS; ++q)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_x, (lds_void*)(to + (q * WAVES + wave) * 1024), 16, (int)(x_off[q] | dead), from, 0, 0);
    if (BWD) {
      const int rows = max(0, min(I8_STEP, k_end - k0));
      const uint32_t bytes = rows > 0 ? (uint32_t)rows * (uint32_t)p.N - (uint32_t)n0 : 0u;
      const __amdgpu_buffer_rsrc_t rs_w = tile_rsrc(w_base + (size_t)min(k0, p.K) * p.N, bytes);
#pragma unroll
      for (int q = 0; q < W_LOADS; ++q)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, (lds_void*)(to + X_TILE + (q * WAVES + wave) * 1024), 16, (int)w_off[q], 0, 0, POLICY);
    } else {
      const __amdgpu_buffer_rsrc_t rs_w = tile_rsrc(w_base, w_rows * (uint32_t)p.K);
#pragma unroll
      for (int q = 0; q < W_LOADS; ++q)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, (lds_void*)(to + X_TILE + (q * WAVES + wave) * 1024), 16, (int)(w_off[q] | dead), from, 0, POLICY);
    }
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b) acc[a][b] = i32x4{0, 0, 0, 0};

  const int fr = lane & 15, fc = lane >> 4;  // a fragment's row, and its chunk of K
  const int frag_row = ((fr >> 1) << 8) | ((fr & 1) << 7);  // its byte in sixteen rows, but for the place of chunk 4 u + fc
  const int frag_place[2] = {(fc ^ (fr >> 1)) << 4, ((4 + fc) ^ (fr >> 1)) << 4};
  auto x_frag = [&](const int8_t* s, int u, int b) {
    return *reinterpret_cast<const i32x4*>(s + (wm * TM + b) * 2048 + frag_row + frag_place[u]);
  };
  auto w_frag = [&](const int8_t* s, int u, int a) {
    return *reinterpret_cast<const i32x4*>(s + X_TILE + (wn * TN + a) * 2048 + frag_row + frag_place[u]);
  };
  // Backward: sixteen lanes take eight rows (of K) by sixteen columns; a lane's address is half a row's, what it gets is a column.
  const uint32_t turn_row = (16 * fc + (fr >> 1)) * BN + 8 * (fr & 1), turn_place = (fr >> 1) | ((fc & 1) << 3);
  auto w_turned = [&](const int8_t* s, auto u_c, i32x4(&w)[TN]) {
    const uint32_t base = (uint32_t)(uintptr_t)(lds_i8*)(s + X_TILE) + turn_row;
    uint32_t at[TN];
#pragma unroll
    for (int a = 0; a < TN; ++a) at[a] = base + ((((uint32_t)(wn * TN + a)) ^ (turn_place % (BN / 16))) << 4);
    read_turned<64 * decltype(u_c)::value * BN, 8 * BN>(at, w);
  };

  // The products of 64 of K come in two halves of the wavefront's columns.  While the first half is worked on, the second half's weights
  // are read; while the second half is, the next tokens and first half of weights.  Behind a step's last reads its stage is filled again,
  // for the step STAGES later.
  static_assert(TN >= 2, "two halves");
  constexpr int LOADS = X_LOADS + W_LOADS, HN = TN / 2;
  i32x4 xf[2][TM], wf[2][TN - HN];
  auto first_half = [&](const int8_t* s, int u, i32x4(&x)[TM]) {
#pragma unroll
    for (int a = 0; a < HN; ++a) wf[0][a] = w_frag(s, u, a);
#pragma unroll
    for (int b = 0; b < TM; ++b) x[b] = x_frag(s, u, b);
  };
  auto second_half = [&](const int8_t* s, int u) {
#pragma unroll
    for (int a = 0; a < TN - HN; ++a) wf[1][a] = w_frag(s, u, HN + a);
  };
  auto multiply = [&](int half, const i32x4(&x)[TM]) {
#pragma unroll
    for (int a = 0; a < (half ? TN - HN : HN); ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b)
        acc[half * HN + a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[half][a], x[b], acc[half * HN + a][b], 0, 0, 0);
  };
  // the tile of the next stage has landed, for every wavefront, and no read of this one is on its way
  auto meet = [&](auto in_flight) {
    constexpr int n = decltype(in_flight)::value;
    __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | ((n >> 4) << 14));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  using AllButOne = std::integral_constant<int, LOADS*(STAGES - 1)>;
  using AllButTwo = std::integral_constant<int, LOADS*(STAGES - 2)>;
  [[maybe_unused]] i32x4 wt[2][TN];
  auto multiply_all = [&](int u) {
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wt[u][a], xf[u][b], acc[a][b], 0, 0, 0);
  };
  auto tokens_of = [&](const int8_t* s, int u) {
#pragma unroll
    for (int b = 0; b < TM; ++b) xf[u][b] = x_frag(s, u, b);
  };
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;
  auto step = [&](int it, int8_t* s, const int8_t* next) {
    if constexpr (BWD) {
      w_turned(s, Second{}, wt[1]);
      tokens_of(s, 1);
      multiply_all(0);
      meet(AllButTwo{});
      request(it + STAGES, s);
      w_turned(next, First{}, wt[0]);
      tokens_of(next, 0);
      multiply_all(1);
      return;
    }
    second_half(s, 0);
    multiply(0, xf[0]);
    first_half(s, 1, xf[1]);
    multiply(1, xf[0]);
    second_half(s, 1);
    multiply(0, xf[1]);
    meet(AllButTwo{});
    request(it + STAGES, s);
    first_half(next, 0, xf[0]);  // (past the last step: of zeros, never used)
    multiply(1, xf[1]);
  };
  with_stages<STAGES>(lds, STAGE, [&](auto... stage) {
    int8_t* const at[STAGES] = {stage...};
#pragma unroll
    for (int s = 0; s < STAGES; ++s) request(s, at[s]);
    meet(AllButOne{});
    if constexpr (BWD) {
      w_turned(at[0], First{}, wt[0]);
      tokens_of(at[0], 0);
    } else {
      first_half(at[0], 0, xf[0]);
    }
    for (int it = 0;; ) {
#pragma unroll
      for (int s = 0; s < STAGES; ++s) {
        step(it, at[s], at[(s + 1) % STAGES]);
        if (++it >= steps) return;
      }
    }
  });
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // (the requests past the last step)
  __syncthreads();

  if (p.partial) {
#pragma unroll
    for (int a = 0; a < TN; ++a) {
      const int n = n0 + (wn * TN + a) * 16 + 4 * fc;
#pragma unroll
      for (int b = 0; b < TM; ++b) {
        const int m = m0 + (wm * TM + b) * 16 + fr;
        if (n < p.N && m < p.M) *reinterpret_cast<i32x4*>(p.partial + ((size_t)blockIdx.y * p.M + m) * p.N + n) = acc[a][b];
      }
    }
    return;
  }

  // ---- epilogue: a wavefront turns its own part of the tile in LDS, some tokens at a time, scaled to fp32, so that it stores whole
  // rows of it: a lane has eight columns, the same ones of every row it comes to.  The place of sixteen bytes in a row is
  // exclusive-ored with the row, so that neither the writes (sixteen rows at once) nor the reads meet in a bank.
  constexpr int CW = 16 * TN, PIECES = CW / 4, MASK = (PIECES % 16 == 0 ? 16 : PIECES % 8 == 0 ? 8 : 4) - 1;
  constexpr int LPR = CW / 8, ROWS_AT_ONCE = 64 / LPR;  // (where 64 lanes are not whole rows, the last few have none)
  constexpr int ROOM = STAGES * STAGE / WAVES / (16 * CW * 4);  // of tiles' rows
  constexpr int PB = ROOM >= TM ? TM : (ROOM >= TM / 2 ? TM / 2 : TM / 4);
  static_assert(PB >= 1 && PB <= ROOM && TM % PB == 0, "whole passes");
  char* stage_lds = reinterpret_cast<char*>(lds) + wave * (PB * 16 * CW * 4);
  f32x4 by[TN];
#pragma unroll
  for (int a = 0; a < TN; ++a) {
    const int n = n0 + (wn * TN + a) * 16 + 4 * fc;
    by[a] = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
    if (!BWD && n < p.N) by[a] = *reinterpret_cast<const f32x4*>(p.col_scale + n);
  }
  float sc[TM];
#pragma unroll
  for (int b = 0; b < TM; ++b) sc[b] = p.row_scale[min(p.M - 1, m0 + (wm * TM + b) * 16 + fr)];
  const int ch = lane % LPR, col = n0 + wn * CW + 8 * ch, row_in = lane / LPR;
  const bool col_ok = col < p.N && row_in < ROWS_AT_ONCE;  // (N is a multiple of eight)
  // (without a bias -0 is added, which leaves every sum as it is, one of -0 too: what the other kernels, which add nothing, give)
  f32x4 bias[2] = {f32x4{-0.0f, -0.0f, -0.0f, -0.0f}, f32x4{-0.0f, -0.0f, -0.0f, -0.0f}};
  if (p.epi.bias && col_ok) {
    bias[0] = reinterpret_cast<const f32x4*>(p.epi.bias + col)[0];
    bias[1] = reinterpret_cast<const f32x4*>(p.epi.bias + col)[1];
  }
  // The other operands of a thread's next rows are asked for while the rows before are finished.
  constexpr int ROWS = ceil_div(PB * 16, ROWS_AT_ONCE), BATCH = ROWS < 4 ? ROWS : 4, ROUND = ceil_div(ROWS, BATCH) * BATCH;
  // (a thread's rows of a pass; how many are on their way)
  EpilogueOperands coming[BATCH];
  auto ask = [&](int pass, int row, EpilogueOperands& o) {
    const int rl = row_in + row * ROWS_AT_ONCE, m = m0 + (wm * TM + pass * PB) * 16 + rl;
    if (col_ok && rl < PB * 16 && m < p.M) request_operands(p.epi, (size_t)m * p.N + col, p.out_bf16, o);
  };
#pragma unroll
  for (int k = 0; k < BATCH; ++k) ask(0, k, coming[k]);
#pragma unroll
  for (int pass = 0; pass < TM / PB; ++pass) {
#pragma unroll
    for (int k = 0; k < PB; ++k) {
      const int b = pass * PB + k;
#pragma unroll
      for (int a = 0; a < TN; ++a) {
        *reinterpret_cast<f32x4*>(stage_lds + (k * 16 + fr) * CW * 4 + (((4 * a + fc) ^ (fr & MASK)) << 4)) = scaled_sums(acc[a][b], sc[b], by[a]);
      }
    }
    const int base = m0 + (wm * TM + pass * PB) * 16;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma nounroll
    for (int first = 0; first < ROWS; first += BATCH) {
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const EpilogueOperands now = coming[k];
        const int next = first + k + BATCH;
        if (next < ROWS) ask(pass, next, coming[k]);
        else if (next >= ROUND && pass + 1 < TM / PB) ask(pass + 1, next - ROUND, coming[k]);
        const int rl = row_in + (first + k) * ROWS_AT_ONCE;
        if (!col_ok || rl >= PB * 16 || base + rl >= p.M) continue;
        const char* src = stage_lds + rl * CW * 4;
        const f32x4 s0 = *reinterpret_cast<const f32x4*>(src + (((2 * ch) ^ (rl & MASK)) << 4)) + bias[0];
        const f32x4 s1 = *reinterpret_cast<const f32x4*>(src + (((2 * ch + 1) ^ (rl & MASK)) << 4)) + bias[1];
        const size_t at = (size_t)(base + rl) * p.N + col;
        float v[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
        apply_epilogue8(p.epi, now, v, at, p.out_bf16);
        if (p.out_bf16) {
          *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at) =
              uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        } else {
          f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at);
          o[0] = f32x4{v[0], v[1], v[2], v[3]};
          o[1] = f32x4{v[4], v[5], v[6], v[7]};
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the pass has been read out
  }
}

// Tile t of tiles_m x tiles_n: rows of tiles are walked in bands of four across the columns.
__device__ __forceinline__ int2 tile_place(int t, int tiles_m, int tiles_n) {
  constexpr int BAND = 4;
  const int band = t / (BAND * tiles_n), in_band = t - band * BAND * tiles_n, rows = min(BAND, tiles_m - band * BAND);
  return int2{band * BAND + in_band % rows, in_band / rows};
}
template <bool BWD, int BM, int BN, int WM, int WN, int STAGES, bool ONCE>
__global__ __launch_bounds__(WM* WN * 64) void gemm_i8_kernel(const Int8GemmArgs p) {
  extern __shared__ __align__(1024) int8_t lds[];
  const int tiles_m = ceil_div(p.M, BM), tiles_n = ceil_div(p.N, BN);
  const int2 at = tile_place(xcd_run(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n);
  gemm_i8_tile<BWD, BM, BN, WM, WN, STAGES, ONCE>(p, lds, at.x * BM, at.y * BN);
}
// 256 x 256 tiles of the first columns and 256 x NARROW ones of the rest: see int8_mixed.  Half of the narrow ones come first: the
// compute units that get them are then out of step with the others, and do not all come to the ends of their tiles, where only memory
// works, at the same time (4096 x 11008 x 4096 with silu, product and z: 219 us, and 227 with all tiles alike; without 180 and 183 to 210).
template <bool BWD, int NARROW>
__global__ __launch_bounds__(512) void gemm_i8_mixed_kernel(const Int8GemmArgs p, int wide_n) {
  extern __shared__ __align__(1024) int8_t lds[];
  const int tiles_m = ceil_div(p.M, 256), narrow_n = ceil_div(p.N - wide_n * 256, NARROW);
  const int wide = tiles_m * wide_n, narrow = tiles_m * narrow_n, first = int8_narrow_first(narrow), b = blockIdx.x;
  if (b >= first && b < first + wide) {
    const int2 at = tile_place(xcd_run(b - first, wide), tiles_m, wide_n);
    gemm_i8_tile<BWD, 256, 256, 2, 4, 2, false>(p, lds, at.x * 256, at.y * 256);
  } else {
    const int t = b < first ? xcd_run(b, first) : first + xcd_run(b - first - wide, narrow - first);
    const int2 at = tile_place(t, tiles_m, narrow_n);
    gemm_i8_tile<BWD, 256, NARROW, 4, 2, 2, false>(p, lds, at.x * 256, wide_n * 256 + at.y * NARROW);
  }
}

// The sum over the slices of K, and what follows it: four columns of a token to a thread.
__global__ __launch_bounds__(256) void gemm_i8_sum_kernel(const Int8GemmArgs p, int slices) {
  const size_t n = (size_t)p.M * p.N, stride = (size_t)gridDim.x * 1024;
  for (size_t at = (blockIdx.x * 256ull + threadIdx.x) * 4; at < n; at += stride) {
    i32x4 acc = *reinterpret_cast<const i32x4*>(p.partial + at);
    int s = 1;
    for (; s + 3 < slices; s += 4) {
      i32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const i32x4*>(p.partial + (s + k) * n + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) acc += v[k];
    }
    for (; s < slices; ++s) acc += *reinterpret_cast<const i32x4*>(p.partial + s * n + at);
    const int m = (int)(at / p.N), col = (int)(at % p.N);
    const float sc = p.row_scale[m];
    f32x4 by = {1.0f, 1.0f, 1.0f, 1.0f};
    if (p.col_scale) by = *reinterpret_cast<const f32x4*>(p.col_scale + col);
    const f32x4 v = apply_epilogue(p.epi, scaled_sums(acc, sc, by), at, col, p.out_bf16);
    if (p.out_bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    else
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = v;
  }
}

template <bool BWD, int BM, int BN, int WM, int WN, int STAGES, bool ONCE = false>
static hipError_t launch_tile(const Int8GemmArgs& a, int slices, hipStream_t st) {
  auto kernel = gemm_i8_kernel<BWD, BM, BN, WM, WN, STAGES, ONCE>;
  constexpr int bytes = STAGES * (BM + BN) * I8_STEP;
  static std::atomic<uint64_t> granted{0};  // per instantiation
  if (hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, granted); e != hipSuccess) return e;
  kernel<<<dim3((unsigned)((size_t)ceil_div(a.M, BM) * ceil_div(a.N, BN)), slices), WM * WN * 64, bytes, st>>>(a);
  return hipGetLastError();
}

template <bool BWD, int NARROW>
static hipError_t launch_mixed(const Int8GemmArgs& a, int wide_n, hipStream_t st) {
  auto kernel = gemm_i8_mixed_kernel<BWD, NARROW>;
  constexpr int bytes = 2 * 512 * I8_STEP;
  static std::atomic<uint64_t> granted{0};  // per instantiation
  if (hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, granted); e != hipSuccess) return e;
  const int tiles_m = ceil_div(a.M, 256);
  kernel<<<(unsigned)(tiles_m * (wide_n + ceil_div(a.N - wide_n * 256, NARROW))), 512, bytes, st>>>(a, wide_n);
  return hipGetLastError();
}

// Forward, a weight that one row of tiles reads goes past the caches (16 x 22016 x 8192: 36.7 us, 40.8 through them; 61 x 13824 x 5120: 20
// and 21.2); backward, where a tile's rows of the weight are parts of lines, that gains nothing.
template <bool BWD>
static hipError_t launch_planned(const Int8GemmArgs& a, const Int8Plan& plan, hipStream_t st) {
  const int s = plan.slices;
  switch (plan.tile) {
    case I8_256x256:
      if (const Int8Mixed m = int8_mixed(a.M, a.N, s, BWD); m.narrow == 128) return launch_mixed<BWD, 128>(a, m.wide_n, st);
      else if constexpr (!BWD) {
        if (m.narrow == 192) return launch_mixed<false, 192>(a, m.wide_n, st);
      }
      return launch_tile<BWD, 256, 256, 2, 4, 2>(a, s, st);
    case I8_192x256: return launch_tile<BWD, 192, 256, 2, 4, 2>(a, s, st);
    case I8_128x256: return launch_tile<BWD, 128, 256, 2, 4, 3>(a, s, st);
    case I8_128x128: return launch_tile<BWD, 128, 128, 4, 2, 2>(a, s, st);
    case I8_64x128: return launch_tile<BWD, 64, 128, 2, 2, 3>(a, s, st);
    default: break;
  }
  if constexpr (BWD) {
    return plan.tile == I8_32x128 ? launch_tile<true, 32, 128, 1, 4, 3>(a, s, st) : launch_tile<true, 16, 128, 1, 2, 3>(a, s, st);
  } else {
    const bool once = a.M <= kInt8Tiles[plan.tile].rows;
    switch (plan.tile) {
      case I8_128x64: return launch_tile<false, 128, 64, 4, 2, 3>(a, s, st);
      case I8_64x64: return once ? launch_tile<false, 64, 64, 2, 2, 4, true>(a, s, st) : launch_tile<false, 64, 64, 2, 2, 4>(a, s, st);
      case I8_32x64: return once ? launch_tile<false, 32, 64, 1, 2, 4, true>(a, s, st) : launch_tile<false, 32, 64, 1, 2, 4>(a, s, st);
      default: return once ? launch_tile<false, 16, 64, 1, 2, 4, true>(a, s, st) : launch_tile<false, 16, 64, 1, 2, 4>(a, s, st);
    }
  }
}

hipError_t launch_gemm_i8(const Int8GemmArgs& args, hipStream_t st) {
  Int8GemmArgs a = args;
  const Int8Plan plan = int8_plan(a.M, a.N, a.K, a.back);
  if (plan.slices == 1) a.partial = nullptr;
  if (hipError_t e = a.back ? launch_planned<true>(a, plan, st) : launch_planned<false>(a, plan, st); e != hipSuccess || !a.partial) return e;
  const size_t blocks = ((size_t)a.M * a.N / 4 + 255) / 256;
  gemm_i8_sum_kernel<<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, st>>>(a, plan.slices);
  return hipGetLastError();
}

}  // namespace qalora
