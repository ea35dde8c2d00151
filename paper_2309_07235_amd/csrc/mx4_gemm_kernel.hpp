// C = A*B^T and C += A*B^T with both operands in microscaled 4-bit floating point.
#pragma once
#include <type_traits>
#include "mx4_tile.hpp"

namespace dla {

// What a launch computes: C (a.rows x b.rows), `steps` times 128 terms; with splits > 1 the sums of each share go to parts.
struct MxGemmArgs {
  Mx4View a, b;
  void* c;
  float* parts;
  int64_t ldc;
  int steps, splits, tiles_m, tiles_n;
  dla_dtype dt;
  bool onto;
};

// Few rows: what bounds the call is reading B once (one row by 8192 x 8192: 8.8 us, 4.1 TB/s).  The WV waves of a workgroup share the sum over k, each with a run of steps and LDS
// of its own, to which both operands are loaded D steps ahead.  Through LDS, because the matrix instructions want neighbouring
// lanes in different rows, and such a load takes 64 cycles where one of whole rows takes 16.
template <int MB, int D, int WV>
__global__ void __launch_bounds__(WV * 64) mx4_gemm_direct_kernel(MxGemmArgs g) {
  constexpr int NB = 2, F = MB + NB, TM = MB * 16, TN = NB * 16;
  constexpr int RING = D * F * 64 + 2 * F * 16;  // units of 16 bytes: the steps, and the scales of twice four
  static_assert(WV * RING * 16 <= 160 * 1024 && RING * 16 >= TM * TN * 4, "LDS");
  __shared__ u32x4_t lds[WV * RING];
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x % tiles;
  const int m0 = tile % g.tiles_m * TM, n0 = tile / g.tiles_m * TN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l15 = lane & 15, l4 = lane >> 4;
  const int share = split * WV + wave, shares = g.splits * WV;
  const int begin = (int)((int64_t)g.steps * share / shares), end = (int)((int64_t)g.steps * (share + 1) / shares);
  u32x4_t* const ring = lds + wave * RING;
  const unsigned int at_q = lds_offset(ring), at_s = at_q + D * F * 1024;

  // A's blocks of 16 rows, then B's.  A load fills one block's rows of 64 bytes, chunk c of row r at c ^ (r / 4) % 4 (a wave's read of them
  // takes LDS 8 clocks; from neighbouring places 4).
  const uint8_t* const aq = g.a.q + (int64_t)m0 * g.a.ldq;
  const uint8_t* const bq = g.b.q + (int64_t)n0 * g.b.ldq;
  const uint8_t* const as = g.a.s + (int64_t)m0 * g.a.lds;
  const uint8_t* const bs = g.b.s + (int64_t)n0 * g.b.lds;
  unsigned int qoff[F];
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const int r = lane / 4;
    qoff[f] = (unsigned int)(f < MB ? min(f * 16 + r, g.a.rows - 1 - m0) * (int)g.a.ldq : min((f - MB) * 16 + r, g.b.rows - 1 - n0) * (int)g.b.ldq) +
              ((lane & 3) ^ (lane >> 4)) * 16;
  }
  // the scales: rows of A (MB * 16 lanes), rows of B (NB * 16)
  const unsigned int aoff = (unsigned int)(min(lane, g.a.rows - 1 - m0) * (int)g.a.lds), boff = (unsigned int)(min(lane & 31, g.b.rows - 1 - n0) * (int)g.b.lds);
  // (loads past the end repeat its last step, so that their number in flight is always the same)
  auto load = [&](int s, int slot) {
    const int64_t from = (int64_t)min(s, end - 1) * 64;
#pragma unroll
    for (int f = 0; f < F; ++f) load_to_lds((f < MB ? aq : bq) + from, qoff[f], at_q + (slot * F + f) * 1024);
  };
  // of four steps, 16 bytes a row, moved back to begin at most four steps before the row's end
  auto scales_from = [&](int chunk) { return min(begin + chunk * 4, g.steps - 4); };
  auto load_s = [&](int chunk) {
    const int64_t from = (int64_t)scales_from(chunk) * 4;
    const unsigned int to = at_s + (chunk & 1) * F * 256;
    if (lane < TM) load_to_lds(as + from, aoff, to);
    if (lane < TN) load_to_lds(bs + from, boff, to + MB * 256);
  };
  float4_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
  if (begin < end) {
    if (g.steps >= 4) {
      load_s(0);
    } else {
      u32x4_t a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (begin + i < end) {
          a[i] = *reinterpret_cast<const unsigned int*>(as + aoff + (begin + i) * 4);
          b[i] = *reinterpret_cast<const unsigned int*>(bs + boff + (begin + i) * 4);
        }
      if (lane < TM) ring[D * F * 64 + lane] = a;
      if (lane < TN) ring[D * F * 64 + TM + lane] = b;
    }
#pragma unroll
    for (int i = 0; i < D; ++i) load(begin + i, i);
    int slot = 0;
    for (int s = begin; s < end; ++s) {
      const int i = s - begin, chunk = i >> 2;
      wait_loads<(D - 1) * F>();
      const u32x4_t* const qr = ring + slot * F * 64;
      const unsigned int* const sr = reinterpret_cast<const unsigned int*>(ring + D * F * 64 + (chunk & 1) * F * 16) + (g.steps >= 4 ? s - scales_from(chunk) : i);
      i32x4_t q[F];
      int sc[F];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        q[f] = __builtin_bit_cast(i32x4_t, qr[f * 64 + l15 * 4 + (l4 ^ (l15 >> 2))]);
        sc[f] = (int)(sr[(f * 16 + l15) * 4] >> (8 * l4));
      }
      wait_lds();  // (before what was read is overwritten)
      if ((i & 3) == 0 && s + 4 < end) load_s(chunk + 1);
      load(s + D, slot);
      slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[a][b] = mx_mma16(q[a], q[MB + b], acc[a][b], sc[a], sc[MB + b]);
    }
  }
  wait_loads_and_barrier<0>();  // (nothing may arrive in LDS after this)
  float* const part = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) part[wave * TM * TN + (i * 16 + l4 * 4 + v) * TN + j * 16 + l15] = acc[i][j][v];
  __syncthreads();
  for (int e = threadIdx.x; e < TM * TN; e += WV * 64) {
    const int r = m0 + e / TN, c = n0 + e % TN;
    if (r >= g.a.rows || c >= g.b.rows) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WV; ++w) sum += part[w * TM * TN + e];
    if (g.splits > 1)
      g.parts[((int64_t)split * g.a.rows + r) * g.b.rows + c] = sum;
    else
      store_value(g.c, (int64_t)r * g.ldc + c, sum, g.dt, g.onto);
  }
}

// A tile.  An operation costs a quarter of bf16's here, an operand byte as much as ever: a tile of 256 x 256 takes 128 terms, 32 KB of
// operands, in 1024 clocks of the matrix pipes, which is 32 bytes a clock into LDS and 96 out of it for eight waves of 128 x 64.  Hence
// the largest tile the registers hold, operands that go to LDS without a register in between, four steps ahead, and LDS reads one half
// step ahead, each between two products.  8192 x 8192, k = 8192: 276 to 290 us by the clocks, 3.8 PFLOP/s (operands of zeros, for which the clocks stay up, 245 us).
// Tried and no better: more steps ahead, padded rows, loads to LDS between the products, four waves of 128 x 128, which read a third less
// from LDS (313 us).  The tile of 128 x 128 is for results of few tiles: 1600 x 1800, k = 2000, fp32, in 10.4 us, operands in the caches.
template <int TM, int TN, int WM, int WN, typename T>
__global__ void __launch_bounds__(WM* WN * 64) mx4_gemm_tile_kernel(MxGemmArgs g) {
  constexpr int NT = WM * WN * 64, FM = TM / WM / 32, FN = TN / WN / 32;
  constexpr int LA = TM * 4 / NT, LB = TN * 4 / NT;  // loads of 16 bytes per thread and step
  static_assert(TM + TN == NT, "one thread per row loads its scales");
  static_assert((TM + TN) * 16 >= WM * WN * kMxRoom<TM / WM, TN / WN>, "room for the result");
  constexpr int STAGE = (TM + TN) * 4;               // a step's rows of both operands, in units of 16 bytes
  __shared__ u32x4_t rows[4 * STAGE];
  __shared__ u32x4_t scales[2][TM + TN];             // those of four steps at a time, 16 bytes a row
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = (int)blockIdx.x / tiles;
  int ti, tj;
  tile_at(xcd_contiguous_id((int)blockIdx.x % tiles, tiles), g.tiles_m, g.tiles_n, &ti, &tj);
  const int m0 = ti * TM, n0 = tj * TN;
  const int first = (int)((int64_t)g.steps * split / g.splits), steps = (int)((int64_t)g.steps * (split + 1) / g.splits) - first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l31 = lane & 31, l5 = lane >> 5;
  const int wm0 = wave / WN * (TM / WM), wn0 = wave % WN * (TN / WN);

  // A load instruction fills 16 rows of 64 bytes; chunk c of row r lies at c ^ (r / 4) % 4, so that a wave's read of 32 rows takes LDS 4
  // clocks, as from neighbouring places.  (The scales' reads, 4 bytes 16 apart, take 8, and 2 from neighbouring places: in a tile of 256 x 256
  // six of them a step, which is as long as its twelve reads of operands.)  Rows past the last repeat it.
  const uint8_t* const aq = g.a.q + (int64_t)m0 * g.a.ldq + (int64_t)first * 64;
  const uint8_t* const bq = g.b.q + (int64_t)n0 * g.b.ldq + (int64_t)first * 64;
  unsigned int off[LA + LB];
#pragma unroll
  for (int i = 0; i < LA + LB; ++i) {
    const int r = i < LA ? (wave * LA + i) * 16 + lane / 4 : (wave * LB + i - LA) * 16 + lane / 4;
    const int c = (lane & 3) ^ ((r >> 2) & 3);
    off[i] = (unsigned int)(i < LA ? min(r, g.a.rows - 1 - m0) * (int)g.a.ldq : min(r, g.b.rows - 1 - n0) * (int)g.b.ldq) + c * 16;
  }
  const unsigned int lds_rows = lds_offset(rows), lds_scales = lds_offset(scales);
  // Loads past the last step repeat it, into a stage that nobody reads any more: the number of loads in flight is then the same
  // in every step, and a wait can count them.
  auto load = [&](int s, int stage) {
    const int64_t at = (int64_t)min(s, steps - 1) * 64;
    const unsigned int to = lds_rows + stage * STAGE * 16;
#pragma unroll
    for (int i = 0; i < LA; ++i) load_to_lds(aq + at, off[i], to + (wave * LA + i) * 1024);
#pragma unroll
    for (int i = 0; i < LB; ++i) load_to_lds(bq + at, off[LA + i], to + TM * 64 + (wave * LB + i) * 1024);
  };
  // The scales of steps 4 chunk .. 4 chunk + 3, a thread a row (a wave's rows are all A's or all B's); moved back to begin at most
  // four steps before the row's end.
  const bool of_a = wave * 64 < TM;
  const uint8_t* const sp = of_a ? g.a.s + (int64_t)m0 * g.a.lds : g.b.s + (int64_t)n0 * g.b.lds;
  const unsigned int soff = of_a ? (unsigned int)(min(tid, g.a.rows - 1 - m0) * (int)g.a.lds) : (unsigned int)(min(tid - TM, g.b.rows - 1 - n0) * (int)g.b.lds);
  auto scales_from = [&](int chunk) { return min(first + chunk * 4, g.steps - 4); };
  auto load_scales = [&](int chunk) {
    load_to_lds(sp + (int64_t)scales_from(chunk) * 4, soff, lds_scales + (chunk & 1) * (TM + TN) * 16 + wave * 1024);
  };

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  // Operands of half a step, and a step's scales.  The result is computed transposed (B's rows are the instruction's rows), so that
  // a lane holds neighbouring columns of C.
  struct Half {
    i32x4_t a[FM], b[FN];
  };
  struct Scales {
    int a[FM], b[FN];
  };
  auto read = [&](int stage, int h) {
    const u32x4_t* const st = rows + stage * STAGE;
    auto at = [&](int r) { return __builtin_bit_cast(i32x4_t, st[r * 4 + ((h * 2 + l5) ^ ((r >> 2) & 3))]); };
    Half f;
#pragma unroll
    for (int j = 0; j < FN; ++j) f.b[j] = at(TM + wn0 + j * 32 + l31);
#pragma unroll
    for (int i = 0; i < FM; ++i) f.a[i] = at(wm0 + i * 32 + l31);
    return f;
  };
  auto read_scales = [&](int s) {
    const unsigned int* const w = reinterpret_cast<const unsigned int*>(scales[(s >> 2) & 1]) + (g.steps >= 4 ? first + s - scales_from(s >> 2) : s);
    Scales f;
#pragma unroll
    for (int j = 0; j < FN; ++j) f.b[j] = (int)(w[(TM + wn0 + j * 32 + l31) * 4] >> (8 * l5));
#pragma unroll
    for (int i = 0; i < FM; ++i) f.a[i] = (int)(w[(wm0 + i * 32 + l31) * 4] >> (8 * l5));
    return f;
  };
  auto multiply = [&](const Half& f, const Scales& w, auto h) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mx_mma32<decltype(h)::value * 2>(f.b[j], f.a[i], acc[i][j], w.b[j], w.a[i]);
    // each read between two products: with the reads in front, all waves would wait for LDS and then all for the products
#pragma unroll
    for (int i = 0; i < FM * FN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    // (an empty use of the sums: what follows is not moved in front of the products)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j]));
  };

  if (g.steps >= 4) {
    load_scales(0);
  } else {
    u32x4_t w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < steps) w[i] = *reinterpret_cast<const unsigned int*>(sp + soff + (first + i) * 4);
    scales[0][tid] = w;
  }
  // Up to four steps are on their way.  The operands of the next half step are read from LDS while this one's are multiplied; in
  // the middle of a step the waves meet: the next step has arrived, and nobody reads this one any more.
  constexpr int L = LA + LB;
  load(0, 0);
  load(1, 1);
  load(2, 2);
  load(3, 3);
  wait_loads_and_barrier<3 * L>();
  Half x = read(0, 0);
  Scales w = read_scales(0);
  auto step = [&](int s, int stage) {
    const Half y = read(stage, 1);
    multiply(x, w, std::integral_constant<int, 0>());
    wait_loads_and_barrier<2 * L>();
    x = read((stage + 1) & 3, 0);
    const Scales next = read_scales(min(s + 1, steps - 1));
    multiply(y, w, std::integral_constant<int, 1>());
    if ((s & 3) == 0 && s + 4 < steps) load_scales(s / 4 + 1);  // its buffer was last read before step s - 1's barrier
    load(s + 4, stage);
    w = next;
  };
  for (int s = 0;; s += 4) {
    step(s, 0);
    if (s + 1 >= steps) break;
    step(s + 1, 1);
    if (s + 2 >= steps) break;
    step(s + 2, 2);
    if (s + 3 >= steps) break;
    step(s + 3, 3);
    if (s + 4 >= steps) break;
  }
  wait_loads_and_barrier<0>();  // (nothing may arrive in LDS after this)

  u32x4_t* const room = rows + wave * kMxRoom<TM / WM, TN / WN>;
  if (g.splits > 1)
    mx_store_tile<TM / WM, TN / WN, float>(room, acc, lane, g.parts + (int64_t)split * g.a.rows * g.b.rows, g.b.rows, m0 + wm0, n0 + wn0, g.a.rows, g.b.rows,
                                           false);
  else if (g.onto)
    mx_store_tile<TM / WM, TN / WN, float>(room, acc, lane, static_cast<T*>(g.c), g.ldc, m0 + wm0, n0 + wn0, g.a.rows, g.b.rows, true);
  else
    mx_store_tile<TM / WM, TN / WN, T>(room, acc, lane, static_cast<T*>(g.c), g.ldc, m0 + wm0, n0 + wn0, g.a.rows, g.b.rows, false);
}

}  // namespace dla
