// Y = X*W^T and Y = X*W with W in microscaled 4-bit floating point and X in ordinary floating point.
#pragma once
#include <type_traits>
#include "mx4_tile.hpp"

namespace dla {

struct MxApplyArgs {
  const void* x;         // rows aligned to 16 bytes, whole steps of 128 terms; planes of bf16 terms, `plane` elements apart
  Mx4View w;
  void* y;
  float* parts;
  int64_t ldx, plane, ldy;
  int m, steps;          // Y m x w.rows, steps of 128 terms
  int splits, tiles_m, tiles_n;
  dla_dtype dt_y;
};

// Eight elements of X as bf16 terms.
template <typename T, int TERMS>
__device__ __forceinline__ void mx_terms_of(T __attribute__((ext_vector_type(8))) r, bf16x8_t* t) {
  if constexpr (TERMS == 1) {
    t[0] = r;
  } else {
    union {
      unsigned short u[8];
      bf16x8_t v;
    } o[TERMS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned short s[TERMS];
      mx_terms<TERMS>((float)r[i], s);
#pragma unroll
      for (int j = 0; j < TERMS; ++j) o[j].u[i] = s[j];
    }
#pragma unroll
    for (int j = 0; j < TERMS; ++j) t[j] = o[j].v;
  }
}

// Scales of 2^126 and 2^127 (no weight that mx4_quantize writes has them) take elements from 4 and from 2 on out of bf16's range: they go
// into the products as infinities, and all sums of their column become infinities or, where a term of X is zero, NaN.  So a wave
// with a finite sum in each column has met none.  Any other looks for such scales, and if it finds one computes its
// values again, each by itself from memory, in fp32 and with weights 2^-4 as large as they are.  (Looking for them in the main loop made
// gradients 2 to 5 % slower; 1024 rows by 4096 x 4096 with a scale of 2^127 in each tile take 9 ms, the gradient 33.)

// Whether no sum of some column is finite.  A lane's registers are N times 16 columns (of M blocks of 32 rows, ACROSS, 32 lanes), or rows of N columns
// (of M blocks of 16, every sixteenth lane).
template <bool ACROSS, typename V, int M, int N>
__device__ __forceinline__ bool mx_column_lost(const V (&acc)[M][N]) {
  constexpr int R = (int)(sizeof(V) / 4);
  float any = 0.0f;  // (a product with zero is zero or a NaN)
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int v = 0; v < R; ++v) any = __builtin_fmaf(acc[i][j][v], 0.0f, any);
  if (__builtin_expect(!__any(any != 0.0f), 1)) return false;
  bool lost = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    unsigned long long all = ~0ull;
#pragma unroll
    for (int v = 0; v < R; ++v) {
#pragma unroll
      for (int i = 0; i < M; ++i) all &= __ballot(acc[i][j][v] * 0.0f != 0.0f);
      if (ACROSS) {
        lost |= (unsigned int)all == ~0u || (unsigned int)(all >> 32) == ~0u;
        all = ~0ull;
      }
    }
    if (!ACROSS) lost |= (all & all >> 16 & all >> 32 & all >> 48 & 0xffffu) != 0;
  }
  return lost;
}

// Whether one of the scales of rows r0 .. r1 - 1 of W, blocks b0 .. b1 - 1, is such a one; b0 is a multiple of four, and so is the end
// of a row with its padding, whose scales are zero.
__device__ __forceinline__ bool mx_beyond_along(const Mx4View& w, int lane, int r0, int r1, int b0, int b1) {
  bool found = false;
  for (int b = b0 + lane * 4; b < b1; b += 256)
#pragma unroll 4
    for (int r = r0; r < min(r1, w.rows); ++r) {
      const unsigned int four = *reinterpret_cast<const unsigned int*>(w.s + (int64_t)r * w.lds + b);
      for (int i = 0; i < 32; i += 8) found |= (four >> i & 255u) - 253u < 2u;
    }
  return __any(found);
}

// The same of many rows and the one or two blocks of C columns from c0 (a multiple of C; past w_cols, W's columns with their padding, the last).
template <int C>
__device__ __forceinline__ bool mx_beyond_down(const Mx4View& w, int lane, int r0, int r1, int c0, int w_cols) {
  static_assert(C == 32 || C == 64, "one load a row");
  typedef typename std::conditional<C == 64, uint16_t, uint8_t>::type load_t;
  const uint8_t* s = w.s + min(c0, w_cols - C) / 32 + (int64_t)(r0 + lane) * w.lds;
  bool found = false;
#pragma unroll 4
  for (int r = r0 + lane; r < r1; r += 64, s += 64 * w.lds) {
    const unsigned int v = *reinterpret_cast<const load_t*>(s);
    found |= (v & 255u) - 253u < 2u;
    if (C == 64) found |= (v >> 8) - 253u < 2u;
  }
  return __any(found);
}

// Row x times row `row` of W, blocks b0 .. b1 - 1.
template <int TERMS>
__device__ __forceinline__ float mx_again_along(const __bf16* x, int64_t plane, const Mx4View& w, int row, int b0, int b1) {
  typedef __bf16 run_t __attribute__((ext_vector_type(8)));
  const unsigned int* const q = reinterpret_cast<const unsigned int*>(w.q + (int64_t)row * w.ldq);
  const uint8_t* const s = w.s + (int64_t)row * w.lds;
  float sum = 0.0f;
#pragma unroll 1
  for (int j = b0 * 4; j < b1 * 4; ++j) {
    const float f = mx_scale_value(s[j / 4]) * 0.0625f;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      const run_t r = *reinterpret_cast<const run_t*>(x + t * plane + (int64_t)j * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += (float)r[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(v[i], __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[j] >> (4 * i), 1.0f, 0)[0] * f, sum);
  }
  return sum * 16.0f;
}

// Row x times column `col` of W, rows r0 .. r1 - 1.
template <int TERMS>
__device__ __forceinline__ float mx_again_down(const __bf16* x, int64_t plane, const Mx4View& w, int col, int r0, int r1) {
  float sum = 0.0f;
#pragma unroll 1
  for (int r = r0; r < r1; ++r) {
    float v = 0.0f;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) v += (float)x[t * plane + r];
    const unsigned int e = w.q[(int64_t)r * w.ldq + col / 2] >> (col & 1) * 4;
    const float f = mx_scale_value(w.s[(int64_t)r * w.lds + col / 32]) * 0.0625f;
    sum = __builtin_fmaf(v, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, 1.0f, 0)[0] * f, sum);
  }
  return sum * 16.0f;
}

// Few rows of X: what bounds the call is reading W once.  The WV waves of a workgroup share the sum over k, each with a run of
// steps of 128 terms and LDS of its own, to which W is loaded DW steps ahead and X DX.  Through LDS, because the matrix instructions
// want neighbouring lanes in different rows, and such a load takes 64 cycles where one of whole rows takes 16 (16384 x 4096 weights,
// one row, bf16: 9.2 us, 3.9 TB/s; 16 us with loads to registers).  With 48 rows of fp16 by 8192 x 8192, 16 to 18 us, it is X too, which each of
// 256 workgroups reads, and the scaling of the products' sums.
//   bf16, fp32   a lane's block of W is made bf16 with its scale; X is one plane of bf16 or, for fp32, three that add up to it (made by a
//                launch in front: made here, by every workgroup, they cost more than the rest of the call); instruction b takes
//                eight elements of every lane's block;
//   fp16         lanes exchange dwords so that instruction b takes block b, whose elements are made fp16 without the scale (with it
//                they would leave the type's range); the sum is scaled on its way to the running one, in fp32.
// XI: loads of X a plane and step, of four rows each: one where there are at most four rows, whose place the others of the instruction read
// too (they reach rows of the result that are not stored).
template <typename T, int TERMS, int MB, int XI, int WV, int DW, int DX>
__global__ void __launch_bounds__(WV * 64) mx4_apply_direct_kernel(MxApplyArgs g) {
  constexpr int NB = 2, TM = MB * 16, TN = NB * 16, XR = XI * 4;
  constexpr bool F16 = std::is_same<T, _Float16>::value;
  static_assert(sizeof(T) == 2 && (XR == TM || XR == 4) && (!F16 || TERMS == 1), "rows of 256 bytes a step, all of them or four");
  constexpr int W_RING = DW * NB * 64, X_STAGE = TERMS * XR * 16, RING = W_RING + DX * X_STAGE + 2 * TN;  // units of 16 bytes
  static_assert(WV * RING * 16 <= 160 * 1024 && RING * 16 >= TM * TN * 4, "LDS");
  typedef T run_t __attribute__((ext_vector_type(8)));
  __shared__ u32x4_t lds[WV * RING];
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x % tiles;
  const int m0 = tile % g.tiles_m * TM, n0 = tile / g.tiles_m * TN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l15 = lane & 15, l4 = lane >> 4;
  const int share = split * WV + wave, shares = g.splits * WV;
  const int begin = (int)((int64_t)g.steps * share / shares), end = (int)((int64_t)g.steps * (share + 1) / shares);
  u32x4_t* const ring = lds + wave * RING;
  const unsigned int at_w = lds_offset(ring), at_x = at_w + W_RING * 16, at_s = at_x + DX * X_STAGE * 16;

  // W: a load fills 16 rows of 64 bytes, chunk c of row r at c ^ (r / 4) % 4; X: 4 rows of 256 bytes, chunk c of row r at c ^ r % 16
  // (a wave's read of 1 KB of either takes LDS 8 clocks; from neighbouring places 4)
  const uint8_t* const wq = g.w.q + (int64_t)n0 * g.w.ldq;
  const uint8_t* const ws = g.w.s + (int64_t)n0 * g.w.lds;
  const T* const x = static_cast<const T*>(g.x) + (int64_t)m0 * g.ldx;
  unsigned int woff[NB], xoff[XI];
#pragma unroll
  for (int j = 0; j < NB; ++j)
    woff[j] = (unsigned int)(min(j * 16 + lane / 4, g.w.rows - 1 - n0) * (int)g.w.ldq) + ((lane & 3) ^ (lane >> 4)) * 16;
#pragma unroll
  for (int i = 0; i < XI; ++i) {
    const int r = i * 4 + lane / 16;
    xoff[i] = (unsigned int)min(r, g.m - 1 - m0) * (unsigned int)(g.ldx * 2) + ((lane & 15) ^ (r & 15)) * 16;
  }
  const unsigned int soff = (unsigned int)(min(lane & 31, g.w.rows - 1 - n0) * (int)g.w.lds);
  // (loads past the end repeat its last step, so that their number in flight is always the same)
  auto load_w = [&](int s, int slot) {
    const int64_t from = (int64_t)min(s, end - 1) * 64;
#pragma unroll
    for (int j = 0; j < NB; ++j) load_to_lds(wq + from, woff[j], at_w + (slot * NB + j) * 1024);
  };
  auto load_x = [&](int s, int slot) {
    const T* const from = x + (int64_t)min(s, end - 1) * kMxStep;
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < XI; ++i) load_to_lds(from + t * g.plane, xoff[i], at_x + slot * X_STAGE * 16 + (t * XI + i) * 1024);
  };
  // the scales of four steps, 16 bytes a row, moved back to begin at most four steps before the row's end
  auto scales_from = [&](int chunk) { return min(begin + chunk * 4, g.steps - 4); };
  auto load_s = [&](int chunk) {
    if (lane < TN) load_to_lds(ws + (int64_t)scales_from(chunk) * 4, soff, at_s + (chunk & 1) * TN * 16);
  };

  float4_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = float4_t{0, 0, 0, 0};

  if (begin < end) {
    if (g.steps >= 4) {
      load_s(0);
    } else if (lane < TN) {
      u32x4_t w = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (begin + i < end) w[i] = *reinterpret_cast<const unsigned int*>(ws + soff + (begin + i) * 4);
      ring[W_RING + DX * X_STAGE + lane] = w;
    }
    // (a step's loads are X's DX steps ahead, then W's DW ahead: here those of the steps before `begin`)
#pragma unroll
    for (int i = 0; i < DW; ++i) {
      if (i >= DW - DX) load_x(begin + i - (DW - DX), i - (DW - DX));
      load_w(begin + i, i);
    }
    int slot = 0;
    for (int s = begin; s < end; ++s) {
      const int i = s - begin, chunk = i >> 2;
      wait_loads<(DX - 1) * TERMS * XI + (DW > DX ? DX : DX - 1) * NB>();  // this step's X and W have arrived
      const u32x4_t* const wr = ring + slot * NB * 64;
      const u32x4_t* const xr = ring + W_RING + i % DX * X_STAGE;
      const unsigned int* const sr = reinterpret_cast<const unsigned int*>(ring + W_RING + DX * X_STAGE + (chunk & 1) * TN) + (g.steps >= 4 ? s - scales_from(chunk) : i);
      unsigned int w[NB][4], sc[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const u32x4_t q = wr[j * 64 + l15 * 4 + (l4 ^ (l15 >> 2))];
#pragma unroll
        for (int b = 0; b < 4; ++b) w[j][b] = q[b];
        sc[j] = sr[(j * 16 + l15) * 4];
      }
      run_t xv[4][TERMS][MB];
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
          for (int k = 0; k < MB; ++k) {
            const int r = XR < 16 ? l15 & (XR - 1) : k * 16 + l15, c = F16 ? b * 4 + l4 : l4 * 4 + b;
            xv[b][t][k] = __builtin_bit_cast(run_t, xr[(t * XR + r) * 16 + (c ^ (r & 15))]);
          }
      wait_lds();  // (before what was read is overwritten)
      if ((i & 3) == 0 && s + 4 < end) load_s(chunk + 1);
      load_x(s + DX, i % DX);
      load_w(s + DW, slot);
      slot = slot + 1 == DW ? 0 : slot + 1;

      float own[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if constexpr (F16) {
          swap_halves(w[j][0], w[j][2]);
          swap_halves(w[j][1], w[j][3]);
          swap_rows(w[j][0], w[j][1]);
          swap_rows(w[j][2], w[j][3]);
        } else {
          own[j] = mx_scale(sc[j] >> (8 * l4));
        }
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if constexpr (F16) {
            const f16x8_t wv = mx_values_f16(w[j][b]);
            const float f = mx_scale_value(sc[j] >> (8 * b));
#pragma unroll
            for (int k = 0; k < MB; ++k) {
              const float4_t sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[b][0][k], wv, float4_t{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
              for (int v = 0; v < 4; ++v) acc[k][j][v] = __builtin_fmaf(sum[v], f, acc[k][j][v]);
            }
          } else {
            const bf16x8_t wv = mx_values(w[j][b], own[j]);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
              for (int k = 0; k < MB; ++k) acc[k][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[b][t][k], wv, acc[k][j], 0, 0, 0);
          }
        }
      }
    }
  }
  wait_loads_and_barrier<0>();  // (nothing may arrive in LDS after this)
  float* const part = reinterpret_cast<float*>(lds);
  bool again = false;
  if constexpr (!F16) again = mx_column_lost<false>(acc) && mx_beyond_along(g.w, lane, n0, n0 + TN, begin * 4, end * 4);
  if (again) {
    if constexpr (!F16) {
#pragma unroll 1
      for (int e = lane; e < TM * TN; e += 64)
        part[wave * TM * TN + e] = mx_again_along<TERMS>(static_cast<const T*>(g.x) + (int64_t)min(m0 + e / TN, g.m - 1) * g.ldx, g.plane, g.w,
                                                         min(n0 + e % TN, g.w.rows - 1), begin * 4, end * 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) part[wave * TM * TN + (i * 16 + l4 * 4 + v) * TN + j * 16 + l15] = acc[i][j][v];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < TM * TN; e += WV * 64) {
    const int r = m0 + e / TN, c = n0 + e % TN;
    if (r >= g.m || c >= g.w.rows) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WV; ++w) sum += part[w * TM * TN + e];
    if (g.splits > 1)
      g.parts[((int64_t)split * g.m + r) * g.w.rows + c] = sum;
    else
      store_value(g.y, (int64_t)r * g.ldy + c, sum, g.dt_y, false);
  }
}

// X in aligned rows of `per_row` runs of eight, zeros behind its columns: what the direct kernel reads where X's own are not so.
template <typename T>
__global__ void __launch_bounds__(256) mx4_copy_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int per_row, T* to) {
  typedef T run_t __attribute__((ext_vector_type(8)));
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row, chunk = at % (unsigned int)per_row;
  if (row >= rows) return;
  run_t r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = chunk * 8 + i < cols ? x[row * ldx + chunk * 8 + i] : (T)0.0f;
  *reinterpret_cast<run_t*>(to + (row * per_row + chunk) * 8) = r;
}

// X as TERMS planes of bf16 that add up to it, rows of `wide` (a multiple of 64) with zeros behind `cols`: what the tile kernel
// multiplies where X itself is not bf16 in whole, aligned rows.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) mx4_planes_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int per_row, bf16x8_t* planes) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row, chunk = at % (unsigned int)per_row;
  if (row >= rows) return;
  typedef T run_t __attribute__((ext_vector_type(8)));
  typedef T load_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));  // (one access of eight needs no more alignment than one element)
  const T* const p = x + row * ldx + chunk * 8;
  const int64_t left = cols - chunk * 8;
  run_t r;
  if (left >= 8) {
    r = *reinterpret_cast<const load_t*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = i < left ? p[i] : (T)0.0f;
  }
  bf16x8_t t[TERMS];
  mx_terms_of<T, TERMS>(r, t);
#pragma unroll
  for (int i = 0; i < TERMS; ++i) planes[(i * rows + row) * per_row + chunk] = t[i];
}

struct MxApplyTileArgs {
  const __bf16* x;  // TERMS planes, `plane` elements apart
  Mx4View w;
  void* y;
  float* parts;
  int64_t ldx, plane, ldy;
  int m, out, w_cols;   // rows and columns of Y; W's columns with their padding
  int steps, splits, tiles_m, tiles_n;  // steps of 64 terms
};

// A wave's part of the result, R x C from row r0 and column c0, its values those of value(row, col).
template <int R, int C, typename TY, typename F>
__device__ __forceinline__ void mx_store_again(const MxApplyTileArgs& g, int split, int lane, int r0, int c0, F value) {
#pragma unroll 1
  for (int e = lane; e < R * C; e += 64) {
    const int row = r0 + e / C, col = c0 + e % C;
    if (row >= g.m || col >= g.out) continue;
    const float v = value(row, col);
    if (g.splits > 1)
      g.parts[((int64_t)split * g.m + row) * g.out + col] = v;
    else
      store_value_as<TY>(g.y, (int64_t)row * g.ldy + col, v, false);
  }
}

// How many steps of a tile of Y = X*W^T the LDS holds: up to six where two workgroups of a unit can have them, else as many as one can.
constexpr int apply_depth(int tm, int tn, int terms) {
  const int stage = tm * 128 * terms + tn * 32, scales = tn * 32;
  const int shared = (80 * 1024 - scales) / stage, alone = (160 * 1024 - scales) / stage;
  return shared >= 3 ? (shared > 6 ? 6 : shared) : (alone > 4 ? 4 : alone);
}

// A tile of Y = X*W^T, bound by the bf16 matrix pipes and the power they draw: 4096 rows of bf16 by 8192 x 8192 in 401 to 430 us by the clocks, 1320 TFLOP/s (a
// library product of bf16 operands of 8192 x 8192 reaches 1410).  X's rows and W's go to LDS as they are, a ring of D steps of 64 terms; a wave makes its part of W bf16 as it
// takes it to its registers (every element in WM waves).  A lane holds one block of a row of W, instruction j takes its elements
// 8 j .. 8 j + 7, and X's likewise.
template <int TM, int TN, int WM, int WN, int TERMS, typename TY>
__global__ void __launch_bounds__(WM* WN * 64) mx4_apply_tile_kernel(MxApplyTileArgs g) {
  constexpr int NW = WM * WN, FM = TM / WM / 32, FN = TN / WN / 32, D = apply_depth(TM, TN, TERMS);
  constexpr int LX = TM / 8 / NW, LW = TN / 32 / NW;             // loads of X (a plane) and of W per wave and step
  static_assert(LX * NW * 8 == TM && LW * NW * 32 == TN && TN <= NW * 64 && D >= 2, "whole loads");
  constexpr int XS = TM * 8, WS = TN * 2, STAGE = TERMS * XS + WS;  // units of 16 bytes
  __shared__ u32x4_t lds[D * STAGE + 2 * TN];                     // the steps; the scales of twice eight steps, 16 bytes a row
  static_assert(D * STAGE + 2 * TN >= NW * kMxRoom<TM / WM, TN / WN>, "room for the result");
  const int tiles = g.tiles_m * g.tiles_n, split = (int)blockIdx.x / tiles;
  int ti, tj;
  tile_at(xcd_contiguous_id((int)blockIdx.x % tiles, tiles), g.tiles_m, g.tiles_n, &ti, &tj);
  const int m0 = ti * TM, n0 = tj * TN;
  const int pairs = (g.steps + 1) / 2;  // a share begins at a whole 128 terms
  const int first = 2 * (int)((int64_t)pairs * split / g.splits), steps = min(g.steps, 2 * (int)((int64_t)pairs * (split + 1) / g.splits)) - first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l31 = lane & 31, l5 = lane >> 5;
  const int wm0 = wave / WN * (TM / WM), wn0 = wave % WN * (TN / WN);

  // X: a load fills eight rows, chunk c of row r at c ^ r / 2 % 8 (a wave's read of 1 KB then takes LDS 4 clocks, as from neighbouring places).
  // W: 32 rows of two chunks (8 clocks a read, and 8 for the scales, bytes 16 apart; of each there is one for four of X's or more).
  const __bf16* const xb = g.x + (int64_t)m0 * g.ldx + (int64_t)first * 64;
  const uint8_t* const wb = g.w.q + (int64_t)n0 * g.w.ldq + (int64_t)first * 32;
  unsigned int xoff[LX], woff[LW];
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int r = (wave * LX + i) * 8 + lane / 8;
    xoff[i] = (unsigned int)min(r, g.m - 1 - m0) * (unsigned int)(g.ldx * 2) + ((lane & 7) ^ ((r >> 1) & 7)) * 16;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) woff[i] = (unsigned int)(min((wave * LW + i) * 32 + lane / 2, g.w.rows - 1 - n0) * (int)g.w.ldq) + (lane & 1) * 16;
  const unsigned int lds0 = lds_offset(lds);
  // (loads past the last step repeat it, so that their number in flight is always the same)
  auto load = [&](int s, int slot) {
    const int64_t at = min(s, steps - 1);
    const unsigned int to = lds0 + slot * STAGE * 16;
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < LX; ++i) load_to_lds(xb + t * g.plane + at * 64, xoff[i], to + (t * XS + (wave * LX + i) * 64) * 16);
#pragma unroll
    for (int i = 0; i < LW; ++i) load_to_lds(wb + at * 32, woff[i], to + (TERMS * XS + (wave * LW + i) * 64) * 16);
  };
  // the scales of eight steps, a thread a row, moved back to begin at most sixteen bytes before the row's end
  const bool scaler = wave * 64 < TN;
  const uint8_t* const sp = g.w.s + (int64_t)n0 * g.w.lds;
  const unsigned int soff = (unsigned int)(min(tid, g.w.rows - 1 - n0) * (int)g.w.lds);
  const int blocks = pairs * 4;         // of 32 terms in a row with its padding
  auto scales_from = [&](int chunk) { return min(first * 2 + chunk * 16, blocks - 16); };
  auto load_scales = [&](int chunk) {
    if (scaler) load_to_lds(sp + scales_from(chunk), soff, lds0 + (D * STAGE + (chunk & 1) * TN + wave * 64) * 16);
  };

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  struct Part {
    bf16x8_t x[TERMS][FM];
  };
  struct Weights {
    u32x4_t q[FN];
    float s[FN];
  };
  auto read_x = [&](int slot, int j) {
    Part f;
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int r = wm0 + i * 32 + l31;
        f.x[t][i] = __builtin_bit_cast(bf16x8_t, lds[slot * STAGE + t * XS + r * 8 + ((l5 * 4 + j) ^ ((r >> 1) & 7))]);
      }
    return f;
  };
  auto read_w = [&](int s, int slot) {
    Weights f;
    const uint8_t* const sc = reinterpret_cast<const uint8_t*>(lds + D * STAGE + ((s >> 3) & 1) * TN) + (blocks >= 16 ? (first + s) * 2 - scales_from(s >> 3) : s * 2) + l5;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int r = wn0 + j * 32 + l31;
      f.q[j] = lds[slot * STAGE + TERMS * XS + r * 2 + l5];
      f.s[j] = mx_scale(sc[r * 16]);
    }
    return f;
  };
  auto multiply = [&](const Part& f, const Weights& w, int j) {
    bf16x8_t b[FN];
#pragma unroll
    for (int n = 0; n < FN; ++n) b[n] = mx_values(w.q[n][j], w.s[n]);
#pragma unroll
    for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int n = 0; n < FN; ++n) acc[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[n], f.x[t][i], acc[i][n], 0, 0, 0);
    // (an empty use of the sums: what follows is not moved in front of the products)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int n = 0; n < FN; ++n) asm volatile("" : "+v"(acc[i][n]));
  };

  if (blocks >= 16) {
    load_scales(0);
  } else if (tid < TN) {
    u32x4_t w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i * 2 < steps) w[i] = *reinterpret_cast<const unsigned int*>(sp + soff + first * 2 + i * 4);
    lds[D * STAGE + tid] = w;
  }
  // D steps are on their way; the waves meet in the last quarter of a step, when the next one has arrived and nobody reads this one any more
  constexpr int L = TERMS * LX + LW;
#pragma unroll
  for (int i = 0; i < D; ++i) load(i, i);
  wait_loads_and_barrier<(D - 1) * L>();
  Weights w = read_w(0, 0);
  Part even = read_x(0, 0), odd;
  int slot = 0;
  for (int s = 0; s < steps; ++s) {
    odd = read_x(slot, 1);
    multiply(even, w, 0);
    even = read_x(slot, 2);
    multiply(odd, w, 1);
    odd = read_x(slot, 3);
    multiply(even, w, 2);
    wait_loads_and_barrier<(D - 2) * L>();
    if ((s & 7) == 0 && s + 8 < steps) load_scales(s / 8 + 1);  // its buffer was last read before step s - 1's barrier
    load(s + D, slot);
    slot = slot + 1 == D ? 0 : slot + 1;
    const Weights next = read_w(min(s + 1, steps - 1), slot);
    even = read_x(slot, 0);
    multiply(odd, w, 3);
    w = next;
  }
  wait_loads_and_barrier<0>();  // (nothing may arrive in LDS after this)
  if (mx_column_lost<true>(acc) && mx_beyond_along(g.w, lane, n0 + wn0, n0 + wn0 + TN / WN, first * 2, (first + steps) * 2)) {
    mx_store_again<TM / WM, TN / WN, TY>(g, split, lane, m0 + wm0, n0 + wn0, [&](int row, int col) {
      return mx_again_along<TERMS>(g.x + row * g.ldx, g.plane, g.w, col, first * 2, (first + steps) * 2);
    });
    return;
  }
  u32x4_t* const room = lds + wave * kMxRoom<TM / WM, TN / WN>;
  if (g.splits > 1)
    mx_store_tile<TM / WM, TN / WN, float>(room, acc, lane, g.parts + (int64_t)split * g.m * g.out, g.out, m0 + wm0, n0 + wn0, g.m, g.out, false);
  else
    mx_store_tile<TM / WM, TN / WN, TY>(room, acc, lane, static_cast<TY*>(g.y), g.ldy, m0 + wm0, n0 + wn0, g.m, g.out, false);
}

// How many steps of a tile of Y = X*W are in LDS or on their way there.
constexpr int grad_depth(int tm, int tn, int terms) {
  const int stage = tm * 128 * terms + tn * 32 + tn * 2, fixed = 2 * tn * 128;
  const int shared = (80 * 1024 - fixed) / stage, alone = (160 * 1024 - fixed) / stage;
  return shared >= 2 ? (shared > 4 ? 4 : shared) : (alone > 3 ? 3 : alone);
}

// A tile of Y = X*W: 2048 rows of bf16 by 8192 x 8192 in 225 to 240 us by the clocks, 1180 TFLOP/s; what a thread does to turn W over takes issue slots from the
// products.  X's rows and W's go to LDS as they are, a ring of D steps of 64 terms (rows of W).  The terms of the sum are the rows of W,
// so what a lane needs of it is a column: a step ahead, threads turn blocks of 4 rows by 8 columns over in registers, make them bf16
// and leave them in LDS with the terms as neighbours, once per workgroup.
template <int TM, int TN, int WM, int WN, int TERMS, typename TY>
__global__ void __launch_bounds__(WM* WN * 64) mx4_apply_grad_kernel(MxApplyTileArgs g) {
  constexpr int NW = WM * WN, NT = NW * 64, FM = TM / WM / 32, FN = TN / WN / 32, D = grad_depth(TM, TN, TERMS);
  constexpr int LX = TM / 8 / NW;                     // loads of X per plane, wave and step; of W's elements and scales one each
  static_assert(LX * NW * 8 == TM && TN * 2 == NT && D >= 2, "a thread takes 32 elements of W a step");
  constexpr int XS = TM * 8, RS = TN * 2, SS = TN / 8;   // units of 16 bytes: X's rows, W's, and the scales
  constexpr int STAGE = TERMS * XS + RS + SS, WS = TN * 8;
  __shared__ u32x4_t lds[D * STAGE + 2 * WS];
  static_assert(D * STAGE + 2 * WS >= NW * kMxRoom<TM / WM, TN / WN>, "room for the result");
  const int tiles = g.tiles_m * g.tiles_n, split = (int)blockIdx.x / tiles;
  int ti, tj;
  tile_at(xcd_contiguous_id((int)blockIdx.x % tiles, tiles), g.tiles_m, g.tiles_n, &ti, &tj);
  const int m0 = ti * TM, n0 = tj * TN;
  const int first = (int)((int64_t)g.steps * split / g.splits), steps = (int)((int64_t)g.steps * (split + 1) / g.splits) - first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l31 = lane & 31, l5 = lane >> 5;
  const int wm0 = wave / WN * (TM / WM), wn0 = wave % WN * (TN / WN);

  // Chunk c of 16 bytes of row r lies at c ^ turn(r), so that neither rows that are read at the same chunk nor the columns 8 l + i that
  // the lanes write lie in the same banks throughout.  It halves what LDS can do: a wave's read of 16 bytes a lane takes 8 clocks and its write
  // of 8 bytes too, from neighbouring places 4 each (what is taken at a time is not 16 neighbouring lanes).
  auto turn = [](int r) { return ((r >> 1) ^ (r >> 3)) & 7; };

  // X: a load fills eight rows
  const __bf16* const xb = g.x + (int64_t)m0 * g.ldx + (int64_t)first * 64;
  unsigned int xoff[LX];
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int r = (wave * LX + i) * 8 + lane / 8;
    xoff[i] = (unsigned int)min(r, g.m - 1 - m0) * (unsigned int)(g.ldx * 2) + ((lane & 7) ^ turn(r)) * 16;
  }
  // W: a wave's load fills 64 / RCH rows of RCH chunks.  Row 4 a + b of each 16 lies at 4 b + a, so that the threads of four rows each, which
  // read row 4 a + b together, do so from neighbouring rows.  Columns past the padding repeat the last.
  constexpr int RCH = TN / 32, RPL = 64 / RCH;
  const int wslot = wave * RPL + lane / RCH, wrow = (wslot & ~15) | (wslot & 3) * 4 | (wslot >> 2 & 3);
  const int wcol = min(n0 / 2 + lane % RCH * 16, g.w_cols / 2 - 16);
  // and its scales: TN / 32 bytes of each of 64 rows, 16 lanes of every wave
  constexpr int SPR = TN / 128;                       // dwords of a row
  const int srow = (wave * 16 + (lane & 15)) / SPR, scol = min(n0 / 32 + (lane & 15) % SPR * 4, g.w_cols / 32 - 4);
  const unsigned int lds0 = lds_offset(lds);
  // (loads past the last step or row repeat it: the number in flight is always the same; what lies behind W's rows is made zero below)
  auto load_x = [&](int s, int slot) {
    const int64_t at = (int64_t)min(s, steps - 1) * 64;
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < LX; ++i) load_to_lds(xb + t * g.plane + at, xoff[i], lds0 + (slot * STAGE + t * XS + (wave * LX + i) * 64) * 16);
  };
  auto load_w = [&](int s, int slot) {
    const int r0 = (first + min(s, steps - 1)) * 64, last = g.w.rows - 1 - r0;
    const unsigned int to = lds0 + (slot * STAGE + TERMS * XS) * 16;
    load_to_lds(g.w.q + (int64_t)r0 * g.w.ldq, (unsigned int)(min(wrow, last) * (int)g.w.ldq + wcol), to + wave * 1024);
    if (lane < 16) load4_to_lds(g.w.s + (int64_t)r0 * g.w.lds, (unsigned int)(min(srow, last) * (int)g.w.lds + scol), to + RS * 16 + wave * 64);
  };
  // W of a step, made bf16 and turned over: columns 8 wc .. 8 wc + 7 of rows wr .. wr + 3
  constexpr int LPR = TN / 8;
  const int wc = tid % LPR, wr = tid / LPR * 4;
  struct Block {
    u32x4_t v[4];
  };
  auto take = [&](int s, int slot) {
    const unsigned int* const q = reinterpret_cast<const unsigned int*>(lds + slot * STAGE + TERMS * XS);
    const uint8_t* const sc = reinterpret_cast<const uint8_t*>(lds + slot * STAGE + TERMS * XS + RS);
    const int left = g.w.rows - (first + s) * 64;
    Block f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wr + i, at = (r & ~15) | (r & 3) * 4 | (r >> 2 & 3);
      const unsigned int e = q[at * (TN / 8) + wc], x = sc[r * (TN / 32) + wc / 4];
      const u32x4_t v = __builtin_bit_cast(u32x4_t, mx_values(e, mx_scale(x)));
      f.v[i] = r < left ? v : u32x4_t{0, 0, 0, 0};
    }
    return f;
  };
  auto turn_over = [&](const Block& f, int s, int from, int to_column) {
    u32x4_t* const to = lds + D * STAGE + (s & 1) * WS;
#pragma unroll
    for (int i = from; i < to_column; ++i) {
      const int c = wc * 8 + i;
      const unsigned int sel = i & 1 ? 0x07060302u : 0x05040100u;
      const u32x2_t w = {__builtin_amdgcn_perm(f.v[1][i / 2], f.v[0][i / 2], sel), __builtin_amdgcn_perm(f.v[3][i / 2], f.v[2][i / 2], sel)};
      reinterpret_cast<u32x2_t*>(to + c * 8 + ((wr / 8) ^ turn(c)))[wr / 4 & 1] = w;
    }
  };

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  struct Part {
    bf16x8_t x[TERMS][FM], w[FN];
  };
  auto read = [&](int s, int slot, int k) {
    Part f;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int r = wn0 + j * 32 + l31;
      f.w[j] = __builtin_bit_cast(bf16x8_t, lds[D * STAGE + (s & 1) * WS + r * 8 + ((k * 2 + l5) ^ turn(r))]);
    }
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int r = wm0 + i * 32 + l31;
        f.x[t][i] = __builtin_bit_cast(bf16x8_t, lds[slot * STAGE + t * XS + r * 8 + ((k * 2 + l5) ^ turn(r))]);
      }
    return f;
  };
  auto multiply = [&](const Part& f) {
#pragma unroll
    for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.w[j], f.x[t][i], acc[i][j], 0, 0, 0);
    // what a thread does for the next step between the products
#pragma unroll
    for (int i = 0; i < TERMS * FM * FN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
      __builtin_amdgcn_sched_group_barrier(0x300, 2, 0);
    }
    // (an empty use of the sums: what follows is not moved in front of the products)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j]));
  };

  // Loads go in groups of X of one step and W of the next; D groups are on their way.  The waves meet in the last quarter of a step:
  // the next step's X and W, and the one's after in LDS, are there, and nobody reads this one's any more.
  constexpr int L = TERMS * LX + 2;
  load_w(0, 0);
#pragma unroll
  for (int i = 0; i < D - 1; ++i) {
    load_x(i, i);
    load_w(i + 1, i + 1);
  }
  wait_loads_and_barrier<(D - 1) * L>();
  turn_over(take(0, 0), 0, 0, 8);
  wait_loads_and_barrier<(D - 1) * L>();
  load_x(D - 1, D - 1);
  load_w(D, 0);
  wait_loads_and_barrier<(D - 1) * L>();
  Part even = read(0, 0, 0), odd;
  int slot = 0;
  for (int s = 0; s < steps; ++s) {
    const int after = slot + 1 == D ? 0 : slot + 1;
    odd = read(s, slot, 1);
    const Block next = take(s + 1, after);
    multiply(even);
    even = read(s, slot, 2);
    turn_over(next, s + 1, 0, 4);
    multiply(odd);
    odd = read(s, slot, 3);
    turn_over(next, s + 1, 4, 8);
    multiply(even);
    wait_loads_and_barrier<(D - 2) * L>();
    load_x(s + D, slot);
    load_w(s + 1 + D, after);
    slot = after;
    even = read(s + 1, slot, 0);
    multiply(odd);
  }
  wait_loads_and_barrier<0>();  // (nothing may arrive in LDS after this)
  const int last = min((first + steps) * 64, g.w.rows);
  if (mx_column_lost<true>(acc) && mx_beyond_down<TN / WN>(g.w, lane, first * 64, last, n0 + wn0, g.w_cols)) {
    mx_store_again<TM / WM, TN / WN, TY>(g, split, lane, m0 + wm0, n0 + wn0,
                                         [&](int row, int col) { return mx_again_down<TERMS>(g.x + row * g.ldx, g.plane, g.w, col, first * 64, last); });
    return;
  }
  u32x4_t* const room = lds + wave * kMxRoom<TM / WM, TN / WN>;
  if (g.splits > 1)
    mx_store_tile<TM / WM, TN / WN, float>(room, acc, lane, g.parts + (int64_t)split * g.m * g.out, g.out, m0 + wm0, n0 + wn0, g.m, g.out, false);
  else
    mx_store_tile<TM / WM, TN / WN, TY>(room, acc, lane, static_cast<TY*>(g.y), g.ldy, m0 + wm0, n0 + wn0, g.m, g.out, false);
}

}  // namespace dla
