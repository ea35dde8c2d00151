// Y = X*W^T and Y = X*W with W in microscaled 4-bit floating point and X in ordinary floating point.
#pragma once
#include "mx4_tile.hpp"

namespace dla {

struct MxApplyArgs {
  const void* x;
  Mx4View w;
  void* y;
  float* parts;
  int64_t ldx, ldy;
  int m, n, k;  // X m x k and Y m x n for op 0, X m x n and Y m x k for op 1; W n x k
  int splits, tiles_m, tiles_n;
  bool vec;     // rows of X are aligned to 16 bytes
};

// Eight elements of X as bf16 terms, those from `valid` on zero.
template <typename T, int TERMS>
__device__ __forceinline__ void mx_load_terms(const T* p, int valid, bool vec, bf16x8_t* t) {
  typedef T run_t __attribute__((ext_vector_type(8)));
  union {
    unsigned short u[8];
    bf16x8_t v;
  } o[TERMS];
  run_t r;
  if (vec && valid >= 8) {
    r = *reinterpret_cast<const run_t*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = i < valid ? p[i] : (T)0.0f;
  }
  if constexpr (TERMS == 1) {
    o[0].v = r;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned short s[TERMS];
      mx_terms<TERMS>((float)r[i], s);
#pragma unroll
      for (int j = 0; j < TERMS; ++j) o[j].u[i] = s[j];
    }
  }
#pragma unroll
  for (int j = 0; j < TERMS; ++j) t[j] = o[j].v;
}

constexpr int kMxApplyWaves = 8;

// Few rows: operands go from memory to the matrix instructions, the eight waves of a workgroup share the sum.  A lane holds 32
// neighbouring elements of a row of W, one block; instruction j of a step of 128 takes its elements 8j .. 8j + 7, and X's likewise.
template <typename T, int TERMS, typename TY>
__global__ void __launch_bounds__(kMxApplyWaves * 64) mx4_apply_direct_kernel(MxApplyArgs g) {
  constexpr int TM = 16, TN = 16;
  __shared__ float part[kMxApplyWaves][TM * TN];
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x % tiles;
  const int m0 = tile % g.tiles_m * TM, n0 = tile / g.tiles_m * TN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l15 = lane & 15, l4 = lane >> 4;
  const int steps = (g.k + kMxStep - 1) / kMxStep;
  const int share = split * kMxApplyWaves + wave, shares = g.splits * kMxApplyWaves;
  const int begin = (int)((int64_t)steps * share / shares), end = (int)((int64_t)steps * (share + 1) / shares);
  const T* const x = static_cast<const T*>(g.x) + (int64_t)min(m0 + l15, g.m - 1) * g.ldx + l4 * 32;
  const int64_t row = min(n0 + l15, g.n - 1);
  const uint8_t* const wq = g.w.q + row * g.w.ldq + l4 * 16;
  const uint8_t* const ws = g.w.s + row * g.w.lds + l4;
  float4_t acc = {0, 0, 0, 0};
  for (int s = begin; s < end; ++s) {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(wq + (int64_t)s * 64);
    const float sc = mx_scale(ws[(int64_t)s * 4]);
    const int left = g.k - s * kMxStep - l4 * 32;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x8_t t[TERMS];
      mx_load_terms<T, TERMS>(x + (int64_t)s * kMxStep + 8 * j, left - 8 * j, g.vec, t);
      const bf16x8_t b = mx_values(w[j], sc);
#pragma unroll
      for (int i = TERMS - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], b, acc, 0, 0, 0);
    }
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) part[wave][(l4 * 4 + v) * TN + l15] = acc[v];
  __syncthreads();
  for (int e = threadIdx.x; e < TM * TN; e += kMxApplyWaves * 64) {
    const int r = m0 + e / TN, c = n0 + e % TN;
    if (r >= g.m || c >= g.n) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kMxApplyWaves; ++w) sum += part[w][e];
    if (g.splits > 1)
      g.parts[((int64_t)split * g.m + r) * g.n + c] = sum;
    else
      static_cast<TY*>(g.y)[r * g.ldy + c] = (TY)sum;
  }
}

// X as TERMS planes of bf16 that add up to it, rows of `wide` (a multiple of 64) with zeros behind `cols`: what the tile kernel
// multiplies where X itself is not bf16 in whole, aligned rows.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) mx4_planes_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int per_row, bool vec, bf16x8_t* planes) {
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row, chunk = at % (unsigned int)per_row;
  if (row >= rows) return;
  bf16x8_t t[TERMS];
  const int64_t left = cols - chunk * 8;
  mx_load_terms<T, TERMS>(x + row * ldx + chunk * 8, left > 8 ? 8 : (int)left, vec, t);
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

// A tile of Y.  X's rows go to LDS as they are; W's elements become bf16 on their way there, once per workgroup, with the terms of
// the sum neighbours in a row in both operations: GRAD turns blocks of 4 rows by 8 columns over in registers.
template <int TM, int TN, int WM, int WN, int TERMS, bool GRAD, typename TY>
__global__ void __launch_bounds__(WM* WN * 64) mx4_apply_tile_kernel(MxApplyTileArgs g) {
  constexpr int NT = WM * WN * 64, FM = TM / WM / 32, FN = TN / WN / 32;
  constexpr int LX = TM * 8 / NT;                     // loads of 16 bytes per thread, step and plane
  static_assert(TN * 2 == NT, "one thread takes one block of 32 elements of W a step");
  constexpr int XS = TM * 8, WS = TN * 8;             // units of 16 bytes: a row is 64 terms
  __shared__ u32x4_t lds[2 * (TERMS * XS + WS)];
  static_assert(2 * (TERMS * XS + WS) >= WM * WN * 1024, "16 KB a wave for the result");
  const int tiles = g.tiles_m * g.tiles_n, split = (int)blockIdx.x / tiles;
  int ti, tj;
  tile_at(xcd_contiguous_id((int)blockIdx.x % tiles, tiles), g.tiles_m, g.tiles_n, &ti, &tj);
  const int m0 = ti * TM, n0 = tj * TN;
  const int first = (int)((int64_t)g.steps * split / g.splits), steps = (int)((int64_t)g.steps * (split + 1) / g.splits) - first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l31 = lane & 31, l5 = lane >> 5;
  const int wm0 = wave / WN * (TM / WM), wn0 = wave % WN * (TN / WN);

  // Chunk c of 16 bytes of row r lies at c ^ turn(r): 16 rows that are read at the same chunk take all banks, and so do the
  // columns 8 l + i that GRAD's lanes write.
  auto turn = [](int r) { return ((r >> 1) ^ (r >> 3)) & 7; };

  // X: a load instruction fills eight rows
  const __bf16* const xb = g.x + (int64_t)m0 * g.ldx + (int64_t)first * 64;
  unsigned int xoff[LX];
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int r = (wave * LX + i) * 8 + lane / 8;
    xoff[i] = (unsigned int)min(r, g.m - 1 - m0) * (unsigned int)(g.ldx * 2) + ((lane & 7) ^ turn(r)) * 16;
  }
  const unsigned int lds0 = lds_offset(lds);
  auto load_x = [&](int s, int stage) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < LX; ++i)
        load_to_lds(xb + t * g.plane + (int64_t)s * 64, xoff[i], lds0 + ((stage * TERMS + t) * XS + (wave * LX + i) * 64) * 16);
  };

  // W, not GRAD: thread 2 r + h takes block h of row r.  GRAD: a thread takes columns 8 wc .. 8 wc + 7 of four rows.
  constexpr int LPR = TN / 8;
  const int wc = tid % LPR, wr = tid / LPR * 4;
  const int64_t wrow = min(n0 + tid / 2, g.w.rows - 1);
  const int wcol = min(n0 + wc * 8, g.w_cols - 8);
  struct Raw {
    u32x4_t q;
    unsigned int s[GRAD ? 4 : 1];
  };
  auto load_w = [&](int s) {
    Raw f;
    if constexpr (GRAD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = (first + s) * 64 + wr + i;
        const bool there = r < g.w.rows;
        const int64_t at = there ? r : g.w.rows - 1;
        f.q[i] = *reinterpret_cast<const unsigned int*>(g.w.q + at * g.w.ldq + wcol / 2);
        f.s[i] = g.w.s[at * g.w.lds + wcol / 32];
        if (!there) f.q[i] = f.s[i] = 0;
      }
    } else {
      f.q = *reinterpret_cast<const u32x4_t*>(g.w.q + wrow * g.w.ldq + (int64_t)(first + s) * 32 + (tid & 1) * 16);
      f.s[0] = g.w.s[wrow * g.w.lds + (int64_t)(first + s) * 2 + (tid & 1)];
    }
    return f;
  };
  auto store_w = [&](const Raw& f, int stage) {
    u32x4_t* const to = lds + 2 * TERMS * XS + stage * WS;
    if constexpr (GRAD) {
      u32x4_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(u32x4_t, mx_values(f.q[i], mx_scale(f.s[i])));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = wc * 8 + i;
        const unsigned int sel = i & 1 ? 0x07060302u : 0x05040100u;
        const u32x2_t w = {__builtin_amdgcn_perm(v[1][i / 2], v[0][i / 2], sel), __builtin_amdgcn_perm(v[3][i / 2], v[2][i / 2], sel)};
        reinterpret_cast<u32x2_t*>(to + c * 8 + ((wr / 8) ^ turn(c)))[wr / 4 & 1] = w;
      }
    } else {
      const float sc = mx_scale(f.s[0]);
      const int r = tid / 2;
#pragma unroll
      for (int j = 0; j < 4; ++j) to[r * 8 + (((tid & 1) * 4 + j) ^ turn(r))] = __builtin_bit_cast(u32x4_t, mx_values(f.q[j], sc));
    }
  };

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  auto multiply = [&](int stage) {
    const u32x4_t* const xs = lds + stage * TERMS * XS;
    const u32x4_t* const ws = lds + 2 * TERMS * XS + stage * WS;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      bf16x8_t b[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int r = wn0 + j * 32 + l31;
        b[j] = __builtin_bit_cast(bf16x8_t, ws[r * 8 + ((k * 2 + l5) ^ turn(r))]);
      }
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const int r = wm0 + i * 32 + l31;
          const bf16x8_t a = __builtin_bit_cast(bf16x8_t, xs[t * XS + r * 8 + ((k * 2 + l5) ^ turn(r))]);
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a, acc[i][j], 0, 0, 0);
        }
    }
  };

  // X of the next step is on its way and W's becomes bf16 while this step is multiplied; W's of the one after is in registers
  load_x(0, 0);
  Raw raw = load_w(0);
  store_w(raw, 0);
  raw = load_w(min(1, steps - 1));
  for (int s = 0; s < steps; ++s) {
    wait_loads_and_barrier<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(raw.q[i]));  // (the compiler's own wait for these, before more is loaded)
#pragma unroll
    for (int i = 0; i < (GRAD ? 4 : 1); ++i) asm volatile("" : "+v"(raw.s[i]));
    const Raw now = raw;
    load_x(min(s + 1, steps - 1), (s + 1) & 1);
    raw = load_w(min(s + 2, steps - 1));
    store_w(now, (s + 1) & 1);
    multiply(s & 1);
  }
  wait_loads_and_barrier<0>();
  u32x4_t* const room = lds + wave * 1024;
  if (g.splits > 1)
    mx_store_tile<TM / WM, TN / WN, float>(room, acc, lane, g.parts + (int64_t)split * g.m * g.out, g.out, m0 + wm0, n0 + wn0, g.m, g.out, false);
  else
    mx_store_tile<TM / WM, TN / WN, TY>(room, acc, lane, static_cast<TY*>(g.y), g.ldy, m0 + wm0, n0 + wn0, g.m, g.out, false);
}

// The gradient: a column of W at a time, element by element.
template <typename T, int TERMS, typename TY>
__global__ void __launch_bounds__(64) mx4_apply_grad_direct_kernel(MxApplyArgs g) {
  const int tiles = g.tiles_m * g.tiles_n, split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x % tiles;
  const int m0 = tile % g.tiles_m * 16, c0 = tile / g.tiles_m * 16;
  const int steps = (g.n + 31) / 32;
  const int begin = (int)((int64_t)steps * split / g.splits), end = (int)((int64_t)steps * (split + 1) / g.splits);
  const int lane = threadIdx.x & 63, l15 = lane & 15, l4 = lane >> 4;
  const T* const x = static_cast<const T*>(g.x) + (int64_t)min(m0 + l15, g.m - 1) * g.ldx;
  const int col = min(c0 + l15, g.k - 1);
  float4_t acc = {0, 0, 0, 0};
  for (int s = begin * 32; s < end * 32; s += 32) {
    bf16x8_t t[TERMS];
    const int left = g.n - s - l4 * 8;
    mx_load_terms<T, TERMS>(x + s + l4 * 8, left, g.vec, t);
    union {
      bf16x8_t v;
      __bf16 e[8];
    } b;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      b.e[i] = (__bf16)0.0f;
      if (i < left) {
        const int64_t r = s + l4 * 8 + i;
        const unsigned int byte = g.w.q[r * g.w.ldq + col / 2];
        const bf16x2_t p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(byte >> (col & 1) * 4, mx_scale(g.w.s[r * g.w.lds + col / 32]), 0);
        b.e[i] = p[0];
      }
    }
#pragma unroll
    for (int i = TERMS - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], b.v, acc, 0, 0, 0);
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int r = m0 + l4 * 4 + v;
    if (r >= g.m || c0 + l15 >= g.k) continue;
    if (g.splits > 1)
      g.parts[((int64_t)split * g.m + r) * g.k + c0 + l15] = acc[v];
    else
      static_cast<TY*>(g.y)[r * g.ldy + c0 + l15] = (TY)acc[v];
  }
}

}  // namespace dla
