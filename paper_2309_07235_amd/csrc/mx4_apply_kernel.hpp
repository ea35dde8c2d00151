// Y = X*W^T and Y = X*W with W in microscaled 4-bit floating point and X in ordinary floating point.
#pragma once
#include "mx4_common.hpp"

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
