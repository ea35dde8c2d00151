// C = A*B^T and C += A*B^T with both operands in microscaled 4-bit floating point.
#pragma once
#include "mx4_common.hpp"

namespace dla {

// What a launch computes: C (a.rows x b.rows), `steps` times 128 terms; with splits > 1 the sums of each share go to parts.
struct MxGemmArgs {
  Mx4View a, b;
  void* c;
  float* parts;
  int64_t ldc;
  int steps, splits, tiles_m, tiles_n;
  bool onto;
};

constexpr int kMxDirectWaves = 8;

// Few rows: the operands go from memory to the matrix instructions, and the eight waves of a workgroup share the sum.
template <int MB, int NB, typename T>
__global__ void __launch_bounds__(kMxDirectWaves * 64) mx4_gemm_direct_kernel(MxGemmArgs g) {
  constexpr int TM = MB * 16, TN = NB * 16;
  __shared__ float part[kMxDirectWaves][TM * TN];
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x % tiles;
  const int m0 = tile % g.tiles_m * TM, n0 = tile / g.tiles_m * TN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l15 = lane & 15, l4 = lane >> 4;
  const int share = split * kMxDirectWaves + wave, shares = g.splits * kMxDirectWaves;
  const int begin = (int)((int64_t)g.steps * share / shares), end = (int)((int64_t)g.steps * (share + 1) / shares);

  const uint8_t *aq[MB], *as[MB], *bq[NB], *bs[NB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int64_t r = min(m0 + i * 16 + l15, g.a.rows - 1);
    aq[i] = g.a.q + r * g.a.ldq + l4 * 16;
    as[i] = g.a.s + r * g.a.lds;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t r = min(n0 + j * 16 + l15, g.b.rows - 1);
    bq[j] = g.b.q + r * g.b.ldq + l4 * 16;
    bs[j] = g.b.s + r * g.b.lds;
  }
  float4_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
  for (int k = begin; k < end; ++k) {
    i32x4_t a[MB], b[NB];
    int sa[MB], sb[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      a[i] = *reinterpret_cast<const i32x4_t*>(aq[i] + (int64_t)k * 64);
      sa[i] = (int)(*reinterpret_cast<const unsigned int*>(as[i] + (int64_t)k * 4) >> (8 * l4));
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      b[j] = *reinterpret_cast<const i32x4_t*>(bq[j] + (int64_t)k * 64);
      sb[j] = (int)(*reinterpret_cast<const unsigned int*>(bs[j] + (int64_t)k * 4) >> (8 * l4));
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = mx_mma16(a[i], b[j], acc[i][j], sa[i], sb[j]);
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) part[wave][(i * 16 + l4 * 4 + v) * TN + j * 16 + l15] = acc[i][j][v];
  __syncthreads();
  for (int e = threadIdx.x; e < TM * TN; e += kMxDirectWaves * 64) {
    const int r = m0 + e / TN, c = n0 + e % TN;
    if (r >= g.a.rows || c >= g.b.rows) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kMxDirectWaves; ++w) sum += part[w][e];
    if (g.splits > 1) {
      g.parts[((int64_t)split * g.a.rows + r) * g.b.rows + c] = sum;
    } else {
      T* const out = static_cast<T*>(g.c) + r * g.ldc + c;
      *out = (T)(g.onto ? (float)*out + sum : sum);
    }
  }
}

}  // namespace dla
