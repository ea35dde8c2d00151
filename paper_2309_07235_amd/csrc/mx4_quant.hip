// Microscaled 4-bit floating point: conversion to it, along rows, along columns or both in one pass, and back; and the joining
// of split sums.  All are bound by memory traffic.
#include "mx4_host.hpp"

namespace dla {
namespace {

template <typename T>
struct Run8 {  // eight elements as accesses of 16 bytes
  typedef T type __attribute__((ext_vector_type(8)));
};

// Elements 0 .. valid - 1 of eight from p, the rest zero.  vec: p is aligned to 16 bytes.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int valid, bool vec, float* v) {
  if (vec && valid >= 8) {
    const typename Run8<T>::type r = *reinterpret_cast<const typename Run8<T>::type*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)r[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? (float)p[i] : 0.0f;
  }
}

__device__ __forceinline__ unsigned int magnitude8(const float* v) {
  unsigned int most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
  return most;
}

// The largest magnitude's bits give the scale: its exponent field less 2, the exponent of the largest element (6 = 1.5 * 2^2).
__device__ __forceinline__ unsigned int scale_of(unsigned int most) {
  const unsigned int e = most >> 23;
  return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}

// Eight elements in one dword.  The instruction rounds to nearest, ties to even, and saturates: compared with the table of
// borders over all elements' neighbourhoods at the lowest, highest and middle scales.
__device__ __forceinline__ unsigned int elements8(const float* v, unsigned int s) {
  const float f = __uint_as_float(s << 23);
  unsigned int w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], f, 3);
  return s == 255u ? 0u : w;
}

// The largest of four neighbouring lanes, in all four.
__device__ __forceinline__ unsigned int max_of_four(unsigned int x) {
  x = max(x, (unsigned int)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));
  return max(x, (unsigned int)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));
}

// Along the rows: a lane takes eight neighbours, four lanes a block.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int per_row, bool vec,
                                                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds) {
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row;
  const int64_t chunk = at % (unsigned int)per_row;
  if (row >= rows) return;
  float v[8];
  const int64_t left = cols - chunk * 8;
  load8(x + row * ldx + chunk * 8, left > 8 ? 8 : (int)left, vec, v);
  const unsigned int sc = scale_of(max_of_four(magnitude8(v)));
  *reinterpret_cast<unsigned int*>(q + row * ldq + chunk * 4) = elements8(v, sc);
  if ((threadIdx.x & 3) == 0) s[row * lds + (chunk >> 2)] = (uint8_t)sc;
}

// Across the rows, and along them too where q is given: a tile of 128 x 128 goes through LDS.  Its columns are rotated by 16
// per 32 rows, so that 16 columns of four row blocks, which is what a wave reads at a time, lie in 64 banks.
template <typename T>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int tiles_c, bool vec,
                                                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, uint8_t* qt, int64_t ldqt,
                                                            uint8_t* st, int64_t ldst) {
  __shared__ float tile[128 * 128];
  const int64_t r0 = (int64_t)(blockIdx.x / (unsigned int)tiles_c) * 128, c0 = (int64_t)(blockIdx.x % (unsigned int)tiles_c) * 128;
  const int tid = threadIdx.x, c = (tid & 15) * 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = (tid >> 4) + 16 * i;
    float v[8];
    const int64_t left = r0 + r < rows ? cols - c0 - c : 0;
    load8(x + (r0 + r) * ldx + c0 + c, left > 8 ? 8 : (int)left, vec, v);
    const int at = r * 128 + ((c + 16 * (r >> 5)) & 127);
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[at + j] = v[j];
    if (q) {
      const unsigned int sc = scale_of(max_of_four(magnitude8(v)));
      if (r0 + r < rows) {
        *reinterpret_cast<unsigned int*>(q + (r0 + r) * ldq + (c0 + c) / 2) = elements8(v, sc);
        if ((tid & 3) == 0) s[(r0 + r) * lds + (c0 + c) / 32] = (uint8_t)sc;
      }
    }
  }
  __syncthreads();
  const int lane = tid & 63, block = lane >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (tid >> 6) * 32 + i * 16 + (lane & 15);
    float v[32];
    const float* p = tile + block * 32 * 128 + ((col + 16 * block) & 127);
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] = p[r * 128];
    const unsigned int sc = scale_of(max(max(magnitude8(v), magnitude8(v + 8)), max(magnitude8(v + 16), magnitude8(v + 24))));
    if (c0 + col < cols) {
      u32x4_t w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = elements8(v + 8 * j, sc);
      *reinterpret_cast<u32x4_t*>(qt + (c0 + col) * ldqt + r0 / 2 + block * 16) = w;
      st[(c0 + col) * ldst + r0 / 32 + block] = (uint8_t)sc;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(Mx4View w, int64_t cols, int per_row, bool vec, T* y, int64_t ldy) {
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row;
  const int64_t chunk = at % (unsigned int)per_row;
  if (row >= w.rows) return;
  const unsigned int e = *reinterpret_cast<const unsigned int*>(w.q + row * w.ldq + chunk * 4);
  const float sc = mx_scale(w.s[row * w.lds + (chunk >> 2)]);
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2_t p = i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 0)
                       : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 1)
                       : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 2)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 3);
    v[2 * i] = p[0];
    v[2 * i + 1] = p[1];
  }
  T* const out = y + row * ldy + chunk * 8;
  const int64_t left = cols - chunk * 8;
  if (vec && left >= 8) {
    typename Run8<T>::type r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)v[i];
    *reinterpret_cast<typename Run8<T>::type*>(out) = r;
  } else {
    for (int i = 0; i < 8; ++i)
      if (i < left) out[i] = (T)v[i];
  }
}

// C = or += the sum of the parts, PER neighbours a thread (4 where the columns are a multiple of 4).
template <typename T, int PER>
__global__ void __launch_bounds__(256) join_kernel(const float* parts, int splits, int64_t total, int64_t n, T* c, int64_t ldc, bool onto) {
  typedef float run_t __attribute__((ext_vector_type(PER)));
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * PER;
  if (i >= total) return;
  run_t sum = *reinterpret_cast<const run_t*>(parts + i);
#pragma unroll 4
  for (int p = 1; p < splits; ++p) sum += *reinterpret_cast<const run_t*>(parts + p * total + i);
  T* const out = c + (i / n) * ldc + i % n;
#pragma unroll
  for (int v = 0; v < PER; ++v) out[v] = (T)(onto ? (float)out[v] + sum[v] : sum[v]);
}

template <typename T>
__global__ void __launch_bounds__(256) zero_kernel(T* c, int64_t ldc, int64_t total, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < total) c[(i / n) * ldc + i % n] = (T)0.0f;
}

bool aligned16(const void* p, int64_t ld, int size) { return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0; }

// Workgroups for `items`, or 0 where they are more than a launch can have.
unsigned int grid_for(int64_t items, int64_t per_group) {
  const int64_t groups = (items + per_group - 1) / per_group;
  return groups > 0x7fffffff ? 0u : (unsigned int)groups;
}

template <typename T>
int quantize_typed(const T* x, int64_t ldx, int64_t rows, int64_t cols, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, uint8_t* qt,
                   int64_t ldqt, uint8_t* st, int64_t ldst, hipStream_t stream) {
  const bool vec = aligned16(x, ldx, sizeof(T));
  if (qt) {
    const int64_t tiles_c = (cols + 127) / 128, tiles = tiles_c * ((rows + 127) / 128);
    const unsigned int grid = grid_for(tiles, 1);
    if (!grid) return DLA_ERR_TOO_LARGE;
    hipLaunchKernelGGL(quantize_tile_kernel<T>, dim3(grid), dim3(256), 0, stream, x, ldx, rows, cols, (int)tiles_c, vec, q, ldq, s, lds, qt,
                       ldqt, st, ldst);
  } else {
    const int64_t per_row = (cols + kMxStep - 1) / kMxStep * (kMxStep / 8);
    const unsigned int grid = grid_for(rows * per_row, 256);
    if (!grid) return DLA_ERR_TOO_LARGE;
    hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3(grid), dim3(256), 0, stream, x, ldx, rows, cols, (int)per_row, vec, q, ldq, s, lds);
  }
  return launch_status(__func__);
}

template <typename T>
int dequantize_typed(const Mx4View& w, int64_t cols, T* y, int64_t ldy, hipStream_t stream) {
  const int64_t per_row = (cols + 7) / 8;
  const unsigned int grid = grid_for(w.rows * per_row, 256);
  if (!grid) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(dequantize_kernel<T>, dim3(grid), dim3(256), 0, stream, w, cols, (int)per_row, aligned16(y, ldy, sizeof(T)), y, ldy);
  return launch_status(__func__);
}

template <typename T>
int join_typed(const float* parts, int splits, int64_t m, int64_t n, T* c, int64_t ldc, bool onto, hipStream_t stream) {
  const int per = n % 4 == 0 ? 4 : 1;
  const unsigned int grid = grid_for(m * n, 256 * per);
  if (!grid) return DLA_ERR_TOO_LARGE;
  if (per == 4)
    hipLaunchKernelGGL((join_kernel<T, 4>), dim3(grid), dim3(256), 0, stream, parts, splits, m * n, n, c, ldc, onto);
  else
    hipLaunchKernelGGL((join_kernel<T, 1>), dim3(grid), dim3(256), 0, stream, parts, splits, m * n, n, c, ldc, onto);
  return launch_status(__func__);
}

template <typename T>
int zero_typed(T* c, int64_t ldc, int64_t m, int64_t n, hipStream_t stream) {
  const unsigned int grid = grid_for(m * n, 256);
  if (!grid) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(zero_kernel<T>, dim3(grid), dim3(256), 0, stream, c, ldc, m * n, n);
  return launch_status(__func__);
}

}  // namespace

int mx4_quantize_launch(const void* x, int64_t ldx, int64_t rows, int64_t cols, dla_dtype dt, uint8_t* q, int64_t ldq, uint8_t* s,
                        int64_t lds, uint8_t* qt, int64_t ldqt, uint8_t* st, int64_t ldst, hipStream_t stream) {
  if (dt == DLA_F32) return quantize_typed((const float*)x, ldx, rows, cols, q, ldq, s, lds, qt, ldqt, st, ldst, stream);
  if (dt == DLA_BF16) return quantize_typed((const __bf16*)x, ldx, rows, cols, q, ldq, s, lds, qt, ldqt, st, ldst, stream);
  return quantize_typed((const _Float16*)x, ldx, rows, cols, q, ldq, s, lds, qt, ldqt, st, ldst, stream);
}

int mx4_dequantize_launch(const Mx4View& w, int64_t cols, dla_dtype dt, void* y, int64_t ldy, hipStream_t stream) {
  if (dt == DLA_F32) return dequantize_typed(w, cols, (float*)y, ldy, stream);
  if (dt == DLA_BF16) return dequantize_typed(w, cols, (__bf16*)y, ldy, stream);
  return dequantize_typed(w, cols, (_Float16*)y, ldy, stream);
}

int mx4_join_launch(const float* parts, int splits, int64_t m, int64_t n, void* c, int64_t ldc, dla_dtype dt, bool onto, hipStream_t stream) {
  if (dt == DLA_F32) return join_typed(parts, splits, m, n, (float*)c, ldc, onto, stream);
  if (dt == DLA_BF16) return join_typed(parts, splits, m, n, (__bf16*)c, ldc, onto, stream);
  return join_typed(parts, splits, m, n, (_Float16*)c, ldc, onto, stream);
}

int mx4_fill_zero_launch(void* c, int64_t ldc, int64_t m, int64_t n, dla_dtype dt, hipStream_t stream) {
  if (dt == DLA_F32) return zero_typed((float*)c, ldc, m, n, stream);
  return zero_typed((_Float16*)c, ldc, m, n, stream);  // zero has the same bits in both 16-bit types
}

}  // namespace dla
