// Microscaled 4-bit floating point: conversion to it, along rows, along columns or both in one pass, and back; and the joining
// of split sums.  All are bound by memory traffic; rates below are of all bytes read and written, X in no cache, beside 5.2 TB/s of a large copy.
#include "mx4_host.hpp"

namespace dla {
namespace {

// Elements 0 .. valid - 1 of eight from p, the rest zero.  (One access of eight needs no more alignment than one element.)
template <typename T>
__device__ __forceinline__ void load8(const T* p, int valid, float* v) {
  typedef T run_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  if (valid >= 8) {
    const run_t r = *reinterpret_cast<const run_t*>(p);
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

// Along the rows: a lane takes eight neighbours, four lanes a block, whose largest magnitude they exchange without LDS.
// 8192 x 8192: fp32 54 us (5.7 TB/s), bf16 36 us (4.8 TB/s); 1 x 4096: 2.1 us, a launch.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int per_row,
                                                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds) {
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row;
  const int64_t chunk = at % (unsigned int)per_row;
  if (row >= rows) return;
  float v[8];
  const int64_t left = cols - chunk * 8;
  load8(x + row * ldx + chunk * 8, left > 8 ? 8 : (int)left, v);
  const unsigned int sc = scale_of(max_of_four(magnitude8(v)));
  *reinterpret_cast<unsigned int*>(q + row * ldq + chunk * 4) = elements8(v, sc);
  if ((threadIdx.x & 3) == 0) s[row * lds + (chunk >> 2)] = (uint8_t)sc;
}

// Across the rows, and along them too where q is given, a tile of 128 x 128 a workgroup.  A wave takes 32 rows, which are one block of every column,
// a lane 8 x 8 of them: everything that belongs to one block is in 4 lanes, neighbours for a row's block, 16 apart for a
// column's.  What a lane has for a column is eight rows' elements, a dword; they and the scales of the four waves meet in LDS.
// Both forms of 8192 x 8192, X read once for the two and in no cache: fp32 67 us (5.1 TB/s), bf16 40 us (5.1 TB/s), call after call; 96 us (fp32) where
// 500 MB that other kernels have just written are on their way to memory.  The tile itself through LDS, a column's 32 rows then read by one lane,
// took 81 and 79 us where this took 73 and 46.
template <typename T>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const T* x, int64_t ldx, int64_t rows, int64_t cols, int tiles_c, uint8_t* q, int64_t ldq,
                                                            uint8_t* s, int64_t lds, uint8_t* qt, int64_t ldqt, uint8_t* st, int64_t ldst) {
  typedef T run_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  __shared__ u32x4_t turned[128 * 4];
  __shared__ unsigned int scales[128];
  // Workgroups go round the eight XCDs.  Two neighbours of a row of tiles share lines of q, two of a column lines of qt, and an L2 that
  // has both writes them whole.  Where a row has a multiple of 64 tiles or up to two more or fewer, eight neighbours go to one XCD, and so does
  // most often the tile below.  Time over that of the plain order, 4096 and 8192 rows: 62 to 66 tiles bf16 0.85 to 0.96, fp32 0.92 to 0.98, 127
  // to 129 tiles 0.84 to 0.99 (1000 rows of 62 tiles 1.02 to 1.05, of 63 to 66 0.93 to 1.01).  Other numbers stay as they come: multiples of eight,
  // whose columns are one XCD's already, 0.95 to 1.15 (the least of them 120 tiles of 8192 rows, 0.92), multiples of four 0.97 to 1.14; odd ones
  // from 9 to 47 gain up to 0.88 in one type and size and nothing in the next.
  const unsigned int part = blockIdx.x / 64u * 64u, in = blockIdx.x % 64u;
  const bool near = tiles_c >= 62 && (tiles_c + 2) % 64 <= 4;
  const unsigned int id = near && part + 64u <= gridDim.x ? part + in % 8u * 8u + in / 8u : blockIdx.x;
  const int64_t r0 = (int64_t)(id / (unsigned int)tiles_c) * 128, c0 = (int64_t)(id % (unsigned int)tiles_c) * 128;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> 4;
  const int64_t row = r0 + wave * 32 + group * 8, col = c0 + (lane & 15) * 8;
  float v[8][8];
  const T* const p = x + row * ldx + col;
  if (r0 + 128 <= rows && c0 + 128 <= cols) {
    run_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = *reinterpret_cast<const run_t*>(p + i * ldx);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (float)r[i][j];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t left = row + i < rows ? cols - col : 0;
      if (left >= 8) {
        const run_t r = *reinterpret_cast<const run_t*>(p + i * ldx);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = (float)r[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = j < left ? (float)p[i * ldx + j] : 0.0f;
      }
    }
  }
  if (q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned int sc = scale_of(max_of_four(magnitude8(v[i])));
      const unsigned int w = elements8(v[i], sc);
      if (row + i < rows) {
        *reinterpret_cast<unsigned int*>(q + (row + i) * ldq + col / 2) = w;
        if ((lane & 3) == 0) s[(row + i) * lds + col / 32] = (uint8_t)sc;
      }
    }
  }
  // the columns' largest magnitudes, two columns' halves put together at a time: in the end lane group g has columns of its own
  unsigned int most[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    most[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most[j] = max(most[j], __float_as_uint(v[i][j]) & 0x7fffffffu);
  }
  unsigned int sc[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned int* const m = most + 4 * h;
    swap_halves(m[0], m[2]);  // m[0]: columns 0 and 2 of the lower half's rows, m[2]: of the upper half's
    swap_halves(m[1], m[3]);
    unsigned int a = max(m[0], m[2]), b = max(m[1], m[3]);
    swap_rows(a, b);          // a: groups 0, 2 hold column 0 and 2 of their even groups' rows, 1 and 3 column 1 and 3
    const unsigned int own = scale_of(max(a, b));
    // and back to all lanes: columns 0 and 2, 1 and 3, then each
    unsigned int even = own, odd = own;
    swap_rows(even, odd);
    unsigned int c0l = even, c2l = even, c1l = odd, c3l = odd;
    swap_halves(c0l, c2l);
    swap_halves(c1l, c3l);
    sc[4 * h] = c0l;
    sc[4 * h + 1] = c1l;
    sc[4 * h + 2] = c2l;
    sc[4 * h + 3] = c3l;
    reinterpret_cast<uint8_t*>(scales)[((lane & 15) * 8 + 4 * h + (group >> 1) * 2 + (group & 1)) * 4 + wave] = (uint8_t)own;
  }
  // A column's 64 bytes are put together in LDS: column 8 l + j at slot 16 j + l, wave w's 16 bytes of it at chunk w ^ l / 4.  A wave's read
  // takes LDS 4 clocks, as from neighbouring places, its write of a dword 4 where it is 2 there.
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = v[i][j];
    reinterpret_cast<unsigned int*>(turned + (j * 16 + (lane & 15)) * 4 + (wave ^ (lane >> 2 & 3)))[group] = elements8(c, sc[j]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int slot = (threadIdx.x >> 2) + 64 * i, w = threadIdx.x & 3, l = slot & 15, c = l * 8 + (slot >> 4);
    if (c0 + c < cols) *reinterpret_cast<u32x4_t*>(qt + (c0 + c) * ldqt + r0 / 2 + w * 16) = turned[slot * 4 + (w ^ (l >> 2))];
  }
  if (threadIdx.x < 128 && c0 + threadIdx.x < cols) *reinterpret_cast<unsigned int*>(st + (c0 + threadIdx.x) * ldst + r0 / 32) = scales[threadIdx.x];
}

// A lane takes eight neighbours; there are `per_row` such runs a row.  8192 x 8192 to fp32 63 us (4.9 TB/s), to bf16 37 us (4.6 TB/s); in
// fp32 four neighbours a lane, so that a wave writes whole lines at a time, were slower (70).
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(Mx4View w, int64_t cols, int per_row, T* y, int64_t ldy) {
  typedef T run_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / per_row;
  const unsigned int at = (unsigned int)(first - row0 * per_row) + threadIdx.x;
  const int64_t row = row0 + at / (unsigned int)per_row;
  const int64_t run = at % (unsigned int)per_row;
  if (row >= w.rows) return;
  const unsigned int e = *reinterpret_cast<const unsigned int*>(w.q + row * w.ldq + run * 4);
  const float sc = mx_scale(w.s[row * w.lds + (run >> 2)]);
  float2_t v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e, sc, 3);
  T* const out = y + row * ldy + run * 8;
  const int64_t left = cols - run * 8;
  if (left >= 8) {
    run_t r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)v[i / 2][i % 2];
    *reinterpret_cast<run_t*>(out) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) out[i] = (T)v[i / 2][i % 2];
  }
}

// C = or += the sum of the parts in their order, which no timing changes, four neighbours a thread, which may lie in two rows.  (There are fewer
// than 2^32 values.)  Parts come from the caches: 333 x 1801, three of them, 4 us.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const float* parts, int splits, unsigned int total, unsigned int n, T* c, int64_t ldc, bool onto) {
  typedef float run_t __attribute__((ext_vector_type(4), aligned(4)));
  const unsigned int i = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= total) return;
  run_t sum;
  if (total - i >= 4) {
    sum = *reinterpret_cast<const run_t*>(parts + i);
#pragma unroll 4
    for (int p = 1; p < splits; ++p) sum += *reinterpret_cast<const run_t*>(parts + (int64_t)p * total + i);
  } else {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sum[v] = 0.0f;
      for (int p = 0; v < (int)(total - i) && p < splits; ++p) sum[v] += parts[(int64_t)p * total + i + v];
    }
  }
  unsigned int row = i / n, col = i - row * n;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    if (i + v < total) {
      T* const out = c + (int64_t)row * ldc + col;
      *out = (T)(onto ? (float)*out + sum[v] : sum[v]);
    }
    if (++col == n) {
      col = 0;
      ++row;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) zero_kernel(T* c, int64_t ldc, int64_t total, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < total) c[(i / n) * ldc + i % n] = (T)0.0f;
}

template <typename T>
int quantize_typed(const T* x, int64_t ldx, int64_t rows, int64_t cols, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, uint8_t* qt,
                   int64_t ldqt, uint8_t* st, int64_t ldst, hipStream_t stream) {
  if (qt) {
    const int64_t tiles_c = (cols + 127) / 128, tiles = tiles_c * ((rows + 127) / 128);
    const unsigned int grid = mx4_grid_for(tiles, 1);
    if (!grid) return DLA_ERR_TOO_LARGE;
    hipLaunchKernelGGL(quantize_tile_kernel<T>, dim3(grid), dim3(256), 0, stream, x, ldx, rows, cols, (int)tiles_c, q, ldq, s, lds, qt, ldqt, st,
                       ldst);
  } else {
    const int64_t per_row = (cols + kMxStep - 1) / kMxStep * (kMxStep / 8);
    const unsigned int grid = mx4_grid_for(rows * per_row, 256);
    if (!grid) return DLA_ERR_TOO_LARGE;
    hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3(grid), dim3(256), 0, stream, x, ldx, rows, cols, (int)per_row, q, ldq, s, lds);
  }
  return launch_status(__func__);
}

template <typename T>
int dequantize_typed(const Mx4View& w, int64_t cols, T* y, int64_t ldy, hipStream_t stream) {
  const int64_t per_row = (cols + 7) / 8;
  const unsigned int grid = mx4_grid_for(w.rows * per_row, 256);
  if (!grid) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(dequantize_kernel<T>, dim3(grid), dim3(256), 0, stream, w, cols, (int)per_row, y, ldy);
  return launch_status(__func__);
}

template <typename T>
int join_typed(const float* parts, int splits, int64_t m, int64_t n, T* c, int64_t ldc, bool onto, hipStream_t stream) {
  const unsigned int grid = mx4_grid_for(m * n, 1024);
  if (!grid) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(join_kernel<T>, dim3(grid), dim3(256), 0, stream, parts, splits, (unsigned int)(m * n), (unsigned int)n, c, ldc, onto);
  return launch_status(__func__);
}

template <typename T>
int zero_typed(T* c, int64_t ldc, int64_t m, int64_t n, hipStream_t stream) {
  const unsigned int grid = mx4_grid_for(m * n, 256);
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
