// What the tile kernels of the microscaled products share: loads to LDS, the order of tiles, and the way of results to memory.
#pragma once
#include "mx4_common.hpp"

namespace dla {

// 16 bytes of every lane from memory (base + off) to LDS without a register in between: lane l's go to byte lds + 16 l; base and
// lds are the same in all lanes.  Assembly, because the compiler lets every later LDS read wait for all such loads, whatever they
// write; so the waits are wait_loads_and_barrier's, and nothing else that a kernel's main loop loads may be in flight beside them.
// There is no register for the load to come back to; the wait state is the one between a write of M0 and its use (nothing else in
// these kernels uses M0).
__device__ __forceinline__ void load_to_lds(const void* base, unsigned int off, unsigned int lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base)
               : "memory");
}

// The same with 4 bytes of every lane, lane l's to byte lds + 4 l.
__device__ __forceinline__ void load4_to_lds(const void* base, unsigned int off, unsigned int lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base)
               : "memory");
}

// Where an array in LDS starts, for load_to_lds.
__device__ __forceinline__ unsigned int lds_offset(const void* p) {
  return __builtin_amdgcn_readfirstlane((unsigned int)(uintptr_t)(const __attribute__((address_space(3))) void*)p);
}

// Waits until at most N of the wave's loads are in flight; until its LDS accesses are done.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Waits until at most N of the wave's loads are in flight and all its LDS accesses are done, then for the other waves.
template <int N>
__device__ __forceinline__ void wait_loads_and_barrier() {
  static_assert(N < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Tile `id` of a grid of tiles: four rows of tiles are walked column by column, so that the workgroups of an XCD, which are
// neighbours in id, share operands in its L2 (its 32 at a time are 4 x 8; with eight rows 1 % slower, with sixteen 3 %).
__device__ __forceinline__ void tile_at(int id, int tiles_m, int tiles_n, int* ti, int* tj) {
  const int band = 4 * tiles_n, first = id / band * 4, height = min(4, tiles_m - first), in = id % band;
  *ti = first + in % height;
  *tj = in / height;
}

template <int R, int C>
constexpr int kMxRoom = R * C / 4 < 1024 ? R * C / 4 : 1024;

// A wave's part of the result, R x C in 32 x 32 blocks whose lanes hold neighbouring columns, to rows r0.. and columns c0.. of a
// matrix of `rows` x `cols`; `lds` is the wave's own room, kMxRoom<R, C> units of 16 bytes.  It goes through LDS as S, rounded to T (or in
// fp32 where it is added onto C, which is rounded once), so that rows are written 16 bytes a lane.
template <int R, int C, typename S, typename T>
__device__ __forceinline__ void mx_store_tile(u32x4_t* lds, const f32x16_t (&acc)[R / 32][C / 32], int lane, T* c, int64_t ldc, int r0, int c0, int rows,
                                              int cols, bool onto) {
  constexpr int PER = 16 / (int)sizeof(S);                              // elements of 16 bytes
  constexpr int WIDE = C * R * (int)sizeof(S) <= 16384 ? C : 16384 / (R * (int)sizeof(S));  // columns at a time
  constexpr int CH = WIDE / PER, RPB = CH >= 16 ? 1 : 16 / CH;          // 16-byte chunks of a row; rows of 256 bytes
  static_assert(WIDE % 32 == 0 && C % WIDE == 0, "whole blocks");
  typedef S run_t __attribute__((ext_vector_type(PER)));
  typedef T out_t __attribute__((ext_vector_type(PER)));
  typedef S quad_t __attribute__((ext_vector_type(4)));
  const int l31 = lane & 31, l5 = lane >> 5;
  const bool vec = (uintptr_t)c % sizeof(out_t) == 0 && ldc % PER == 0 && cols >= PER;
  // chunk c of a row lies at c ^ (r / RPB) % CH.  A wave's read of 1 KB takes LDS 4 clocks, as from neighbouring places; a write 8 clocks in rows
  // of 16 chunks, as there, and twice as long as there in rows of 8 and of 4.
  auto place = [&](int r, int chunk) { return r * CH + (chunk ^ ((r / RPB) & (CH - 1))); };
  auto in_order = [] {  // what other lanes of the wave have written
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
#pragma unroll
  for (int p = 0; p < C / WIDE; ++p) {
#pragma unroll
    for (int i = 0; i < R / 32; ++i)
#pragma unroll
      for (int j = 0; j < WIDE / 32; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = j * 32 + 8 * q + 4 * l5;
          quad_t t;
#pragma unroll
          for (int v = 0; v < 4; ++v) t[v] = (S)acc[i][p * (WIDE / 32) + j][4 * q + v];
          reinterpret_cast<quad_t*>(lds + place(i * 32 + l31, col / PER))[col % PER / 4] = t;
        }
    in_order();
    const int first = c0 + p * WIDE;
    // A lane's N accesses, U at a time so that U loads of what is added to are on their way, without a branch around each (C += A*B^T,
    // 1600 x 1800, k = 2000, fp32, the largest part of it: 21 us with branches, 16 without): as many as the registers hold.
    constexpr int N = R * CH / 64, MOST = R * C > 4096 ? 4 : 128 / (int)sizeof(out_t), U = N < MOST ? N : MOST;
    static_assert(N % U == 0, "whole turns");
#pragma unroll 1
    for (int from = 0; from < N; from += U) {
      out_t o[U];
      if (onto && vec) {  // (past the end the last row or whole run, which is not used there and may just be written)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int e = (from + u) * 64 + lane, row = min(r0 + e / CH, rows - 1), col = min(first + e % CH * PER, cols / PER * PER - PER);
          o[u] = *reinterpret_cast<const out_t*>(c + (int64_t)row * ldc + col);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = (from + u) * 64 + lane, r = e / CH, chunk = e % CH, row = r0 + r, col = first + chunk * PER;
        const run_t t = __builtin_bit_cast(run_t, lds[place(r, chunk)]);
        if (row >= rows || col >= cols) continue;
        T* const out = c + (int64_t)row * ldc + col;
        if (vec && col + PER <= cols) {
#pragma unroll
          for (int v = 0; v < PER; ++v) o[u][v] = (T)(onto ? (float)o[u][v] + (float)t[v] : (float)t[v]);
          *reinterpret_cast<out_t*>(out) = o[u];
        } else {
#pragma unroll
          for (int v = 0; v < PER; ++v)
            if (col + v < cols) out[v] = (T)(onto ? (float)out[v] + (float)t[v] : (float)t[v]);
        }
      }
    }
    in_order();
  }
}

}  // namespace dla
