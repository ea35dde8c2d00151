// Host side of microscaled weights applied to ordinary rows: the tile menu, the choice of a schedule and the launches.
#include "mx4_apply_kernel.hpp"
#include "mx4_schedule.hpp"

namespace dla {
namespace {

constexpr int kDirect = 32;  // columns of a direct kernel's tile

// The tiles.  The direct kernels are for op 0; more than 16 rows of fp32 there, and two or three terms of 256 rows, do not fit the LDS.  The
// costs are fitted to 8000 timings of 390 products (1 to 4096 rows, 128 to 8192 columns and terms, every tile, 1 to 32 splits): the choice takes
// 1 to 6 % longer in the mean than the best of them, by operation and type.
const MxTileCost kForwardBf16[] = {
    {16, 32, 4.94f, 4.38f, 0.0397f, 0.0881f, 0.916f},
    {32, 32, 3.46f, 5.91f, 0.0355f, 0.15f, 2.25f},
    {48, 32, 2.43f, 6.68f, 0.0651f, 0.186f, 2.79f},
    {64, 32, 0.967f, 8.39f, 0.0789f, 0.213f, 3.52f},
    {32, 128, 6.73f, 1.25f, 0.464f, 0.345f, 0.912f},
    {64, 128, 6.98f, 2.09f, 0.28f, 0.54f, 0.877f},
    {128, 128, 6.9f, 1.34f, 0.929f, 0.74f, 1.26f},
    {256, 256, 9.24f, 2.73f, 0.432f, 2.34f, 1.04f},
};
const MxTileCost kForwardF16[] = {
    {16, 32, 5.2f, 3.94f, 0.0511f, 0.106f, 0.749f},
    {32, 32, 1.93f, 7.79f, 0.0108f, 0.18f, 2.39f},
    {48, 32, 1.55f, 7.34f, 0.0771f, 0.209f, 3.11f},
    {64, 32, 7.06f, 1.72f, 0.167f, 0.256f, 1.0f},
    {32, 128, 8.07f, 1.59f, 0.583f, 0.504f, 1.16f},
    {64, 128, 7.98f, 2.99f, 0.385f, 0.834f, 1.0f},
    {128, 128, 9.22f, 2.26f, 0.48f, 1.74f, 1.0f},
};
const MxTileCost kForwardF32[] = {
    {16, 32, 3.15f, 8.18f, 0.0402f, 0.198f, 2.19f},
    {32, 128, 8.07f, 2.88f, 0.262f, 0.742f, 0.683f},
    {64, 128, 5.85f, 4.54f, 0.841f, 1.32f, 2.73f},
    {128, 128, 6.45f, 3.0f, 0.5f, 2.32f, 3.31f},
};
const MxTileCost kGradBf16[] = {
    {32, 128, 5.51f, 2.2f, 0.862f, 0.748f, 1.01f},
    {64, 128, 6.77f, 1.03f, 1.04f, 0.869f, 0.746f},
    {128, 128, 5.78f, 2.28f, 1.13f, 1.04f, 1.01f},
    {256, 256, 8.44f, 2.95f, 0.507f, 2.73f, 0.766f},
};
const MxTileCost kGradF16[] = {
    {32, 128, 7.15f, 2.77f, 0.568f, 1.11f, 1.27f},
    {64, 128, 7.99f, 1.94f, 1.2f, 1.39f, 1.0f},
    {128, 128, 8.13f, 2.9f, 1.68f, 2.31f, 1.02f},
};
const MxTileCost kGradF32[] = {
    {32, 128, 6.87f, 4.18f, 0.343f, 1.16f, 1.0f},
    {64, 128, 3.06f, 7.51f, 0.907f, 1.86f, 4.29f},
    {128, 128, 7.26f, 4.54f, 1.05f, 2.97f, 1.03f},
};

struct Menu {
  const MxTileCost* tiles;
  int count;
};
template <int N>
Menu menu(const MxTileCost (&t)[N]) {
  return {t, N};
}
Menu menu_of(int op, dla_dtype dt) {
  if (op == 0) return dt == DLA_F32 ? menu(kForwardF32) : dt == DLA_BF16 ? menu(kForwardBf16) : menu(kForwardF16);
  return dt == DLA_F32 ? menu(kGradF32) : dt == DLA_BF16 ? menu(kGradBf16) : menu(kGradF16);
}

int64_t wide(int64_t terms) { return (terms + 63) / 64 * 64; }

// X as it is: bf16 in aligned rows, no terms behind the last whole step of 64.
bool whole(const void* x, int64_t ldx, dla_dtype dt, int64_t terms) {
  return dt == DLA_BF16 && (uintptr_t)x % 16 == 0 && ldx % 8 == 0 && terms % 64 == 0 && ldx <= kMxMaxLd / 2;
}

// X as the direct kernel takes it: 16-bit, aligned rows of whole steps (and offsets inside a tile of 64 rows in 32 bits).
bool direct_takes(const void* x, int64_t ldx, dla_dtype dt, int64_t terms) {
  return dt != DLA_F32 && (uintptr_t)x % 16 == 0 && ldx % 8 == 0 && terms % kMxStep == 0 && ldx <= (int64_t)1 << 24;
}

// The room for what a kernel reads instead of X.
size_t copy_bytes(const MxPlan& plan, int64_t m, int64_t terms, dla_dtype dt) {
  const int64_t count = plan.tile_n == kDirect ? (terms + kMxStep - 1) / kMxStep * kMxStep * 2 * (dt == DLA_F32 ? 3 : 1)
                                               : wide(terms) * 2 * (dt == DLA_F32 ? 3 : dt == DLA_F16 ? 2 : 1);
  return ((size_t)(m * count) + 255) / 256 * 256;
}

template <typename T, int TERMS, int MB, int XI, int WV, int DW, int DX>
int launch_direct_as(const MxApplyArgs& g, hipStream_t stream) {
  hipLaunchKernelGGL((mx4_apply_direct_kernel<T, TERMS, MB, XI, WV, DW, DX>), dim3((unsigned)(g.tiles_m * g.tiles_n * g.splits)), dim3(WV * 64), 0, stream, g);
  return launch_status(__func__);
}

// How many waves and how far ahead is what the LDS holds.  Up to 16 rows of 16 bits (4 of fp32): eight waves where there is one workgroup
// for each of the 256 units at most, and four, so that several fit a unit, where there are more.  Above, eight waves with one step of
// X ahead rather than four with two, so that one wave's products hide what the other of its SIMD waits for: 48 rows of fp16 by
// 8192 x 8192 17.5 us for 19.8, 64 by 4096 x 4096 10.9 for 13.2 (bf16, which has half the work between its loads, the same in both).
template <typename T, int TERMS>
int launch_direct(const MxApplyArgs& g, int tile_m, hipStream_t stream) {
  const bool many = (int64_t)g.tiles_m * g.tiles_n * g.splits > 256;
  if (tile_m == 16 && g.m <= 4) return many ? launch_direct_as<T, TERMS, 1, 1, 4, 4, 2>(g, stream) : launch_direct_as<T, TERMS, 1, 1, 8, 4, 2>(g, stream);
  if constexpr (TERMS == 3) {
    return launch_direct_as<T, TERMS, 1, 4, 4, 4, 2>(g, stream);
  } else {
    switch (tile_m) {
      case 16: return many ? launch_direct_as<T, 1, 1, 4, 4, 4, 2>(g, stream) : launch_direct_as<T, 1, 1, 4, 8, 4, 2>(g, stream);
      case 32: return launch_direct_as<T, 1, 2, 8, 8, 4, 1>(g, stream);
      case 48: return launch_direct_as<T, 1, 3, 12, 8, 3, 1>(g, stream);
      default: return launch_direct_as<T, 1, 4, 16, 8, 1, 1>(g, stream);
    }
  }
}

template <typename T>
int launch_copy(const T* x, int64_t ldx, int64_t m, int64_t terms, int64_t to_ld, T* to, hipStream_t stream) {
  const int64_t per_row = to_ld / 8;
  const unsigned int groups = mx4_grid_for(m * per_row, 256);
  if (!groups) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(mx4_copy_kernel<T>, dim3(groups), dim3(256), 0, stream, x, ldx, m, terms, (int)per_row, to);
  return launch_status(__func__);
}

template <dla_dtype DT>
int launch_planes(const void* x, int64_t ldx, int64_t m, int64_t terms, int64_t to_ld, void* planes, hipStream_t stream) {
  using T = typename MxType<DT>::type;
  const int64_t per_row = to_ld / 8;
  const unsigned int groups = mx4_grid_for(m * per_row, 256);
  if (!groups) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL((mx4_planes_kernel<T, MxType<DT>::kTerms>), dim3(groups), dim3(256), 0, stream, static_cast<const T*>(x), ldx, m, terms,
                     (int)per_row, static_cast<bf16x8_t*>(planes));
  return launch_status(__func__);
}

template <int TM, int TN, int WM, int WN, int TERMS, typename TY>
int launch_tile(int op, const MxApplyTileArgs& g, hipStream_t stream) {
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits)), block(WM * WN * 64);
  if (op == 0)
    hipLaunchKernelGGL((mx4_apply_tile_kernel<TM, TN, WM, WN, TERMS, TY>), grid, block, 0, stream, g);
  else
    hipLaunchKernelGGL((mx4_apply_grad_kernel<TM, TN, WM, WN, TERMS, TY>), grid, block, 0, stream, g);
  return launch_status(__func__);
}

template <dla_dtype DT, typename TY>
int launch_typed(int op, const void* x, int64_t ldx, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy, const MxPlan& plan, void* workspace,
                 hipStream_t stream) {
  const int64_t out = op == 0 ? w.rows : k, terms = op == 0 ? k : w.rows;
  const int tiles_m = (int)((m + plan.tile_m - 1) / plan.tile_m), tiles_n = (int)((out + plan.tile_n - 1) / plan.tile_n);
  float* const parts = static_cast<float*>(workspace);
  MxApplyTileArgs g = {static_cast<const __bf16*>(x), w, y, parts, ldx, 0, ldy, (int)m, (int)out, (int)((k + kMxStep - 1) / kMxStep * kMxStep),
                       (int)(wide(terms) / 64), plan.splits, tiles_m, tiles_n};
  if (!whole(x, ldx, DT, terms)) {
    void* const planes = static_cast<char*>(workspace) + mx4_parts_bytes(m, out, plan);
    const int rc = launch_planes<DT>(x, ldx, m, terms, wide(terms), planes, stream);
    if (rc != DLA_SUCCESS) return rc;
    g.x = static_cast<const __bf16*>(planes);
    g.ldx = wide(terms);
    g.plane = m * g.ldx;
  }
  if constexpr (DT == DLA_BF16) {
    if (plan.tile_m == 256) return launch_tile<256, 256, 2, 4, 1, TY>(op, g, stream);
  }
  if (plan.tile_m == 32) return launch_tile<32, 128, 1, 4, MxType<DT>::kTerms, TY>(op, g, stream);
  if (plan.tile_m == 64) return launch_tile<64, 128, 1, 4, MxType<DT>::kTerms, TY>(op, g, stream);
  return launch_tile<128, 128, 2, 2, MxType<DT>::kTerms, TY>(op, g, stream);
}

template <dla_dtype DT>
int launch_to(int op, const void* x, int64_t ldx, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy, dla_dtype dt_y, const MxPlan& plan,
              void* workspace, hipStream_t stream) {
  using T = typename MxType<DT>::type;
  if (plan.tile_n == kDirect) {
    const int64_t steps = (k + kMxStep - 1) / kMxStep, to_ld = steps * kMxStep;
    MxApplyArgs g = {x, w, y, static_cast<float*>(workspace), ldx, 0, ldy, (int)m, (int)steps, plan.splits, (int)((m + plan.tile_m - 1) / plan.tile_m),
                     (w.rows + kDirect - 1) / kDirect, dt_y};
    if (!direct_takes(x, ldx, DT, k)) {
      void* const to = static_cast<char*>(workspace) + mx4_parts_bytes(m, w.rows, plan);
      int rc;
      if constexpr (DT == DLA_F32)
        rc = launch_planes<DT>(x, ldx, m, k, to_ld, to, stream);
      else
        rc = launch_copy<T>(static_cast<const T*>(x), ldx, m, k, to_ld, static_cast<T*>(to), stream);
      if (rc != DLA_SUCCESS) return rc;
      g.x = to;
      g.ldx = to_ld;
      g.plane = m * to_ld;
    }
    if constexpr (DT == DLA_F32)
      return launch_direct<__bf16, 3>(g, plan.tile_m, stream);
    else
      return launch_direct<T, 1>(g, plan.tile_m, stream);
  }
  if (dt_y == DLA_F32) return launch_typed<DT, float>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  if (dt_y == DLA_BF16) return launch_typed<DT, __bf16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  return launch_typed<DT, _Float16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
}

}  // namespace

int mx4_apply_menu(int op, dla_dtype dt, mx4_params* out, int cap) {
  const Menu m = menu_of(op, dt);
  for (int i = 0; i < m.count && i < cap && out; ++i) out[i] = mx4_params{m.tiles[i].m, m.tiles[i].n, 0};
  return m.count;
}

int mx4_apply_plan(int op, int64_t m, int64_t n, int64_t k, dla_dtype dt, const mx4_params* p, MxPlan* plan) {
  const Menu t = menu_of(op, dt);
  const int64_t terms = op == 0 ? k : n, out = op == 0 ? n : k;
  if (terms > kMxMaxLd / 2) return DLA_ERR_TOO_LARGE;
  return mx4_choose(t.tiles, t.count, m, out, terms, p, plan);
}

size_t mx4_apply_bytes(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, int64_t n, int64_t k, const MxPlan& plan) {
  const int64_t terms = op == 0 ? k : n;
  const bool as_it_is = plan.tile_n == kDirect ? direct_takes(x, ldx, dt, terms) : whole(x, ldx, dt, terms);
  return mx4_parts_bytes(m, op == 0 ? n : k, plan) + (as_it_is ? 0 : copy_bytes(plan, m, terms, dt));
}

int mx4_apply_launch(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy, dla_dtype dt_y,
                     const MxPlan& plan, void* workspace, hipStream_t stream) {
  const int rc = dt == DLA_F32 ? launch_to<DLA_F32>(op, x, ldx, m, w, k, y, ldy, dt_y, plan, workspace, stream)
                 : dt == DLA_BF16 ? launch_to<DLA_BF16>(op, x, ldx, m, w, k, y, ldy, dt_y, plan, workspace, stream)
                                  : launch_to<DLA_F16>(op, x, ldx, m, w, k, y, ldy, dt_y, plan, workspace, stream);
  if (rc != DLA_SUCCESS || plan.splits == 1) return rc;
  return mx4_join_launch((const float*)workspace, plan.splits, m, op == 0 ? w.rows : k, y, ldy, dt_y, false, stream);
}

}  // namespace dla
