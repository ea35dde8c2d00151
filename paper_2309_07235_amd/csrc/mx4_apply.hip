// Host side of microscaled weights applied to ordinary rows: the tile menu, the choice of a schedule and the launches.
#include "mx4_apply_kernel.hpp"
#include "mx4_host.hpp"

namespace dla {
namespace {

constexpr int kMaxSplits = 32;
constexpr int kDirect = 16;  // the tile of the direct kernels

struct Tile {
  int m, n;
};
const Tile kTiles[] = {{kDirect, kDirect}, {128, 128}, {256, 256}};

bool legal(const Tile& t, dla_dtype dt) { return t.m < 256 || dt == DLA_BF16; }  // two or three terms of 256 rows do not fit the LDS

int64_t wide(int64_t terms) { return (terms + 63) / 64 * 64; }

// X as it is: bf16 in aligned rows, no terms behind the last whole step of 64.
bool whole(const void* x, int64_t ldx, dla_dtype dt, int64_t terms) {
  return dt == DLA_BF16 && (uintptr_t)x % 16 == 0 && ldx % 8 == 0 && terms % 64 == 0 && ldx <= kMxMaxLd / 2;
}

size_t planes_bytes(int64_t m, int64_t terms, dla_dtype dt) {
  const int64_t count = dt == DLA_F32 ? 3 : dt == DLA_F16 ? 2 : 1;
  return ((size_t)(count * m * wide(terms)) * 2 + 255) / 256 * 256;
}

template <dla_dtype DT, typename TY>
int launch_direct(int op, const MxApplyArgs& g, hipStream_t stream) {
  using T = typename MxType<DT>::type;
  constexpr int TERMS = MxType<DT>::kTerms;
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits));
  if (op == 0)
    hipLaunchKernelGGL((mx4_apply_direct_kernel<T, TERMS, TY>), grid, dim3(kMxApplyWaves * 64), 0, stream, g);
  else
    hipLaunchKernelGGL((mx4_apply_grad_direct_kernel<T, TERMS, TY>), grid, dim3(64), 0, stream, g);
  return launch_status(__func__);
}

template <dla_dtype DT>
int launch_planes(const void* x, int64_t ldx, int64_t m, int64_t terms, void* planes, hipStream_t stream) {
  using T = typename MxType<DT>::type;
  const int64_t per_row = wide(terms) / 8, groups = (m * per_row + 255) / 256;
  if (groups > 0x7fffffff) return DLA_ERR_TOO_LARGE;
  const bool vec = (uintptr_t)x % 16 == 0 && ldx * (int64_t)sizeof(T) % 16 == 0;
  hipLaunchKernelGGL((mx4_planes_kernel<T, MxType<DT>::kTerms>), dim3((unsigned)groups), dim3(256), 0, stream, static_cast<const T*>(x), ldx, m, terms,
                     (int)per_row, vec, static_cast<bf16x8_t*>(planes));
  return launch_status(__func__);
}

template <int TM, int TN, int WM, int WN, int TERMS, typename TY>
int launch_tile(int op, const MxApplyTileArgs& g, hipStream_t stream) {
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits)), block(WM * WN * 64);
  if (op == 0)
    hipLaunchKernelGGL((mx4_apply_tile_kernel<TM, TN, WM, WN, TERMS, false, TY>), grid, block, 0, stream, g);
  else
    hipLaunchKernelGGL((mx4_apply_tile_kernel<TM, TN, WM, WN, TERMS, true, TY>), grid, block, 0, stream, g);
  return launch_status(__func__);
}

template <dla_dtype DT, typename TY>
int launch_typed(int op, const void* x, int64_t ldx, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy, const MxPlan& plan, void* workspace,
                 hipStream_t stream) {
  const int64_t out = op == 0 ? w.rows : k, terms = op == 0 ? k : w.rows;
  const int tiles_m = (int)((m + plan.tile_m - 1) / plan.tile_m), tiles_n = (int)((out + plan.tile_n - 1) / plan.tile_n);
  float* const parts = static_cast<float*>(workspace);
  if (plan.tile_m == kDirect) {
    const bool vec = (uintptr_t)x % 16 == 0 && ldx * (int64_t)sizeof(typename MxType<DT>::type) % 16 == 0;
    const MxApplyArgs g = {x, w, y, parts, ldx, ldy, (int)m, w.rows, (int)k, plan.splits, tiles_m, tiles_n, vec};
    return launch_direct<DT, TY>(op, g, stream);
  }
  MxApplyTileArgs g = {static_cast<const __bf16*>(x), w, y, parts, ldx, 0, ldy, (int)m, (int)out, (int)((k + kMxStep - 1) / kMxStep * kMxStep),
                       (int)(wide(terms) / 64), plan.splits, tiles_m, tiles_n};
  if (!whole(x, ldx, DT, terms)) {
    void* const planes = static_cast<char*>(workspace) + mx4_parts_bytes(m, out, plan);
    const int rc = launch_planes<DT>(x, ldx, m, terms, planes, stream);
    if (rc != DLA_SUCCESS) return rc;
    g.x = static_cast<const __bf16*>(planes);
    g.ldx = wide(terms);
    g.plane = m * g.ldx;
  }
  if constexpr (DT == DLA_BF16) {
    if (plan.tile_m == 256) return launch_tile<256, 256, 2, 4, 1, TY>(op, g, stream);
  }
  return launch_tile<128, 128, 2, 2, MxType<DT>::kTerms, TY>(op, g, stream);
}

template <dla_dtype DT>
int launch_to(int op, const void* x, int64_t ldx, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy, dla_dtype dt_y, const MxPlan& plan,
              void* workspace, hipStream_t stream) {
  if (dt_y == DLA_F32) return launch_typed<DT, float>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  if (dt_y == DLA_BF16) return launch_typed<DT, __bf16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  return launch_typed<DT, _Float16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
}

}  // namespace

int mx4_apply_menu(int, dla_dtype dt, mx4_params* out, int cap) {
  int count = 0;
  for (const Tile& t : kTiles) {
    if (!legal(t, dt)) continue;
    if (out && count < cap) out[count] = mx4_params{t.m, t.n, 0};
    ++count;
  }
  return count;
}

int mx4_apply_plan(int op, int64_t m, int64_t n, int64_t k, dla_dtype dt, const mx4_params* p, MxPlan* plan) {
  MxPlan r = {0, 0, 0};
  if (p) r = MxPlan{p->tile_m, p->tile_n, p->splits};
  const int64_t terms = op == 0 ? k : n, out = op == 0 ? n : k;
  if (r.tile_m < 0 || r.tile_n < 0 || r.splits < 0 || r.splits > kMaxSplits || r.splits > (terms + kMxStep - 1) / kMxStep) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.tile_m == 0 && r.tile_n == 0) r.tile_m = r.tile_n = m <= 32 ? 16 : (m < 1024 || dt != DLA_BF16) ? 128 : 256;
  bool found = false;
  for (const Tile& t : kTiles) found |= t.m == r.tile_m && t.n == r.tile_n && legal(t, dt);
  if (!found) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.splits == 0) r.splits = 1;
  const int64_t tiles = ((m + r.tile_m - 1) / r.tile_m) * ((out + r.tile_n - 1) / r.tile_n);
  if (tiles * r.splits > 0x7fffffff || terms > kMxMaxLd / 2) return DLA_ERR_TOO_LARGE;
  *plan = r;
  return DLA_SUCCESS;
}

size_t mx4_apply_bytes(int op, int64_t m, int64_t n, int64_t k, dla_dtype dt, const MxPlan& plan) {
  return mx4_parts_bytes(m, op == 0 ? n : k, plan) + (plan.tile_m == kDirect ? 0 : planes_bytes(m, op == 0 ? k : n, dt));
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
