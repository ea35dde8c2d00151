// Host side of microscaled weights applied to ordinary rows: the tile menu, the choice of a schedule and the launch.
#include "mx4_apply_kernel.hpp"
#include "mx4_host.hpp"

namespace dla {
namespace {

constexpr int kMaxSplits = 32;

template <dla_dtype DT, typename TY>
int launch_typed(int op, const MxApplyArgs& g, hipStream_t stream) {
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
int launch_to(int op, const MxApplyArgs& g, dla_dtype dt_y, hipStream_t stream) {
  if (dt_y == DLA_F32) return launch_typed<DT, float>(op, g, stream);
  if (dt_y == DLA_BF16) return launch_typed<DT, __bf16>(op, g, stream);
  return launch_typed<DT, _Float16>(op, g, stream);
}

}  // namespace

int mx4_apply_menu(int, mx4_params* out, int cap) {
  if (out && cap > 0) out[0] = mx4_params{16, 16, 0};
  return 1;
}

int mx4_apply_plan(int op, int64_t m, int64_t n, int64_t k, dla_dtype, const mx4_params* p, MxPlan* plan) {
  MxPlan r = {0, 0, 0};
  if (p) r = MxPlan{p->tile_m, p->tile_n, p->splits};
  const int64_t terms = op == 0 ? k : n, out = op == 0 ? n : k;
  if (r.tile_m < 0 || r.tile_n < 0 || r.splits < 0 || r.splits > kMaxSplits || r.splits > (terms + kMxStep - 1) / kMxStep) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.tile_m == 0 && r.tile_n == 0) r.tile_m = r.tile_n = 16;
  if (r.tile_m != 16 || r.tile_n != 16) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.splits == 0) r.splits = 1;
  const int64_t tiles = ((m + r.tile_m - 1) / r.tile_m) * ((out + r.tile_n - 1) / r.tile_n);
  if (tiles * r.splits > 0x7fffffff) return DLA_ERR_TOO_LARGE;
  *plan = r;
  return DLA_SUCCESS;
}

size_t mx4_apply_bytes(int op, int64_t m, int64_t n, int64_t k, dla_dtype, const MxPlan& plan) {
  return mx4_parts_bytes(m, op == 0 ? n : k, plan);
}

int mx4_apply_launch(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy,
                     dla_dtype dt_y, const MxPlan& plan, void* workspace, hipStream_t stream) {
  const int size = dt == DLA_F32 ? 4 : 2;
  const int64_t out = op == 0 ? w.rows : k;
  const MxApplyArgs g = {x, w, y, (float*)workspace, ldx, ldy, (int)m, w.rows, (int)k, plan.splits, (int)((m + plan.tile_m - 1) / plan.tile_m),
                         (int)((out + plan.tile_n - 1) / plan.tile_n), (uintptr_t)x % 16 == 0 && ldx * size % 16 == 0};
  const int rc = dt == DLA_F32 ? launch_to<DLA_F32>(op, g, dt_y, stream)
                 : dt == DLA_BF16 ? launch_to<DLA_BF16>(op, g, dt_y, stream) : launch_to<DLA_F16>(op, g, dt_y, stream);
  if (rc != DLA_SUCCESS || plan.splits == 1) return rc;
  return mx4_join_launch((const float*)workspace, plan.splits, m, out, y, ldy, dt_y, false, stream);
}

}  // namespace dla
