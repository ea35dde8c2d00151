// Host side of the microscaled product: its tile menu, the choice of a schedule and the launch.
#include "mx4_gemm_kernel.hpp"
#include "mx4_host.hpp"

namespace dla {
namespace {

struct Tile {
  int m, n;
};
const Tile kTiles[] = {{16, 32}, {32, 32}, {48, 32}, {64, 32}, {128, 128}, {256, 256}};  // 32 columns: the direct kernels
constexpr int kNumTiles = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
constexpr int kMaxSplits = 32;

int steps_of(int64_t k) { return (int)((k + kMxStep - 1) / kMxStep); }

// Eight waves a workgroup where there is one for each of the 256 units at most; four, so that two workgroups fit a unit's LDS, where
// there are more (one row by 16384 x 4096 DIRECT_A us against DIRECT_B, by 8192 x 8192 DIRECT_C against DIRECT_D).
template <int MB, int D8, int D4>
int launch_direct(const MxGemmArgs& g, hipStream_t stream) {
  const unsigned grid = (unsigned)(g.tiles_m * g.tiles_n * g.splits);
  if (grid <= 256)
    hipLaunchKernelGGL((mx4_gemm_direct_kernel<MB, D8, 8>), dim3(grid), dim3(512), 0, stream, g);
  else
    hipLaunchKernelGGL((mx4_gemm_direct_kernel<MB, D4, 4>), dim3(grid), dim3(256), 0, stream, g);
  return launch_status(__func__);
}

template <int TM, int TN, int WM, int WN, typename T>
int launch_tile(const MxGemmArgs& g, hipStream_t stream) {
  hipLaunchKernelGGL((mx4_gemm_tile_kernel<TM, TN, WM, WN, T>), dim3((unsigned)(g.tiles_m * g.tiles_n * g.splits)), dim3(WM * WN * 64), 0, stream,
                     g);
  return launch_status(__func__);
}

template <typename T>
int launch_typed(const MxGemmArgs& g, const MxPlan& plan, hipStream_t stream) {
  if (plan.tile_m == 128) return launch_tile<128, 128, 2, 2, T>(g, stream);
  return launch_tile<256, 256, 2, 4, T>(g, stream);
}

int launch(const MxGemmArgs& g, const MxPlan& plan, hipStream_t stream) {
  switch (plan.tile_m) {
    case 16: return launch_direct<1, 4, 4>(g, stream);
    case 32: return launch_direct<2, 4, 4>(g, stream);
    case 48: return launch_direct<3, 3, 3>(g, stream);
    case 64: return launch_direct<4, 2, 2>(g, stream);
  }
  return g.dt == DLA_F32 ? launch_typed<float>(g, plan, stream) : g.dt == DLA_BF16 ? launch_typed<__bf16>(g, plan, stream) : launch_typed<_Float16>(g, plan, stream);
}

}  // namespace

int mx4_gemm_menu(mx4_params* out, int cap) {
  for (int i = 0; i < kNumTiles && i < cap && out; ++i) out[i] = mx4_params{kTiles[i].m, kTiles[i].n, 0};
  return kNumTiles;
}

int mx4_gemm_plan(int64_t m, int64_t n, int64_t k, const mx4_params* p, MxPlan* plan) {
  MxPlan r = {0, 0, 0};
  if (p) r = MxPlan{p->tile_m, p->tile_n, p->splits};
  if (r.tile_m < 0 || r.tile_n < 0 || r.splits < 0 || r.splits > kMaxSplits || r.splits > steps_of(k)) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.tile_m == 0 && r.tile_n == 0) {
    r.tile_m = m <= 64 ? (int)(m + 15) / 16 * 16 : m < 2048 ? 128 : 256;
    r.tile_n = m <= 64 ? 32 : r.tile_m;
  }
  bool found = false;
  for (const Tile& t : kTiles) found |= t.m == r.tile_m && t.n == r.tile_n;
  if (!found) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.splits == 0) r.splits = 1;
  const int64_t tiles = ((m + r.tile_m - 1) / r.tile_m) * ((n + r.tile_n - 1) / r.tile_n);
  if (tiles * r.splits > 0x7fffffff) return DLA_ERR_TOO_LARGE;
  *plan = r;
  return DLA_SUCCESS;
}

int mx4_gemm_launch(bool onto, const Mx4View& a, const Mx4View& b, void* c, int64_t ldc, int64_t k, dla_dtype dt, const MxPlan& plan,
                    float* parts, hipStream_t stream) {
  const MxGemmArgs g = {a, b, c, parts, ldc, steps_of(k), plan.splits, (a.rows + plan.tile_m - 1) / plan.tile_m,
                        (b.rows + plan.tile_n - 1) / plan.tile_n, dt, onto};
  const int rc = launch(g, plan, stream);
  if (rc != DLA_SUCCESS || plan.splits == 1) return rc;
  return mx4_join_launch(parts, plan.splits, a.rows, b.rows, c, ldc, dt, onto, stream);
}

}  // namespace dla
