// Host side of the microscaled product: its tile menu, the choice of a schedule and the launch.
#include "mx4_gemm_kernel.hpp"
#include "mx4_schedule.hpp"

namespace dla {
namespace {

// The tiles; 32 columns: the direct kernels.  The costs are fitted to 1725 timings of 78 products (1 to 8192 rows, 128 to 8192 columns and
// terms, every tile, 1 to 32 splits): the choice takes 4 % longer in the mean than the best of them.
const MxTileCost kTiles[] = {
    {16, 32, 3.56f, 3.96f, 0.0208f, 0.0524f, 0.853f},
    {32, 32, 3.07f, 4.35f, 0.0207f, 0.0758f, 1.15f},
    {48, 32, 2.06f, 5.32f, 0.024f, 0.101f, 1.45f},
    {64, 32, 2.4f, 5.07f, 0.0227f, 0.113f, 1.54f},
    {128, 128, 2.59f, 4.99f, 0.0726f, 0.247f, 2.72f},
    {256, 256, 1.4f, 2.47f, 0.674f, 0.574f, 7.47f},
};
constexpr int kNumTiles = (int)(sizeof(kTiles) / sizeof(kTiles[0]));

int steps_of(int64_t k) { return (int)((k + kMxStep - 1) / kMxStep); }

// Eight waves a workgroup where there is one for each of the 256 units at most; four, so that two workgroups fit a unit's LDS, where
// there are more (one row by 16384 x 4096, 512 workgroups: 8.6 us with four waves, 10.2 with eight; by 8192 x 8192, 256 workgroups
// of eight waves: 9.1 us, by 8320 x 8192, 260 of four: 11.0).
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
  if (g.dt == DLA_F32) return launch_typed<float>(g, plan, stream);
  return g.dt == DLA_BF16 ? launch_typed<__bf16>(g, plan, stream) : launch_typed<_Float16>(g, plan, stream);
}

}  // namespace

int mx4_gemm_menu(mx4_params* out, int cap) {
  for (int i = 0; i < kNumTiles && i < cap && out; ++i) out[i] = mx4_params{kTiles[i].m, kTiles[i].n, 0};
  return kNumTiles;
}

int mx4_gemm_plan(int64_t m, int64_t n, int64_t k, const mx4_params* p, MxPlan* plan) { return mx4_choose(kTiles, kNumTiles, m, n, k, p, plan); }

int mx4_gemm_launch(bool onto, const Mx4View& a, const Mx4View& b, void* c, int64_t ldc, int64_t k, dla_dtype dt, const MxPlan& plan,
                    float* parts, hipStream_t stream) {
  const MxGemmArgs g = {a, b, c, parts, ldc, steps_of(k), plan.splits, (a.rows + plan.tile_m - 1) / plan.tile_m,
                        (b.rows + plan.tile_n - 1) / plan.tile_n, dt, onto};
  const int rc = launch(g, plan, stream);
  if (rc != DLA_SUCCESS || plan.splits == 1) return rc;
  return mx4_join_launch(parts, plan.splits, a.rows, b.rows, c, ldc, dt, onto, stream);
}

}  // namespace dla
