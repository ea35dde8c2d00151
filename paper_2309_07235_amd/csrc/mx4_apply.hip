// Host side of microscaled weights applied to ordinary rows: the tile menu, the choice of a schedule and the launches.
#include "mx4_apply_kernel.hpp"
#include "mx4_host.hpp"

namespace dla {
namespace {

constexpr int kMaxSplits = 32;
constexpr int kDirect = 32;  // columns of a direct kernel's tile

struct Tile {
  int m, n;
};
const Tile kTiles[] = {{16, kDirect}, {32, kDirect}, {48, kDirect}, {64, kDirect}, {32, 128}, {64, 128}, {128, 128}, {256, 256}};

// The direct kernels are for op 0; more than 32 rows of fp32, or two or three terms of 256 rows, do not fit the LDS.
bool legal(const Tile& t, int op, dla_dtype dt) {
  return t.n == kDirect ? op == 0 && (t.m <= 32 || dt != DLA_F32) : t.m < 256 || dt == DLA_BF16;
}

int64_t wide(int64_t terms) { return (terms + 63) / 64 * 64; }

// X as it is: bf16 in aligned rows, no terms behind the last whole step of 64.
bool whole(const void* x, int64_t ldx, dla_dtype dt, int64_t terms) {
  return dt == DLA_BF16 && (uintptr_t)x % 16 == 0 && ldx % 8 == 0 && terms % 64 == 0 && ldx <= kMxMaxLd / 2;
}

// X as the direct kernel takes it: aligned rows of whole steps (and offsets inside a tile of 64 rows in 32 bits).
bool direct_takes(const void* x, int64_t ldx, int size, int64_t terms) {
  return (uintptr_t)x % 16 == 0 && ldx * size % 16 == 0 && terms % kMxStep == 0 && ldx * size <= (int64_t)1 << 25;
}

// The room for what a kernel reads instead of X.
size_t copy_bytes(const MxPlan& plan, int64_t m, int64_t terms, dla_dtype dt) {
  const int64_t count = plan.tile_n == kDirect ? (terms + kMxStep - 1) / kMxStep * kMxStep * (dt == DLA_F32 ? 4 : 2)
                                               : wide(terms) * 2 * (dt == DLA_F32 ? 3 : dt == DLA_F16 ? 2 : 1);
  return ((size_t)(m * count) + 255) / 256 * 256;
}

template <typename T, int MB, int XI, int WV, int DW>
int launch_direct_as(const MxApplyArgs& g, hipStream_t stream) {
  hipLaunchKernelGGL((mx4_apply_direct_kernel<T, MB, XI, WV, DW>), dim3((unsigned)(g.tiles_m * g.tiles_n * g.splits)), dim3(WV * 64), 0, stream, g);
  return launch_status(__func__);
}

// How many waves and how far ahead is what the LDS holds: of 16-bit rows up to 16, eight waves where there is one workgroup for each
// of the 256 units at most, and four, so that two fit a unit, where there are more.  A load of X takes four rows of 16-bit
// elements or two of fp32.
template <typename T>
int launch_direct(const MxApplyArgs& g, int tile_m, hipStream_t stream) {
  if constexpr (sizeof(T) == 4) {
    if (tile_m == 16) return g.m <= 2 ? launch_direct_as<T, 1, 1, 4, 4>(g, stream) : launch_direct_as<T, 1, 8, 4, 4>(g, stream);
    return launch_direct_as<T, 2, 16, 4, 3>(g, stream);
  } else {
    const bool many = (int64_t)g.tiles_m * g.tiles_n * g.splits > 256;
    switch (tile_m) {
      case 16:
        if (g.m <= 4) return many ? launch_direct_as<T, 1, 1, 4, 4>(g, stream) : launch_direct_as<T, 1, 1, 8, 4>(g, stream);
        return many ? launch_direct_as<T, 1, 4, 4, 4>(g, stream) : launch_direct_as<T, 1, 4, 8, 4>(g, stream);
      case 32: return launch_direct_as<T, 2, 8, 4, 6>(g, stream);
      case 48: return launch_direct_as<T, 3, 12, 4, 6>(g, stream);
      default: return launch_direct_as<T, 4, 16, 4, 3>(g, stream);
    }
  }
}

template <typename T>
int launch_copy(const T* x, int64_t ldx, int64_t m, int64_t terms, int64_t to_ld, T* to, hipStream_t stream) {
  const int64_t per_row = to_ld / 8, groups = (m * per_row + 255) / 256;
  if (groups > 0x7fffffff) return DLA_ERR_TOO_LARGE;
  hipLaunchKernelGGL(mx4_copy_kernel<T>, dim3((unsigned)groups), dim3(256), 0, stream, x, ldx, m, terms, (int)per_row, to);
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
    const int rc = launch_planes<DT>(x, ldx, m, terms, planes, stream);
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
    const int64_t steps = (k + kMxStep - 1) / kMxStep;
    MxApplyArgs g = {x, w, y, static_cast<float*>(workspace), ldx, ldy, (int)m, (int)steps, plan.splits, (int)((m + plan.tile_m - 1) / plan.tile_m),
                     (w.rows + kDirect - 1) / kDirect, dt_y};
    if (!direct_takes(x, ldx, sizeof(T), k)) {
      T* const to = reinterpret_cast<T*>(static_cast<char*>(workspace) + mx4_parts_bytes(m, w.rows, plan));
      const int rc = launch_copy<T>(static_cast<const T*>(x), ldx, m, k, steps * kMxStep, to, stream);
      if (rc != DLA_SUCCESS) return rc;
      g.x = to;
      g.ldx = steps * kMxStep;
    }
    return launch_direct<T>(g, plan.tile_m, stream);
  }
  if (dt_y == DLA_F32) return launch_typed<DT, float>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  if (dt_y == DLA_BF16) return launch_typed<DT, __bf16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
  return launch_typed<DT, _Float16>(op, x, ldx, m, w, k, y, ldy, plan, workspace, stream);
}

}  // namespace

int mx4_apply_menu(int op, dla_dtype dt, mx4_params* out, int cap) {
  int count = 0;
  for (const Tile& t : kTiles) {
    if (!legal(t, op, dt)) continue;
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
  if (r.tile_m == 0 && r.tile_n == 0) {
    const bool direct = op == 0 && m <= (dt == DLA_F32 ? 32 : 64);
    r.tile_m = direct ? (int)(m + 15) / 16 * 16 : m <= 32 ? 32 : m <= 64 ? 64 : m < 1024 || dt != DLA_BF16 ? 128 : 256;
    r.tile_n = direct ? kDirect : r.tile_m < 128 ? 128 : r.tile_m;
  }
  bool found = false;
  for (const Tile& t : kTiles) found |= t.m == r.tile_m && t.n == r.tile_n && legal(t, op, dt);
  if (!found) return DLA_ERR_UNSUPPORTED_PARAMS;
  if (r.splits == 0) r.splits = 1;
  const int64_t tiles = ((m + r.tile_m - 1) / r.tile_m) * ((out + r.tile_n - 1) / r.tile_n);
  if (tiles * r.splits > 0x7fffffff || terms > kMxMaxLd / 2) return DLA_ERR_TOO_LARGE;
  *plan = r;
  return DLA_SUCCESS;
}

size_t mx4_apply_bytes(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, int64_t n, int64_t k, const MxPlan& plan) {
  const int64_t terms = op == 0 ? k : n;
  const bool as_it_is = plan.tile_n == kDirect ? direct_takes(x, ldx, dt == DLA_F32 ? 4 : 2, terms) : whole(x, ldx, dt, terms);
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
