// Which schedule a microscaled product runs where the caller names none.
#pragma once
#include "mx4_host.hpp"

namespace dla {

// A tile and what a launch of it costs, in us (at the clocks of short calls: a product of many tiles, for which the power that they draw brings
// the clocks down, takes longer, 4096 x 8192 x 8192 of mx4_apply in bf16 414 to 430 us for 311 here; only the order of tiles counts): start + max(first + step * steps, each * (more + unit * steps)) for workgroups of `steps` times 128
// terms, `each` of them to a compute unit (their number over 256, rounded up): the chain of one workgroup's steps, or the units' work.
struct MxTileCost {
  int m, n;
  float start, first, step, unit, more;
};

constexpr int kMxMaxSplits = 32;

// Joining split sums costs a launch and the parts' way to memory and back, at 4 TB/s.
constexpr float kMxJoin = 2.0f, kMxJoinPerByte = 0.25e-6f;

// Fills in what the caller left 0: the tile of `tiles` (`count` of them, all legal) and the splits with the least cost.  rows x cols: the
// result; terms: of the sum.
inline int mx4_choose(const MxTileCost* tiles, int count, int64_t rows, int64_t cols, int64_t terms, const mx4_params* p, MxPlan* plan) {
  MxPlan r = {0, 0, 0};
  if (p) r = MxPlan{p->tile_m, p->tile_n, p->splits};
  const int64_t steps = (terms + kMxStep - 1) / kMxStep;
  if (r.tile_m < 0 || r.tile_n < 0 || r.splits < 0 || r.splits > kMxMaxSplits || r.splits > steps) return DLA_ERR_UNSUPPORTED_PARAMS;
  static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  float best = 0.0f;
  bool found = false, large = false;
  for (int i = 0; i < count; ++i) {
    const MxTileCost& t = tiles[i];
    if ((r.tile_m || r.tile_n) && (t.m != r.tile_m || t.n != r.tile_n)) continue;
    const int64_t groups = ((rows + t.m - 1) / t.m) * ((cols + t.n - 1) / t.n);
    for (int s : kSplits) {
      if (r.splits) s = r.splits;
      // (launches have fewer than 2^32 threads: up to 512 a tile here, one to an element where parts are joined; parts of more than
      // 2^26 values are not chosen, but may be named)
      const double values = (double)rows * (double)cols * s;
      const bool fits = groups * s < (int64_t)1 << 23 && (s == 1 || (values < 4.0e9 * s && (r.splits || values <= (double)(1 << 26))));
      if (s <= steps && fits) {
        const float each = (float)((groups * s + 255) / 256), n = (float)((steps + s - 1) / s);
        const float chain = t.first + t.step * n, work = each * (t.more + t.unit * n);
        float cost = t.start + (chain > work ? chain : work);
        if (s > 1) cost += kMxJoin + kMxJoinPerByte * (float)rows * (float)cols * (4.0f * s + 6.0f);
        if (!found || cost < best) {
          best = cost;
          *plan = MxPlan{t.m, t.n, s};
        }
        found = true;
      } else if (s <= steps) {
        large = true;
      }
      if (r.splits || groups >= 2048) break;
    }
  }
  return found ? DLA_SUCCESS : large ? DLA_ERR_TOO_LARGE : DLA_ERR_UNSUPPORTED_PARAMS;
}

}  // namespace dla
