// Host side of the mx4_ kernels: what the entry points (mx4_api.hip) hand to the launch functions.
#pragma once
#include "host_common.hpp"
#include "mx4_common.hpp"

namespace dla {

// A schedule with everything filled in.
struct MxPlan {
  int tile_m, tile_n, splits;
};

// A launch has fewer than 2^32 threads; what needs more is refused.  Workgroups of 256 threads for `items`, or 0.
inline unsigned int mx4_grid_for(int64_t items, int64_t per_group) {
  const int64_t groups = (items + per_group - 1) / per_group;
  return groups < (int64_t)1 << 24 ? (unsigned int)groups : 0;
}

int mx4_quantize_launch(const void* x, int64_t ldx, int64_t rows, int64_t cols, dla_dtype dt, uint8_t* q, int64_t ldq, uint8_t* s,
                        int64_t lds, uint8_t* qt, int64_t ldqt, uint8_t* st, int64_t ldst, hipStream_t stream);
int mx4_dequantize_launch(const Mx4View& w, int64_t cols, dla_dtype dt, void* y, int64_t ldy, hipStream_t stream);

// C (m x n) = or += the sum over `splits` of parts (each m x n, fp32), in their order.
int mx4_join_launch(const float* parts, int splits, int64_t m, int64_t n, void* c, int64_t ldc, dla_dtype dt, bool onto, hipStream_t stream);
int mx4_fill_zero_launch(void* c, int64_t ldc, int64_t m, int64_t n, dla_dtype dt, hipStream_t stream);

int mx4_gemm_menu(mx4_params* out, int cap);
int mx4_gemm_plan(int64_t m, int64_t n, int64_t k, const mx4_params* p, MxPlan* plan);
int mx4_gemm_launch(bool onto, const Mx4View& a, const Mx4View& b, void* c, int64_t ldc, int64_t k, dla_dtype dt, const MxPlan& plan,
                    float* parts, hipStream_t stream);

int mx4_apply_menu(int op, dla_dtype dt, mx4_params* out, int cap);
int mx4_apply_plan(int op, int64_t m, int64_t n, int64_t k, dla_dtype dt, const mx4_params* p, MxPlan* plan);
int mx4_apply_launch(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, const Mx4View& w, int64_t k, void* y, int64_t ldy,
                     dla_dtype dt_y, const MxPlan& plan, void* workspace, hipStream_t stream);
size_t mx4_apply_bytes(int op, const void* x, int64_t ldx, dla_dtype dt, int64_t m, int64_t n, int64_t k, const MxPlan& plan);

inline size_t mx4_parts_bytes(int64_t m, int64_t n, const MxPlan& plan) {
  return plan.splits > 1 ? ((size_t)plan.splits * (size_t)m * (size_t)n * 4 + 255) / 256 * 256 : 0;
}

}  // namespace dla
