// C-ABI entry points of the microscaled operators (see include/dla.h): argument checks, schedules, workspaces.
#include "mx4_host.hpp"

using namespace dla;

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30;

int type_size(dla_dtype dt) { return dt == DLA_F32 ? 4 : dt == DLA_BF16 || dt == DLA_F16 ? 2 : 0; }
int64_t padded(int64_t cols) { return (cols + kMxStep - 1) / kMxStep * kMxStep; }

// 0, or which of (q, ldq, s, lds) is wrong (1 .. 4), or -1: a row too long for the kernels' offsets.
int check_mx(const void* q, int64_t ldq, const void* s, int64_t lds, int64_t rows, int64_t cols) {
  const bool empty = rows == 0 || cols == 0;
  if (!empty && (!q || (uintptr_t)q % 16)) return 1;
  if (ldq < padded(cols) / 2 || (!empty && ldq % 16)) return 2;
  if (!empty && (!s || (uintptr_t)s % 4)) return 3;
  if (lds < padded(cols) / 32 || (!empty && lds % 4)) return 4;
  if (ldq > kMxMaxLd || lds > kMxMaxLd) return -1;
  return 0;
}

bool bad_values(const void* x, dla_dtype dt) { return !x || (uintptr_t)x % (size_t)type_size(dt); }

}  // namespace

extern "C" {

int64_t mx4_padded(int64_t cols) { return cols > 0 && cols <= kMaxDim ? padded(cols) : 0; }

int mx4_quantize(const void* d_x, int64_t ldx, int64_t rows, int64_t cols, dla_dtype dt, void* d_q, int64_t ldq, void* d_s,
                 int64_t lds, void* d_qt, int64_t ldqt, void* d_st, int64_t ldst, void* hip_stream) {
  if (rows < 0) return -3;
  if (cols < 0) return -4;
  if (!type_size(dt)) return -5;
  if (rows > kMaxDim || cols > kMaxDim) return DLA_ERR_TOO_LARGE;
  const bool empty = rows == 0 || cols == 0;
  if (!empty && bad_values(d_x, dt)) return -1;
  if (ldx < (cols > 0 ? cols : 1)) return -2;
  const bool along = d_q || d_s, across = d_qt || d_st;
  int bad;
  if (along || !across) {
    if ((bad = check_mx(d_q, ldq, d_s, lds, rows, cols)) != 0) return bad < 0 ? DLA_ERR_TOO_LARGE : -5 - bad;
  }
  if (across) {
    if ((bad = check_mx(d_qt, ldqt, d_st, ldst, cols, rows)) != 0) return bad < 0 ? DLA_ERR_TOO_LARGE : -9 - bad;
  }
  if (empty) return DLA_SUCCESS;
  hip_clear_stale_error();
  return mx4_quantize_launch(d_x, ldx, rows, cols, dt, (uint8_t*)d_q, ldq, (uint8_t*)d_s, lds, (uint8_t*)d_qt, ldqt, (uint8_t*)d_st,
                             ldst, static_cast<hipStream_t>(hip_stream));
}

int mx4_dequantize(const void* d_q, int64_t ldq, const void* d_s, int64_t lds, int64_t rows, int64_t cols, dla_dtype dt, void* d_y,
                   int64_t ldy, void* hip_stream) {
  if (rows < 0) return -5;
  if (cols < 0) return -6;
  if (!type_size(dt)) return -7;
  if (rows > kMaxDim || cols > kMaxDim) return DLA_ERR_TOO_LARGE;
  const int bad = check_mx(d_q, ldq, d_s, lds, rows, cols);
  if (bad) return bad < 0 ? DLA_ERR_TOO_LARGE : -bad;
  const bool empty = rows == 0 || cols == 0;
  if (!empty && bad_values(d_y, dt)) return -8;
  if (ldy < (cols > 0 ? cols : 1)) return -9;
  if (empty) return DLA_SUCCESS;
  hip_clear_stale_error();
  const Mx4View w = {(const uint8_t*)d_q, (const uint8_t*)d_s, ldq, lds, (int)rows};
  return mx4_dequantize_launch(w, cols, dt, d_y, ldy, static_cast<hipStream_t>(hip_stream));
}

size_t mx4_gemm_workspace_bytes(int64_t m, int64_t n, int64_t k, const mx4_params* p) {
  MxPlan plan;
  if (m <= 0 || n <= 0 || k <= 0 || m > kMaxDim || n > kMaxDim || k > kMaxDim) return 0;
  if (mx4_gemm_plan(m, n, k, p, &plan) != DLA_SUCCESS) return 0;
  return mx4_parts_bytes(m, n, plan);
}

int mx4_gemm(int op, const void* d_a, int64_t lda, const void* d_sa, int64_t ldsa, const void* d_b, int64_t ldb, const void* d_sb,
             int64_t ldsb, void* d_c, int64_t ldc, int64_t m, int64_t n, int64_t k, dla_dtype dt, const mx4_params* p,
             void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (op != 0 && op != 1) return -1;
  if (m < 0) return -12;
  if (n < 0) return -13;
  if (k < 0) return -14;
  if (!type_size(dt)) return -15;
  if (m > kMaxDim || n > kMaxDim || k > kMaxDim) return DLA_ERR_TOO_LARGE;
  const bool empty = m == 0 || n == 0;
  int bad;
  if ((bad = check_mx(d_a, lda, d_sa, ldsa, n ? m : 0, k)) != 0) return bad < 0 ? DLA_ERR_TOO_LARGE : -1 - bad;
  if ((bad = check_mx(d_b, ldb, d_sb, ldsb, m ? n : 0, k)) != 0) return bad < 0 ? DLA_ERR_TOO_LARGE : -5 - bad;
  if (!empty && bad_values(d_c, dt)) return -10;
  if (ldc < (n > 0 ? n : 1)) return -11;
  MxPlan plan = {0, 0, 1};
  const int rc = mx4_gemm_plan(m > 0 ? m : 1, n > 0 ? n : 1, k > 0 ? k : 1, p, &plan);
  if (rc != DLA_SUCCESS) return rc;
  if (empty) return DLA_SUCCESS;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (k == 0) {
    hip_clear_stale_error();
    return op == 0 ? mx4_fill_zero_launch(d_c, ldc, m, n, dt, st) : DLA_SUCCESS;
  }
  const size_t need = mx4_parts_bytes(m, n, plan);
  if (need && (!d_workspace || (uintptr_t)d_workspace % 256 || workspace_bytes < need)) return DLA_ERR_WORKSPACE;
  hip_clear_stale_error();
  const Mx4View a = {(const uint8_t*)d_a, (const uint8_t*)d_sa, lda, ldsa, (int)m}, b = {(const uint8_t*)d_b, (const uint8_t*)d_sb, ldb, ldsb, (int)n};
  ProfileScope scope(PHASE_GEMM, 2.0 * (double)m * (double)n * (double)k, st);
  return mx4_gemm_launch(op == 1, a, b, d_c, ldc, k, dt, plan, (float*)d_workspace, st);
}

size_t mx4_apply_workspace_bytes(int op, const void* d_x, int64_t ldx, dla_dtype dt, int64_t m, int64_t n, int64_t k, const mx4_params* p) {
  MxPlan plan;
  if ((op != 0 && op != 1) || m <= 0 || n <= 0 || k <= 0 || m > kMaxDim || n > kMaxDim || k > kMaxDim || !type_size(dt)) return 0;
  if (mx4_apply_plan(op, m, n, k, dt, p, &plan) != DLA_SUCCESS) return 0;
  return mx4_apply_bytes(op, d_x, ldx, dt, m, n, k, plan);
}

int mx4_apply(int op, const void* d_x, int64_t ldx, dla_dtype dt, const void* d_w, int64_t ldw, const void* d_sw, int64_t ldsw,
              void* d_y, int64_t ldy, dla_dtype dt_y, int64_t m, int64_t n, int64_t k, const mx4_params* p, void* d_workspace,
              size_t workspace_bytes, void* hip_stream) {
  if (op != 0 && op != 1) return -1;
  if (!type_size(dt)) return -4;
  if (!type_size(dt_y)) return -11;
  if (m < 0) return -12;
  if (n < 0) return -13;
  if (k < 0) return -14;
  if (m > kMaxDim || n > kMaxDim || k > kMaxDim) return DLA_ERR_TOO_LARGE;
  const int64_t terms = op == 0 ? k : n, out = op == 0 ? n : k;
  const bool empty = m == 0 || out == 0;
  if (!empty && terms > 0 && bad_values(d_x, dt)) return -2;
  if (ldx < (terms > 0 ? terms : 1)) return -3;
  const int bad = check_mx(d_w, ldw, d_sw, ldsw, m ? n : 0, k);
  if (bad) return bad < 0 ? DLA_ERR_TOO_LARGE : -4 - bad;
  if (!empty && bad_values(d_y, dt_y)) return -9;
  if (ldy < (out > 0 ? out : 1)) return -10;
  MxPlan plan = {0, 0, 1};
  const int rc = mx4_apply_plan(op, m > 0 ? m : 1, n > 0 ? n : 1, k > 0 ? k : 1, dt, p, &plan);
  if (rc != DLA_SUCCESS) return rc;
  if (empty) return DLA_SUCCESS;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (terms == 0) {
    hip_clear_stale_error();
    return mx4_fill_zero_launch(d_y, ldy, m, out, dt_y, st);
  }
  const size_t need = mx4_apply_bytes(op, d_x, ldx, dt, m, n, k, plan);
  if (need && (!d_workspace || (uintptr_t)d_workspace % 256 || workspace_bytes < need)) return DLA_ERR_WORKSPACE;
  hip_clear_stale_error();
  const Mx4View w = {(const uint8_t*)d_w, (const uint8_t*)d_sw, ldw, ldsw, (int)n};
  ProfileScope scope(PHASE_GEMM, 2.0 * (double)m * (double)n * (double)k, st);
  return mx4_apply_launch(op, d_x, ldx, dt, m, w, k, d_y, ldy, dt_y, plan, d_workspace, st);
}

int mx4_enumerate_tiles(int kernel, int op, dla_dtype dt, mx4_params* out, int cap) {
  if ((op != 0 && op != 1) || !type_size(dt)) return 0;
  if (kernel == DLA_KERNEL_MX4_GEMM) return mx4_gemm_menu(out, cap);
  if (kernel == DLA_KERNEL_MX4_APPLY) return mx4_apply_menu(op, dt, out, cap);
  return 0;
}

int mx4_default_params(int kernel, int op, int64_t m, int64_t n, int64_t k, dla_dtype dt, mx4_params* out) {
  if (kernel != DLA_KERNEL_MX4_GEMM && kernel != DLA_KERNEL_MX4_APPLY) return -1;
  if (op != 0 && op != 1) return -2;
  if (m < 1 || m > kMaxDim) return -3;
  if (n < 1 || n > kMaxDim) return -4;
  if (k < 1 || k > kMaxDim) return -5;
  if (!type_size(dt)) return -6;
  if (!out) return -7;
  MxPlan plan;
  const int rc = kernel == DLA_KERNEL_MX4_GEMM ? mx4_gemm_plan(m, n, k, nullptr, &plan) : mx4_apply_plan(op, m, n, k, dt, nullptr, &plan);
  if (rc == DLA_SUCCESS) *out = mx4_params{plan.tile_m, plan.tile_n, plan.splits};
  return rc;
}

}  // extern "C"
