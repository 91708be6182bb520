// Entry points of the 8-bit layer's operators (include/stq.h): checks of the arguments, and one launch or two each.  Nothing is
// allocated, uploaded or waited for, and of the context only its device is used.
#include <cmath>

#include "stq_host.h"
#include "stq_operators.h"

using namespace stq;

namespace {

constexpr uint64_t kMost = 0x7FFFFFFFull;  // rows or columns

struct Wanted {
  uint64_t rows, cols;
  bool f32, bf16, q8;
  bool by_row;  // an 8-bit matrix with one scale for each row
};
constexpr Wanted floats(uint64_t rows, uint64_t cols) { return {rows, cols, true, true, false, false}; }
constexpr Wanted codes(uint64_t rows, uint64_t cols, bool by_row) { return {rows, cols, false, false, true, by_row}; }
constexpr Wanted any(uint64_t rows, uint64_t cols) { return {rows, cols, true, true, true, false}; }
Wanted of_type(uint64_t rows, uint64_t cols, uint32_t dtype) { return {rows, cols, dtype == STQ_F32, dtype == STQ_BF16, dtype == STQ_Q8, false}; }

// The size of the operator: that of one of its matrices.
int check_size(const stq_matrix* m) {
  if (!m) return STQ_EINVAL;
  return m->cols == 0 || m->cols > kMost || m->rows > kMost ? STQ_ESHAPE : STQ_OK;
}

int take(const stq_matrix* m, const Wanted& want, Mat* out) {
  if (!m) return STQ_EINVAL;
  const bool known = m->dtype == STQ_F32 || m->dtype == STQ_BF16 || m->dtype == STQ_Q8;
  if (!known || !(m->dtype == STQ_F32 ? want.f32 : (m->dtype == STQ_BF16 ? want.bf16 : want.q8))) return STQ_EDTYPE;
  if (m->rows != want.rows || m->cols != want.cols || m->stride < m->cols) return STQ_ESHAPE;
  uint64_t bytes;
  if (__builtin_mul_overflow(m->stride, (m->rows ? m->rows : 1) * 4, &bytes) || bytes > (1ull << 62)) return STQ_ESHAPE;
  const bool q8 = m->dtype == STQ_Q8;
  if (q8 && m->block != 0 && (want.by_row || lg_block(m->block) < 0)) return STQ_EBLOCK;
  if (m->rows && (!m->data || (q8 && !m->scales))) return STQ_EINVAL;
  if (!aligned(m->data, m->dtype == STQ_F32 ? 4 : (q8 ? 1 : 2)) || (q8 && !aligned(m->scales, 4))) return STQ_EALIGN;
  out->p = m->data;
  out->s = q8 ? m->scales : nullptr;
  out->stride = m->stride;
  out->lg = q8 && m->block ? static_cast<uint32_t>(lg_block(m->block)) : 0u;
  out->per_row = out->lg ? static_cast<uint32_t>((m->cols + m->block - 1) >> out->lg) : 1u;
  return STQ_OK;
}
int take_optional(const stq_matrix* m, const Wanted& want, Mat* out) {
  *out = Mat{};
  return m ? take(m, want, out) : STQ_OK;
}
// A vector or workspace on the device.
int check_buffer(const void* p, uintptr_t alignment) {
  if (!p) return STQ_EINVAL;
  return aligned(p, alignment) ? STQ_OK : STQ_EALIGN;
}
int launched(int error) { return error == 0 ? STQ_OK : STQ_EHIP; }

}  // namespace

extern "C" {

int stq_quantize_rows(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* out, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  RowsArgs a;
  if (int e = take(x, floats(x->rows, x->cols), &a.x)) return e;
  if (int e = take(out, codes(x->rows, x->cols, false), &a.out)) return e;
  a.rows = static_cast<uint32_t>(x->rows);
  a.cols = static_cast<uint32_t>(x->cols);
  if (!a.rows) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_quantize_rows(a, x->dtype, ctx->n_cu, stream));
}

int stq_dequantize_rows(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* out, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  RowsArgs a;
  if (int e = take(x, codes(x->rows, x->cols, false), &a.x)) return e;
  if (int e = take(out, floats(x->rows, x->cols), &a.out)) return e;
  a.rows = static_cast<uint32_t>(x->rows);
  a.cols = static_cast<uint32_t>(x->cols);
  if (!a.rows) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_dequantize_rows(a, out->dtype, ctx->n_cu, stream));
}

int stq_rms_norm(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* residual, const float* weight, float eps,
                 const stq_matrix* sum, const stq_matrix* y, const stq_matrix* saved, float* rstd, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  const uint64_t rows = x->rows, cols = x->cols;
  NormArgs a;
  if (int e = take(x, floats(rows, cols), &a.x)) return e;
  if (int e = take_optional(residual, of_type(rows, cols, x->dtype), &a.residual)) return e;
  if (int e = check_buffer(weight, 4)) return e;
  if (!(eps > 0.0f) || !std::isfinite(eps)) return STQ_EINVAL;
  if (int e = take_optional(sum, of_type(rows, cols, x->dtype), &a.sum)) return e;
  if (int e = take(y, codes(rows, cols, true), &a.y)) return e;
  if (int e = take_optional(saved, codes(rows, cols, false), &a.saved)) return e;
  if (!aligned(rstd, 4)) return STQ_EALIGN;
  a.weight = weight;
  a.rstd = rstd;
  a.eps = eps;
  a.rows = static_cast<uint32_t>(rows);
  a.cols = static_cast<uint32_t>(cols);
  if (!a.rows) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_rms_norm(a, x->dtype, ctx->n_cu, stream));
}

int stq_rms_norm_grad_bytes(uint64_t rows, uint64_t cols, uint64_t* bytes) {
  if (!bytes) return STQ_EINVAL;
  if (cols == 0 || cols > kMost || rows > kMost) return STQ_ESHAPE;
  *bytes = 4ull * norm_grad_groups(rows, static_cast<uint32_t>(cols)) * cols;
  return STQ_OK;
}

int stq_rms_norm_grad(stq_ctx* ctx, const stq_matrix* sum, const float* weight, const float* rstd, const stq_matrix* dy,
                      const stq_matrix* dresidual, const stq_matrix* dx, float* dweight, void* workspace,
                      uint64_t workspace_bytes, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(sum)) return e;
  const uint64_t rows = sum->rows, cols = sum->cols;
  NormGradArgs a;
  if (int e = take(sum, any(rows, cols), &a.sum)) return e;
  if (int e = check_buffer(weight, 4)) return e;
  if (int e = rows ? check_buffer(rstd, 4) : STQ_OK) return e;
  if (int e = take(dy, floats(rows, cols), &a.dy)) return e;
  if (int e = take_optional(dresidual, of_type(rows, cols, dy->dtype), &a.dres)) return e;
  if (int e = take(dx, of_type(rows, cols, dy->dtype), &a.dx)) return e;
  if (int e = check_buffer(dweight, 4)) return e;
  uint64_t need = 0;
  if (int e = stq_rms_norm_grad_bytes(rows, cols, &need)) return e;
  if (need) {
    if (workspace_bytes < need) return STQ_EINVAL;
    if (int e = check_buffer(workspace, 16)) return e;
  }
  a.weight = weight;
  a.rstd = rstd;
  a.dweight = dweight;
  a.partial = static_cast<float*>(workspace);
  a.rows = static_cast<uint32_t>(rows);
  a.cols = static_cast<uint32_t>(cols);
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_rms_norm_grad(a, sum->dtype, dy->dtype, stream));
}

int stq_gated_silu(stq_ctx* ctx, const stq_matrix* gate, const stq_matrix* up, const stq_matrix* y,
                   const stq_matrix* saved_gate, const stq_matrix* saved_up, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(gate)) return e;
  const uint64_t rows = gate->rows, cols = gate->cols;
  GatedArgs a;
  if (int e = take(gate, floats(rows, cols), &a.gate)) return e;
  if (int e = take(up, of_type(rows, cols, gate->dtype), &a.up)) return e;
  if (int e = take(y, codes(rows, cols, true), &a.y)) return e;
  if (!saved_gate != !saved_up) return STQ_EINVAL;
  if (int e = take_optional(saved_gate, codes(rows, cols, false), &a.saved_gate)) return e;
  if (int e = take_optional(saved_up, codes(rows, cols, false), &a.saved_up)) return e;
  if (saved_gate && saved_gate->block != saved_up->block) return STQ_EBLOCK;
  a.rows = static_cast<uint32_t>(rows);
  a.cols = static_cast<uint32_t>(cols);
  if (!a.rows) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_gated(a, gate->dtype, ctx->n_cu, stream));
}

int stq_gated_silu_grad(stq_ctx* ctx, const stq_matrix* gate, const stq_matrix* up, const stq_matrix* dy,
                        const stq_matrix* dgate, const stq_matrix* dup, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(gate)) return e;
  const uint64_t rows = gate->rows, cols = gate->cols;
  GatedGradArgs a;
  if (int e = take(gate, any(rows, cols), &a.gate)) return e;
  if (int e = take(up, of_type(rows, cols, gate->dtype), &a.up)) return e;
  if (gate->dtype == STQ_Q8 && gate->block != up->block) return STQ_EBLOCK;
  if (int e = take(dy, floats(rows, cols), &a.dy)) return e;
  if (int e = take(dgate, of_type(rows, cols, dy->dtype), &a.dgate)) return e;
  if (int e = take(dup, of_type(rows, cols, dy->dtype), &a.dup)) return e;
  a.rows = static_cast<uint32_t>(rows);
  a.cols = static_cast<uint32_t>(cols);
  if (!a.rows) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_gated_grad(a, gate->dtype, dy->dtype, ctx->n_cu, stream));
}

int stq_matmul(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* w, const stq_matrix* out, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  if (int e = check_size(w)) return e;
  if (w->rows == 0 || x->cols > STQ_MAX_INNER) return STQ_ESHAPE;
  MatmulArgs a;
  if (int e = take(x, codes(x->rows, x->cols, true), &a.a)) return e;
  if (int e = take(w, codes(w->rows, x->cols, true), &a.b)) return e;
  if (int e = take(out, floats(x->rows, w->rows), &a.out)) return e;
  a.m = static_cast<uint32_t>(x->rows);
  a.n = static_cast<uint32_t>(w->rows);
  a.k = static_cast<uint32_t>(x->cols);
  if (!a.m) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_matmul(a, out->dtype, ctx->n_cu, stream));
}

int stq_matmul_grad_input(stq_ctx* ctx, const stq_matrix* dy, const stq_matrix* w, const stq_matrix* dx, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(dy)) return e;
  if (int e = check_size(w)) return e;
  MatmulArgs a;
  if (int e = take(dy, floats(dy->rows, dy->cols), &a.a)) return e;
  if (int e = take(w, codes(dy->cols, w->cols, true), &a.b)) return e;
  if (int e = take(dx, floats(dy->rows, w->cols), &a.out)) return e;
  a.m = static_cast<uint32_t>(dy->rows);
  a.n = static_cast<uint32_t>(dy->cols);
  a.k = static_cast<uint32_t>(w->cols);
  if (!a.m) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_matmul_grad_input(a, dy->dtype, dx->dtype, stream));
}

int stq_matmul_grad_weight_bytes(uint64_t tokens, uint64_t outputs, uint64_t inputs, uint64_t* bytes) {
  if (!bytes) return STQ_EINVAL;
  if (tokens > kMost || outputs == 0 || outputs > kMost || inputs == 0 || inputs > kMost) return STQ_ESHAPE;
  *bytes = grad_weight_bytes(tokens, outputs, inputs);
  return STQ_OK;
}

int stq_matmul_grad_weight(stq_ctx* ctx, const stq_matrix* dy, const stq_matrix* x, const stq_matrix* dw, void* workspace,
                           uint64_t workspace_bytes, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(dy)) return e;
  if (int e = check_size(x)) return e;
  MatmulArgs a;
  if (int e = take(dy, floats(dy->rows, dy->cols), &a.a)) return e;
  if (int e = take(x, codes(dy->rows, x->cols, true), &a.b)) return e;
  if (int e = take(dw, floats(dy->cols, x->cols), &a.out)) return e;
  uint64_t need = 0;
  if (int e = stq_matmul_grad_weight_bytes(dy->rows, dy->cols, x->cols, &need)) return e;
  if (need) {
    if (workspace_bytes < need) return STQ_EINVAL;
    if (int e = check_buffer(workspace, 16)) return e;
  }
  a.m = static_cast<uint32_t>(dy->rows);
  a.n = static_cast<uint32_t>(dy->cols);
  a.k = static_cast<uint32_t>(x->cols);
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_matmul_grad_weight(a, dy->dtype, dw->dtype, need ? static_cast<float*>(workspace) : nullptr, stream));
}

int stq_cross_entropy_bytes(uint64_t tokens, uint64_t classes, uint64_t inputs, uint64_t* bytes) {
  if (!bytes) return STQ_EINVAL;
  if (tokens > kMost || classes == 0 || classes > kMost || inputs == 0 || inputs > STQ_MAX_INNER) return STQ_ESHAPE;
  *bytes = loss_bytes(tokens, classes);
  return STQ_OK;
}

int stq_cross_entropy(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* w, const int64_t* targets, float* loss, float* lse,
                      void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  if (int e = check_size(w)) return e;
  if (w->rows == 0 || x->cols > STQ_MAX_INNER) return STQ_ESHAPE;
  LossArgs a;
  if (int e = take(x, codes(x->rows, x->cols, true), &a.x)) return e;
  if (int e = take(w, codes(w->rows, x->cols, true), &a.w)) return e;
  if (!x->rows) return STQ_OK;
  if (int e = check_buffer(targets, 8)) return e;
  if (int e = check_buffer(loss, 4)) return e;
  if (int e = check_buffer(lse, 4)) return e;
  uint64_t need = 0;
  if (int e = stq_cross_entropy_bytes(x->rows, w->rows, x->cols, &need)) return e;
  if (workspace_bytes < need) return STQ_EINVAL;
  if (int e = check_buffer(workspace, 16)) return e;
  a.targets = targets;
  a.loss = loss;
  a.lse = lse;
  a.tokens = static_cast<uint32_t>(x->rows);
  a.classes = static_cast<uint32_t>(w->rows);
  a.inputs = static_cast<uint32_t>(x->cols);
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_loss(a, workspace, ctx->n_cu, stream));
}

int stq_cross_entropy_grad_bytes(uint64_t tokens, uint64_t classes, uint64_t inputs, uint64_t* bytes) {
  if (!bytes) return STQ_EINVAL;
  if (tokens > kMost || classes == 0 || classes > kMost || inputs == 0 || inputs > STQ_MAX_INNER) return STQ_ESHAPE;
  *bytes = loss_grad_bytes(tokens, classes, inputs);
  return STQ_OK;
}

int stq_cross_entropy_grad(stq_ctx* ctx, const stq_matrix* x, const stq_matrix* w, const int64_t* targets, const float* loss,
                           const float* lse, const float* dloss, const float* dlse, const stq_matrix* dx, const stq_matrix* dw,
                           void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!ctx) return STQ_EINVAL;
  if (int e = check_size(x)) return e;
  if (int e = check_size(w)) return e;
  if (w->rows == 0 || x->cols > STQ_MAX_INNER) return STQ_ESHAPE;
  LossGradArgs a{};
  if (int e = take(x, codes(x->rows, x->cols, true), &a.x)) return e;
  if (int e = take(w, codes(w->rows, x->cols, true), &a.w)) return e;
  if (!dx && !dw) return STQ_EINVAL;
  if (int e = take_optional(dx, floats(x->rows, x->cols), &a.dx)) return e;
  if (int e = take_optional(dw, floats(w->rows, x->cols), &a.dw)) return e;
  if (x->rows) {
    if (int e = check_buffer(targets, 8)) return e;
    if (int e = check_buffer(loss, 4)) return e;
    if (int e = check_buffer(lse, 4)) return e;
    if (int e = check_buffer(dloss, 4)) return e;
    if (!aligned(dlse, 4)) return STQ_EALIGN;
    uint64_t need = 0;
    if (int e = stq_cross_entropy_grad_bytes(x->rows, w->rows, x->cols, &need)) return e;
    if (workspace_bytes < need) return STQ_EINVAL;
    if (int e = check_buffer(workspace, 16)) return e;
  }
  a.targets = targets;
  a.loss = loss;
  a.lse = lse;
  a.dloss = dloss;
  a.dlse = dlse;
  a.tokens = static_cast<uint32_t>(x->rows);
  a.classes = static_cast<uint32_t>(w->rows);
  a.inputs = static_cast<uint32_t>(x->cols);
  if (!a.tokens && !dw) return STQ_OK;
  DeviceGuard g(ctx->device);
  if (!g.ok) return STQ_EHIP;
  return launched(launch_loss_grad(a, dx ? dx->dtype : 0u, dw ? dw->dtype : 0u, workspace, ctx->n_cu, stream));
}

}  // extern "C"
