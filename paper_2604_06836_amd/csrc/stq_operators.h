// What the host side and the kernels of the 8-bit layer's operators share.
#pragma once
#include <cstdint>

namespace stq {

enum MatrixType : uint32_t { kF32 = 0, kBF16 = 1, kQ8 = 2 };

// A matrix as the kernels see it: rows of `stride` elements; the scales of an 8-bit one, `per_row` for each row, one for
// each 2^lg columns (lg = 0: per_row = 1, one for the row).
struct Mat {
  void* p;
  float* s;
  uint64_t stride;
  uint32_t per_row, lg;
};

struct RowsArgs {  // quantize, dequantize
  Mat x, out;
  uint32_t rows, cols;
};
struct NormArgs {
  Mat x, residual, sum, y, saved;  // p null: not there
  const float* weight;
  float* rstd;
  float eps;
  uint32_t rows, cols;
};
struct NormGradArgs {
  Mat sum, dy, dres, dx;
  const float* weight;
  const float* rstd;
  float* dweight;
  float* partial;   // [groups][cols]
  uint32_t rows, cols;
};
struct GatedArgs {
  Mat gate, up, y, saved_gate, saved_up;
  uint32_t rows, cols;
};
struct GatedGradArgs {
  Mat gate, up, dy, dgate, dup;
  uint32_t rows, cols;
};
// out[m][n] = sum over k of a[m][k] b[n][k] and its gradients: m tokens, n outputs, k inputs.
struct MatmulArgs {
  Mat a, b, out;
  uint32_t m, n, k;
};

// Workgroups of the norm's gradients, each of which leaves a part of dweight: as many as have 16 waves on each of 256 CUs.
inline uint32_t norm_grad_groups(uint64_t rows, uint32_t cols) {
  const uint64_t at_once = cols <= 512 ? 4 : 1, need = (rows + at_once - 1) / at_once;  // (rows of a workgroup, see with_rows)
  const uint32_t waves = cols <= 512 ? 4 : (cols <= 8192 ? (cols + 511) / 512 : 16), most = 4096 / waves;
  return need < most ? static_cast<uint32_t>(need) : most;
}

// Launchers; `stream` is a hipStream_t.  Return a hipError_t as int.  rows, m > 0.
int launch_quantize_rows(const RowsArgs& a, uint32_t type, uint32_t n_cu, void* stream);
int launch_dequantize_rows(const RowsArgs& a, uint32_t type, uint32_t n_cu, void* stream);
int launch_rms_norm(const NormArgs& a, uint32_t type, uint32_t n_cu, void* stream);
int launch_rms_norm_grad(NormGradArgs a, uint32_t sum_type, uint32_t type, void* stream);
int launch_gated(const GatedArgs& a, uint32_t type, uint32_t n_cu, void* stream);
int launch_gated_grad(const GatedGradArgs& a, uint32_t kept_type, uint32_t type, uint32_t n_cu, void* stream);
int launch_matmul(const MatmulArgs& a, uint32_t out_type, uint32_t n_cu, void* stream);
int launch_matmul_grad_input(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, void* stream);
int launch_matmul_grad_weight(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, float* workspace, void* stream);
uint64_t grad_weight_bytes(uint64_t m, uint64_t n, uint64_t k);

}  // namespace stq
