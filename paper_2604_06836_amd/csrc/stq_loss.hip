// gfx950 kernels of the softmax cross entropy over 8-bit codes.  The classes are taken in pieces, of which the logits lie in the
// workspace: each leaves a maximum and a sum for every token, which a last kernel joins.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_vectors.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

constexpr uint32_t kNoTarget = 0xFFFFFFFFu;
constexpr float kLog2e = 1.44269504088896340736f;

// The class of a token's target, or kNoTarget; one beyond the classes comes out as no class either, and is told apart by `beyond`.
__device__ __forceinline__ uint32_t target_of(const int64_t* targets, uint32_t token, uint32_t classes, bool* beyond) {
  const int64_t t = as_global(targets)[token];
  *beyond = t >= static_cast<int64_t>(classes);
  return t < 0 || *beyond ? kNoTarget : static_cast<uint32_t>(t);
}

// Largest element and sum over a workgroup of four waves.
__device__ __forceinline__ float group_max(float x, float* held) {
  for (int o = 1; o < 64; o *= 2) x = fmaxf(x, __shfl_xor(x, o));
  if ((threadIdx.x & 63) == 0) held[threadIdx.x >> 6] = x;
  __syncthreads();
  x = fmaxf(fmaxf(held[0], held[1]), fmaxf(held[2], held[3]));
  __syncthreads();
  return x;
}
__device__ __forceinline__ float group_sum(float x, float* held) {
  for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o);
  if ((threadIdx.x & 63) == 0) held[threadIdx.x >> 6] = x;
  __syncthreads();
  x = (held[0] + held[1]) + (held[2] + held[3]);
  __syncthreads();
  return x;
}

// A workgroup to a token's logits of a piece, classes first .. first + n - 1: their maximum and the sum of exp(z - maximum), both without
// the target, and the target's logit if it is one of them.
__global__ __launch_bounds__(256) void piece_kernel(const float* z, uint32_t first, uint32_t n, uint32_t classes, const int64_t* targets, float2* part, float* at_target) {
  __shared__ float held[4];
  const uint32_t token = blockIdx.x;
  bool beyond;
  const uint32_t target = target_of(targets, token, classes, &beyond) - first;
  const STQ_GLOBAL float* row = as_global(z) + static_cast<uint64_t>(token) * n;
  float most = -INFINITY;
  bool nan = false;
  for (uint32_t c = threadIdx.x; c < n; c += 256) {
    const float x = row[c];
    nan |= __builtin_isnan(x);
    if (c == target) at_target[token] = x;
    else most = fmaxf(most, x);
  }
  most = group_max(most, held);
  float sum = 0.0f;
  for (uint32_t c = threadIdx.x; c < n; c += 256)
    if (c != target) sum += __builtin_amdgcn_exp2f((row[c] - most) * kLog2e);
  if (nan) sum = NAN;
  sum = group_sum(sum, held);
  if (threadIdx.x == 0) part[token] = make_float2(most, most == -INFINITY && !__builtin_isnan(sum) ? 0.0f : sum);
}

// The parts of each token's sum in one order, its loss and its log-sum.
__global__ __launch_bounds__(256) void join_kernel(const float2* part, const float* at_target, uint32_t parts, uint32_t tokens, uint32_t classes, const int64_t* targets,
                                                   float* loss, float* lse) {
  const uint32_t token = blockIdx.x * 256 + threadIdx.x;
  if (token >= tokens) return;
  float most = -INFINITY;
  for (uint32_t p = 0; p < parts; ++p) most = fmaxf(most, part[static_cast<uint64_t>(p) * tokens + token].x);
  float sum = 0.0f;
  for (uint32_t p = 0; p < parts; ++p) {
    const float2 v = part[static_cast<uint64_t>(p) * tokens + token];
    sum += v.y * (v.x == most ? 1.0f : __builtin_amdgcn_exp2f((v.x - most) * kLog2e));
  }
  const float others = sum == 0.0f ? -INFINITY : most + logf(sum);
  bool beyond;
  if (target_of(targets, token, classes, &beyond) == kNoTarget) {
    lse[token] = others;
    loss[token] = beyond ? NAN : 0.0f;
    return;
  }
  // log(1 + exp(d)), d = others - target
  const float z = at_target[token], d = others - z, small = log1pf(expf(-fabsf(d)));
  loss[token] = fmaxf(d, 0.0f) + small;
  lse[token] = d == d ? fmaxf(others, z) + small : d;
}

// What a token's gradients need: lse, dloss + dlse, the gradient of the target's logit and the target's class; and the scale of its
// codes, or 0 where the token takes no part.
__global__ __launch_bounds__(256) void tokens_kernel(LossGradArgs a) {
  const uint32_t token = blockIdx.x * 256 + threadIdx.x;
  if (token >= a.tokens) return;
  bool beyond;
  const uint32_t target = target_of(a.targets, token, a.classes, &beyond);
  const float dlse = a.dlse ? as_global(a.dlse)[token] : 0.0f, dloss = beyond ? NAN : (target == kNoTarget ? 0.0f : as_global(a.dloss)[token]);
  const float loss = as_global(a.loss)[token];
  const bool part = !(dlse == 0.0f && dloss == 0.0f);
  static_cast<float4*>(a.token)[token] = make_float4(as_global(a.lse)[token], part ? dloss + dlse : 0.0f, dlse * expf(-loss) + dloss * expm1f(-loss), u2f(part ? target : kNoTarget));
  a.scale[token] = part ? as_global(a.x.s)[token] : 0.0f;
}

// Logits of a piece to their gradients.
__global__ __launch_bounds__(256) void softmax_grad_kernel(float* z, uint32_t first, uint32_t n, const float4* tokens) {
  const float4 t = tokens[blockIdx.x];
  const uint32_t target = f2u(t.w) - first;
  float* row = z + static_cast<uint64_t>(blockIdx.x) * n;
  for (uint32_t c = threadIdx.x; c < n; c += 256) {
    const float g = t.y * __builtin_amdgcn_exp2f((row[c] - t.x) * kLog2e);
    row[c] = t.y == 0.0f ? 0.0f : g;
    if (c == target) row[c] = t.z;
  }
}

// out[i][j] (+)= sum over c of g(i, c) * s(c) * q(c, j), a thread to an element: with respect to x i is the token and c the class, with
// respect to w (WEIGHT) i is the class and c the token.  g: [tokens][n].
template <bool WEIGHT, uint32_t TO>
__global__ __launch_bounds__(256) void product_kernel(const float* g, uint32_t n, const Mat q, const Mat out, float* sum, bool first, bool last, uint32_t ni, uint32_t nj, uint32_t nc) {
  using T = typename Elem<TO>::type;
  const uint64_t total = static_cast<uint64_t>(ni) * nj;
  for (uint64_t t = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; t < total; t += static_cast<uint64_t>(gridDim.x) * 256) {
    const uint64_t i = t / nj, j = t % nj;
    float v = first ? 0.0f : sum[t];
    for (uint64_t c = 0; c < nc; ++c)
      v = fmaf(as_global(g)[WEIGHT ? c * n + i : i * n + c] * as_global(q.s)[c], static_cast<float>(as_global(static_cast<const int8_t*>(q.p))[c * q.stride + j]), v);
    if (last) as_global(static_cast<T*>(out.p))[i * out.stride + j] = static_cast<T>(v);
    else sum[t] = v;
  }
}
template <bool WEIGHT>
void product(uint32_t to, const float* g, uint32_t n, const Mat& q, const Mat& out, float* sum, bool first, bool last, uint32_t ni, uint32_t nj, uint32_t nc, hipStream_t st) {
  const uint64_t groups = (static_cast<uint64_t>(ni) * nj + 255) / 256;
  const uint32_t grid = static_cast<uint32_t>(groups < 65536 ? groups : 65536);
  if (to == kF32) product_kernel<WEIGHT, kF32><<<grid, 256, 0, st>>>(g, n, q, out, sum, first, last, ni, nj, nc);
  else product_kernel<WEIGHT, kBF16><<<grid, 256, 0, st>>>(g, n, q, out, sum, first, last, ni, nj, nc);
}

// Classes of a piece: of as many logits as 256 MiB hold in fp32, and of one size.
constexpr uint64_t kPieceLogits = 1ull << 26, kLeastPiece = 1024;
uint64_t piece_of(uint64_t tokens, uint64_t classes) {
  uint64_t most = kPieceLogits / (tokens ? tokens : 1);
  if (most < kLeastPiece) most = kLeastPiece;
  const uint64_t pieces = (classes + most - 1) / most, each = (classes + pieces - 1) / pieces;
  return each < classes ? (each + 255) / 256 * 256 : classes;
}
uint64_t whole(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

struct Arena {  // parts of the workspace
  char* at;
  template <class T>
  T* take(uint64_t n) {
    T* const p = reinterpret_cast<T*>(at);
    at += whole(n * sizeof(T));
    return p;
  }
};
Mat rows_from(const Mat& m, uint64_t row) {
  Mat r = m;
  r.p = static_cast<int8_t*>(m.p) + row * m.stride;
  r.s = m.s + row;
  return r;
}

}  // namespace

uint64_t loss_bytes(uint64_t tokens, uint64_t classes) {
  const uint64_t piece = piece_of(tokens, classes), parts = (classes + piece - 1) / piece;
  return tokens ? whole(8 * parts * tokens) + whole(4 * tokens) + whole(4 * piece * tokens) : 0;
}

int launch_loss(const LossArgs& a, void* workspace, uint32_t n_cu, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t piece = static_cast<uint32_t>(piece_of(a.tokens, a.classes)), parts = (a.classes + piece - 1) / piece;
  Arena arena{static_cast<char*>(workspace)};
  float2* const part = arena.take<float2>(static_cast<uint64_t>(parts) * a.tokens);
  float* const at_target = arena.take<float>(a.tokens);
  float* const z = arena.take<float>(static_cast<uint64_t>(piece) * a.tokens);
  for (uint32_t p = 0; p < parts; ++p) {
    const uint32_t first = p * piece, n = a.classes - first < piece ? a.classes - first : piece;
    const MatmulArgs m{a.x, rows_from(a.w, first), Mat{z, nullptr, n, 0, 0}, a.tokens, n, a.inputs};
    if (int e = launch_matmul(m, kF32, n_cu, stream)) return e;
    piece_kernel<<<a.tokens, 256, 0, st>>>(z, first, n, a.classes, a.targets, part + static_cast<uint64_t>(p) * a.tokens, at_target);
  }
  join_kernel<<<(a.tokens + 255) / 256, 256, 0, st>>>(part, at_target, parts, a.tokens, a.classes, a.targets, a.loss, a.lse);
  return hipGetLastError();
}

uint64_t loss_grad_bytes(uint64_t tokens, uint64_t classes, uint64_t inputs) {
  const uint64_t piece = piece_of(tokens, classes);
  return tokens ? whole(16 * tokens) + whole(4 * tokens) + whole(4 * piece * tokens) + whole(4 * tokens * inputs) : 0;
}

int launch_loss_grad(LossGradArgs a, uint32_t dx_type, uint32_t dw_type, void* workspace, uint32_t n_cu, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t piece = static_cast<uint32_t>(piece_of(a.tokens, a.classes)), parts = (a.classes + piece - 1) / piece;
  Arena arena{static_cast<char*>(workspace)};
  a.token = arena.take<float4>(a.tokens);
  a.scale = arena.take<float>(a.tokens);
  float* const z = arena.take<float>(static_cast<uint64_t>(piece) * a.tokens);
  float* const sum = arena.take<float>(static_cast<uint64_t>(a.tokens) * a.inputs);
  if (a.tokens) tokens_kernel<<<(a.tokens + 255) / 256, 256, 0, st>>>(a);
  Mat x = a.x;
  x.s = a.scale;
  for (uint32_t p = 0; p < parts; ++p) {
    const uint32_t first = p * piece, n = a.classes - first < piece ? a.classes - first : piece;
    const Mat g{z, nullptr, n, 0, 0}, w = rows_from(a.w, first);
    if (a.tokens) {
      if (int e = launch_matmul(MatmulArgs{a.x, w, g, a.tokens, n, a.inputs}, kF32, n_cu, stream)) return e;
      softmax_grad_kernel<<<a.tokens, 256, 0, st>>>(z, first, n, static_cast<const float4*>(a.token));
    }
    if (a.dx.p && a.tokens) product<false>(dx_type, z, n, w, a.dx, sum, p == 0, p + 1 == parts, a.tokens, a.inputs, n, st);
    if (a.dw.p) {
      Mat dw = a.dw;
      dw.p = static_cast<char*>(a.dw.p) + static_cast<uint64_t>(first) * a.dw.stride * (dw_type == kF32 ? 4 : 2);
      product<true>(dw_type, z, n, x, dw, nullptr, true, true, n, a.inputs, a.tokens, st);
    }
  }
  return hipGetLastError();
}

}  // namespace stq
