// gfx950 kernels of the 8-bit layer that work on rows: conversion to codes and back, the root-mean-square norm with the
// residual's addition and its gradients, the gated activation and its gradients.
//
// All are bound by memory: every matrix is read once and written once.  A thread owns vectors of eight neighbouring columns, so
// that a vector has one scale (blocks are 64, 128 or 256 columns) and is one load of 8 (codes), 16 (bf16) or 32 bytes.  Kernels
// that need a maximum or a sum over a row hold the row in registers between the two: a wave for a row of up to 1024 columns,
// without any barrier, a workgroup of 256 to 1024 threads for longer ones, with one barrier for a row.  Unaligned vectors are the
// hardware's to split; only the last vector of a row whose columns are no multiple of eight goes element by element.  Rows of over
// 16384 columns are not held but read again, out of the caches.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "stq_operators.h"
#include "stq_wave.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

constexpr float kLeast = 0x1p-100f;  // what a group's largest magnitude counts as at least
constexpr uint32_t kInf = 0x7F800000u;

// ---------------------------------------------------------------------------------------------- vectors of eight columns
template <uint32_t TY> struct Elem;
template <> struct Elem<kF32> { using type = float; };
template <> struct Elem<kBF16> { using type = __bf16; };
template <> struct Elem<kQ8> { using type = int8_t; };

// Columns c .. c+7 of a row, as they are stored; beyond the row's end zeros, and nothing is read there.
template <class T>
struct Raw { T e[8]; };
template <class T>
__device__ __forceinline__ Raw<T> load_raw(const T* row, uint32_t c, uint32_t cols) {
  Raw<T> r;
  const STQ_GLOBAL T* p = as_global(row) + c;
  if (c + 8 <= cols) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) r.e[i] = c + i < cols ? p[i] : static_cast<T>(0);
  }
  return r;
}
template <class T>
__device__ __forceinline__ void store_raw(T* row, uint32_t c, uint32_t cols, const Raw<T>& r) {
  STQ_GLOBAL T* p = as_global(row) + c;
  if (c + 8 <= cols) {
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (c + i < cols) p[i] = r.e[i];
  }
}
template <class T>
__device__ __forceinline__ T* row_of(const Mat& m, uint32_t row) { return static_cast<T*>(m.p) + static_cast<uint64_t>(row) * m.stride; }
__device__ __forceinline__ float* scale_of(const Mat& m, uint32_t row, uint32_t c) {
  return m.s + static_cast<uint64_t>(row) * m.per_row + (m.lg ? c >> m.lg : 0u);
}

template <uint32_t TY>
__device__ __forceinline__ void load8(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, float (&v)[8]) {
  using T = typename Elem<TY>::type;
  const Raw<T> r = load_raw(row_of<T>(m, row), c, cols);
  if constexpr (TY == kQ8) {
    const float s = c < cols ? as_global(scale_of(m, row, c))[0] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = s * static_cast<float>(r.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(r.e[i]);
  }
}
template <uint32_t TY>
__device__ __forceinline__ void store8(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, const float (&v)[8]) {
  using T = typename Elem<TY>::type;
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.e[i] = static_cast<T>(v[i]);
  store_raw(row_of<T>(m, row), c, cols, r);
}
// v as the matrix' type holds it
template <uint32_t TY>
__device__ __forceinline__ float rounded(float v) {
  if constexpr (TY == kBF16) return static_cast<float>(static_cast<__bf16>(v));
  return v;
}

// ---------------------------------------------------------------------------------------------- codes
// Largest magnitudes are kept as bit patterns: as whole numbers they are ordered as the values are, with infinities and NaN above
// every finite value, so that one comparison at the end sees them all.
__device__ __forceinline__ uint32_t magnitude(float v) { return f2u(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t largest8(const float (&v)[8]) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, magnitude(v[i]));
  return a;
}

// How a group's elements become codes: q = rint(x * inv); scale = largest / 127.
struct Coder { float inv, scale; uint32_t keep; };
__device__ __forceinline__ Coder coder_of(uint32_t largest) {
  const float a = fmaxf(u2f(largest), kLeast);
  const bool finite = largest < kInf;
  return {127.0f / a, finite ? a / 127.0f : __builtin_nanf(""), finite ? 0xFFFFFFFFu : 0u};
}
// rint by the addition of 1.5 * 2^23: the low byte of the sum is the code in two's complement
__device__ __forceinline__ uint32_t code_byte(float x, float inv) { return f2u(x * inv + 12582912.0f); }
__device__ __forceinline__ uint32_t codes4(const float* x, float inv, uint32_t keep) {
  const uint32_t lo = __builtin_amdgcn_perm(code_byte(x[1], inv), code_byte(x[0], inv), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(code_byte(x[3], inv), code_byte(x[2], inv), 0x04000C0Cu);
  return (lo | hi) & keep;
}
__device__ __forceinline__ void store_codes(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, const float (&v)[8], const Coder& k) {
  const uint32_t w[2] = {codes4(v, k.inv, k.keep), codes4(v + 4, k.inv, k.keep)};
  Raw<int8_t> r;
  __builtin_memcpy(&r, w, 8);
  store_raw(row_of<int8_t>(m, row), c, cols, r);
}
// Codes with a scale for each block: the maximum over the block's 8, 16 or 32 neighbouring threads (all lanes take part).
__device__ __forceinline__ void store_block_codes(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, const float (&v)[8]) {
  uint32_t a = octet_max(largest8(v));
  if (m.lg > 6) a = max(a, dpp_u32<kDppMirror>(a));
  if (m.lg > 7) a = max(a, static_cast<uint32_t>(__shfl_xor(static_cast<int>(a), 16)));
  const Coder k = coder_of(a);
  if (c < cols) {
    store_codes(m, row, c, cols, v, k);
    if ((c & ((1u << m.lg) - 1u)) == 0) as_global(scale_of(m, row, c))[0] = k.scale;
  }
}

// ---------------------------------------------------------------------------------------------- reductions over a row
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = row_max(x);
  const uint32_t a = max(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16));
  const uint32_t b = max(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48));
  return max(a, b);
}
__device__ __forceinline__ float wave_sum(float x) {
  x += u2f(dpp_u32<kDppXor1>(f2u(x)));
  x += u2f(dpp_u32<kDppXor2>(f2u(x)));
  x += u2f(dpp_u32<kDppHalfMirror>(f2u(x)));
  x += u2f(dpp_u32<kDppMirror>(f2u(x)));
  const uint32_t u = f2u(x);
  const float a = u2f(__builtin_amdgcn_readlane(u, 0)) + u2f(__builtin_amdgcn_readlane(u, 16));
  const float b = u2f(__builtin_amdgcn_readlane(u, 32)) + u2f(__builtin_amdgcn_readlane(u, 48));
  return a + b;
}

// A sum and M maxima over the T threads of a row, left in all of them.  The T > 64 threads of a workgroup exchange them through
// `box`: two sets in turn, so that one barrier a row is enough (a wave that is a row ahead writes the other set, and cannot be two
// ahead).
template <int T, int M>
struct RowReducer {
  static constexpr int kWaves = T / 64;
  struct Box { float sum[kWaves]; uint32_t largest[M ? M : 1][kWaves]; };
  Box* box;       // [2], in LDS
  uint32_t turn;
  __device__ __forceinline__ void reduce(float& sum, uint32_t* largest) {
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < M; ++i) largest[i] = wave_max(largest[i]);
    if constexpr (T > 64) {
      Box& b = box[turn];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        b.sum[threadIdx.x >> 6] = sum;
#pragma unroll
        for (int i = 0; i < M; ++i) b.largest[i][threadIdx.x >> 6] = largest[i];
      }
      __syncthreads();
      sum = b.sum[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) sum += b.sum[w];
#pragma unroll
      for (int i = 0; i < M; ++i) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) largest[i] = max(largest[i], b.largest[i][w]);
      }
    }
  }
};

// The rows of a workgroup of kernels that go over a row twice: T threads for a row.
template <int T> struct Rows {
  static constexpr int kThreads = T < 256 ? 256 : T;
  static constexpr uint32_t kPerGroup = kThreads / T;
  __device__ static __forceinline__ uint32_t first() { return blockIdx.x * kPerGroup + (T < 256 ? threadIdx.x / T : 0); }
  __device__ static __forceinline__ uint32_t step() { return gridDim.x * kPerGroup; }
  __device__ static __forceinline__ uint32_t column() { return (threadIdx.x & (T - 1)) * 8; }
};
// f(first column, place in registers) for each vector of the thread: V of them that are held, or (V = 0) any number that are not.
// All lanes of a wave take part in every call, also those beyond the row's end.
template <int T, int V, class F>
__device__ __forceinline__ void each_vector(uint32_t cols, F f) {
  if constexpr (V > 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) f(Rows<T>::column() + static_cast<uint32_t>(j) * T * 8, j);
  } else {
    for (uint32_t base = 0; base < cols; base += T * 8) f(base + Rows<T>::column(), 0);
  }
}
template <int V> constexpr int kHeld = V ? V : 1;

// ---------------------------------------------------------------------------------------------- conversion
template <uint32_t TY, int T, int V>
__global__ __launch_bounds__(Rows<T>::kThreads) void quantize_kernel(const RowsArgs a) {
  __shared__ typename RowReducer<T, 1>::Box box[2];
  RowReducer<T, 1> red{box, 0};
  for (uint32_t row = Rows<T>::first(); row < a.rows; row += Rows<T>::step()) {
    float v[kHeld<V>][8];
    uint32_t largest = 0;
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      load8<TY>(a.x, row, c, a.cols, v[at]);
      if (a.out.lg) store_block_codes(a.out, row, c, a.cols, v[at]);
      else largest = max(largest, largest8(v[at]));
    });
    if (a.out.lg) continue;
    float none = 0.0f;
    red.reduce(none, &largest);
    const Coder k = coder_of(largest);
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) load8<TY>(a.x, row, c, a.cols, v[at]);
      store_codes(a.out, row, c, a.cols, v[at], k);
    });
    if (Rows<T>::column() == 0) as_global(a.out.s)[row] = k.scale;
  }
}

// Elementwise kernels: 2^lg_t threads for a row, blockIdx.x along the row, blockIdx.y over the rows.
struct Flat {
  uint32_t c, row, step;
  __device__ __forceinline__ explicit Flat(uint32_t lg_t) {
    c = (blockIdx.x * (1u << lg_t) + (threadIdx.x & ((1u << lg_t) - 1u))) * 8;
    row = blockIdx.y * (256u >> lg_t) + (threadIdx.x >> lg_t);
    step = gridDim.y * (256u >> lg_t);
  }
};

template <uint32_t TY>
__global__ __launch_bounds__(256) void dequantize_kernel(const RowsArgs a, uint32_t lg_t) {
  const Flat f(lg_t);
  if (f.c >= a.cols) return;
  for (uint32_t row = f.row; row < a.rows; row += f.step) {
    float v[8];
    load8<kQ8>(a.x, row, f.c, a.cols, v);
    store8<TY>(a.out, row, f.c, a.cols, v);
  }
}

// ---------------------------------------------------------------------------------------------- norm
// One pass: with h the sum, the scale of y is rstd * max|h w| / 127 and its codes are rint(h w * (127 / max|h w|)), free of rstd, so
// that the sum of squares and the maxima are reduced together.
template <uint32_t TY, int T, int V>
__global__ __launch_bounds__(Rows<T>::kThreads) void rms_norm_kernel(const NormArgs a) {
  __shared__ typename RowReducer<T, 2>::Box box[2];
  RowReducer<T, 2> red{box, 0};
  for (uint32_t row = Rows<T>::first(); row < a.rows; row += Rows<T>::step()) {
    float h[kHeld<V>][8];
    float squares = 0.0f;
    uint32_t largest[2] = {0, 0};  // of h * weight, of h
    auto add = [&](uint32_t c, float (&v)[8]) {  // h of a vector
      load8<TY>(a.x, row, c, a.cols, v);
      if (!a.residual.p) return;
      float r[8];
      load8<TY>(a.residual, row, c, a.cols, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = rounded<TY>(v[i] + r[i]);
    };
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      add(c, h[at]);
      if (a.sum.p && c < a.cols) store8<TY>(a.sum, row, c, a.cols, h[at]);
      const Raw<float> w = load_raw(a.weight, c, a.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        squares = fmaf(h[at][i], h[at][i], squares);
        largest[0] = max(largest[0], magnitude(h[at][i] * w.e[i]));
        largest[1] = max(largest[1], magnitude(h[at][i]));
      }
      if (a.saved.p && a.saved.lg) store_block_codes(a.saved, row, c, a.cols, h[at]);
    });
    red.reduce(squares, largest);
    // squares that are not finite (an element that is not, or more than fp32 holds) make the row NaN
    const bool finite = magnitude(squares) < kInf;
    const float rstd = finite ? 1.0f / __fsqrt_rn(squares / static_cast<float>(a.cols) + a.eps) : __builtin_nanf("");
    const Coder k = coder_of(finite ? largest[0] : kInf), ks = coder_of(largest[1]);
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) {  // sum may have taken x's or residual's place
        if (a.sum.p) load8<TY>(a.sum, row, c, a.cols, h[at]);
        else add(c, h[at]);
      }
      const Raw<float> w = load_raw(a.weight, c, a.cols);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[at][i] * w.e[i];
      store_codes(a.y, row, c, a.cols, y, k);
      if (a.saved.p && !a.saved.lg) store_codes(a.saved, row, c, a.cols, h[at], ks);
    });
    if (Rows<T>::column() == 0) {
      as_global(a.y.s)[row] = k.scale * rstd;
      if (a.rstd) as_global(a.rstd)[row] = rstd;
      if (a.saved.p && !a.saved.lg) as_global(a.saved.s)[row] = ks.scale;
    }
  }
}

// Gradients of the norm.  A workgroup goes through rows of its own and adds up its part of dweight, in registers (for rows that are
// not held: in `partial` itself, each of whose columns has one thread); the second kernel sums the parts in one order.
template <uint32_t TS, uint32_t TY, int T, int V>
__global__ __launch_bounds__(Rows<T>::kThreads) void rms_norm_grad_kernel(const NormGradArgs a) {
  __shared__ typename RowReducer<T, 0>::Box box[2];
  RowReducer<T, 0> red{box, 0};
  float* const part = a.partial + static_cast<uint64_t>(blockIdx.x) * a.cols;
  float dw[kHeld<V>][8];
#pragma unroll
  for (int j = 0; j < kHeld<V>; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
  for (uint32_t row = Rows<T>::first(); row < a.rows; row += Rows<T>::step()) {
    const float rstd = as_global(a.rstd)[row];
    float n[kHeld<V>][8], g[kHeld<V>][8], dot = 0.0f;
    auto take = [&](uint32_t c, int at) {  // n = sum * rstd and dy
      load8<TS>(a.sum, row, c, a.cols, n[at]);
      load8<TY>(a.dy, row, c, a.cols, g[at]);
#pragma unroll
      for (int i = 0; i < 8; ++i) n[at][i] *= rstd;
    };
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      take(c, at);
      const Raw<float> w = load_raw(a.weight, c, a.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(g[at][i] * w.e[i], n[at][i], dot);
    });
    red.reduce(dot, nullptr);
    const float mean = dot / static_cast<float>(a.cols);
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) {
        take(c, at);
        if (row != Rows<T>::first()) {
          const Raw<float> r = load_raw(part, c, a.cols);
#pragma unroll
          for (int i = 0; i < 8; ++i) dw[at][i] = r.e[i];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) dw[at][i] = 0.0f;
        }
      }
      const Raw<float> w = load_raw(a.weight, c, a.cols);
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dw[at][i] = fmaf(g[at][i], n[at][i], dw[at][i]);
        d[i] = rstd * (g[at][i] * w.e[i] - n[at][i] * mean);
      }
      if (a.dres.p) {
        float r[8];
        load8<TY>(a.dres, row, c, a.cols, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += r[i];
      }
      store8<TY>(a.dx, row, c, a.cols, d);
      if (!V) store8<kF32>(Mat{part, nullptr, 0, 0, 0}, 0, c, a.cols, dw[at]);
    });
  }
  if (!V) return;
  if constexpr (T < 256) {  // the rows of several waves
    __shared__ float of_wave[3][kHeld<V>][64][9];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wave) {
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) of_wave[wave - 1][j][lane][i] = dw[j][i];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[j][i] += (of_wave[0][j][lane][i] + of_wave[1][j][lane][i]) + of_wave[2][j][lane][i];
  }
  each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
    if (c < a.cols) store8<kF32>(Mat{part, nullptr, 0, 0, 0}, 0, c, a.cols, dw[at]);
  });
}
// dweight[c] = the sum of the parts of column c: 64 columns and 8 waves a workgroup, which take the parts in turn.
__global__ __launch_bounds__(512) void sum_parts_kernel(const float* partial, float* out, uint32_t groups, uint32_t cols) {
  __shared__ float box[8][64];
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (uint32_t g = wave; g < groups; g += 8) s += as_global(partial)[static_cast<uint64_t>(g) * cols + c];
  }
  box[wave][lane] = s;
  __syncthreads();
  if (wave || c >= cols) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) s += box[w][lane];
  as_global(out)[c] = s;
}

// ---------------------------------------------------------------------------------------------- gated activation
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

template <uint32_t TY, int T, int V>
__global__ __launch_bounds__(Rows<T>::kThreads) void gated_kernel(const GatedArgs a) {
  __shared__ typename RowReducer<T, 3>::Box box[2];
  RowReducer<T, 3> red{box, 0};
  for (uint32_t row = Rows<T>::first(); row < a.rows; row += Rows<T>::step()) {
    float y[kHeld<V>][8], g[kHeld<V>][8], u[kHeld<V>][8];
    uint32_t largest[3] = {0, 0, 0};  // of y, gate, up
    auto take = [&](uint32_t c, int at) {
      load8<TY>(a.gate, row, c, a.cols, g[at]);
      load8<TY>(a.up, row, c, a.cols, u[at]);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[at][i] = g[at][i] * sigmoid(g[at][i]) * u[at][i];
    };
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      take(c, at);
      largest[0] = max(largest[0], largest8(y[at]));
      if (!a.saved_gate.p) return;
      if (a.saved_gate.lg) {
        store_block_codes(a.saved_gate, row, c, a.cols, g[at]);
        store_block_codes(a.saved_up, row, c, a.cols, u[at]);
      } else {
        largest[1] = max(largest[1], largest8(g[at]));
        largest[2] = max(largest[2], largest8(u[at]));
      }
    });
    float none = 0.0f;
    red.reduce(none, largest);
    const bool rows_saved = a.saved_gate.p && !a.saved_gate.lg;
    const Coder k = coder_of(largest[0]), kg = coder_of(largest[1]), ku = coder_of(largest[2]);
    each_vector<T, V>(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) take(c, at);
      store_codes(a.y, row, c, a.cols, y[at], k);
      if (!rows_saved) return;
      store_codes(a.saved_gate, row, c, a.cols, g[at], kg);
      store_codes(a.saved_up, row, c, a.cols, u[at], ku);
    });
    if (Rows<T>::column() == 0) {
      as_global(a.y.s)[row] = k.scale;
      if (rows_saved) {
        as_global(a.saved_gate.s)[row] = kg.scale;
        as_global(a.saved_up.s)[row] = ku.scale;
      }
    }
  }
}

template <uint32_t TS, uint32_t TY>
__global__ __launch_bounds__(256) void gated_grad_kernel(const GatedGradArgs a, uint32_t lg_t) {
  const Flat f(lg_t);
  if (f.c >= a.cols) return;
  for (uint32_t row = f.row; row < a.rows; row += f.step) {
    float g[8], u[8], d[8], dg[8], du[8];
    load8<TS>(a.gate, row, f.c, a.cols, g);
    load8<TS>(a.up, row, f.c, a.cols, u);
    load8<TY>(a.dy, row, f.c, a.cols, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = sigmoid(g[i]);
      dg[i] = d[i] * (u[i] * (s * (1.0f + g[i] * (1.0f - s))));
      du[i] = d[i] * (g[i] * s);
    }
    store8<TY>(a.dgate, row, f.c, a.cols, dg);
    store8<TY>(a.dup, row, f.c, a.cols, du);
  }
}

// ---------------------------------------------------------------------------------------------- launches
// Threads and vectors for a row of `cols` columns: f(T, V) as compile-time constants.
template <int T_, int V_> struct Shape { static constexpr int T = T_, V = V_; };
template <class F>
void with_shape(uint32_t cols, F f) {
  if (cols <= 1024) f(Shape<64, 2>{});
  else if (cols <= 4096) f(Shape<256, 2>{});
  else if (cols <= 8192) f(Shape<512, 2>{});
  else if (cols <= 16384) f(Shape<1024, 2>{});
  else f(Shape<1024, 0>{});
}
template <class F>
void with_type(uint32_t type, F f) {
  if (type == kF32) f(std::integral_constant<uint32_t, kF32>{});
  else f(std::integral_constant<uint32_t, kBF16>{});
}
template <class F>
void with_kept(uint32_t type, F f) {
  if (type == kQ8) f(std::integral_constant<uint32_t, kQ8>{});
  else with_type(type, f);
}
// Workgroups for rows held by T threads: as many as fit the card at once, which then go through the rows.
template <int T>
uint32_t groups_of(uint32_t rows, uint32_t n_cu) {
  const uint32_t need = (rows + Rows<T>::kPerGroup - 1) / Rows<T>::kPerGroup, fit = n_cu * (2048 / Rows<T>::kThreads);
  return need < fit ? need : fit;
}
// Launch shape of the elementwise kernels.
struct FlatShape { uint32_t lg_t; dim3 grid; };
FlatShape flat_shape(uint32_t rows, uint32_t cols) {
  const uint32_t vectors = (cols - 1) / 8 + 1;
  uint32_t lg = 3;
  while (lg < 8 && (1u << lg) < vectors) ++lg;
  const uint32_t per_group = 256u >> lg, y = (rows - 1) / per_group + 1;
  return {lg, dim3(((vectors - 1) >> lg) + 1, y < 16384u ? y : 16384u)};
}

}  // namespace

int launch_quantize_rows(const RowsArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_shape(a.cols, [&](auto s) { with_type(type, [&](auto ty) {
    quantize_kernel<ty(), s.T, s.V><<<groups_of<s.T>(a.rows, n_cu), Rows<s.T>::kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_dequantize_rows(const RowsArgs& a, uint32_t type, void* stream) {
  const FlatShape f = flat_shape(a.rows, a.cols);
  with_type(type, [&](auto ty) { dequantize_kernel<ty()><<<f.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, f.lg_t); });
  return hipGetLastError();
}
int launch_rms_norm(const NormArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_shape(a.cols, [&](auto s) { with_type(type, [&](auto ty) {
    rms_norm_kernel<ty(), s.T, s.V><<<groups_of<s.T>(a.rows, n_cu), Rows<s.T>::kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_rms_norm_grad(NormGradArgs a, uint32_t sum_type, uint32_t type, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  a.groups = norm_grad_groups(a.rows, a.cols);
  if (a.groups) {
    with_shape(a.cols, [&](auto s) { with_kept(sum_type, [&](auto ts) { with_type(type, [&](auto ty) {
      rms_norm_grad_kernel<ts(), ty(), s.T, s.V><<<a.groups, Rows<s.T>::kThreads, 0, st>>>(a);
    }); }); });
    if (const hipError_t e = hipGetLastError()) return e;
  }
  sum_parts_kernel<<<(a.cols - 1) / 64 + 1, 512, 0, st>>>(a.partial, a.dweight, a.groups, a.cols);
  return hipGetLastError();
}
int launch_gated(const GatedArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_shape(a.cols, [&](auto s) { with_type(type, [&](auto ty) {
    gated_kernel<ty(), s.T, s.V><<<groups_of<s.T>(a.rows, n_cu), Rows<s.T>::kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_gated_grad(const GatedGradArgs& a, uint32_t kept_type, uint32_t type, void* stream) {
  const FlatShape f = flat_shape(a.rows, a.cols);
  with_kept(kept_type, [&](auto ts) { with_type(type, [&](auto ty) {
    gated_grad_kernel<ts(), ty()><<<f.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, f.lg_t);
  }); });
  return hipGetLastError();
}

}  // namespace stq
