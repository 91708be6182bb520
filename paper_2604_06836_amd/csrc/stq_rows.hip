// gfx950 kernels of the 8-bit layer that work on rows: conversion to codes and back, the root-mean-square norm with the
// residual's addition and its gradients, the gated activation and its gradients.
//
// All are bound by memory: every matrix is read once and written once.  A thread owns vectors of eight neighbouring columns, so
// that a vector has one scale (blocks are 64, 128 or 256 columns) and is one load of 8 (codes), 16 (bf16) or 32 bytes.  Kernels
// that need a maximum or a sum over a row hold the row in registers between the two: a wave for a row of up to 1024 columns,
// without any barrier, a workgroup of just the waves that it takes for longer ones, with one barrier for a row.  They go through the
// rows with the next row's loads under way.  Only the last vector of a row whose columns are no multiple of eight goes element by element.  Longer
// rows (over 16384 columns; 8192 for the norm's gradients) are not held but read again, out of the caches.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "stq_vectors.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

constexpr float kLeast = 0x1p-100f;  // what a group's largest magnitude counts as at least
constexpr uint32_t kInf = 0x7F800000u;

// ---------------------------------------------------------------------------------------------- rows and vectors
template <class T>
__device__ __forceinline__ T* row_of(const Mat& m, uint32_t row) { return static_cast<T*>(m.p) + static_cast<uint64_t>(row) * m.stride; }
__device__ __forceinline__ float* scale_of(const Mat& m, uint32_t row, uint32_t c) {
  return m.s + static_cast<uint64_t>(row) * m.per_row + (m.lg ? c >> m.lg : 0u);
}
// A vector as it was loaded, with the scale of codes.
template <uint32_t TY>
struct Loaded {
  Packed<typename Elem<TY>::type> v;
  float s;
  __device__ __forceinline__ void from(const Mat& m, uint32_t row, uint32_t c, uint32_t cols) {
    v = load_ending(row_of<typename Elem<TY>::type>(m, row), c, cols);
    if constexpr (TY == kQ8) s = as_global(scale_of(m, row, min(c, cols - 1)))[0];
  }
  __device__ __forceinline__ float at(uint32_t e) const {
    if constexpr (TY == kQ8) return s * v.at(e);
    return v.at(e);
  }
};
template <uint32_t TY>
__device__ __forceinline__ void store8(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, const float (&v)[8]) {
  using T = typename Elem<TY>::type;
  store_ending(row_of<T>(m, row), c, cols, pack<T>(v));
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

// How a group's elements become codes: scale = largest * (1 / 127), q = rint(x * (127 * (1 / largest))), every step rounded as it is
// written, so that codes are the same wherever they are computed so.  (The compiler's divisions for each block were a sixth of the
// gated kernel's instructions; a reciprocal of a hardware one is rounded after one step.)  Above 2^64 it is taken of a smaller number.
struct Coder { float inv, scale; uint32_t keep; };
__device__ __forceinline__ Coder coder_of(uint32_t largest) {
  const float a = fmaxf(u2f(largest), kLeast);
  const bool finite = largest < kInf, far = a > 0x1p64f;
  const float d = far ? a * 0x1p-64f : a, r = __builtin_amdgcn_rcpf(d), inv = 127.0f * fmaf(fmaf(-d, r, 1.0f), r, r);
  return {far ? inv * 0x1p-64f : inv, finite ? a * (1.0f / 127.0f) : __builtin_nanf(""), finite ? 0xFFFFFFFFu : 0u};
}
// rint by the addition of 1.5 * 2^23: the low byte of the sum is the code in two's complement
__device__ __forceinline__ uint32_t code_byte(float x, float inv) { return f2u(x * inv + 12582912.0f); }
__device__ __forceinline__ uint32_t codes4(const float* x, float inv, uint32_t keep) {
  const uint32_t lo = __builtin_amdgcn_perm(code_byte(x[1], inv), code_byte(x[0], inv), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(code_byte(x[3], inv), code_byte(x[2], inv), 0x04000C0Cu);
  return (lo | hi) & keep;
}
__device__ __forceinline__ void store_codes(const Mat& m, uint32_t row, uint32_t c, uint32_t cols, const float (&v)[8], const Coder& k) {
  const Packed<int8_t> r = {{codes4(v, k.inv, k.keep), codes4(v + 4, k.inv, k.keep)}};
  store_ending(row_of<int8_t>(m, row), c, cols, r);
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
__device__ __forceinline__ float row_total(float x) {  // over each 16 lanes
  x += u2f(dpp_u32<kDppXor1>(f2u(x)));
  x += u2f(dpp_u32<kDppXor2>(f2u(x)));
  x += u2f(dpp_u32<kDppHalfMirror>(f2u(x)));
  x += u2f(dpp_u32<kDppMirror>(f2u(x)));
  return x;
}
__device__ __forceinline__ float first_of(float x) { return u2f(__builtin_amdgcn_readfirstlane(f2u(x))); }
__device__ __forceinline__ float wave_sum(float x) {
  const uint32_t u = f2u(row_total(x));
  const float a = u2f(__builtin_amdgcn_readlane(u, 0)) + u2f(__builtin_amdgcn_readlane(u, 16));
  const float b = u2f(__builtin_amdgcn_readlane(u, 32)) + u2f(__builtin_amdgcn_readlane(u, 48));
  return a + b;
}

// The rows of a workgroup of kernels that go over a row twice.  WAVES: a wave for a row, else the workgroup, of up to 16 waves.  V: the
// vectors of a thread, which are held, or 0: any number, which are not.
constexpr uint32_t kMostWaves = 16;
template <bool WAVES_, int V_>
struct Rows {
  static constexpr bool WAVES = WAVES_;
  static constexpr int V = V_, kHeld = V ? V : 1;
  static constexpr uint32_t kPerGroup = WAVES ? 4 : 1;
  __device__ static __forceinline__ uint32_t first() { return blockIdx.x * kPerGroup + (WAVES ? threadIdx.x >> 6 : 0); }
  __device__ static __forceinline__ uint32_t step() { return gridDim.x * kPerGroup; }
  __device__ static __forceinline__ uint32_t thread() { return WAVES ? threadIdx.x & 63 : threadIdx.x; }
  // f(first column, place in registers) for each vector of the thread.  All lanes of a wave take part in every call, also those beyond
  // the row's end.
  template <class F>
  __device__ static __forceinline__ void each(uint32_t cols, F f) {
    const uint32_t threads = WAVES ? 64 : blockDim.x;
    if constexpr (V > 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) f((thread() + j * threads) * 8, j);
    } else {
      for (uint32_t base = 0; base < cols; base += threads * 8) f(base + thread() * 8, 0);
    }
  }
};

// A sum and M maxima over the threads of a row, left in all of them.  The waves of a workgroup exchange theirs through `box`: two sets in
// turn, so that one barrier is enough (a wave that is an exchange ahead writes the other set, and cannot be two ahead).
template <class R, int M>
struct RowReducer {
  struct Box { float sum[kMostWaves]; uint32_t largest[M ? M : 1][kMostWaves]; };
  Box* box;  // [2], in LDS
  uint32_t turn;
  template <bool SUM = true>
  __device__ __forceinline__ void reduce(float& sum, uint32_t* largest) {
    if (SUM) sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < M; ++i) largest[i] = wave_max(largest[i]);
    if constexpr (!R::WAVES) {
      Box& b = box[turn];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        if (SUM) b.sum[threadIdx.x >> 6] = sum;
#pragma unroll
        for (int i = 0; i < M; ++i) b.largest[i][threadIdx.x >> 6] = largest[i];
      }
      __syncthreads();
      // a lane of sixteen for each wave
      const uint32_t w = threadIdx.x & 15;
      const bool there = w < blockDim.x >> 6;
      if (SUM) sum = first_of(row_total(there ? b.sum[w] : 0.0f));
#pragma unroll
      for (int i = 0; i < M; ++i) largest[i] = __builtin_amdgcn_readfirstlane(row_max(there ? b.largest[i][w] : 0u));
    }
  }
  __device__ __forceinline__ void most(uint32_t* largest) {
    float none;
    reduce<false>(none, largest);
  }
};
#define STQ_ROWS_KERNEL __global__ __launch_bounds__(R::WAVES ? 256 : 64 * kMostWaves) void

// ---------------------------------------------------------------------------------------------- conversion
// 11008 x 4096 from fp32: 39 us, 5.7 TB/s.
template <uint32_t TY, class R>
STQ_ROWS_KERNEL quantize_kernel(const RowsArgs a) {
  constexpr int V = R::V;
  __shared__ typename RowReducer<R, 1>::Box box[2];
  RowReducer<R, 1> red{box, 0};
  Loaded<TY> next[R::kHeld];
  const auto fetch = [&](uint32_t row) {
    if (V && row < a.rows) R::each(a.cols, [&](uint32_t c, int at) { next[at].from(a.x, row, c, a.cols); });
  };
  fetch(R::first());
  for (uint32_t row = R::first(); row < a.rows; row += R::step()) {
    float v[R::kHeld][8];
    uint32_t largest = 0;
    const auto take = [&](uint32_t c, int at) {
      if (!V) next[at].from(a.x, row, c, a.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[at][i] = next[at].at(i);
    };
    if (V) {
      R::each(a.cols, take);
      fetch(row + R::step());
    }
    R::each(a.cols, [&](uint32_t c, int at) {
      if (!V) take(c, at);
      if (a.out.lg) store_block_codes(a.out, row, c, a.cols, v[at]);
      else largest = max(largest, largest8(v[at]));
    });
    if (a.out.lg) continue;
    red.most(&largest);
    const Coder k = coder_of(largest);
    R::each(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) take(c, at);
      store_codes(a.out, row, c, a.cols, v[at], k);
    });
    if (R::thread() == 0) as_global(a.out.s)[row] = k.scale;
  }
}

// Elementwise kernels (codes of 16384 x 4096 to bf16: 32 us, 6.2 TB/s): 2^lg_t threads for a row, blockIdx.x along the row, blockIdx.y
// over the rows, four of which a thread has under way together.
constexpr uint32_t kTogether = 4;
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
  for (uint32_t row = f.row; row < a.rows; row += kTogether * f.step) {
    Loaded<kQ8> x[kTogether];
#pragma unroll
    for (uint32_t k = 0; k < kTogether; ++k)
      if (row + k * f.step < a.rows) x[k].from(a.x, row + k * f.step, f.c, a.cols);
#pragma unroll
    for (uint32_t k = 0; k < kTogether; ++k) {
      if (row + k * f.step >= a.rows) break;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = x[k].at(i);
      store8<TY>(a.out, row + k * f.step, f.c, a.cols, v);
    }
  }
}

// ---------------------------------------------------------------------------------------------- norm
// Two exchanges a row, of the squares and then of max|y|.  (The codes are free of rstd, and with max|h w| in place of max|y| one exchange
// would do, in the same time; but its roundings are others than the formula's, and so are codes next to a half.)  Bound by memory: 16384 x
// 4096 in bf16 with the residual, the sum kept in 8 bits, 104 us, 5.2 TB/s (an addition in place of 4 GiB reaches 5.9).
template <uint32_t TY, class R>
STQ_ROWS_KERNEL rms_norm_kernel(const NormArgs a) {
  constexpr int V = R::V;
  __shared__ typename RowReducer<R, 1>::Box box[2];
  RowReducer<R, 1> red{box, 0};
  Loaded<TY> next[R::kHeld], next_r[R::kHeld];
  Loaded<kF32> w[R::kHeld];
  const Mat weight{const_cast<float*>(a.weight), nullptr, 0, 0, 0};
  const auto load = [&](uint32_t row, uint32_t c, int at) {
    next[at].from(a.x, row, c, a.cols);
    if (a.residual.p) next_r[at].from(a.residual, row, c, a.cols);
  };
  const auto fetch = [&](uint32_t row) {
    if (V && row < a.rows) R::each(a.cols, [&](uint32_t c, int at) { load(row, c, at); });
  };
  fetch(R::first());
  if (V) R::each(a.cols, [&](uint32_t c, int at) { w[at].from(weight, 0, c, a.cols); });
  for (uint32_t row = R::first(); row < a.rows; row += R::step()) {
    float h[R::kHeld][8];
    float squares = 0.0f;
    uint32_t largest = 0;  // of h
    const auto add = [&](uint32_t c, int at) {  // h of a vector
      if (!V) {
        load(row, c, at);
        w[at].from(weight, 0, c, a.cols);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) h[at][i] = a.residual.p ? rounded<TY>(next[at].at(i) + next_r[at].at(i)) : next[at].at(i);
    };
    if (V) {
      R::each(a.cols, add);
      fetch(row + R::step());
    }
    R::each(a.cols, [&](uint32_t c, int at) {
      if (!V) add(c, at);
      if (a.sum.p && c < a.cols) store8<TY>(a.sum, row, c, a.cols, h[at]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        squares = fmaf(h[at][i], h[at][i], squares);
        largest = max(largest, magnitude(h[at][i]));
      }
      if (a.saved.p && a.saved.lg) store_block_codes(a.saved, row, c, a.cols, h[at]);
    });
    red.reduce(squares, &largest);
    // squares that are not finite (an element that is not, or more than fp32 holds) make the row NaN
    const bool finite = magnitude(squares) < kInf;
    const float rstd = finite ? 1.0f / __fsqrt_rn(squares / static_cast<float>(a.cols) + a.eps) : __builtin_nanf("");
    const Coder ks = coder_of(largest);
    uint32_t largest_y = f2u(rstd * kLeast);  // 2^-100 in the measure of h w, so that a row of zeros has a scale in it
    const auto again = [&](uint32_t c, int at) {  // h and weight of a vector that is not held; the sum may have taken x's or residual's place
      if (V) return;
      if (!a.sum.p) return add(c, at);
      Loaded<TY> t;
      t.from(a.sum, row, c, a.cols);
      w[at].from(weight, 0, c, a.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[at][i] = t.at(i);
    };
    R::each(a.cols, [&](uint32_t c, int at) {
      again(c, at);
#pragma unroll
      for (int i = 0; i < 8; ++i) largest_y = max(largest_y, magnitude(h[at][i] * rstd * w[at].at(i)));
    });
    red.most(&largest_y);
    const Coder k = coder_of(finite ? largest_y : kInf);
    R::each(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      again(c, at);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[at][i] * rstd * w[at].at(i);
      store_codes(a.y, row, c, a.cols, y, k);
      if (a.saved.p && !a.saved.lg) store_codes(a.saved, row, c, a.cols, h[at], ks);
    });
    if (R::thread() == 0) {
      as_global(a.y.s)[row] = k.scale;
      if (a.rstd) as_global(a.rstd)[row] = rstd;
      if (a.saved.p && !a.saved.lg) as_global(a.saved.s)[row] = ks.scale;
    }
  }
}

// Gradients of the norm.  A workgroup goes through rows of its own and adds up its part of dweight, in registers (for rows that are
// not held: in `partial` itself, each of whose columns has one thread); the second kernel sums the parts in one order.  16384 x 4096 from
// codes: 88 us, 5.3 TB/s; 8192 x 1600: 26 us, of which the second kernel takes 4.4 and the way there of the parts a seventh.
template <uint32_t TS, uint32_t TY, class R>
STQ_ROWS_KERNEL rms_norm_grad_kernel(const NormGradArgs a) {
  constexpr int V = R::V;
  __shared__ typename RowReducer<R, 0>::Box box[2];
  RowReducer<R, 0> red{box, 0};
  float* const part = a.partial + static_cast<uint64_t>(blockIdx.x) * a.cols;
  const Mat to_part{part, nullptr, 0, 0, 0}, weight{const_cast<float*>(a.weight), nullptr, 0, 0, 0};
  float dw[R::kHeld][8];
#pragma unroll
  for (int j = 0; j < R::kHeld; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
  Loaded<TS> next_n[R::kHeld];
  Loaded<TY> next_g[R::kHeld], next_r[R::kHeld];
  Loaded<kF32> w[R::kHeld];
  const auto load = [&](uint32_t row, uint32_t c, int at) {
    next_n[at].from(a.sum, row, c, a.cols);
    next_g[at].from(a.dy, row, c, a.cols);
    if (a.dres.p) next_r[at].from(a.dres, row, c, a.cols);
  };
  const auto fetch = [&](uint32_t row) {
    if (V && row < a.rows) R::each(a.cols, [&](uint32_t c, int at) { load(row, c, at); });
  };
  fetch(R::first());
  if (V) R::each(a.cols, [&](uint32_t c, int at) { w[at].from(weight, 0, c, a.cols); });
  for (uint32_t row = R::first(); row < a.rows; row += R::step()) {
    const float rstd = as_global(a.rstd)[row];
    Loaded<TS> n[R::kHeld];
    Loaded<TY> g[R::kHeld], r[R::kHeld];
    float dot = 0.0f;
    const auto take = [&](uint32_t c, int at) {
      if (!V) {
        load(row, c, at);
        w[at].from(weight, 0, c, a.cols);
      }
      n[at] = next_n[at];
      g[at] = next_g[at];
      r[at] = next_r[at];
    };
    if (V) {
      R::each(a.cols, take);
      fetch(row + R::step());
    }
    R::each(a.cols, [&](uint32_t c, int at) {
      if (!V) take(c, at);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(g[at].at(i) * w[at].at(i), n[at].at(i) * rstd, dot);
    });
    red.reduce(dot, nullptr);
    const float mean = dot / static_cast<float>(a.cols);
    R::each(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      if (!V) {
        take(c, at);
        Loaded<kF32> t;
        if (row != R::first()) t.from(to_part, 0, c, a.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[at][i] = row != R::first() ? t.at(i) : 0.0f;
      }
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = n[at].at(i) * rstd;
        dw[at][i] = fmaf(g[at].at(i), x, dw[at][i]);
        d[i] = rstd * (g[at].at(i) * w[at].at(i) - x * mean);
        if (a.dres.p) d[i] += r[at].at(i);
      }
      store8<TY>(a.dx, row, c, a.cols, d);
      if (!V) store8<kF32>(to_part, 0, c, a.cols, dw[at]);
    });
  }
  if (!V) return;
  if constexpr (R::WAVES) {  // the rows of several waves
    __shared__ float of_wave[3][R::kHeld][64][9];
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
  R::each(a.cols, [&](uint32_t c, int at) {
    if (c < a.cols) store8<kF32>(to_part, 0, c, a.cols, dw[at]);
  });
}
// dweight[c] = the sum of the parts of column c: 16 columns a workgroup, of whose 64 threads for each a part goes to each in turn.
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float* partial, float* out, uint32_t groups, uint32_t cols) {
  __shared__ float box[64][17];
  const uint32_t turn = threadIdx.x >> 4, lane = threadIdx.x & 15, c = group_number() * 16 + lane;
  float s = 0.0f;
  if (c < cols) {
#pragma unroll 16
    for (uint32_t g = turn; g < groups; g += 64) s += as_global(partial)[static_cast<uint64_t>(g) * cols + c];
  }
  box[turn][lane] = s;
#pragma unroll
  for (uint32_t n = 64; n > 1; n /= 4) {  // four to one
    __syncthreads();
    if (turn < n / 4) {
      s = (box[turn][lane] + box[turn + n / 4][lane]) + (box[turn + n / 2][lane] + box[turn + n / 4 * 3][lane]);
      box[turn][lane] = s;
    }
  }
  if (turn == 0 && c < cols) as_global(out)[c] = s;
}

// ---------------------------------------------------------------------------------------------- gated activation
// (the gradients': off by up to (2 |x| + 10) 2^-24, since the exponential's argument is rounded)
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
// The forward pass rounds as its formula x / (1 + exp(-x)) is written, where codes are decided by the last bit: the exponential to fp32's
// precision, and a quotient that is rounded after one step, of a quarter of both sides, so that the reciprocal of a finite denominator is
// a normal number.  The fixup has the quotients of what is not finite: where the exponential passes fp32's range, 0 of any finite gate.
__device__ __forceinline__ float silu(float x) {
  const float d = fmaf(expf(-x), 0.25f, 0.25f), n = x * 0.25f, r = __builtin_amdgcn_rcpf(d), q = n * r;
  return __builtin_amdgcn_div_fixupf(fmaf(fmaf(-d, q, n), r, q), d, n);
}

// The vector unit more than memory: about 40 instructions an element, a third of them the exponential and the quotient as rounded.  8192 x
// 11008 in bf16 with both inputs kept: 161 us, 4.0 TB/s (126 with a silu and codes to a few units in the last place).  No
// row is loaded ahead here: more waves hide more than a row of each would (164 us with, 141 without, when codes were divisions).
template <class R> constexpr uint32_t kGatedWaves = R::V == 2 ? 6 : 8;  // of a SIMD
template <uint32_t TY, class R>
__global__ __launch_bounds__(R::WAVES ? 256 : 64 * kMostWaves, kGatedWaves<R>) void gated_kernel(const GatedArgs a) {
  constexpr int V = R::V;
  __shared__ typename RowReducer<R, 3>::Box box[2];
  RowReducer<R, 3> red{box, 0};
  for (uint32_t row = R::first(); row < a.rows; row += R::step()) {
    float y[R::kHeld][8];
    Loaded<TY> g[R::kHeld], u[R::kHeld];
    uint32_t largest[3] = {0, 0, 0};  // of y, gate, up
    const auto take = [&](uint32_t c, int at) {
      g[at].from(a.gate, row, c, a.cols);
      u[at].from(a.up, row, c, a.cols);
    };
    const auto product = [&](int at, float (&gate)[8], float (&up)[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        gate[i] = g[at].at(i);
        up[i] = u[at].at(i);
        y[at][i] = silu(gate[i]) * up[i];
      }
    };
    if (V) R::each(a.cols, take);
    R::each(a.cols, [&](uint32_t c, int at) {
      if (!V) take(c, at);
      float gate[8], up[8];
      product(at, gate, up);
      largest[0] = max(largest[0], largest8(y[at]));
      if (!a.saved_gate.p) return;
      if (a.saved_gate.lg) {
        store_block_codes(a.saved_gate, row, c, a.cols, gate);
        store_block_codes(a.saved_up, row, c, a.cols, up);
      } else {
        largest[1] = max(largest[1], largest8(gate));
        largest[2] = max(largest[2], largest8(up));
      }
    });
    red.most(largest);
    const bool rows_saved = a.saved_gate.p && !a.saved_gate.lg;
    const Coder k = coder_of(largest[0]), kg = coder_of(largest[1]), ku = coder_of(largest[2]);
    R::each(a.cols, [&](uint32_t c, int at) {
      if (c >= a.cols) return;
      float gate[8], up[8];
      if (!V) {
        take(c, at);
        product(at, gate, up);
      }
      store_codes(a.y, row, c, a.cols, y[at], k);
      if (!rows_saved) return;
      if (V) take(c, at);  // again, out of the caches: held, they would cost waves also where they are not needed
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        gate[i] = g[at].at(i);
        up[i] = u[at].at(i);
      }
      store_codes(a.saved_gate, row, c, a.cols, gate, kg);
      store_codes(a.saved_up, row, c, a.cols, up, ku);
    });
    if (R::thread() == 0) {
      as_global(a.y.s)[row] = k.scale;
      if (rows_saved) {
        as_global(a.saved_gate.s)[row] = kg.scale;
        as_global(a.saved_up.s)[row] = ku.scale;
      }
    }
  }
}

// 8192 x 11008 from codes: 135 us, 5.4 TB/s.
template <uint32_t TS, uint32_t TY>
__global__ __launch_bounds__(256) void gated_grad_kernel(const GatedGradArgs a, uint32_t lg_t) {
  constexpr uint32_t kRowsNow = kTogether / 2;  // (of three inputs)
  const Flat f(lg_t);
  if (f.c >= a.cols) return;
  for (uint32_t row = f.row; row < a.rows; row += kRowsNow * f.step) {
    Loaded<TS> gate[kRowsNow], up[kRowsNow];
    Loaded<TY> dy[kRowsNow];
#pragma unroll
    for (uint32_t k = 0; k < kRowsNow; ++k)
      if (row + k * f.step < a.rows) {
        gate[k].from(a.gate, row + k * f.step, f.c, a.cols);
        up[k].from(a.up, row + k * f.step, f.c, a.cols);
        dy[k].from(a.dy, row + k * f.step, f.c, a.cols);
      }
#pragma unroll
    for (uint32_t k = 0; k < kRowsNow; ++k) {
      if (row + k * f.step >= a.rows) break;
      float dg[8], du[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float g = gate[k].at(i), d = dy[k].at(i), s = sigmoid(g);
        dg[i] = d * (up[k].at(i) * (s * (1.0f + g * (1.0f - s))));
        du[i] = d * (g * s);
      }
      store8<TY>(a.dgate, row + k * f.step, f.c, a.cols, dg);
      store8<TY>(a.dup, row + k * f.step, f.c, a.cols, du);
    }
  }
}

// ---------------------------------------------------------------------------------------------- launches
// The shape for rows of `cols` columns: f(Rows<WAVES, V>, threads of a workgroup).  A vector a thread where a workgroup can have so many
// (norm of 16384 x 4096: 114 us; with two, and no registers for a row ahead, 156), two beyond; a wave for what it can hold, without a
// barrier.  TWO: whether a thread may hold two vectors (the norm's gradients have no registers for that).
template <bool TWO, class F>
void with_rows(uint32_t cols, F f) {
  const uint32_t vectors = (cols - 1) / 8 + 1, most = 64 * kMostWaves;
  const auto threads = [&](uint32_t v) { return ((vectors + v - 1) / v + 63) / 64 * 64; };
  if (vectors <= 64) return f(Rows<true, 1>{}, 256u);
  if constexpr (TWO) {
    if (vectors <= 128) return f(Rows<true, 2>{}, 256u);
    if (vectors > most && vectors <= 2 * most) return f(Rows<false, 2>{}, threads(2));
  }
  if (vectors <= most) f(Rows<false, 1>{}, threads(1));
  else f(Rows<false, 0>{}, most);
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
// Workgroups for rows that are held: as many as fit the card at once, which then go through the rows.
template <class R>
uint32_t groups_of(uint32_t rows, uint32_t threads, uint32_t n_cu, uint32_t waves = R::V == 1 ? 5 : 4) {  // of a SIMD
  const uint32_t need = (rows + R::kPerGroup - 1) / R::kPerGroup, fit = n_cu * (waves * 256 / threads);
  return need < fit ? need : fit;
}
// Launch shape of the elementwise kernels: of 32 to 256 threads for a row (8 for the narrowest) those that leave few without
// work; 16 workgroups on a CU, which go through the rows.
struct FlatShape { uint32_t lg_t; dim3 grid; };
FlatShape flat_shape(uint32_t rows, uint32_t cols, uint32_t n_cu) {
  const uint32_t vectors = (cols - 1) / 8 + 1;
  const auto whole = [&](uint32_t lg) { return (((vectors - 1) >> lg) + 1) << lg; };
  uint32_t lg = vectors <= 8 ? 3 : (vectors <= 16 ? 4 : 8);
  for (uint32_t l = 7; lg > 4 && l >= 5; --l)
    if (whole(l) * 16 < whole(lg) * 15) lg = l;
  const uint32_t x = whole(lg) >> lg, per_group = 256u >> lg, need = (rows - 1) / per_group + 1;
  const uint32_t fit = (n_cu * 16 - 1) / x + 1;
  const uint32_t y = need < fit ? need : fit;
  return {lg, dim3(x, y < 65535u ? y : 65535u)};
}

}  // namespace

int launch_quantize_rows(const RowsArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_rows<true>(a.cols, [&](auto r, uint32_t threads) { with_type(type, [&](auto ty) {
    using R = decltype(r);
    quantize_kernel<ty(), R><<<groups_of<R>(a.rows, threads, n_cu), threads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_dequantize_rows(const RowsArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  const FlatShape f = flat_shape(a.rows, a.cols, n_cu);
  with_type(type, [&](auto ty) { dequantize_kernel<ty()><<<f.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, f.lg_t); });
  return hipGetLastError();
}
int launch_rms_norm(const NormArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_rows<true>(a.cols, [&](auto r, uint32_t threads) { with_type(type, [&](auto ty) {
    using R = decltype(r);
    rms_norm_kernel<ty(), R><<<groups_of<R>(a.rows, threads, n_cu), threads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_rms_norm_grad(NormGradArgs a, uint32_t sum_type, uint32_t type, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t groups = norm_grad_groups(a.rows, a.cols);
  if (groups) {
    with_rows<false>(a.cols, [&](auto r, uint32_t threads) { with_kept(sum_type, [&](auto ts) { with_type(type, [&](auto ty) {
      using R = decltype(r);
      rms_norm_grad_kernel<ts(), ty(), R><<<groups, threads, 0, st>>>(a);
    }); }); });
    if (const hipError_t e = hipGetLastError()) return e;
  }
  sum_parts_kernel<<<in_layers((a.cols - 1) / 16 + 1), 1024, 0, st>>>(a.partial, a.dweight, groups, a.cols);
  return hipGetLastError();
}
int launch_gated(const GatedArgs& a, uint32_t type, uint32_t n_cu, void* stream) {
  with_rows<true>(a.cols, [&](auto r, uint32_t threads) { with_type(type, [&](auto ty) {
    using R = decltype(r);
    gated_kernel<ty(), R><<<groups_of<R>(a.rows, threads, n_cu, kGatedWaves<R>), threads, 0, static_cast<hipStream_t>(stream)>>>(a);
  }); });
  return hipGetLastError();
}
int launch_gated_grad(const GatedGradArgs& a, uint32_t kept_type, uint32_t type, uint32_t n_cu, void* stream) {
  const FlatShape f = flat_shape(a.rows, a.cols, n_cu);
  with_kept(kept_type, [&](auto ts) { with_type(type, [&](auto ty) {
    gated_grad_kernel<ts(), ty()><<<f.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, f.lg_t);
  }); });
  return hipGetLastError();
}

}  // namespace stq
