// What the kernels of the cross entropy and those of its gradients share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_tiles.h"

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

// A logit by itself.
__device__ __forceinline__ float logit(const MatmulArgs& a, uint64_t m, uint64_t n) {
  const STQ_GLOBAL int8_t* x = as_global(static_cast<const int8_t*>(a.a.p)) + m * a.a.stride;
  const STQ_GLOBAL int8_t* w = as_global(static_cast<const int8_t*>(a.b.p)) + n * a.b.stride;
  int32_t sum = 0;
  for (uint32_t k = 0; k < a.k; ++k) sum += x[k] * w[k];
  return static_cast<float>(sum) * as_global(a.a.s)[m] * as_global(a.b.s)[n];
}

// ---------------------------------------------------------------------------------------------- on the host
inline uint64_t whole(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

struct Arena {  // parts of a workspace, of 256 bytes each
  char* at;
  template <class T>
  T* take(uint64_t n) {
    T* const p = reinterpret_cast<T*>(at);
    at += whole(n * sizeof(T));
    return p;
  }
};

// Whether operands have the 16 codes that a load takes.
inline bool enough_codes(const MatmulArgs& a) { return (a.m - 1) * a.a.stride + a.k >= 16 && (a.n - 1) * a.b.stride + a.k >= 16; }

}  // namespace
}  // namespace stq
