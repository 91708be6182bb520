// Device code that the 8-bit layer's kernels share: element types, and vectors of eight neighbouring elements.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_operators.h"
#include "stq_wave.h"

namespace stq {
namespace {

// Workgroups of launches that grow with a matrix' size, in layers of 2^21: HIP counts the threads along an axis in 32 bits, and beyond
// that leaves workgroups out without an error.  Those of the last layer whose number is too large have nothing to do.
constexpr uint32_t kLgLayer = 21;
inline dim3 in_layers(uint64_t groups, uint32_t y = 1) {
  const uint64_t most = 1u << kLgLayer;
  return dim3(static_cast<uint32_t>(groups < most ? groups : most), y, static_cast<uint32_t>((groups + most - 1) >> kLgLayer));
}
__device__ __forceinline__ uint32_t group_number() { return blockIdx.z << kLgLayer | blockIdx.x; }

template <uint32_t TY> struct Elem;
template <> struct Elem<kF32> { using type = float; };
template <> struct Elem<kBF16> { using type = __bf16; };
template <> struct Elem<kQ8> { using type = int8_t; };

// Eight elements as they are stored, in whole words: loads that are under way must not be taken apart before they are needed.
template <class T>
struct Packed {
  static constexpr uint32_t kWords = 8 * sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void keep(bool there) {  // or zeros
#pragma unroll
    for (uint32_t i = 0; i < kWords; ++i) w[i] = there ? w[i] : 0u;
  }
  __device__ __forceinline__ void move(uint32_t by) {  // elements by, by+1 .. to the front
    for (; by; --by) {
#pragma unroll
      for (uint32_t i = 0; i + 1 < kWords; ++i) w[i] = sizeof(T) == 4 ? w[i + 1] : __builtin_amdgcn_alignbit(w[i + 1], w[i], 8 * sizeof(T) % 32);
      w[kWords - 1] = sizeof(T) == 4 ? 0u : w[kWords - 1] >> (8 * sizeof(T) % 32);
    }
  }
  __device__ __forceinline__ float at(uint32_t e) const {
    if constexpr (sizeof(T) == 4) return u2f(w[e]);
    else if constexpr (sizeof(T) == 2) return u2f(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);  // bf16
    else return static_cast<float>(static_cast<int8_t>(w[e / 4] >> (e % 4 * 8)));
  }
};
// (Vectors need not be aligned to more than their elements: the hardware splits what is not.)
template <class T>
__device__ __forceinline__ Packed<T> load_packed(const T* p) {
  Packed<T> r;
  __builtin_memcpy(&r, as_global(p), sizeof(r));
  return r;
}
// Elements c .. c+7 of a row; zeros beyond its end, where nothing is read.
template <class T>
__device__ __forceinline__ Packed<T> load_ending(const T* row, uint32_t c, uint32_t cols) {
  if (c + 8 <= cols) return load_packed(row + c);
  T e[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) e[i] = c + i < cols ? as_global(row)[c + i] : static_cast<T>(0);
  Packed<T> r;
  __builtin_memcpy(&r, e, sizeof(r));
  return r;
}
// Stores go past the caches: results are written in one sweep and read by others (16384 x 4096 codes to bf16: 61 us, so 32 us).
template <class T>
__device__ __forceinline__ void store_ending(T* row, uint32_t c, uint32_t cols, const Packed<T>& v) {
  STQ_GLOBAL T* p = as_global(row) + c;
  if (c + 8 <= cols) {
    constexpr uint32_t kWords = Packed<T>::kWords < 4 ? 2 : 4;
    typedef uint32_t Words __attribute__((ext_vector_type(kWords), aligned(1)));
#pragma unroll
    for (uint32_t k = 0; k < Packed<T>::kWords / kWords; ++k) {
      Words w;
      __builtin_memcpy(&w, v.w + k * kWords, sizeof(w));
      __builtin_nontemporal_store(w, (STQ_GLOBAL Words*)p + k);
    }
  } else {
    T e[8];
    __builtin_memcpy(e, &v, sizeof(v));
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (c + i < cols) p[i] = e[i];
  }
}
template <class T>
__device__ __forceinline__ Packed<T> pack(const float (&v)[8]) {
  T e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = static_cast<T>(v[i]);
  Packed<T> r;
  __builtin_memcpy(&r, e, sizeof(r));
  return r;
}

}  // namespace
}  // namespace stq
