// gfx950 kernels of the global gradient norm and of clipping to it: one pass each over all gradients of a call.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_device.h"
#include "stq_vectors.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

constexpr uint32_t kWaves = 8;  // of a workgroup

// The units of a launch go to its waves in turn, so that the card sweeps the gradients front to back.
template <class F>
__device__ __forceinline__ void for_units(const TensorDesc* desc, uint32_t n_tensors, uint32_t total, uint32_t lane, F f) {
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6)), waves = gridDim.x * kWaves;
  TensorDesc d;
  d.tile_begin = d.n_tiles = 0;
  for (uint64_t t = wave; t < total; t += waves) {
    if (t >= static_cast<uint64_t>(d.tile_begin) + d.n_tiles) d = load_desc(desc, find_begin(desc, n_tensors, static_cast<uint32_t>(t), lane));
    f(d, (t - d.tile_begin) * kTile);
  }
}

__device__ __forceinline__ double wave_sum(double x) {
  x = row_sum(x);
  x += __shfl_xor(x, 16);
  x += __shfl_xor(x, 32);
  return x;
}

// Sum over a unit of a tensor of elements T, from `base` on: eight neighbouring ones to a lane at a time.
template <class T>
__device__ __forceinline__ double unit_squares(const TensorDesc& d, uint64_t base, uint32_t lane) {
  const T* p = static_cast<const T*>(d.grad) + base;
  const uint64_t left = d.numel - base;
  Packed<T> v[4];
  if (left >= kTile) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[i] = load_packed(p + 512 * i + 8 * lane);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[i] = load_ending(p, 512 * i + 8 * lane, static_cast<uint32_t>(left));
  }
  double sum = 0.0;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      const double g = static_cast<double>(v[i].at(e));
      sum = __builtin_fma(g, g, sum);
    }
  return sum;
}

// The squares of all elements, in fp64: a product of two fp32 is exact there.  A workgroup leaves its sum in `partial`; the one that
// comes last adds them up, always in the same order, and leaves the counter at zero.
__global__ __launch_bounds__(kWaves * 64) void norm_kernel(const TensorDesc* desc, uint32_t n_tensors, uint32_t total, double* partial,
                                                           uint32_t* counter, double* norm) {
  __shared__ double held[kWaves];
  __shared__ uint32_t last;
  const uint32_t lane = threadIdx.x & 63;
  double sum = 0.0;
  for_units(desc, n_tensors, total, lane, [&](const TensorDesc& d, uint64_t base) {
    sum += d.bm ? unit_squares<__bf16>(d, base, lane) : unit_squares<float>(d, base, lane);
  });
  sum = wave_sum(sum);
  if (lane == 0) held[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = held[0];
#pragma unroll
    for (uint32_t w = 1; w < kWaves; ++w) sum += held[w];
    __hip_atomic_store(partial + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  sum = 0.0;
  for (uint32_t k = threadIdx.x; k < gridDim.x; k += kWaves * 64) sum += __hip_atomic_load(partial + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = wave_sum(sum);
  if (lane == 0) held[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = held[0];
#pragma unroll
    for (uint32_t w = 1; w < kWaves; ++w) sum += held[w];
    norm[0] = sum;
    norm[1] = __builtin_sqrt(sum);
    *counter = 0;
  }
}

template <class T>
__device__ __forceinline__ void clip_unit(const TensorDesc& d, uint64_t base, uint32_t lane, float c, float back) {
  const T* p = static_cast<const T*>(d.grad) + base;
  T* out = reinterpret_cast<T*>(d.param) + base;
  const uint32_t left = static_cast<uint32_t>(min(d.numel - base, static_cast<uint64_t>(kTile)));
  Packed<T> v[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) v[i] = load_ending(p, 512 * i + 8 * lane, left);
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    float g[8];
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) g[e] = v[i].at(e) * c * back;
    store_ending(out, 512 * i + 8 * lane, left, pack<T>(g));
  }
}

__global__ __launch_bounds__(kWaves * 64) void clip_kernel(const TensorDesc* desc, uint32_t n_tensors, uint32_t total, const double* norm, double most) {
  const uint32_t lane = threadIdx.x & 63;
  const double ratio = most / (__builtin_sqrt(norm[0]) + 1e-6);
  // (NaN stays.  A factor below fp32's normal numbers, of gradients near its largest, would lose digits: it is taken 2^64 times as large,
  // and the product brought back.)
  const bool tiny = ratio < 0x1p-126;
  const float c = ratio >= 1.0 ? 1.0f : static_cast<float>(tiny ? ratio * 0x1p64 : ratio), back = tiny ? 0x1p-64f : 1.0f;
  for_units(desc, n_tensors, total, lane, [&](const TensorDesc& d, uint64_t base) {
    if (c == 1.0f && d.param == d.grad) return;
    if (d.bm) clip_unit<__bf16>(d, base, lane, c, back);
    else clip_unit<float>(d, base, lane, c, back);
  });
}

uint32_t groups_of(uint32_t total, uint32_t n_cu) {
  const uint32_t need = (total + kWaves - 1) / kWaves, most = n_cu * 4 < kNormGroups ? n_cu * 4 : kNormGroups;
  return need == 0 ? 1 : (need < most ? need : most);
}

}  // namespace

int launch_grad_norm(const TensorDesc* desc, uint32_t n_tensors, uint32_t total_tiles, double* partial, double* norm, uint32_t n_cu, void* stream) {
  uint32_t* const counter = reinterpret_cast<uint32_t*>(partial + kNormGroups);
  norm_kernel<<<groups_of(total_tiles, n_cu), kWaves * 64, 0, static_cast<hipStream_t>(stream)>>>(desc, n_tensors, total_tiles, partial, counter, norm);
  return static_cast<int>(hipGetLastError());
}

int launch_clip(const TensorDesc* desc, uint32_t n_tensors, uint32_t total_tiles, const double* norm, double most, uint32_t n_cu, void* stream) {
  clip_kernel<<<groups_of(total_tiles, n_cu), kWaves * 64, 0, static_cast<hipStream_t>(stream)>>>(desc, n_tensors, total_tiles, norm, most);
  return static_cast<int>(hipGetLastError());
}

}  // namespace stq
