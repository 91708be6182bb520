// gfx950 matrix products of the 8-bit layer: int8 codes by int8 codes, and the gradients with respect to either operand, bf16 by
// int8 codes, on the matrix cores.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "stq_operators.h"
#include "stq_wave.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
#define STQ_LDS __attribute__((address_space(3)))

template <uint32_t TY> struct Elem;
template <> struct Elem<kF32> { using type = float; };
template <> struct Elem<kBF16> { using type = __bf16; };

// N elements of a row from element c on; those at or beyond `end` are zeros and are not read (nor any, of a row that is not there).
template <int N, class T>
struct Vec { T e[N]; };
template <int N, class T>
__device__ __forceinline__ Vec<N, T> load_vec(const T* row, uint32_t c, uint32_t end, bool there) {
  Vec<N, T> r;
  const STQ_GLOBAL T* p = as_global(row) + c;
  if (there && c + N <= end) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) r.e[i] = there && c + i < end ? p[i] : static_cast<T>(0);
  }
  return r;
}

// ---------------------------------------------------------------------------------------------- codes by codes
// A workgroup's 128 x 128 of the result, its four waves 64 x 64 each; 64 codes of the inner dimension at a time through LDS.
constexpr int kTileM = 128, kTileN = 128, kStepK = 64, kRowI8 = kStepK + 16;

template <uint32_t TO>
__global__ __launch_bounds__(256) void matmul_kernel(const MatmulArgs a) {
  __shared__ __align__(16) int8_t sa[kTileM * kRowI8], sb[kTileN * kRowI8];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t m0 = blockIdx.y * kTileM, n0 = blockIdx.x * kTileN;
  const uint32_t row = threadIdx.x >> 2, col = (threadIdx.x & 3) * 16;  // of a thread's two vectors of either tile, 64 rows apart
  const int8_t* pa = static_cast<const int8_t*>(a.a.p);
  const int8_t* pb = static_cast<const int8_t*>(a.b.p);
  Vec<16, int8_t> va[2], vb[2];
  auto load = [&](uint32_t k) {
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      const uint32_t m = m0 + row + 64 * h, n = n0 + row + 64 * h;
      va[h] = load_vec<16>(pa + m * a.a.stride, k + col, a.k, m < a.m);
      vb[h] = load_vec<16>(pb + n * a.b.stride, k + col, a.k, n < a.n);
    }
  };
  v4i acc[4][4] = {};
  const uint32_t wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  load(0);
  for (uint32_t k = 0; k < a.k; k += kStepK) {
    __syncthreads();
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      __builtin_memcpy(sa + (row + 64 * h) * kRowI8 + col, &va[h], 16);
      __builtin_memcpy(sb + (row + 64 * h) * kRowI8 + col, &vb[h], 16);
    }
    __syncthreads();
    if (k + kStepK < a.k) load(k + kStepK);
    v4i fa[4], fb[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      fa[i] = *reinterpret_cast<const v4i*>(sa + (wm + i * 16 + (lane & 15)) * kRowI8 + (lane >> 4) * 16);
      fb[i] = *reinterpret_cast<const v4i*>(sb + (wn + i * 16 + (lane & 15)) * kRowI8 + (lane >> 4) * 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
  }
  using T = typename Elem<TO>::type;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) {
      const uint32_t m = m0 + wm + i * 16 + (lane >> 4) * 4 + r;
      if (m >= a.m) continue;
      const float s = as_global(a.a.s)[m];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t n = n0 + wn + j * 16 + (lane & 15);
        if (n < a.n)
          as_global(static_cast<T*>(a.out.p))[m * a.out.stride + n] =
              static_cast<T>(static_cast<float>(acc[i][j][r]) * s * as_global(a.b.s)[n]);
      }
    }
}

// ---------------------------------------------------------------------------------------------- gradients
// out[i][j] = sum over c of dy(i, c) * s(c) * q(c, j): with respect to the input (WEIGHT false) i is the token and c the output, and
// dy's rows run along c; with respect to the weight i is the output and c the token, and dy's rows run along i.  The codes' rows run
// along j.  Codes are whole numbers below 2^8 and exact in bf16.  dy * s is rounded to bf16, or with TERMS = 2 to the sum of two, for
// results in fp32: what is left out is then at most 2^-16 of it.  Operands whose rows run along the result's rows or columns are read
// out of LDS transposed, four rows of 16 columns at a time.
constexpr int kTileI = 128, kTileJ = 128, kStepC = 32;
constexpr int kRowC = kStepC + 8;    // LDS row of an operand that runs along c
constexpr int kRowX = kTileI + 16;   // LDS row of one that runs along i or j

// a fragment of 16 columns from x0 on and 32 rows of a [c][x] tile: eight neighbouring rows of one column to a lane
__device__ __forceinline__ v8b transposed(const __bf16* tile, uint32_t x0, uint32_t lane) {
  const __bf16* p = tile + ((lane >> 4) * 8 + ((lane & 15) >> 2)) * kRowX + x0 + (lane & 3) * 4;
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((STQ_LDS v4s*)(p));
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((STQ_LDS v4s*)(p + 4 * kRowX));
  v8b r;
  __builtin_memcpy(&r, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &hi, 8);
  return r;
}

template <bool WEIGHT, uint32_t TY, uint32_t TO>
__global__ __launch_bounds__(256) void grad_kernel(const MatmulArgs a, uint32_t ni, uint32_t nj, uint32_t nc) {
  constexpr int kTerms = TO == kF32 ? 2 : 1;
  constexpr int kSizeA = WEIGHT ? kStepC * kRowX : kTileI * kRowC;
  __shared__ __align__(16) __bf16 sa[kTerms][kSizeA], sb[kStepC * kRowX];
  using T = typename Elem<TY>::type;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t i0 = blockIdx.y * kTileI, j0 = blockIdx.x * kTileJ;
  const T* dy = static_cast<const T*>(a.a.p);
  const int8_t* q = static_cast<const int8_t*>(a.b.p);
  // a thread's two vectors of eight: of a tile along x rows 16 apart, of one along c rows 64 apart
  const uint32_t xr = threadIdx.x >> 4, xc = (threadIdx.x & 15) * 8, cr = threadIdx.x >> 2, cc = (threadIdx.x & 3) * 8;
  Vec<8, T> va[2];
  Vec<8, int8_t> vb[2];
  Vec<8, float> vs;
  auto load = [&](uint32_t c) {
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      const uint32_t row = c + xr + 16 * h;
      vb[h] = load_vec<8>(q + row * a.b.stride, j0 + xc, nj, row < nc);
      if (WEIGHT) {
        va[h] = load_vec<8>(dy + row * a.a.stride, i0 + xc, ni, row < nc);
        vs.e[h] = row < nc ? as_global(a.b.s)[row] : 0.0f;
      } else {
        const uint32_t i = i0 + cr + 64 * h;
        va[h] = load_vec<8>(dy + i * a.a.stride, c + cc, nc, i < ni);
      }
    }
    if (!WEIGHT) vs = load_vec<8>(a.b.s, c + cc, nc, true);
  };
  v4f acc[4][4] = {};
  const uint32_t wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
  load(0);
  for (uint32_t c = 0; c < nc; c += kStepC) {
    __syncthreads();
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      v8b t[kTerms], b;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = static_cast<float>(va[h].e[e]) * (WEIGHT ? vs.e[h] : vs.e[e]);
        t[0][e] = static_cast<__bf16>(x);
        if (kTerms == 2) t[kTerms - 1][e] = static_cast<__bf16>(x - static_cast<float>(t[0][e]));
        b[e] = static_cast<__bf16>(static_cast<float>(vb[h].e[e]));
      }
      const uint32_t at = WEIGHT ? (xr + 16 * h) * kRowX + xc : (cr + 64 * h) * kRowC + cc;
#pragma unroll
      for (int k = 0; k < kTerms; ++k) __builtin_memcpy(&sa[k][at], &t[k], 16);
      __builtin_memcpy(&sb[(xr + 16 * h) * kRowX + xc], &b, 16);
    }
    __syncthreads();
    if (c + kStepC < nc) load(c + kStepC);
    v8b fb[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) fb[j] = transposed(sb, wj + j * 16, lane);
#pragma unroll
    for (int k = 0; k < kTerms; ++k)
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        v8b fa;
        if (WEIGHT) fa = transposed(sa[k], wi + i * 16, lane);
        else __builtin_memcpy(&fa, &sa[k][(wi + i * 16 + (lane & 15)) * kRowC + (lane >> 4) * 8], 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, fb[j], acc[i][j], 0, 0, 0);
      }
  }
  using O = typename Elem<TO>::type;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) {
      const uint32_t row = i0 + wi + i * 16 + (lane >> 4) * 4 + r;
      if (row >= ni) continue;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t col = j0 + wj + j * 16 + (lane & 15);
        if (col < nj) as_global(static_cast<O*>(a.out.p))[row * a.out.stride + col] = static_cast<O>(acc[i][j][r]);
      }
    }
}

template <class F>
void with_type(uint32_t type, F f) {
  if (type == kF32) f(std::integral_constant<uint32_t, kF32>{});
  else f(std::integral_constant<uint32_t, kBF16>{});
}

}  // namespace

int launch_matmul(const MatmulArgs& a, uint32_t out_type, uint32_t n_cu, void* stream) {
  const dim3 grid((a.n - 1) / kTileN + 1, (a.m - 1) / kTileM + 1);
  with_type(out_type, [&](auto to) { matmul_kernel<to()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
  return hipGetLastError();
}
int launch_matmul_grad_input(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, uint32_t n_cu, void* stream) {
  const dim3 grid((a.k - 1) / kTileJ + 1, (a.m - 1) / kTileI + 1);
  with_type(dy_type, [&](auto ty) { with_type(out_type, [&](auto to) {
    grad_kernel<false, ty(), to()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, a.m, a.k, a.n);
  }); });
  return hipGetLastError();
}
int launch_matmul_grad_weight(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, float* workspace, uint32_t n_cu, void* stream) {
  const dim3 grid((a.k - 1) / kTileJ + 1, (a.n - 1) / kTileI + 1);
  with_type(dy_type, [&](auto ty) { with_type(out_type, [&](auto to) {
    grad_kernel<true, ty(), to()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, a.n, a.k, a.m);
  }); });
  return hipGetLastError();
}
uint64_t grad_weight_bytes(uint64_t m, uint64_t n, uint64_t k) { return 0; }

}  // namespace stq
