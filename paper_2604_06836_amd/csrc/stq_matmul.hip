// gfx950 matrix products of the 8-bit layer: int8 codes by int8 codes, and the gradients with respect to either operand, bf16 by
// int8 codes, on the matrix cores.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_vectors.h"

#pragma clang fp contract(off)

namespace stq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
#define STQ_LDS __attribute__((address_space(3)))

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

// What a lane has of a wave's result at a time is four neighbouring columns of one row; 16 bytes of a row, as an output has them.
struct Piece { uint32_t w[4]; };
template <uint32_t TO>
__device__ __forceinline__ void pack4(const float (&v)[4], void* to) {  // in LDS
  if constexpr (TO == kF32) {
    __builtin_memcpy(to, v, 16);
  } else {
    const __bf16 h[4] = {static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]), static_cast<__bf16>(v[2]), static_cast<__bf16>(v[3])};
    uint64_t w;
    __builtin_memcpy(&w, h, 8);
    __builtin_memcpy(to, &w, 8);
  }
}
template <uint32_t TO>
__device__ __forceinline__ void store_piece(const Mat& out, uint32_t row, uint32_t col, uint32_t end, const Piece& v) {
  using T = typename Elem<TO>::type;
  constexpr uint32_t kPer = 16 / sizeof(T);
  STQ_GLOBAL T* p = as_global(static_cast<T*>(out.p)) + row * out.stride + col;
  if (col + kPer <= end) {
    __builtin_memcpy(p, &v, 16);
  } else {
    T e[kPer];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i)
      if (col + i < end) p[i] = e[i];
  }
}
// A wave's result, FI x FJ fragments of 32 x 32 from row0, col0 on, into an output of rows x cols, by way of 32 rows of LDS of its own
// (`box`, 4096 FJ bytes for fp32), so that whole pieces of rows are stored, neighbouring ones together.  value(i, j, p, e): column
// 8 p + 4 (lane / 32) + e of row lane % 32 of fragment i, j.  Pieces lie at the places that their number and the row's give by
// exclusive or.
template <uint32_t TO, uint32_t FI, uint32_t FJ, class F>
__device__ __forceinline__ void store_tile(const Mat& out, uint32_t row0, uint32_t col0, uint32_t rows, uint32_t cols, char* box, uint32_t lane, F value) {
  constexpr uint32_t kSize = TO == kF32 ? 4 : 2, kRow = FJ * 32 * kSize, kPieces = kRow / 16, kShift = kRow == 256 ? 0 : (kRow == 128 ? 1 : 2);
  const auto place = [&](uint32_t row, uint32_t piece) { return row * kRow + ((piece ^ (row >> kShift)) & (kPieces - 1)) * 16; };
#pragma unroll
  for (uint32_t i = 0; i < FI; ++i) {
#pragma unroll
    for (uint32_t j = 0; j < FJ; ++j)
#pragma unroll
      for (uint32_t p = 0; p < 4; ++p) {
        float v[4];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[e] = value(i, j, p, e);
        const uint32_t byte = (j * 32 + p * 8 + (lane >> 5) * 4) * kSize;
        pack4<TO>(v, box + place(lane & 31, byte / 16) + byte % 16);
      }
#pragma unroll
    for (uint32_t h = 0; h < 32 * kPieces / 64; ++h) {
      const uint32_t row = h * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
      Piece v;
      __builtin_memcpy(&v, box + place(row, piece), 16);
      const uint32_t r = row0 + i * 32 + row, c = col0 + piece * (16 / kSize);
      if (r < rows && c < cols) store_piece<TO>(out, r, c, cols, v);
    }
  }
}
// Four elements where they are: for kernels whose results are few.
template <uint32_t TO>
__device__ __forceinline__ void store4(const Mat& out, uint32_t row, uint32_t col, uint32_t end, const float (&v)[4]) {
  using T = typename Elem<TO>::type;
  STQ_GLOBAL T* p = as_global(static_cast<T*>(out.p)) + row * out.stride + col;
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e)
    if (col + e < end) p[e] = static_cast<T>(v[e]);
}

// ---------------------------------------------------------------------------------------------- order of the tiles
// Workgroups go to the card's eight dies in turn, each of which has an L2 of its own: a die takes a run of tiles, in an order that
// goes through patches of up to eight rows of tiles, column by column, so that those at work together share rows and columns.
constexpr uint32_t kDies = 8, kPatch = 8;
struct TileAt { uint32_t row, col; };
__device__ __forceinline__ TileAt tile_at(uint32_t id, uint32_t rows, uint32_t cols) {
  const uint32_t total = rows * cols, each = total / kDies, more = total % kDies;
  const uint32_t die = id % kDies, t = die * each + min(die, more) + id / kDies;
  const uint32_t patch = t / (kPatch * cols), first = patch * kPatch, high = min(kPatch, rows - first);
  const uint32_t in = t - first * cols;
  return {first + in % high, in / high};
}

// ---------------------------------------------------------------------------------------------- codes by codes
// A workgroup's TM x TN of the result, its WM x WN waves a part each.  128 codes of the inner dimension at a time are loaded
// straight into LDS, into one of two buffers while the other is worked on.  A row is 128 bytes there, eight pieces of 16, which lie at
// the places that their number and the row's give by exclusive or, so that the reads of a fragment meet every bank once.
// Rows beyond the matrix' end repeat its last one; a step that goes beyond the rows' end comes through registers, with zeros there.
constexpr uint32_t kStepK = 128;

template <uint32_t TO, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void matmul_tile_kernel(const MatmulArgs a, uint32_t tiles_m, uint32_t tiles_n) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's compiler has no buffer descriptors)
  constexpr uint32_t FM = TM / WM / 32, FN = TN / WN / 32;  // fragments of 32 of a wave
  constexpr uint32_t kAtOnce = WM * WN * 8;                 // rows that a load of all waves fills
  __shared__ __align__(1024) int8_t a0[TM * kStepK], b0[TN * kStepK], a1[TM * kStepK], b1[TN * kStepK];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TileAt at = tile_at(blockIdx.x, tiles_m, tiles_n);
  const uint32_t m0 = at.row * TM, n0 = at.col * TN;
  int8_t* const pa = static_cast<int8_t*>(a.a.p) + m0 * a.a.stride;
  int8_t* const pb = static_cast<int8_t*>(a.b.p) + n0 * a.b.stride;
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(pa, 0, 0x7FFFFFFF, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(pb, 0, 0x7FFFFFFF, 0x00020000);
  // load i of a wave fills rows kAtOnce i + 8 wave .. + 7 of LDS, in lane order
  const uint32_t load_row = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ (load_row >> 1)) & 7;
  uint32_t oa[TM / kAtOnce], ob[TN / kAtOnce];
#pragma unroll
  for (uint32_t i = 0; i < TM / kAtOnce; ++i) oa[i] = min(load_row + kAtOnce * i, a.m - 1 - m0) * static_cast<uint32_t>(a.a.stride) + piece * 16;
#pragma unroll
  for (uint32_t i = 0; i < TN / kAtOnce; ++i) ob[i] = min(load_row + kAtOnce * i, a.n - 1 - n0) * static_cast<uint32_t>(a.b.stride) + piece * 16;
  const uint32_t both_end = (a.k + 2 * kStepK - 1) / (2 * kStepK) * (2 * kStepK);  // of the steps, taken two at a time
  const auto load = [&](uint32_t k, int8_t* la, int8_t* lb) {
    if (k + kStepK <= a.k) {
#pragma unroll
      for (uint32_t i = 0; i < TM / kAtOnce; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (STQ_LDS void*)(la + (i * kAtOnce + wave * 8) * kStepK), 16, oa[i], k, 0, 0);
#pragma unroll
      for (uint32_t i = 0; i < TN / kAtOnce; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (STQ_LDS void*)(lb + (i * kAtOnce + wave * 8) * kStepK), 16, ob[i], k, 0, 0);
    } else if (k < both_end) {
      const auto rest = [&](const int8_t* p, uint64_t stride, uint32_t last, int8_t* to, uint32_t rows) {
#pragma unroll 1
        for (uint32_t r = load_row; r < rows; r += kAtOnce) {
          const Vec<16, int8_t> v = load_vec<16>(p + min(r, last) * stride, k + piece * 16, a.k, true);
          __builtin_memcpy(to + r * kStepK + (lane & 7) * 16, &v, 16);
        }
      };
      rest(pa, a.a.stride, a.m - 1 - m0, la, TM);
      rest(pb, a.b.stride, a.n - 1 - n0, lb, TN);
    }
  };
  v16i acc[FM][FN] = {};
  const uint32_t wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);
  // A step out of la, lb, in units of one fragment of the tokens.  A unit's fragments are read kAhead units ahead, so that those of the
  // last kAhead are there when the workgroup meets: from then on the next step's buffers are full and this step's are free.
  constexpr uint32_t kUnits = kStepK / 32 * FM, kAhead = FM < 4 ? 2 : 4;
  v4i fa[kAhead], fb[2][FN];
  const uint32_t r = lane & 31;
  const auto at_piece = [&](uint32_t row, uint32_t s) { return row * kStepK + (((2 * s + (lane >> 5)) ^ (r >> 1)) & 7) * 16; };
  const auto read = [&](uint32_t u, const int8_t* la, const int8_t* lb) {
    const uint32_t s = u / FM, i = u % FM;
    fa[u % kAhead] = *reinterpret_cast<const v4i*>(la + at_piece(wm + i * 32 + r, s));
    if (i) return;
#pragma unroll
    for (uint32_t j = 0; j < FN; ++j) fb[s & 1][j] = *reinterpret_cast<const v4i*>(lb + at_piece(wn + j * 32 + r, s));
  };
  const auto work = [&](uint32_t k, int8_t* la, int8_t* lb, const int8_t* na, const int8_t* nb) {
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
      if (u == kUnits - kAhead) {
        __syncthreads();
        load(k + 2 * kStepK, la, lb);
      }
#pragma unroll
      for (uint32_t j = 0; j < FN; ++j)
        acc[u % FM][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[u / FM & 1][j], fa[u % kAhead], acc[u % FM][j], 0, 0, 0);
      if (u + kAhead < kUnits) read(u + kAhead, la, lb);
      else read(u + kAhead - kUnits, na, nb);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  load(0, a0, b0);
  __syncthreads();
  load(kStepK, a1, b1);
#pragma unroll
  for (uint32_t u = 0; u < kAhead; ++u) read(u, a0, b0);
  // Two steps at a time, of which the second may lie beyond the rows' end and be one of zeros: with one way out of the loop the sums
  // stay in their registers.  (What the last step reads ahead is not used.)
  for (uint32_t k = 0; k < a.k; k += 2 * kStepK) {
    work(k, a0, b0, a1, b1);
    work(k + kStepK, a1, b1, a0, b0);
  }
  // the scales and the result by way of LDS, into which nothing is loaded any more
  __syncthreads();
  float* const sm = reinterpret_cast<float*>(a1);
  float* const sn = reinterpret_cast<float*>(b1);
  for (uint32_t i = threadIdx.x; i < TM; i += WM * WN * 64) sm[i] = as_global(a.a.s)[min(m0 + i, a.m - 1)];
  for (uint32_t i = threadIdx.x; i < TN; i += WM * WN * 64) sn[i] = as_global(a.b.s)[min(n0 + i, a.n - 1)];
  __syncthreads();
  constexpr uint32_t kBox = 32 * FN * 32 * 4, kHalf = WM * WN / 2;
  static_assert(kHalf * kBox <= TM * kStepK && kHalf * kBox <= TN * kStepK, "a box for each wave");
  char* const box = wave < kHalf ? reinterpret_cast<char*>(a0) + wave * kBox : reinterpret_cast<char*>(b0) + (wave - kHalf) * kBox;
  store_tile<TO, FM, FN>(a.out, m0 + wm, n0 + wn, a.m, a.n, box, lane, [&](uint32_t i, uint32_t j, uint32_t p, uint32_t e) {
    return static_cast<float>(acc[i][j][p * 4 + e]) * sm[wm + i * 32 + (lane & 31)] * sn[wn + j * 32 + p * 8 + (lane >> 5) * 4 + e];
  });
#endif
}

// The same for operands of any alignment and inner size, through registers: 128 x 128 of the result, 64 codes at a time.
constexpr uint32_t kAnyM = 128, kAnyN = 128, kAnyK = 64, kAnyRow = kAnyK + 16;

template <uint32_t TO>
__global__ __launch_bounds__(256) void matmul_any_kernel(const MatmulArgs a, uint32_t tiles_m, uint32_t tiles_n) {
  __shared__ __align__(16) int8_t sa[kAnyM * kAnyRow], sb[kAnyN * kAnyRow];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const TileAt at = tile_at(blockIdx.x, tiles_m, tiles_n);
  const uint32_t m0 = at.row * kAnyM, n0 = at.col * kAnyN;
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
  for (uint32_t k = 0; k < a.k; k += kAnyK) {
    __syncthreads();
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      __builtin_memcpy(sa + (row + 64 * h) * kAnyRow + col, &va[h], 16);
      __builtin_memcpy(sb + (row + 64 * h) * kAnyRow + col, &vb[h], 16);
    }
    __syncthreads();
    if (k + kAnyK < a.k) load(k + kAnyK);
    v4i fa[4], fb[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      fa[i] = *reinterpret_cast<const v4i*>(sa + (wm + i * 16 + (lane & 15)) * kAnyRow + (lane >> 4) * 16);
      fb[i] = *reinterpret_cast<const v4i*>(sb + (wn + i * 16 + (lane & 15)) * kAnyRow + (lane >> 4) * 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t m = m0 + wm + i * 16 + (lane & 15);
    const float s = as_global(a.a.s)[min(m, a.m - 1)];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const uint32_t n = n0 + wn + j * 16 + (lane >> 4) * 4;
      float v[4];
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) v[e] = static_cast<float>(acc[i][j][e]) * s * as_global(a.b.s)[min(n + e, a.n - 1)];
      if (m < a.m) store4<TO>(a.out, m, n, a.n, v);
    }
  }
}

__device__ __forceinline__ v4i load_fragment(const int8_t* p) {
  v4i v;
  __builtin_memcpy(&v, as_global(p), 16);
  return v;
}

// Few tokens: what counts is how fast w's codes arrive.  A workgroup has 16 of w's rows and up to 16 G tokens; its eight waves share
// the inner dimension, a run of 128 codes each in turn, read straight into the fragments, and add up at the end.
template <uint32_t TO, int G>
__global__ __launch_bounds__(512) void matmul_few_kernel(const MatmulArgs a) {
  __shared__ __align__(16) v4i part[8][G][64];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * G;
  const uint32_t row = lane & 15, piece = (lane >> 4) * 16;
  const int8_t* pw = static_cast<const int8_t*>(a.b.p) + min(n0 + row, a.n - 1) * a.b.stride;
  const int8_t* px[G];
#pragma unroll
  for (uint32_t g = 0; g < G; ++g) px[g] = static_cast<const int8_t*>(a.a.p) + min(m0 + g * 16 + row, a.m - 1) * a.a.stride;
  v4i acc[G] = {};
  uint32_t k = wave * 128 + piece;
  constexpr uint32_t kAhead = 4;  // runs whose loads are under way together
  for (; (k & ~127u) + (kAhead - 1) * 1024 + 128 <= a.k; k += kAhead * 1024) {
    v4i fw[2 * kAhead], fx[G][2 * kAhead];
#pragma unroll
    for (uint32_t h = 0; h < 2 * kAhead; ++h) {
      const uint32_t c = k + (h >> 1) * 1024 + (h & 1) * 64;
      fw[h] = load_fragment(pw + c);
#pragma unroll
      for (uint32_t g = 0; g < G; ++g) fx[g][h] = load_fragment(px[g] + c);
    }
#pragma unroll
    for (uint32_t h = 0; h < 2 * kAhead; ++h)
#pragma unroll
      for (uint32_t g = 0; g < G; ++g) acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[h], fx[g][h], acc[g], 0, 0, 0);
  }
  for (; (k & ~127u) < a.k; k += 1024) {
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      const Vec<16, int8_t> w = load_vec<16>(pw, k + h * 64, a.k, true);
      v4i fw;
      __builtin_memcpy(&fw, &w, 16);
#pragma unroll
      for (uint32_t g = 0; g < G; ++g) {
        const Vec<16, int8_t> x = load_vec<16>(px[g], k + h * 64, a.k, true);
        v4i fx;
        __builtin_memcpy(&fx, &x, 16);
        acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, fx, acc[g], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (uint32_t g = 0; g < G; ++g) part[wave][g][lane] = acc[g];
  __syncthreads();
  if (wave >= G) return;
  v4i sum = part[0][wave][lane];
#pragma unroll
  for (uint32_t w = 1; w < 8; ++w) sum += part[w][wave][lane];
  const uint32_t m = m0 + wave * 16 + row, n = n0 + (lane >> 4) * 4;
  if (m >= a.m) return;
  const float s = as_global(a.a.s)[m];
  float v[4];
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) v[e] = static_cast<float>(sum[e]) * s * as_global(a.b.s)[min(n + e, a.n - 1)];
  store4<TO>(a.out, m, n, a.n, v);
}

// ---------------------------------------------------------------------------------------------- gradients
// out[i][j] = sum over c of dy(i, c) * s(c) * q(c, j): with respect to the input (WEIGHT false) i is the token and c the output, and
// dy's rows run along c; with respect to the weight i is the output and c the token, and dy's rows run along i.  The codes' rows run
// along j.  Codes are whole numbers below 2^8 and exact in bf16.  dy * s is rounded to bf16, or for results in fp32 to the sum of
// three, which hold all 24 bits of it.
// A workgroup has TI x TJ of the result, its WI x WJ waves a part each, and takes STEP of c at a time: what a step needs is loaded
// into registers two steps ahead, turned into bf16 and put into one of two LDS buffers one step ahead.  Operands whose rows run along
// i or j are read out of LDS transposed, four rows of 16 columns at a time.
template <uint32_t TO> constexpr int kTerms = TO == kF32 ? 3 : 1;

// A [c][x] tile: rows of X elements, 64 bytes more apart than that, so that the four rows of a transposed read meet every bank once.
template <uint32_t X> constexpr uint32_t kRowX = X + 32;
// A [i][c] tile of C = 32 or 64 elements a row, in pieces of eight which lie at the places that their number and the row's give by
// exclusive or, for the same reason.
template <uint32_t C>
__device__ __forceinline__ uint32_t place_c(uint32_t row, uint32_t piece) {
  return row * C + (C == 32 ? piece ^ ((row >> 2) & 3) : piece ^ ((row >> 1) & 7)) * 8;
}

// The fragment of columns x0 .. x0+31 and rows c0 .. c0+15 of a [c][x] tile: eight neighbouring rows of one column to a lane.
template <uint32_t X>
__device__ __forceinline__ v8b transposed(const __bf16* tile, uint32_t c0, uint32_t x0, uint32_t lane) {
  const __bf16* p = tile + (c0 + (lane >> 5) * 8 + ((lane & 15) >> 2)) * kRowX<X> + x0 + (lane & 16) + (lane & 3) * 4;
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((STQ_LDS v4s*)(p));
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((STQ_LDS v4s*)(p + 4 * kRowX<X>));
  v8b r;
  __builtin_memcpy(&r, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &hi, 8);
  return r;
}

struct GradShape {
  uint32_t ni, nj, nc;      // sizes of the sum
  uint32_t tiles_i, tiles_j;
  uint32_t splits, each;    // parts of c, and their length (a multiple of the step)
  float* partial;           // [splits][ni][nj] where there are several
};

// Elements x .. x+7 of a row of `size`; what lies beyond its end is anything that the row holds (it meets zeros, or results that are
// not stored).
template <class T>
__device__ __forceinline__ Packed<T> load_each(const T* row, uint32_t x, uint32_t size) {
  T e[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) e[i] = as_global(row)[min(x + i, size - 1)];
  Packed<T> r;
  __builtin_memcpy(&r, e, sizeof(r));
  return r;
}

// EIGHTS: the sizes along the operands' rows are multiples of eight, so that a vector is there or is not, and a tile's offsets fit 32
// bits.
template <bool WEIGHT, bool EIGHTS, uint32_t TY, uint32_t TO, int TI, int TJ, int WI, int WJ, int STEP>
__global__ __launch_bounds__(WI * WJ * 64) void grad_kernel(const MatmulArgs a, const GradShape g) {
  constexpr uint32_t kThreads = WI * WJ * 64, FI = TI / WI / 32, FJ = TJ / WJ / 32, T = kTerms<TO>;
  constexpr uint32_t kSizeA = WEIGHT ? STEP * kRowX<TI> : TI * STEP, kSizeB = STEP * kRowX<TJ>;
  constexpr uint32_t VA = TI * STEP / 8 / kThreads, VB = TJ * STEP / 8 / kThreads;  // vectors of eight of a thread
  __shared__ __align__(16) struct { __bf16 a0[T][kSizeA], b0[kSizeB], a1[T][kSizeA], b1[kSizeB]; } tiles;
  using D = typename Elem<TY>::type;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TileAt at = tile_at(blockIdx.x, g.tiles_i, g.tiles_j);
  const uint32_t i0 = at.row * TI, j0 = at.col * TJ;
  const uint32_t first = blockIdx.y * g.each, end = min(g.nc, first + g.each), last = first + (end - 1 - first) / STEP * STEP;
  const D* const dy = static_cast<const D*>(a.a.p);
  const int8_t* const q = static_cast<const int8_t*>(a.b.p);
  const float* const scales = a.b.s;
  // where a thread's vectors lie: of a [c][x] tile kThreads / (X / 8) rows apart, of the [i][c] one kThreads / (STEP / 8)
  constexpr uint32_t kApartB = kThreads / (TJ / 8), kApartA = WEIGHT ? kThreads / (TI / 8) : kThreads / (STEP / 8);
  const uint32_t br = threadIdx.x / (TJ / 8), bc = threadIdx.x % (TJ / 8) * 8;
  const uint32_t ar = threadIdx.x / (WEIGHT ? TI / 8 : STEP / 8), ac = threadIdx.x % (WEIGHT ? TI / 8 : STEP / 8) * 8;
  // EIGHTS: offsets of the vectors and scales from the start of a step, [1]: of the last one, where rows (or, along c, vectors) that
  // are not there repeat the last that is
  uint32_t oa[2][VA], ob[2][VB], os[2][WEIGHT ? VA : 1];
  if (EIGHTS) {
#pragma unroll
    for (uint32_t l = 0; l < 2; ++l) {
      const uint32_t rows = l ? end - 1 - last : STEP - 1;
#pragma unroll
      for (uint32_t h = 0; h < VB; ++h) ob[l][h] = min(br + kApartB * h, rows) * static_cast<uint32_t>(a.b.stride) + min(j0 + bc, g.nj - 8);
#pragma unroll
      for (uint32_t h = 0; h < VA; ++h) {
        const uint32_t r = ar + kApartA * h;
        if (WEIGHT) {
          os[l][h] = min(r, rows);
          oa[l][h] = os[l][h] * static_cast<uint32_t>(a.a.stride) + min(i0 + ac, g.ni - 8);
        } else {
          oa[l][h] = min(r, g.ni - 1 - i0) * static_cast<uint32_t>(a.a.stride) + min(ac, rows - 7);
        }
      }
      if (!WEIGHT) os[l][0] = min(ac, rows - 7);
    }
  }

  Packed<D> va[VA];
  Packed<int8_t> vb[VB];
  float vs[8];  // scales: of each vector of dy's, or (along c) of its elements
  // The loads of piece p, a vector of dy or of the codes, of step c (beyond the last step: of that).
  const auto load = [&](uint32_t c, uint32_t p) {
    c = min(c, last);
    const bool l = c == last;
    if (p < VA) {
      const uint32_t h = p;
      if (EIGHTS) va[h] = load_packed(dy + (WEIGHT ? c : i0) * a.a.stride + (WEIGHT ? 0 : c) + (l ? oa[1][h] : oa[0][h]));
      else if (WEIGHT) va[h] = load_each(dy + min(c + ar + kApartA * h, end - 1) * a.a.stride, i0 + ac, g.ni);
      else va[h] = load_each(dy + min(i0 + ar + kApartA * h, g.ni - 1) * a.a.stride, c + ac, end);
      if (WEIGHT) {
        vs[h] = EIGHTS ? as_global(scales + c)[l ? os[1][h] : os[0][h]] : as_global(scales)[min(c + ar + kApartA * h, end - 1)];
      } else if (h == VA - 1) {
        const Packed<float> t = EIGHTS ? load_packed(scales + c + (l ? os[1][0] : os[0][0])) : load_each(scales, c + ac, end);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) vs[e] = t.at(e);
      }
    } else {
      const uint32_t h = p - VA;
      if (EIGHTS) vb[h] = load_packed(q + c * a.b.stride + (l ? ob[1][h] : ob[0][h]));
      else vb[h] = load_each(q + min(c + br + kApartB * h, end - 1) * a.b.stride, j0 + bc, g.nj);
    }
  };
  // Piece p, which was loaded for step c, into LDS.  What lies beyond the sum's end is zero, whatever was read in its place.
  const auto put = [&](uint32_t c, uint32_t p, __bf16 (*ta)[kSizeA], __bf16* tb) {
    if (p < VA) {
      const uint32_t h = p;
      if (WEIGHT) va[h].keep(c + ar + kApartA * h < end);
      else if (EIGHTS) va[h].keep(c + ac < end);
      v8b t[T];
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        float x = va[h].at(e), s = vs[WEIGHT ? h : e];
        if (!WEIGHT) {  // (the scales repeat, too, and need not be finite)
          const bool there = c + ac + (EIGHTS ? 0 : e) < end;
          x = EIGHTS || there ? x : 0.0f;
          s = there ? s : 0.0f;
        }
        x *= s;
#pragma unroll
        for (uint32_t k = 0; k < T; ++k) {
          t[k][e] = static_cast<__bf16>(x);
          x -= static_cast<float>(t[k][e]);
        }
      }
      const uint32_t row = ar + kApartA * h, to = WEIGHT ? row * kRowX<TI> + ac : place_c<STEP>(row, ac / 8);
#pragma unroll
      for (uint32_t k = 0; k < T; ++k) __builtin_memcpy(&ta[k][to], &t[k], 16);
    } else {
      const uint32_t h = p - VA;
      v8b t;
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) t[e] = static_cast<__bf16>(vb[h].at(e));
      __builtin_memcpy(&tb[(br + kApartB * h) * kRowX<TJ> + bc], &t, 16);
    }
  };
  v16f acc[FI][FJ] = {};
  const uint32_t wi = wave / WJ * (TI / WI), wj = wave % WJ * (TJ / WJ);
  // A step out of ta, tb, in units of one fragment of dy.  A unit's fragments are read two units ahead; on the way, between the matrix
  // instructions, so that the vector unit and LDS work beside the matrix cores, what was loaded for the next step goes into na, nb, and
  // the loads of the step after that begin.  When the workgroup meets, before the last two units, all of this step has been read and all
  // of the next is there.
  constexpr uint32_t kUnits = STEP / 16 * T * FI, kPieces = VA + VB;
  v8b fa[2], fb[2][FJ];
  const auto read = [&](uint32_t u, const __bf16 (*ta)[kSizeA], const __bf16* tb) {
    const uint32_t s = u / (T * FI), k = u / FI % T, i = u % FI;
    if (WEIGHT) fa[u & 1] = transposed<TI>(ta[k], s * 16, wi + i * 32, lane);
    else __builtin_memcpy(&fa[u & 1], &ta[k][place_c<STEP>(wi + i * 32 + (lane & 31), s * 2 + (lane >> 5))], 16);
    if (u % (T * FI)) return;
#pragma unroll
    for (uint32_t j = 0; j < FJ; ++j) fb[s & 1][j] = transposed<TJ>(tb, s * 16, wj + j * 32, lane);
  };
  const auto work = [&](uint32_t c, const __bf16 (*ta)[kSizeA], const __bf16* tb, __bf16 (*na)[kSizeA], __bf16* nb) {
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
      if (u == kUnits - 2) __syncthreads();
#pragma unroll
      for (uint32_t j = 0; j < FJ; ++j)
        acc[u % FI][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[u / (T * FI) & 1][j], fa[u & 1], acc[u % FI][j], 0, 0, 0);
      if (u + 2 < kUnits) read(u + 2, ta, tb);
      else read(u + 2 - kUnits, na, nb);
#pragma unroll
      for (uint32_t p = 0; p < kPieces; ++p)
        if (p * (kUnits - 2) / kPieces == u) {
          put(c + STEP, p, na, nb);
          load(c + 2 * STEP, p);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (uint32_t p = 0; p < kPieces; ++p) load(first, p);
#pragma unroll
  for (uint32_t p = 0; p < kPieces; ++p) put(first, p, tiles.a0, tiles.b0);
#pragma unroll
  for (uint32_t p = 0; p < kPieces; ++p) load(first + STEP, p);
  __syncthreads();
  read(0, tiles.a0, tiles.b0);
  read(1, tiles.a0, tiles.b0);
  // Two steps at a time, of which the second may lie beyond the sum's end and be one of zeros: with one way out of the loop the sums
  // stay in their registers.  (What the last step reads ahead is not used.)
  for (uint32_t c = first; c < end; c += 2 * STEP) {
    work(c, tiles.a0, tiles.b0, tiles.a1, tiles.b1);
    work(c + STEP, tiles.a1, tiles.b1, tiles.a0, tiles.b0);
  }
  __syncthreads();
  const auto value = [&](uint32_t i, uint32_t j, uint32_t p, uint32_t e) { return acc[i][j][p * 4 + e]; };
  constexpr uint32_t kBox = 32 * FJ * 32 * (TI == 256 && TO != kF32 ? 2 : 4);
  static_assert(sizeof(tiles) >= WI * WJ * kBox, "a box for each wave");
  char* const box = reinterpret_cast<char*>(&tiles) + wave * kBox;
  if (TI != 256 && g.splits > 1) {  // (sums taken in parts are of small tiles)
    const Mat part{g.partial + static_cast<uint64_t>(blockIdx.y) * g.ni * g.nj, nullptr, g.nj, 0, 0};
    store_tile<kF32, FI, FJ>(part, i0 + wi, j0 + wj, g.ni, g.nj, box, lane, value);
  } else {
    store_tile<TO, FI, FJ>(a.out, i0 + wi, j0 + wj, g.ni, g.nj, box, lane, value);
  }
}

// The parts of a sum that was taken in parts, in one order.
template <uint32_t TO>
__global__ __launch_bounds__(256) void join_kernel(const Mat out, const float* partial, uint32_t splits, uint32_t ni, uint32_t nj) {
  const uint32_t per_row = (nj + 3) / 4;
  const uint64_t total = static_cast<uint64_t>(ni) * per_row, size = static_cast<uint64_t>(ni) * nj;
  for (uint64_t t = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; t < total; t += static_cast<uint64_t>(gridDim.x) * 256) {
    const uint32_t row = static_cast<uint32_t>(t / per_row), col = static_cast<uint32_t>(t % per_row) * 4;
    float v[4] = {0, 0, 0, 0};
    for (uint32_t k = 0; k < splits; ++k) {
      const Vec<4, float> p = load_vec<4>(partial + k * size + static_cast<uint64_t>(row) * nj, col, nj, true);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += p.e[e];
    }
    store4<TO>(out, row, col, nj, v);
  }
}

uint32_t tiles_of(uint32_t size, uint32_t tile) { return (size - 1) / tile + 1; }

// Whether a matrix' rows can be loaded straight into LDS: 16-byte pieces, a tile's rows within reach of a 31-bit offset.
bool in_pieces(const Mat& x) { return (reinterpret_cast<uintptr_t>(x.p) & 15) == 0 && x.stride % 16 == 0 && x.stride < (1u << 22); }

template <uint32_t TO>
void run_matmul(const MatmulArgs& a, uint32_t n_cu, hipStream_t st) {
  if (a.m <= 64) {
    const uint32_t groups = tiles_of(a.n, 16);
    if (a.m <= 16) matmul_few_kernel<TO, 1><<<groups, 512, 0, st>>>(a);
    else if (a.m <= 32) matmul_few_kernel<TO, 2><<<groups, 512, 0, st>>>(a);
    else matmul_few_kernel<TO, 4><<<groups, 512, 0, st>>>(a);
    return;
  }
  if (!in_pieces(a.a) || !in_pieces(a.b)) {
    const uint32_t rows = tiles_of(a.m, kAnyM), cols = tiles_of(a.n, kAnyN);
    matmul_any_kernel<TO><<<rows * cols, 256, 0, st>>>(a, rows, cols);
    return;
  }
  const auto count = [&](uint32_t t) { return static_cast<uint64_t>(tiles_of(a.m, t)) * tiles_of(a.n, t); };
  const uint32_t t = count(256) >= n_cu ? 256 : (count(128) >= n_cu ? 128 : 64), rows = tiles_of(a.m, t), cols = tiles_of(a.n, t);
  if (t == 256) matmul_tile_kernel<TO, 256, 256, 2, 4><<<rows * cols, 512, 0, st>>>(a, rows, cols);
  else if (t == 128) matmul_tile_kernel<TO, 128, 128, 2, 2><<<rows * cols, 256, 0, st>>>(a, rows, cols);
  else matmul_tile_kernel<TO, 64, 64, 2, 2><<<rows * cols, 256, 0, st>>>(a, rows, cols);
}

// Parts of the tokens for a weight gradient of few tiles: as many as give every CU a workgroup, of 512 tokens at least (a part
// costs a write and a read of the result in fp32).
constexpr uint32_t kCus = 256, kLeastPart = 512;
uint32_t splits_of(uint64_t m, uint64_t n, uint64_t k) {
  const uint64_t tiles = ((n + 127) / 128) * ((k + 127) / 128);
  if (tiles * 2 > kCus || m < 2 * kLeastPart) return 1;
  const uint64_t s = kCus / tiles, most = m / kLeastPart;
  return static_cast<uint32_t>(s < most ? s : most);
}

template <bool WEIGHT, uint32_t TY, uint32_t TO>
void run_grad(const MatmulArgs& a, GradShape g, uint32_t n_cu, hipStream_t st) {
  constexpr int kStepC = 32;
  const auto count = [&](uint32_t t) { return static_cast<uint64_t>(tiles_of(g.ni, t)) * tiles_of(g.nj, t); };
  const bool eights = g.nj % 8 == 0 && (WEIGHT ? g.ni : g.nc) % 8 == 0 && a.a.stride < (1u << 22) && a.b.stride < (1u << 22);
  const uint32_t t = eights && g.splits == 1 && count(256) >= n_cu ? 256 : 128;
  g.tiles_i = tiles_of(g.ni, t);
  g.tiles_j = tiles_of(g.nj, t);
  const auto join = [&] {
    const uint64_t groups = (static_cast<uint64_t>(g.ni) * ((g.nj + 3) / 4) + 255) / 256;
    join_kernel<TO><<<static_cast<uint32_t>(groups < 4096 ? groups : 4096), 256, 0, st>>>(a.out, g.partial, g.splits, g.ni, g.nj);
  };
  if (g.nc == 0) {  // no tokens: a sum of nothing
    g.splits = 0;
    return join();
  }
  g.each = tiles_of(g.nc, g.splits * 64) * 64;
  g.splits = tiles_of(g.nc, g.each);
  const dim3 grid(g.tiles_i * g.tiles_j, g.splits);
  if (!eights) grad_kernel<WEIGHT, false, TY, TO, 128, 128, 2, 2, kStepC><<<grid, 256, 0, st>>>(a, g);
  else if (t == 256) grad_kernel<WEIGHT, true, TY, TO, 256, 256, 2, 4, kStepC><<<grid, 512, 0, st>>>(a, g);
  else grad_kernel<WEIGHT, true, TY, TO, 128, 128, 2, 2, kStepC><<<grid, 256, 0, st>>>(a, g);
  if (g.splits > 1) join();
}
template <bool WEIGHT>
int run_grads(const MatmulArgs& a, const GradShape& g, uint32_t dy_type, uint32_t out_type, uint32_t n_cu, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dy_type == kF32) {
    if (out_type == kF32) run_grad<WEIGHT, kF32, kF32>(a, g, n_cu, st);
    else run_grad<WEIGHT, kF32, kBF16>(a, g, n_cu, st);
  } else {
    if (out_type == kF32) run_grad<WEIGHT, kBF16, kF32>(a, g, n_cu, st);
    else run_grad<WEIGHT, kBF16, kBF16>(a, g, n_cu, st);
  }
  return hipGetLastError();
}

}  // namespace

int launch_matmul(const MatmulArgs& a, uint32_t out_type, uint32_t n_cu, void* stream) {
  if (out_type == kF32) run_matmul<kF32>(a, n_cu, static_cast<hipStream_t>(stream));
  else run_matmul<kBF16>(a, n_cu, static_cast<hipStream_t>(stream));
  return hipGetLastError();
}
int launch_matmul_grad_input(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, uint32_t n_cu, void* stream) {
  return run_grads<false>(a, GradShape{a.m, a.k, a.n, 0, 0, 1, 0, nullptr}, dy_type, out_type, n_cu, stream);
}
int launch_matmul_grad_weight(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, float* workspace, uint32_t n_cu, void* stream) {
  return run_grads<true>(a, GradShape{a.n, a.k, a.m, 0, 0, splits_of(a.m, a.n, a.k), 0, workspace}, dy_type, out_type, n_cu, stream);
}
uint64_t grad_weight_bytes(uint64_t m, uint64_t n, uint64_t k) {
  const uint64_t s = splits_of(m, n, k);
  return s > 1 ? 4 * s * n * k : 0;
}

}  // namespace stq
