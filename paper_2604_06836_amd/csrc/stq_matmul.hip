// gfx950 matrix products of the 8-bit layer: int8 codes by int8 codes, and the gradients with respect to either operand, bf16 by
// int8 codes, on the matrix cores.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

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

__device__ __forceinline__ v4i load_fragment(const int8_t* p) {
  v4i v;
  __builtin_memcpy(&v, as_global(p), 16);
  return v;
}
// 16 codes of which only the first `valid` (any number) are wanted, zeros in place of the others, at offset `at` of a matrix of `total`
// (16 at least): what would lie beyond its end is not read, but 16 that end there, moved into place.
__device__ __forceinline__ v4i load_last(const int8_t* p, int64_t at, int64_t total, int32_t valid) {
  const int64_t from = min(at, total - 16);
  v4i v = load_fragment(p + from);
  if (valid >= 16 && from == at) return v;
  const int32_t far = valid > 0 ? static_cast<int32_t>(at - from) : 0;  // (what is wanted is there: below 16)
  for (int32_t k = 0; k < far; ++k) {
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = __builtin_amdgcn_alignbit(v[i + 1], v[i], 8);
    v[3] = static_cast<int>(static_cast<uint32_t>(v[3]) >> 8);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int32_t n = valid - 4 * i;
    v[i] &= n >= 4 ? -1 : (n <= 0 ? 0 : (1 << (8 * n)) - 1);
  }
  return v;
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
// What the lanes of a wave have put into LDS is there for the others after this, and what they have read may be written over: LDS takes a
// wave's accesses in their order, so that only the compiler has to keep it.
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
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
    lanes_meet();
#pragma unroll
    for (uint32_t h = 0; h < 32 * kPieces / 64; ++h) {
      const uint32_t row = h * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
      Piece v;
      __builtin_memcpy(&v, box + place(row, piece), 16);
      const uint32_t r = row0 + i * 32 + row, c = col0 + piece * (16 / kSize);
      if (r < rows && c < cols) store_piece<TO>(out, r, c, cols, v);
    }
    lanes_meet();
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
// PIECES: whether the rows lie in 16-byte pieces; others come through registers altogether, loaded a step ahead.
// 256 x 256 with eight waves of 128 x 64: as much of w and x in registers as two waves on a SIMD can hold, so that LDS is read for a step
// in less time than the matrix cores take for it.  16384 x 11008 x 4096: 656 to 685 us, 2.25 to 2.16 Pop/s, little below this card's library
// product of int8 codes (2.28 to 2.37 for 8192^3); of zeros 3.3, so that what bounds it is the card's power.
[[maybe_unused]] constexpr uint32_t kStepK = 128;

template <uint32_t TO, int TM, int TN, int WM, int WN, bool PIECES>
__global__ __launch_bounds__(WM * WN * 64) void matmul_tile_kernel(const MatmulArgs a, uint32_t tiles_m, uint32_t tiles_n) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's compiler has no buffer descriptors)
  constexpr uint32_t FM = TM / WM / 32, FN = TN / WN / 32;  // fragments of 32 of a wave
  constexpr uint32_t kAtOnce = WM * WN * 8;                 // rows that a load of all waves fills
  constexpr uint32_t VA = TM / kAtOnce, VB = TN / kAtOnce;
  __shared__ __align__(1024) int8_t a0[TM * kStepK], b0[TN * kStepK], a1[TM * kStepK], b1[TN * kStepK];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (group_number() >= tiles_m * tiles_n) return;
  const TileAt at = tile_at(group_number(), tiles_m, tiles_n);
  const uint32_t m0 = at.row * TM, n0 = at.col * TN;
  int8_t* const pa = static_cast<int8_t*>(a.a.p) + m0 * a.a.stride;
  int8_t* const pb = static_cast<int8_t*>(a.b.p) + n0 * a.b.stride;
  const int64_t total_a = static_cast<int64_t>((a.m - 1 - m0) * a.a.stride + a.k), total_b = static_cast<int64_t>((a.n - 1 - n0) * a.b.stride + a.k);
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(pa, 0, 0x7FFFFFFF, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(pb, 0, 0x7FFFFFFF, 0x00020000);
  // load i of a wave fills rows kAtOnce i + 8 wave .. + 7 of LDS, in lane order
  const uint32_t load_row = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ (load_row >> 1)) & 7, to = load_row * kStepK + (lane & 7) * 16;
  uint32_t oa[VA], ob[VB];
#pragma unroll
  for (uint32_t i = 0; i < VA; ++i) oa[i] = min(load_row + kAtOnce * i, a.m - 1 - m0) * static_cast<uint32_t>(a.a.stride) + piece * 16;
#pragma unroll
  for (uint32_t i = 0; i < VB; ++i) ob[i] = min(load_row + kAtOnce * i, a.n - 1 - n0) * static_cast<uint32_t>(a.b.stride) + piece * 16;
  const uint32_t both_end = (a.k + 2 * kStepK - 1) / (2 * kStepK) * (2 * kStepK);  // of the steps, taken two at a time
  const auto load_pieces = [&](uint32_t k, int8_t* la, int8_t* lb) {
    if (k + kStepK <= a.k) {
#pragma unroll
      for (uint32_t i = 0; i < VA; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (STQ_LDS void*)(la + (i * kAtOnce + wave * 8) * kStepK), 16, oa[i], k, 0, 0);
#pragma unroll
      for (uint32_t i = 0; i < VB; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (STQ_LDS void*)(lb + (i * kAtOnce + wave * 8) * kStepK), 16, ob[i], k, 0, 0);
    } else if (k < both_end) {
      const int32_t valid = static_cast<int32_t>(a.k) - static_cast<int32_t>(k + piece * 16);
#pragma unroll 1
      for (uint32_t i = 0; i < TM / kAtOnce; ++i) {
        const v4i v = load_last(pa, static_cast<int64_t>(min(load_row + kAtOnce * i, a.m - 1 - m0)) * a.a.stride + k + piece * 16, total_a, valid);
        __builtin_memcpy(la + to + i * kAtOnce * kStepK, &v, 16);
      }
#pragma unroll 1
      for (uint32_t i = 0; i < TN / kAtOnce; ++i) {
        const v4i v = load_last(pb, static_cast<int64_t>(min(load_row + kAtOnce * i, a.n - 1 - n0)) * a.b.stride + k + piece * 16, total_b, valid);
        __builtin_memcpy(lb + to + i * kAtOnce * kStepK, &v, 16);
      }
    }
  };
  v4i va[PIECES ? 1 : VA], vb[PIECES ? 1 : VB];
  const auto load_any = [&](uint32_t k) {
    if (k + kStepK <= a.k) {
#pragma unroll
      for (uint32_t i = 0; i < VA; ++i) va[i] = load_fragment(pa + k + oa[i]);
#pragma unroll
      for (uint32_t i = 0; i < VB; ++i) vb[i] = load_fragment(pb + k + ob[i]);
    } else if (k < both_end) {
      const int32_t valid = static_cast<int32_t>(a.k) - static_cast<int32_t>(k + piece * 16);
#pragma unroll
      for (uint32_t i = 0; i < VA; ++i) va[i] = load_last(pa, static_cast<int64_t>(oa[i]) + k, total_a, valid);
#pragma unroll
      for (uint32_t i = 0; i < VB; ++i) vb[i] = load_last(pb, static_cast<int64_t>(ob[i]) + k, total_b, valid);
    }
  };
  const auto put_any = [&](int8_t* la, int8_t* lb) {
#pragma unroll
    for (uint32_t i = 0; i < VA; ++i) __builtin_memcpy(la + to + i * kAtOnce * kStepK, &va[i], 16);
#pragma unroll
    for (uint32_t i = 0; i < VB; ++i) __builtin_memcpy(lb + to + i * kAtOnce * kStepK, &vb[i], 16);
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
  const auto work = [&](uint32_t k, int8_t* la, int8_t* lb, int8_t* na, int8_t* nb) {
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
      if (u == kUnits - kAhead) {
        __syncthreads();
        if (PIECES) load_pieces(k + 2 * kStepK, la, lb);
      }
#pragma unroll
      for (uint32_t j = 0; j < FN; ++j)
        acc[u % FM][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[u / FM & 1][j], fa[u % kAhead], acc[u % FM][j], 0, 0, 0);
      if (u + kAhead < kUnits) read(u + kAhead, la, lb);
      else read(u + kAhead - kUnits, na, nb);
      if (!PIECES && u == 0) {
        put_any(na, nb);
        load_any(k + 2 * kStepK);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (PIECES) {
    load_pieces(0, a0, b0);
  } else {
    load_any(0);
    put_any(a0, b0);
    load_any(kStepK);
  }
  __syncthreads();
  if (PIECES) load_pieces(kStepK, a1, b1);
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

// Few tokens: what counts is how fast w's codes arrive.  A workgroup has 16 R of w's rows and up to 16 G tokens; its eight waves share
// the inner dimension, a run of 128 codes each in turn, read straight into the fragments, and add up at the end.  The loads of A runs
// are under way together.  One token through 11008 x 4096: 11.0 us, of which the codes would take 8.4 at the rate of a large copy; a
// launch and its end are most of the rest (32000 x 4096: 4.8 TB/s).  (Workgroups beyond w's rows, in launches of several layers, repeat its
// last one and store nothing: a way out for them took 0.2 us of every call.)
template <uint32_t TO, int G, int R, int A>
__global__ __launch_bounds__(512) void matmul_few_kernel(const MatmulArgs a) {
  __shared__ __align__(16) v4i part[8][G * R][64];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t n0 = group_number() * 16 * R, row = lane & 15, piece = (lane >> 4) * 16;
  const int8_t* const px = static_cast<const int8_t*>(a.a.p);
  const int8_t* const pw = static_cast<const int8_t*>(a.b.p);
  uint64_t ox[G], ow[R];
#pragma unroll
  for (uint32_t g = 0; g < G; ++g) ox[g] = min(g * 16 + row, a.m - 1) * a.a.stride + piece;
#pragma unroll
  for (uint32_t r = 0; r < R; ++r) ow[r] = min(n0 + r * 16 + row, a.n - 1) * a.b.stride + piece;
  v4i acc[R][G] = {};
  for (uint32_t k0 = wave * 128; k0 < a.k; k0 += A * 1024) {
    v4i fw[A][2][R], fx[A][2][G];
#pragma unroll
    for (uint32_t t = 0; t < A; ++t) {
      const uint32_t k = k0 + t * 1024;
      if (k + 128 > a.k) break;
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h) {
#pragma unroll
        for (uint32_t r = 0; r < R; ++r) fw[t][h][r] = load_fragment(pw + ow[r] + k + h * 64);
#pragma unroll
        for (uint32_t g = 0; g < G; ++g) fx[t][h][g] = load_fragment(px + ox[g] + k + h * 64);
      }
    }
#pragma unroll
    for (uint32_t t = 0; t < A; ++t) {
      if (k0 + t * 1024 + 128 > a.k) break;
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
        for (uint32_t r = 0; r < R; ++r)
#pragma unroll
          for (uint32_t g = 0; g < G; ++g) acc[r][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[t][h][r], fx[t][h][g], acc[r][g], 0, 0, 0);
    }
  }
  if (const uint32_t k = a.k & ~127u; k < a.k && k / 128 % 8 == wave) {  // a run that is no whole one
    const int64_t total_x = static_cast<int64_t>((a.m - 1) * a.a.stride + a.k), total_w = static_cast<int64_t>((a.n - 1) * a.b.stride + a.k);
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
      const int32_t valid = static_cast<int32_t>(a.k) - static_cast<int32_t>(k + h * 64 + piece);
      v4i fw[R], fx[G];
#pragma unroll
      for (uint32_t r = 0; r < R; ++r) fw[r] = load_last(pw, ow[r] + k + h * 64, total_w, valid);
#pragma unroll
      for (uint32_t g = 0; g < G; ++g) fx[g] = load_last(px, ox[g] + k + h * 64, total_x, valid);
#pragma unroll
      for (uint32_t r = 0; r < R; ++r)
#pragma unroll
        for (uint32_t g = 0; g < G; ++g) acc[r][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[r], fx[g], acc[r][g], 0, 0, 0);
    }
  }
#pragma unroll
  for (uint32_t r = 0; r < R; ++r)
#pragma unroll
    for (uint32_t g = 0; g < G; ++g) part[wave][r * G + g][lane] = acc[r][g];
  __syncthreads();
  if (wave >= G * R) return;
  v4i sum = part[0][wave][lane];
#pragma unroll
  for (uint32_t w = 1; w < 8; ++w) sum += part[w][wave][lane];
  const uint32_t m = wave % G * 16 + row, n = n0 + wave / G * 16 + (lane >> 4) * 4;
  if (m >= a.m) return;
  const float s = as_global(a.a.s)[m];
  float v[4];
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) v[e] = static_cast<float>(sum[e]) * s * as_global(a.b.s)[min(n + e, a.n - 1)];
  store4<TO>(a.out, m, n, a.n, v);
}

// Operands of fewer than 16 codes, or of rows too far apart for the offsets of a tile: an element to a thread.
template <uint32_t TO>
__global__ __launch_bounds__(256) void matmul_each_kernel(const MatmulArgs a) {
  const uint64_t total = static_cast<uint64_t>(a.m) * a.n;
  for (uint64_t t = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; t < total; t += static_cast<uint64_t>(gridDim.x) * 256) {
    const uint64_t m = t / a.n, n = t % a.n;
    const STQ_GLOBAL int8_t* x = as_global(static_cast<const int8_t*>(a.a.p)) + m * a.a.stride;
    const STQ_GLOBAL int8_t* w = as_global(static_cast<const int8_t*>(a.b.p)) + n * a.b.stride;
    int32_t sum = 0;
    for (uint32_t k = 0; k < a.k; ++k) sum += x[k] * w[k];
    using T = typename Elem<TO>::type;
    as_global(static_cast<T*>(a.out.p))[m * a.out.stride + n] = static_cast<T>(static_cast<float>(sum) * as_global(a.a.s)[m] * as_global(a.b.s)[n]);
  }
}

// ---------------------------------------------------------------------------------------------- gradients
// out[i][j] = sum over c of dy(i, c) * s(c) * q(c, j): with respect to the input (WEIGHT false) i is the token and c the output, and
// dy's rows run along c; with respect to the weight i is the output and c the token, and dy's rows run along i.  The codes' rows run
// along j.  Codes are whole numbers below 2^8 and exact in bf16.  dy * s enters as the sum of T bf16: three for results in fp32, which
// hold all 24 bits of it; two for results in bf16.  (One would add to them about as much again as their own rounding, 2.3e-3 for 1.7e-3
// of the result's 2-norm, at three fifths of the time; but a small element beside large ones, of an output or token with large
// gradients, it leaves with an error of half of the result's root mean square.)
// A workgroup has TI x TJ of the result, its WI x WJ waves a part each, and takes STEP of c at a time: what a step needs is loaded
// into registers two steps ahead, turned into bf16 and put into one of two LDS buffers one step ahead.  Operands whose rows run along
// i or j are read out of LDS transposed, four rows of 16 columns at a time.  256 x 256 with eight waves of 128 x 64, as above: dx 8192 x
// 4096 x 11008 in bf16 in 1216 to 1301 us, 1.21 to 1.14 Pflop/s of the matrix cores (this card's library reaches 1.33 to 1.41 for a product of two bf16 matrices,
// and would need both factors and both terms in memory first).  What bounds it is the card's power.
// A [c][x] tile: rows of X elements, 64 bytes more apart than that, so that the four rows of a transposed read meet every bank once.
template <uint32_t X> constexpr uint32_t kRowX = X + 32;
// A [i][c] tile of C elements a row, 32 or 64, in pieces of eight which lie at the places that their number and the row's give by
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

constexpr float kMostBF16 = 0x1.FEp127f;  // the largest finite one

struct GradShape {
  uint32_t ni, nj, nc;      // sizes of the sum
  uint32_t tiles_i, tiles_j;
  uint32_t splits, each;    // parts of c, and their length (a multiple of the step)
  float* partial;           // [splits][ni][nj] where there are several
};

// Rows along i and j have eight elements at least, and a tile's offsets fit 32 bits.  What a vector has beyond its row's end is whatever
// comes next in the matrix: it meets zeros, or results that are not stored.  Beyond the matrix' end nothing is read: the vector is then
// one that ends there, moved into place.  EIGHTS: sizes along the rows are multiples of eight, so that there are no such vectors.
// WC: parts of c that a workgroup takes side by side, WI x WJ waves and buffers for each, and adds up at the end: for results of few tiles,
// of which each then has more waves.
template <bool WEIGHT, bool EIGHTS, uint32_t TY, uint32_t TO, int T, int TI, int TJ, int WI, int WJ, int WC, int STEP>
__global__ __launch_bounds__(WC * WI * WJ * 64) void grad_kernel(const MatmulArgs a, const GradShape g) {
  constexpr uint32_t kThreads = WI * WJ * 64, FI = TI / WI / 32, FJ = TJ / WJ / 32;
  constexpr uint32_t kSizeA = WEIGHT ? STEP * kRowX<TI> : TI * STEP, kSizeB = STEP * kRowX<TJ>;
  constexpr uint32_t VA = TI * STEP / 8 / kThreads, VB = TJ * STEP / 8 / kThreads;  // vectors of eight of a thread
  __shared__ __align__(16) struct { __bf16 a0[T][kSizeA], b0[kSizeB], a1[T][kSizeA], b1[kSizeB]; } parts[WC];
  __shared__ uint32_t any_nan;  // a sum of the workgroup's is
  using D = typename Elem<TY>::type;
  const uint32_t lane = threadIdx.x & 63, part = WC == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  const uint32_t thread = threadIdx.x - part * kThreads, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  auto& tiles = parts[part];
  if (group_number() >= g.tiles_i * g.tiles_j) return;
  const TileAt at = tile_at(group_number(), g.tiles_i, g.tiles_j);
  const uint32_t i0 = at.row * TI, j0 = at.col * TJ;
  // (a part may be empty: its steps then lie beyond the sum's end, load the last one and put zeros)
  const uint32_t first = (blockIdx.y * WC + part) * g.each, end = min(g.nc, first + g.each);
  const uint32_t last = first < end ? first + (end - 1 - first) / STEP * STEP : (end - 1) / STEP * STEP;
  const uint32_t length = WC == 1 ? end - first : g.each;
  const D* const dy = static_cast<const D*>(a.a.p);
  const int8_t* const q = static_cast<const int8_t*>(a.b.p);
  const float* const scales = a.b.s;
  // where a thread's vectors lie: of a [c][x] tile kThreads / (X / 8) rows apart, of the [i][c] one kThreads / (STEP / 8)
  constexpr uint32_t kApartB = kThreads / (TJ / 8), kApartA = WEIGHT ? kThreads / (TI / 8) : kThreads / (STEP / 8);
  const uint32_t br = thread / (TJ / 8), bc = thread % (TJ / 8) * 8;
  const uint32_t ar = thread / (WEIGHT ? TI / 8 : STEP / 8), ac = thread % (WEIGHT ? TI / 8 : STEP / 8) * 8;
  // Offsets of the vectors and scales from the start of a step, [1]: of the last one, where rows (or, along c, vectors) that are not
  // there repeat others.  far: by how many elements a vector of the last step ends too early, four bits for each piece.
  int32_t oa[2][VA], ob[2][VB], os[2][WEIGHT ? VA : 1];
  uint32_t far = 0;
#pragma unroll
  for (uint32_t l = 0; l < 2; ++l) {
    const uint32_t rows = l ? end - 1 - last : STEP - 1;
    const auto in_matrix = [&](int32_t& o, uint64_t rest, uint32_t p) {  // rest: elements of the matrix from the step's start on
      const int32_t most = static_cast<int32_t>(min(rest, static_cast<uint64_t>(0x7FFFFFFF))) - 8;
      if (EIGHTS || !l || o <= most) return;
      far |= static_cast<uint32_t>(o - most) << (4 * p);
      o = most;
    };
#pragma unroll
    for (uint32_t h = 0; h < VB; ++h) {
      ob[l][h] = static_cast<int32_t>(min(br + kApartB * h, rows) * static_cast<uint32_t>(a.b.stride) + (j0 + bc < g.nj ? j0 + bc : 0));
      in_matrix(ob[l][h], (g.nc - 1 - last) * a.b.stride + g.nj, VA + h);
    }
#pragma unroll
    for (uint32_t h = 0; h < VA; ++h) {
      const uint32_t r = ar + kApartA * h;
      if (WEIGHT) {
        os[l][h] = static_cast<int32_t>(min(r, rows));
        oa[l][h] = static_cast<int32_t>(min(r, rows) * static_cast<uint32_t>(a.a.stride) + (i0 + ac < g.ni ? i0 + ac : 0));
        in_matrix(oa[l][h], (g.nc - 1 - last) * a.a.stride + g.ni, h);
      } else {
        oa[l][h] = static_cast<int32_t>(min(r, g.ni - 1 - i0) * static_cast<uint32_t>(a.a.stride) + (ac <= rows ? ac : 0));
        in_matrix(oa[l][h], (g.ni - 1 - i0) * a.a.stride + (g.nc - last), h);
      }
    }
    if (!WEIGHT) {
      os[l][0] = static_cast<int32_t>(ac <= rows ? ac : 0);
      in_matrix(os[l][0], g.nc - last, 7);
    }
  }

  Packed<D> va[VA];
  Packed<int8_t> vb[VB];
  float vs[8];  // scales: of each vector of dy's, or (along c) of its elements
  // The loads of piece p, a vector of dy or of the codes, of step c (beyond the last step: of that).
  const auto load = [&](uint32_t c, uint32_t p) __attribute__((always_inline)) {
    c = min(c, last);
    const bool l = c == last;
    if (p < VA) {
      const uint32_t h = p;
      va[h] = load_packed(dy + (WEIGHT ? c : i0) * a.a.stride + (WEIGHT ? 0 : c) + (l ? oa[1][h] : oa[0][h]));
      if (WEIGHT) {
        vs[h] = as_global(scales + c)[l ? os[1][h] : os[0][h]];
      } else if (h == VA - 1) {
        const Packed<float> t = load_packed(scales + c + (l ? os[1][0] : os[0][0]));
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) vs[e] = t.at(e);
      }
    } else {
      const uint32_t h = p - VA;
      vb[h] = load_packed(q + c * a.b.stride + (l ? ob[1][h] : ob[0][h]));
    }
  };
  // Piece p, which was loaded for step c, into LDS.  What lies beyond the sum's end is zero, whatever was read in its place.
  // LARGE: the first terms end at bf16's largest number, so that what is left of more, an infinity and NaN are in the last one.
  const auto put = [&](auto large, uint32_t c, uint32_t p, __bf16 (*ta)[kSizeA], __bf16* tb) __attribute__((always_inline)) {
    constexpr bool LARGE = large();
    if (!EIGHTS && c == last && far) {
      if (p < VA) va[p].move(far >> (4 * p) & 15u);
      else vb[p - VA].move(far >> (4 * p) & 15u);
      if (!WEIGHT && p == 0) {
        for (uint32_t k = far >> 28; k; --k) {
#pragma unroll
          for (uint32_t e = 0; e < 7; ++e) vs[e] = vs[e + 1];
        }
      }
    }
    if (p < VA) {
      const uint32_t h = p;
      const bool row_there = c + ar + kApartA * h < end;
      if (WEIGHT) va[h].keep(row_there);
      else if (EIGHTS) va[h].keep(c + ac < end);
      const float row_scale = row_there ? vs[h] : 0.0f;
      v8b t[T];
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        float x = va[h].at(e), s = WEIGHT ? row_scale : vs[e];  // (the scales repeat, too, and need not be finite)
        if (!WEIGHT) {
          const bool there = c + ac + (EIGHTS ? 0 : e) < end;
          x = EIGHTS || there ? x : 0.0f;
          s = there ? s : 0.0f;
        }
        x *= s;
#pragma unroll
        for (int k = 0; k < T; ++k) {
          t[k][e] = static_cast<__bf16>(LARGE && k + 1 < T ? __builtin_amdgcn_fmed3f(x, -kMostBF16, kMostBF16) : x);
          x -= static_cast<float>(t[k][e]);
        }
      }
      const uint32_t row = ar + kApartA * h, to = WEIGHT ? row * kRowX<TI> + ac : place_c<STEP>(row, ac / 8);
#pragma unroll
      for (int k = 0; k < T; ++k) __builtin_memcpy(&ta[k][to], &t[k], 16);
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
  const auto read = [&](uint32_t u, const __bf16 (*ta)[kSizeA], const __bf16* tb) __attribute__((always_inline)) {
    const uint32_t s = u / (T * FI), k = u / FI % T, i = u % FI;
    if (WEIGHT) fa[u & 1] = transposed<TI>(ta[k], s * 16, wi + i * 32, lane);
    else __builtin_memcpy(&fa[u & 1], &ta[k][place_c<STEP>(wi + i * 32 + (lane & 31), s * 2 + (lane >> 5))], 16);
    if (u % (T * FI)) return;
#pragma unroll
    for (uint32_t j = 0; j < FJ; ++j) fb[s & 1][j] = transposed<TJ>(tb, s * 16, wj + j * 32, lane);
  };
  const auto work = [&](auto large, uint32_t c, const __bf16 (*ta)[kSizeA], const __bf16* tb, __bf16 (*na)[kSizeA], __bf16* nb) __attribute__((always_inline)) {
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
          put(large, c + STEP, p, na, nb);
          load(c + 2 * STEP, p);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto take = [&](auto large, uint32_t from) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) load(from, p);
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) put(large, from, p, tiles.a0, tiles.b0);
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) load(from + STEP, p);
    __syncthreads();
    read(0, tiles.a0, tiles.b0);
    read(1, tiles.a0, tiles.b0);
    // Two steps at a time, of which the second may lie beyond the sum's end and be one of zeros: with one way out of the loop the sums
    // stay in their registers.  (What the last step reads ahead is not used.)
    for (uint32_t c = from; c < from + length; c += 2 * STEP) {
      work(large, c, tiles.a0, tiles.b0, tiles.a1, tiles.b1);
      work(large, c + STEP, tiles.a1, tiles.b1, tiles.a0, tiles.b0);
    }
  };
  if (threadIdx.x == 0) any_nan = 0;
  take(std::false_type{}, first);
  // A factor beyond bf16's largest number, as its first term an infinity, has made its whole row NaN: then the tile again, with LARGE terms,
  // as long as before, or six times where that does not fit the registers (fp32 dy of odd sizes to fp32).  (In every step these would be
  // 2 to 7 % of the time of dx 8192 x 4096 x 11008; so it is 0.2 %, and 1 to 3 % of the time of small results.)
  bool nan = false;
#pragma unroll
  for (uint32_t e = 0; e < FI * FJ * 16; ++e) nan |= __builtin_isnan(acc[e / 16 / FJ][e / 16 % FJ][e % 16]);
  if (__builtin_amdgcn_ballot_w64(nan)) any_nan = 1;
  __syncthreads();
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(any_nan), 0)) {
#pragma unroll
    for (uint32_t e = 0; e < FI * FJ; ++e) acc[e / FJ][e % FJ] = v16f{};
    uint32_t again = first;
    asm volatile("" : "+s"(again));  // (or the registers of what both begin with would be held all along)
    take(std::true_type{}, again);
    __syncthreads();
  }
  const auto value = [&](uint32_t i, uint32_t j, uint32_t p, uint32_t e) { return acc[i][j][p * 4 + e]; };
  if constexpr (WC > 1) {  // the parts' sums, in one order, to the first
    constexpr uint32_t kEach = FI * FJ * 16;
    static_assert(sizeof(parts) >= (WC - 1) * kThreads * kEach * 4, "sums of the parts");
    float* const sums = reinterpret_cast<float*>(&parts);
    if (part)
#pragma unroll
      for (uint32_t e = 0; e < kEach; ++e) sums[((part - 1) * kEach + e) * kThreads + thread] = acc[e / 16 / FJ][e / 16 % FJ][e % 16];
    __syncthreads();
    if (!part)
#pragma unroll
      for (uint32_t p = 0; p < WC - 1; ++p)
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) acc[e / 16 / FJ][e / 16 % FJ][e % 16] += sums[(p * kEach + e) * kThreads + thread];
    __syncthreads();
    if (part) return;
  }
  constexpr uint32_t kBox = 32 * FJ * 32 * (TI == 256 && TO != kF32 ? 2 : 4);
  static_assert(sizeof(parts) >= WI * WJ * kBox, "a box for each wave");
  char* const box = reinterpret_cast<char*>(&parts) + wave * kBox;
  if (TI == 128 && g.splits > 1) {  // (sums that several workgroups take in parts are of these tiles)
    const Mat partial{g.partial + static_cast<uint64_t>(blockIdx.y) * g.ni * g.nj, nullptr, g.nj, 0, 0};
    store_tile<kF32, FI, FJ>(partial, i0 + wi, j0 + wj, g.ni, g.nj, box, lane, value);
  } else {
    store_tile<TO, FI, FJ>(a.out, i0 + wi, j0 + wj, g.ni, g.nj, box, lane, value);
  }
}

// Results or sums of fewer than eight along a side, or rows too far apart for the offsets of a tile: 32 columns of a row to a workgroup,
// with eight threads for each that share c.  2 outputs by 4096 inputs over 16384 tokens: dw in fp32 635 us, dx in bf16 567 (the bytes would take
// 11 and 23).
template <bool WEIGHT, uint32_t TY, uint32_t TO>
__global__ __launch_bounds__(256) void grad_each_kernel(const MatmulArgs a, const GradShape g) {
  __shared__ float part[8][32];
  const uint32_t j = group_number() * 32 + (threadIdx.x & 31), turn = threadIdx.x >> 5;
  const STQ_GLOBAL typename Elem<TY>::type* dy = as_global(static_cast<const typename Elem<TY>::type*>(a.a.p));
  const STQ_GLOBAL int8_t* q = as_global(static_cast<const int8_t*>(a.b.p));
  for (uint32_t i = blockIdx.y; i < g.ni; i += gridDim.y) {
    float sum = 0.0f;
    if (j < g.nj)
      for (uint32_t c = turn; c < g.nc; c += 8)
        sum = fmaf(static_cast<float>(dy[(WEIGHT ? c : i) * a.a.stride + (WEIGHT ? i : c)]) * as_global(a.b.s)[c], static_cast<float>(q[c * a.b.stride + j]), sum);
    part[turn][threadIdx.x & 31] = sum;
    __syncthreads();
    if (turn == 0 && j < g.nj) {
#pragma unroll
      for (int k = 1; k < 8; ++k) sum += part[k][threadIdx.x];
      using T = typename Elem<TO>::type;
      as_global(static_cast<T*>(a.out.p))[i * a.out.stride + j] = static_cast<T>(sum);
    }
    __syncthreads();
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
      const float* p = partial + k * size + static_cast<uint64_t>(row) * nj + col;
      if (col + 4 <= nj) {
        const v4i w = load_fragment(reinterpret_cast<const int8_t*>(p));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u2f(static_cast<uint32_t>(w[e]));
      } else {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
          if (col + e < nj) v[e] += as_global(p)[e];
      }
    }
    store4<TO>(out, row, col, nj, v);
  }
}

uint32_t tiles_of(uint32_t size, uint32_t tile) { return (size - 1) / tile + 1; }

constexpr uint32_t kCus = 256;  // for sizes that must not depend on the device
bool near(const Mat& x) { return x.stride < (1u << 22); }  // a tile's rows within reach of a 31-bit offset
// Whether a matrix' rows can be loaded straight into LDS.
bool in_pieces(const Mat& x) { return (reinterpret_cast<uintptr_t>(x.p) & 15) == 0 && x.stride % 16 == 0; }

template <uint32_t TO>
void run_matmul(const MatmulArgs& a, uint32_t n_cu, hipStream_t st) {
  const auto size = [&](uint32_t rows, const Mat& x) { return (rows - 1) * x.stride + a.k; };
  // Up to 32 tokens, or 64 where a tile kernel would leave half of the CUs without work (64 tokens through 4096 x 4096: 11.6 us, by
  // tiles 16.6; through 11008 x 4096 29.5 and 17.7).
  const bool tiles = near(a.a) && near(a.b), wide = tiles_of(a.n, 16) > 2 * n_cu;
  const bool few = a.m <= 32 || (a.m <= 64 && (!tiles || tiles_of(a.n, 64) * 2 < n_cu));
  if (size(a.m, a.a) < 16 || size(a.n, a.b) < 16 || (!few && !tiles)) {
    const uint64_t groups = (static_cast<uint64_t>(a.m) * a.n + 255) / 256;
    matmul_each_kernel<TO><<<static_cast<uint32_t>(groups < 65536 ? groups : 65536), 256, 0, st>>>(a);
  } else if (few) {
    // Many rows of w: fewer runs ahead, so that all workgroups fit the card (one token through 11008 x 4096 11.7 us, with four 12.6), or,
    // with more tokens, two fragments of rows for each of tokens (32 tokens 17.7 us, with one 19.1; 4096 x 4096 10.0 and 8.4).
    if (a.m <= 16 && wide) matmul_few_kernel<TO, 1, 1, 2><<<in_layers(tiles_of(a.n, 16)), 512, 0, st>>>(a);
    else if (a.m <= 16) matmul_few_kernel<TO, 1, 1, 4><<<in_layers(tiles_of(a.n, 16)), 512, 0, st>>>(a);
    else if (a.m <= 32 && wide) matmul_few_kernel<TO, 2, 2, 2><<<in_layers(tiles_of(a.n, 32)), 512, 0, st>>>(a);
    else if (a.m <= 32) matmul_few_kernel<TO, 2, 1, 2><<<in_layers(tiles_of(a.n, 16)), 512, 0, st>>>(a);
    else matmul_few_kernel<TO, 4, 1, 2><<<in_layers(tiles_of(a.n, 16)), 512, 0, st>>>(a);
  } else {
    const auto count = [&](uint32_t t) { return static_cast<uint64_t>(tiles_of(a.m, t)) * tiles_of(a.n, t); };
    const bool pieces = in_pieces(a.a) && in_pieces(a.b);
    // 256 x 256 from three quarters of a tile for each CU on (3008 x 4096 x 4096: 61.5 us, by 128 x 128 72; 2048 tokens 54.5 and 42.3), 128 x 128
    // from one on (1024 x 4096 x 4096: 27.3 us, by 64 x 64 30.5; 2048 outputs 23.8 and 19.0); rows that are not in pieces by way of registers
    // (8192 x 4096 x 4096: 137 us in pieces, 177 not).
    const uint32_t t = pieces && count(256) * 4 >= 3 * n_cu ? 256 : (count(128) >= n_cu ? 128 : 64), rows = tiles_of(a.m, t), cols = tiles_of(a.n, t);
    const dim3 grid = in_layers(count(t));
    if (t == 256) matmul_tile_kernel<TO, 256, 256, 2, 4, true><<<grid, 512, 0, st>>>(a, rows, cols);
    else if (t == 128 && pieces) matmul_tile_kernel<TO, 128, 128, 2, 2, true><<<grid, 256, 0, st>>>(a, rows, cols);
    else if (t == 128) matmul_tile_kernel<TO, 128, 128, 2, 2, false><<<grid, 256, 0, st>>>(a, rows, cols);
    else if (pieces) matmul_tile_kernel<TO, 64, 64, 2, 2, true><<<grid, 256, 0, st>>>(a, rows, cols);
    else matmul_tile_kernel<TO, 64, 64, 2, 2, false><<<grid, 256, 0, st>>>(a, rows, cols);
  }
}

// Parts of the tokens for a weight gradient of few tiles, of 512 tokens at least.  What a number of parts takes, in units of the time of
// a token of a tile: the tiles that a CU takes one after the other, and for several parts a write and a read of the result in fp32 and
// another launch (measured: 169 tiles of 16384 tokens 319 us, in three parts 249; 36 of 5001 tokens in one 43 us, in seven 29, in nine 35;
// 256 of 4096 90 us, in two 95).
constexpr uint32_t kLeastPart = 512;
uint32_t splits_of(uint64_t m, uint64_t n, uint64_t k) {
  const auto count = [&](uint64_t t) { return ((n + t - 1) / t) * ((k + t - 1) / t); };
  if (n < 8 || k < 8 || count(256) * 2 >= kCus) return 1;
  const uint64_t tiles = count(128);
  uint32_t best = 1;
  double least = 0;
  for (uint32_t s = 1; s == 1 || (s <= 64 && s * kLeastPart <= m); ++s) {
    const double turns = static_cast<double>((tiles * s + kCus - 1) / kCus);
    const double t = turns * static_cast<double>(m) / s + (s > 1 ? 200.0 + 1.1e-4 * static_cast<double>(s * n * k) : 0.0);
    if (s == 1 || t < least) { least = t; best = s; }
  }
  return best;
}

template <uint32_t TO>
void join(const MatmulArgs& a, const GradShape& g, hipStream_t st) {
  const uint64_t groups = (static_cast<uint64_t>(g.ni) * ((g.nj + 3) / 4) + 255) / 256;
  join_kernel<TO><<<static_cast<uint32_t>(groups < 4096 ? groups : 4096), 256, 0, st>>>(a.out, g.partial, g.splits, g.ni, g.nj);
}

template <bool WEIGHT, bool EIGHTS, uint32_t TY, uint32_t TO>
void run_tiles(const MatmulArgs& a, GradShape g, hipStream_t st) {
  const auto count = [&](uint32_t i, uint32_t j) { return static_cast<uint64_t>(tiles_of(g.ni, i)) * tiles_of(g.nj, j); };
  const auto grid = [&](uint32_t i, uint32_t j, uint32_t parts) {
    g.tiles_i = tiles_of(g.ni, i);
    g.tiles_j = tiles_of(g.nj, j);
    g.each = tiles_of(g.nc, g.splits * parts * 64) * 64;
    if (parts == 1) g.splits = tiles_of(g.nc, g.each);
    return in_layers(count(i, j), g.splits);
  };
  // 256 x 256 where more than half of the CUs have a tile (dx 2304 x 4096 x 4096: 180 us, by 128 x 128 221; 8192 tokens 451 and 607; at
  // half, 2048 tokens, 191 and 184), of short sums where all have (dw 2048 x 4096 over 400 tokens: 32 us and 24).  Below, 128 x 128, and
  // where that leaves half of the CUs without one, smaller tiles whose workgroups take parts of c side by side (dx 300 x 1600 x 1600: 16.8
  // us, by 128 x 128 31.8; 2048 tokens 49.8 and 36.5).
  constexpr int kTerms = TO == kF32 ? 3 : 2;
  if (g.splits == 1 && count(256, 256) > (g.nc < 512 ? kCus - 1 : kCus / 2)) {
    const dim3 d = grid(256, 256, 1);
    grad_kernel<WEIGHT, EIGHTS, TY, TO, kTerms, 256, 256, 2, 4, 1, 32><<<d, 512, 0, st>>>(a, g);
  } else if (g.splits > 1 || count(128, 128) * 2 > kCus) {
    const dim3 d = grid(128, 128, 1);
    grad_kernel<WEIGHT, EIGHTS, TY, TO, kTerms, 128, 128, 2, 4, 1, 32><<<d, 512, 0, st>>>(a, g);
    if (g.splits > 1) join<TO>(a, g, st);
  } else if (g.ni <= 32) {
    const dim3 d = grid(32, 64, 4);
    grad_kernel<WEIGHT, EIGHTS, TY, TO, kTerms, 32, 64, 1, 2, 4, 32><<<d, 512, 0, st>>>(a, g);
  } else {
    const dim3 d = grid(64, 64, 2);
    grad_kernel<WEIGHT, EIGHTS, TY, TO, kTerms, 64, 64, 2, 2, 2, 32><<<d, 512, 0, st>>>(a, g);
  }
}
template <bool WEIGHT, uint32_t TY, uint32_t TO>
void run_grad(const MatmulArgs& a, GradShape g, hipStream_t st) {
  if (g.nc == 0) {  // no tokens: a sum of nothing
    g.splits = 0;
    join<TO>(a, g, st);
  } else if (g.ni < 8 || g.nj < 8 || g.nc < 8 || !near(a.a) || !near(a.b)) {
    grad_each_kernel<WEIGHT, TY, TO><<<in_layers(tiles_of(g.nj, 32), g.ni < 65535 ? g.ni : 65535), 256, 0, st>>>(a, g);
  } else if (g.nj % 8 == 0 && (WEIGHT ? g.ni : g.nc) % 8 == 0) {
    run_tiles<WEIGHT, true, TY, TO>(a, g, st);
  } else {
    run_tiles<WEIGHT, false, TY, TO>(a, g, st);
  }
}
template <bool WEIGHT>
int run_grads(const MatmulArgs& a, const GradShape& g, uint32_t dy_type, uint32_t out_type, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dy_type == kF32) {
    if (out_type == kF32) run_grad<WEIGHT, kF32, kF32>(a, g, st);
    else run_grad<WEIGHT, kF32, kBF16>(a, g, st);
  } else {
    if (out_type == kF32) run_grad<WEIGHT, kBF16, kF32>(a, g, st);
    else run_grad<WEIGHT, kBF16, kBF16>(a, g, st);
  }
  return hipGetLastError();
}

}  // namespace

int launch_matmul(const MatmulArgs& a, uint32_t out_type, uint32_t n_cu, void* stream) {
  if (out_type == kF32) run_matmul<kF32>(a, n_cu, static_cast<hipStream_t>(stream));
  else run_matmul<kBF16>(a, n_cu, static_cast<hipStream_t>(stream));
  return hipGetLastError();
}
int launch_matmul_grad_input(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, void* stream) {
  return run_grads<false>(a, GradShape{a.m, a.k, a.n, 0, 0, 1, 0, nullptr}, dy_type, out_type, stream);
}
int launch_matmul_grad_weight(const MatmulArgs& a, uint32_t dy_type, uint32_t out_type, float* workspace, void* stream) {
  return run_grads<true>(a, GradShape{a.n, a.k, a.m, 0, 0, splits_of(a.m, a.n, a.k), 0, workspace}, dy_type, out_type, stream);
}
uint64_t grad_weight_bytes(uint64_t m, uint64_t n, uint64_t k) {
  const uint64_t s = splits_of(m, n, k);
  return s > 1 ? 4 * s * n * k : 0;
}

}  // namespace stq
