// Device code that the matrix products share: fragments of codes, results by way of LDS, the order of the tiles, and a tile of a
// product of codes by codes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "stq_vectors.h"

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
    using T = typename Elem<TO>::type;
    const T h[4] = {static_cast<T>(v[0]), static_cast<T>(v[1]), static_cast<T>(v[2]), static_cast<T>(v[3])};
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

// ending(acc, t): what becomes of the sums; a wave's are those of rows t.m0 + t.wm .. and columns t.n0 + t.wn .., in store_tile's order.
struct CodeTile {
  uint32_t m0, n0, wm, wn;  // of the workgroup, of the wave in it
  uint32_t lane, wave;
  const float* sm;          // in LDS: the scales of the workgroup's rows and columns
  const float* sn;
  char* box;                // of the wave, for store_tile
  char* room;               // of the workgroup: all boxes of the first half of its waves
  char* spare;              // of the workgroup: 64 bytes a row and more beside the boxes
};
template <int TM, int TN, int WM, int WN, bool PIECES, class END>
__device__ __forceinline__ void code_tile(const MatmulArgs& a, uint32_t tiles_m, uint32_t tiles_n, END ending) {
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
  ending(acc, CodeTile{m0, n0, wm, wn, lane, wave, sm, sn, box, reinterpret_cast<char*>(a0), reinterpret_cast<char*>(sm + TM)});
#endif
}

// Few tokens: what counts is how fast w's codes arrive.  A workgroup has 16 R of w's rows and up to 16 G tokens; its eight waves share
// the inner dimension, a run of 128 codes each in turn, read straight into the fragments, and add up at the end.  The loads of A runs
// are under way together.  One token through 11008 x 4096: 11.0 us, of which the codes would take 8.4 at the rate of a large copy; a
// launch and its end are most of the rest (32000 x 4096: 4.8 TB/s).  (Workgroups beyond w's rows, in launches of several layers, repeat its
// last one and store nothing: a way out for them took 0.2 us of every call.)
// ending(sum, m, n): codes' products of token m and the four classes or outputs from n on, of the waves that have them (m or n may lie beyond
// the matrices).
template <int G, int R, int A, class END>
__device__ __forceinline__ void code_few(const MatmulArgs& a, END ending) {
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
  ending(sum, m, n);
}

// ---------------------------------------------------------------------------------------------- on the host
inline uint32_t tiles_of(uint32_t size, uint32_t tile) { return (size - 1) / tile + 1; }

inline bool near(const Mat& x) { return x.stride < (1u << 22); }  // a tile's rows within reach of a 31-bit offset
// Whether a matrix' rows can be loaded straight into LDS.
inline bool in_pieces(const Mat& x) { return (reinterpret_cast<uintptr_t>(x.p) & 15) == 0 && x.stride % 16 == 0; }

}  // namespace
}  // namespace stq
