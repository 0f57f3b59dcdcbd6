// The matrix product of gts_linear and gts_linear_backward on gfx950's matrix cores,
// and its plan.  Instantiated by gts_linear_f32.hip, gts_linear_bf16.hip and
// gts_linear_f16.hip; planned and launched by gts_linear.hip.
//
// C[m][n] = sum over k of A(m, k) B(n, k).  An operand lies with its k axis contiguous
// (x and W in the forward pass) or with its other axis contiguous (W for dx, dz and x
// for dW); both orders are read as they lie, nothing is transposed in memory.
//
// A workgroup computes a tile of C.  Slices of A and B, 128 bytes of each row deep, pass
// through two LDS buffers in turn: while the waves multiply one, the next one is on its
// way from memory.  Each wave holds FM x FN accumulators of 16 x 16.
#pragma once

#include <algorithm>

#include "gts_nn_common.h"

namespace gts {
namespace nn {

struct ProductArgs {
  const void* a;
  int64_t lda;
  const void* b;
  int64_t ldb;
  int64_t m, n, k;
  int64_t k_chunk;       // of k, for each split; a multiple of the slices' depth
  int32_t splits;        // above 1, sums go to part[split][m][n]
  int32_t tiles_m, tiles_n;
  int32_t act;
  int32_t past_l2;       // C is written past the L2s
  float* part;
  const void* bias;
  const void* residual;
  int64_t ld_r;
  void* c;
  int64_t ld_c;
  void* pre;
  int64_t ld_pre;
};

enum Layout : int { kForward = 0, kGradX = 1, kGradW = 2 };
enum Shape : int { kLarge = 0, kLower = 1, kMiddle = 2, kSmall = 3, kNarrow = 4, kMany = 5, kFewRows = 6 };

struct ProductPlan {
  int shape;
  bool direct;           // operands copied to LDS by the memory system, 16 bytes a lane
  bool align;            // what does not lie so is copied to where it does first
  int splits;
  int64_t k_chunk;
  int64_t part_bytes;    // the splits' sums
};

// One operand's copy with rows that start at multiples of 16 bytes and end in zeros; dst
// is null for none.
struct AlignArgs {
  const void* src;
  int64_t ld, rows, width;
  void* dst;
  int64_t ld_dst;
};

// Column sums of part[parts][n] into out[n], where it is not null.
struct ColumnSums {
  const float* part;
  int64_t parts, n;
  void* out;
};

hipError_t launch_product_f32(const ProductArgs& p, Layout layout, const ProductPlan& plan,
                              const AlignArgs (&align)[2], hipStream_t s);
hipError_t launch_product_bf16(const ProductArgs& p, Layout layout, const ProductPlan& plan,
                              const AlignArgs (&align)[2], hipStream_t s);
hipError_t launch_product_f16(const ProductArgs& p, Layout layout, const ProductPlan& plan,
                              const AlignArgs (&align)[2], hipStream_t s);
hipError_t launch_pair_f32(const ProductArgs& x, const ProductArgs& w, int shape, const AlignArgs& align_w,
                           const AlignArgs& align_x, const ColumnSums& sums, hipStream_t s);
hipError_t launch_pair_bf16(const ProductArgs& x, const ProductArgs& w, int shape, const AlignArgs& align_w,
                           const AlignArgs& align_x, const ColumnSums& sums, hipStream_t s);
hipError_t launch_pair_f16(const ProductArgs& x, const ProductArgs& w, int shape, const AlignArgs& align_w,
                           const AlignArgs& align_x, const ColumnSums& sums, hipStream_t s);

constexpr int kSliceBytes = 128;   // depth of a slice, in bytes of k
template <class T>
constexpr int kDepth = kSliceBytes / (int)sizeof(T);

// Tile extents by shape, waves along each, groups of such waves that take every KW-th
// slice, slices of a group held in LDS, waves a SIMD.  Two groups hide each other's waits
// where a compute unit has one tile (2000 x 2048 x 2048 in bf16: 23.1 against 26.7 us);
// where there are more, two smaller workgroups side by side do it better, their starts and
// ends too (8000 x 4096 x 1024: 64 against 77).
template <int S>
struct TileShape;
template <>
struct TileShape<kMiddle> { static constexpr int BM = 128, BN = 128, WM = 2, WN = 2, KW = 2, STAGES = 2, OCC = 2; };
template <>
struct TileShape<kMany> { static constexpr int BM = 128, BN = 128, WM = 2, WN = 2, KW = 1, STAGES = 2, OCC = 2; };
template <>
struct TileShape<kSmall> { static constexpr int BM = 64, BN = 64, WM = 2, WN = 2, KW = 2, STAGES = 2, OCC = 4; };
template <>
struct TileShape<kNarrow> { static constexpr int BM = 64, BN = 32, WM = 2, WN = 2, KW = 2, STAGES = 2, OCC = 4; };

#ifdef __HIP_DEVICE_COMPILE__
#define GTS_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#endif

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of an operand: 8 or 4 elements.
template <class T>
struct Fragment;
template <>
struct Fragment<bf16> { typedef __bf16 type __attribute__((ext_vector_type(8))); };
template <>
struct Fragment<f16> { typedef _Float16 type __attribute__((ext_vector_type(8))); };
template <>
struct Fragment<float> { typedef float type __attribute__((ext_vector_type(4))); };

// acc += X Y^T over the fragments' k, X along acc's registers, Y along its lanes.  A
// lane's 16 bytes are k = (lane / 16) * E ... + E - 1 of row lane % 16; in 32 bits, four
// products take one element of each lane, that is k = j, 4 + j, 8 + j, 12 + j.
__device__ __forceinline__ void multiply(f32x4& acc, Fragment<bf16>::type x, Fragment<bf16>::type y) {
#ifdef __HIP_DEVICE_COMPILE__
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc, 0, 0, 0);
#endif
}
__device__ __forceinline__ void multiply(f32x4& acc, Fragment<f16>::type x, Fragment<f16>::type y) {
#ifdef __HIP_DEVICE_COMPILE__
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, acc, 0, 0, 0);
#endif
}
__device__ __forceinline__ void multiply(f32x4& acc, f32x4 x, f32x4 y) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], acc, 0, 0, 0);
#endif
}

// A value that all lanes agree on, in a scalar register.
__device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// 16 bytes a lane, from byte offset `at` of `buffer` to LDS at lds + 16 lane, without passing
// registers; zeros from past the buffer's end.
template <bool WRITTEN>
__device__ __forceinline__ void copy_to_lds(const char* lds, u32x4 buffer, unsigned at) {
#ifdef __HIP_DEVICE_COMPILE__
  const auto to = GTS_LDS(const_cast<char*>(lds));
  if constexpr (WRITTEN) {
    // the buffer's registers may have been written by a vector instruction just before, which
    // a load has to stand 5 wait states behind; the compiler does not count them in here
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(scalar((uint32_t)reinterpret_cast<uintptr_t>(to))), "v"(at), "s"(buffer)
                 : "memory", "m0");
  } else {
    void* base = reinterpret_cast<void*>((uint64_t)buffer[1] << 32 | buffer[0]);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(base, 0, (int)buffer[2], (int)buffer[3]),
                                             to, 16, at, 0, 0, 0);
  }
#endif
}

// One operand's slices.  OUTER: the axis that is not k is the contiguous one.  R is the
// tile's extent along it, WAVES the waves that copy a slice, each wave's copies 1024
// consecutive bytes of LDS, 16 a lane.
//
// In LDS, a slice of a k-contiguous operand is R rows of 128 bytes, one of an OUTER
// operand kDepth rows of R elements.  The 16-byte pieces of a row are permuted by the row's
// number so that the lanes which read together reach all banks: k-contiguous, 8
// rows at one k hit 8 different pieces; OUTER in 16 bits, where a transposing read takes
// 32 bytes of 4 rows (and another four, 8 rows further), those fall on different
// 32-byte pieces; OUTER in 32 bits, 4 rows, 4 apart, on different 64-byte pieces.
template <class T, bool OUTER, int R, int WAVES>
struct Slices {
  static constexpr int E = kVec<T>, D = kDepth<T>;
  static constexpr int kBytes = R * kSliceBytes;
  static constexpr int kRowBytes = OUTER ? R * (int)sizeof(T) : kSliceBytes;
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kCopies = kBytes / 1024 / WAVES;
  static_assert(kCopies * WAVES * 1024 == kBytes, "whole copies a wave");
  static_assert(!OUTER || kPieces % ((sizeof(T) == 4 && R >= 64) || R % 128 == 0 ? 16 : 8) == 0, "place() stays in its row");
  static constexpr unsigned kNowhere = 0x80000000u;

  // A piece's place in row `row`, and the other way round.
  __device__ static __forceinline__ int place(int piece, int row) {
    if constexpr (!OUTER) return piece ^ (row & 7);
    else if constexpr (sizeof(T) == 4) return piece ^ (((row >> 2) & (R >= 64 ? 3 : 1)) << 2);
    else if constexpr (R % 128 == 0) return piece ^ (((row & 3) | ((row >> 1) & 4)) << 1);
    else return piece ^ ((((row >> 1) & 1) | ((row >> 2) & 2)) << 1);
  }

  const T* p;          // the tile's first row or column, k = 0
  int64_t ld;
  int wave, lane;
  int64_t left;        // rows or columns from the tile's first to the operand's end
  unsigned at[kCopies];   // byte offset of the lane's piece from the slice's start

  __device__ __forceinline__ void begin(const void* base, int64_t ld_, int64_t first, int64_t extent,
                                        int wave_) {
    ld = ld_;
    wave = wave_;
    left = extent - first;
    p = static_cast<const T*>(base) + (OUTER ? first : first * ld);
    lane = threadIdx.x % 64;
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const int row = row_of(j), piece = piece_of(j);
      const bool there = OUTER ? piece * E < left : row < left;
      at[j] = there ? (unsigned)(row * ld * (int64_t)sizeof(T)) + piece * 16 : kNowhere;
    }
  }
  __device__ __forceinline__ int row_of(int j) const { return ((wave * kCopies + j) * 64 + lane) / kPieces; }
  __device__ __forceinline__ int piece_of(int j) const {
    return place(((wave * kCopies + j) * 64 + lane) % kPieces, row_of(j));
  }

  // The address of slice k0.
  __device__ __forceinline__ const T* slice(int64_t k0) const { return p + (OUTER ? k0 * ld : k0); }

  // Copies slice k0 of k < end to lds without passing registers.  Pieces outside read
  // as zero: their offset is past the buffer's end.  (Of an OUTER operand a piece may
  // reach past the last column, by less than its 16 bytes, into columns of C that do not
  // exist.)
  //
  // Around the builtin, the compiler lets every transposing read of LDS wait for all copies;
  // WRITTEN as assembly they are waited for by wait_copies alone, at the cost of some
  // scheduling.  Tiles of 128 x 128 in bf16, written against not: dw of 10000 x 1024 x 4096
  // 122 against 160 us, dx 110 against 132; without transposing reads 103 against 97, and the
  // large tiles, whose reads and copies have their turns, 840 against 800 at 8192^3.
  template <bool WRITTEN>
  __device__ __forceinline__ void copy(char* lds, int64_t k0, int64_t end) const {
    // a buffer of 2^31 bytes from the slice's start on
    const uint64_t from = reinterpret_cast<uint64_t>(slice(k0));
    const u32x4 buffer = {scalar((uint32_t)from), scalar((uint32_t)(from >> 32) & 0xffffu), kNowhere, 0x00027000u};
    const int deep = (int)scalar((uint32_t)min(end - k0, (int64_t)D));
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const bool there = OUTER ? row_of(j) < deep : piece_of(j) * E < deep;
      copy_to_lds<WRITTEN>(lds + (wave * kCopies + j) * 1024, buffer, there ? at[j] : kNowhere);
    }
  }

  // The same through registers, for operands whose rows do not start at multiples of 16
  // bytes or whose k ends within a piece.
  typedef typename Fragment<T>::type Piece;
  __device__ __forceinline__ void fetch(Piece (&held)[kCopies], int64_t k0, int64_t end) const {
    const T* from = slice(k0);
    const int64_t deep = end - k0;
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const int row = row_of(j), piece = piece_of(j);
      const int64_t n = OUTER ? (row < deep ? left - piece * E : 0) : (row < left ? deep - piece * E : 0);
      const T* q = from + row * ld + piece * E;
      if (n >= E) {
        held[j] = *reinterpret_cast<const typename Unaligned<T, E>::type*>(q);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) held[j][i] = i < n ? q[i] : (T)0.0f;
      }
    }
  }
  __device__ __forceinline__ void put(char* lds, const Piece (&held)[kCopies]) const {
#pragma unroll
    for (int j = 0; j < kCopies; ++j)
      *reinterpret_cast<Piece*>(lds + (wave * kCopies + j) * 1024 + lane * 16) = held[j];
  }

  // The fragment of rows (columns) first ... first + 15 at k step `step` of the slice
  // (half a slice each).
  __device__ static __forceinline__ Piece read(const char* lds, int first, int step) {
    const int lane = threadIdx.x % 64, q = lane / 16, i = lane % 16;
    if constexpr (!OUTER) {
      const int row = first + i;
      return *reinterpret_cast<const Piece*>(lds + row * kSliceBytes + place(step * 4 + q, row) * 16);
    } else if constexpr (sizeof(T) == 4) {
      Piece x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = step * 16 + 4 * q + j, col = first + i;
        x[j] = *reinterpret_cast<const float*>(lds + row * kRowBytes + place(col / 4, row) * 16 + col % 4 * 4);
      }
      return x;
    } else {
      // lane i of 16 reads 8 bytes of row i / 4 and receives column i of the four rows
      s16x4 half[2] = {};
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = step * 32 + q * 8 + h * 4 + i / 4, col = first + i % 4 * 4;
        const char* at = lds + row * kRowBytes + place(col / 8, row) * 16 + col % 8 * 2;
        half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)GTS_LDS(const_cast<char*>(at)));
      }
#endif
      const s16x8 both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(Piece, both);
    }
  }
};

// Waits until at most LEFT of this wave's copies to LDS (and other loads) are on their way.
template <int LEFT>
__device__ __forceinline__ void wait_copies() {
  // the counters' fields: vmcnt in bits 0-3 and 14-15, the others at their ends
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4 | 15 << 8);
}

// Nothing is moved across: neither memory accesses nor, by the scheduler, anything else.
__device__ __forceinline__ void pin() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A barrier that, other than __syncthreads, leaves copies on their way.
__device__ __forceinline__ void barrier() {
  pin();
  __builtin_amdgcn_s_barrier();
  pin();
}

__device__ __forceinline__ unsigned tile_count(const ProductArgs& p) {
  return (unsigned)p.tiles_m * (unsigned)p.tiles_n * (unsigned)p.splits;
}

// The tile that workgroup `id` of `count` takes.  Workgroups go round the 8 XCDs, each
// with an L2 of its own, so every XCD gets a contiguous range of tiles; in it, 8 tiles of
// rows run through the columns together, so that the slices they share are in that L2.
__device__ __forceinline__ void tile_of(const ProductArgs& p, unsigned id, unsigned count, int& tm,
                                        int& tn, int& split) {
  const unsigned q = count / 8, r = count % 8, xcd = id % 8;
  unsigned t = xcd * q + min(xcd, r) + id / 8;
  const unsigned tiles = (unsigned)p.tiles_m * (unsigned)p.tiles_n;
  split = (int)(t / tiles);
  t %= tiles;
  const unsigned group = 8u * (unsigned)p.tiles_n, g = t / group;
  const unsigned rows = min(8u, (unsigned)p.tiles_m - g * 8u);
  t -= g * group;
  tm = (int)(g * 8u + t % rows);
  tn = (int)(t / rows);
}

// Orders a wave's LDS accesses before against those after: what one lane wrote, another
// reads.  (The hardware takes a wave's LDS accesses in order.)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The epilogue of R pieces of N consecutive columns of C, in rows m[], at column n: bias (read
// once by the caller), activation, residual.  Rows that are -1 do not exist.
template <class T, int R, int N>
__device__ __forceinline__ void finish(const ProductArgs& p, const int64_t (&m)[R], int64_t n,
                                       const float (&bias)[N], float (&z)[R][N]) {
  const int64_t left = p.n - n;
  float res[R][N];
  if (p.residual != nullptr)   // all on their way before the first is used
#pragma unroll
    for (int r = 0; r < R; ++r)
      load_vec<T, N>(res[r], static_cast<const T*>(p.residual) + m[r] * p.ld_r + n, m[r] >= 0 ? left : 0);
  if (p.bias != nullptr)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < N; ++i) z[r][i] += bias[i];
  if (p.pre != nullptr)
#pragma unroll
    for (int r = 0; r < R; ++r)
      store_vec<T, N>(static_cast<T*>(p.pre) + m[r] * p.ld_pre + n, z[r], m[r] >= 0 ? left : 0);
  with_act(p.act, [&](auto a) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < N; ++i) z[r][i] = act_value<decltype(a)::value>(z[r][i]);
  });
  if (p.residual != nullptr)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < N; ++i) z[r][i] += res[r][i];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    T* to = static_cast<T*>(p.c) + m[r] * p.ld_c + n;
    if (p.past_l2 && m[r] >= 0 && left >= N) {
      typename Unaligned<T, N>::type v;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (T)z[r][i];
      __builtin_nontemporal_store(v, reinterpret_cast<typename Unaligned<T, N>::type*>(to));
    } else {
      store_vec<T, N>(to, z[r], m[r] >= 0 ? left : 0);
    }
  }
}

template <class T, int N>
__device__ __forceinline__ void load_bias(const ProductArgs& p, int64_t n, float (&bias)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = 0.0f;
  if (p.bias != nullptr) load_vec<T, N>(bias, static_cast<const T*>(p.bias) + n, p.n - n);
}

// Of an accumulator, a lane holds columns 4 (lane / 16) ... + 3 of row lane % 16.  Through
// LDS a wave gets its sums as 16-byte pieces of C's rows, so that memory is written in whole
// lines.  Pieces of 4 sums are permuted by their row against bank conflicts.

// FN accumulators side by side, to rows `first` ... + 15 of a wave's sums.
template <int FN>
__device__ __forceinline__ void put_sums(float* own, int first, const f32x4 (&acc)[FN], int lane) {
  constexpr int COLS = FN * 16, PIECES = COLS / 4;
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int row = first + lane % 16, piece = (j * 4 + lane / 16) ^ (row & (PIECES - 1));
    *reinterpret_cast<f32x4*>(own + row * COLS + piece * 4) = acc[j];
  }
}

// Rows of a wave's sums, every `by`-th handful from the `from`-th on, to C at m0, n0: the
// sums of KW groups, `apart` floats apart, added.
template <class T, int FN, int KW>
__device__ __forceinline__ void write_rows(const ProductArgs& p, const float* own, int apart, int rows, int from,
                                           int by, int64_t m0, int64_t n0, int split, int lane) {
  constexpr int E = kVec<T>, COLS = FN * 16, PIECES = COLS / 4;
  constexpr int LPR = COLS / E, RPP = 64 / LPR;   // lanes a row, rows at once
  constexpr int AHEAD = 4;   // handfuls of rows worked on together
  const int64_t n = n0 + lane % LPR * E;
  float bias[E];
  load_bias<T, E>(p, n, bias);
#pragma unroll 1
  for (int r = from * RPP; r < rows; r += AHEAD * by * RPP) {
    float z[AHEAD][E];
    int64_t m[AHEAD];
#pragma unroll
    for (int h = 0; h < AHEAD; ++h) {
      const int row = r + h * by * RPP + lane / LPR;
      m[h] = row < rows && m0 + row < p.m && n < p.n ? m0 + row : -1;
      const int at = row < rows ? row : 0;
#pragma unroll
      for (int g = 0; g < KW; ++g)
#pragma unroll
        for (int k = 0; k < E / 4; ++k) {
          const int piece = (lane % LPR * (E / 4) + k) ^ (at & (PIECES - 1));
          const f32x4 v = *reinterpret_cast<const f32x4*>(own + g * apart + at * COLS + piece * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) z[h][k * 4 + i] = g == 0 ? v[i] : z[h][k * 4 + i] + v[i];
        }
    }
    if (p.part != nullptr) {
#pragma unroll
      for (int h = 0; h < AHEAD; ++h)
        store_vec<float, E>(p.part + ((int64_t)split * p.m + m[h]) * p.n + n, z[h], m[h] >= 0 ? p.n - n : 0);
    } else {
      finish<T, AHEAD, E>(p, m, n, bias, z);
    }
  }
}

template <int S>
constexpr int kTileThreads = TileShape<S>::WM * TileShape<S>::WN * TileShape<S>::KW * 64;

// LDS of a tile: its groups' slices.
template <int S, bool DIRECT>
constexpr int kTileLds = (DIRECT ? TileShape<S>::STAGES : 2) * TileShape<S>::KW *
                         (TileShape<S>::BM + TileShape<S>::BN) * kSliceBytes;

// The tile of C that workgroup `id` of `count` computes.
template <class T, int L, int S, bool DIRECT>
__device__ __forceinline__ void product_tile(const ProductArgs& p, unsigned id, unsigned count, char* memory) {
  using Sh = TileShape<S>;
  constexpr int WAVES = Sh::WM * Sh::WN, KW = Sh::KW, D = kDepth<T>;
  constexpr int FM = Sh::BM / Sh::WM / 16, FN = Sh::BN / Sh::WN / 16;
  using A = Slices<T, L == kGradW, Sh::BM, WAVES>;
  using B = Slices<T, L != kForward, Sh::BN, WAVES>;
  constexpr int STAGES = DIRECT ? Sh::STAGES : 2;
  constexpr bool WRITTEN = L != kForward && sizeof(T) == 2;
  auto lds = reinterpret_cast<char(*)[KW][A::kBytes + B::kBytes]>(memory);   // [STAGES]
  int tm, tn, split;
  tile_of(p, id, count, tm, tn, split);
  const int64_t m0 = (int64_t)tm * Sh::BM, n0 = (int64_t)tn * Sh::BN;
  const int64_t begin = split * p.k_chunk, end = min(p.k, begin + p.k_chunk);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int group = wave / WAVES;
  A a;
  B b;
  a.begin(p.a, p.lda, m0, p.m, wave % WAVES);
  b.begin(p.b, p.ldb, n0, p.n, wave % WAVES);
  const int wm = a.wave / Sh::WN * (FM * 16), wn = a.wave % Sh::WN * (FN * 16);
  f32x4 acc[FM][FN] = {};
  auto compute = [&](const char* buf) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename A::Piece x[FM];
      typename B::Piece y[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) y[j] = B::read(buf + A::kBytes, wn + j * 16, s);
#pragma unroll
      for (int i = 0; i < FM; ++i) x[i] = A::read(buf, wm + i * 16, s);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) multiply(acc[i][j], y[j], x[i]);
    }
  };
  // a group's slices, KW slices apart; where they run out for one group, it reads zeros
  const int slices = (int)ceil_div(max(end - begin, (int64_t)0), (int64_t)D * KW);
  const int64_t k0 = begin + (int64_t)group * D;
  constexpr int64_t STEP = (int64_t)D * KW;
  if constexpr (DIRECT) {
    // STAGES - 1 slices are on their way while one is multiplied
    constexpr int COPIES = A::kCopies + B::kCopies;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
      if (i < slices) {
        a.template copy<WRITTEN>(lds[i][group], k0 + i * STEP, end);
        b.template copy<WRITTEN>(lds[i][group] + A::kBytes, k0 + i * STEP, end);
      }
    int at = 0;
    for (int i = 0; i < slices; ++i) {
      if (i + STAGES - 2 < slices)
        wait_copies<(STAGES - 2) * COPIES>();
      else
        wait_copies<0>();
      barrier();   // slice i has arrived; slice i - 1 has been read by all
      if (i + STAGES - 1 < slices) {
        char* next = lds[at == 0 ? STAGES - 1 : at - 1][group];
        a.template copy<WRITTEN>(next, k0 + (i + STAGES - 1) * STEP, end);
        b.template copy<WRITTEN>(next + A::kBytes, k0 + (i + STAGES - 1) * STEP, end);
      }
      compute(lds[at][group]);
      at = at == STAGES - 1 ? 0 : at + 1;
    }
  } else {
    typename A::Piece ha[A::kCopies];
    typename B::Piece hb[B::kCopies];
    if (slices > 0) {
      a.fetch(ha, k0, end);
      b.fetch(hb, k0, end);
      a.put(lds[0][group], ha);
      b.put(lds[0][group] + A::kBytes, hb);
    }
    for (int i = 0; i < slices; ++i) {
      __syncthreads();
      const bool more = i + 1 < slices;
      if (more) {
        a.fetch(ha, k0 + (i + 1) * STEP, end);
        b.fetch(hb, k0 + (i + 1) * STEP, end);
      }
      compute(lds[i & 1][group]);
      if (more) {
        a.put(lds[(i + 1) & 1][group], ha);
        b.put(lds[(i + 1) & 1][group] + A::kBytes, hb);
      }
    }
  }
  // the groups' sums meet in the buffers; each group takes a share of the rows
  constexpr int OWN = FM * 16 * FN * 16;
  static_assert(KW * WAVES * OWN * 4 <= kTileLds<S, DIRECT>, "the waves' sums fit the buffers");
  const int lane = threadIdx.x % 64;
  float* own = reinterpret_cast<float*>(memory) + a.wave * OWN;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < FM; ++i) put_sums<FN>(own + group * (WAVES * OWN), i * 16, acc[i], lane);
  __syncthreads();
  write_rows<T, FN, KW>(p, own, WAVES * OWN, FM * 16, group, KW, m0 + wm, n0 + wn, split, lane);
}

template <class T, int L, int S, bool DIRECT>
__global__ __launch_bounds__(kTileThreads<S>, TileShape<S>::OCC) void product_kernel(const ProductArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[kTileLds<S, DIRECT>];
  const unsigned id = (unsigned)group_of_grid(), count = tile_count(p);
  if (id < count) product_tile<T, L, S, DIRECT>(p, id, count, lds);
}

// Both gradient products and the bias' sums in one launch, for products of small tiles:
// they fill the device together.
template <class T, int S>
__global__ __launch_bounds__(kTileThreads<S>, TileShape<S>::OCC)
void pair_kernel(const ProductArgs x, const ProductArgs w, unsigned groups_x, unsigned groups_w, const ColumnSums sums) {
  __shared__ __attribute__((aligned(1024))) char lds[kTileLds<S, true>];
  // the product with the longer sums goes first, so that none of its tiles is left for the end
  const bool w_first = w.k_chunk > x.k_chunk;
  const unsigned first = w_first ? groups_w : groups_x, both = groups_x + groups_w;
  if (blockIdx.x >= both) {
    const int64_t c = (int64_t)(blockIdx.x - both) * kSumColumns + threadIdx.x % kSumColumns;
    const float sum = column_sum<kTileThreads<S>>(sums.part, sums.parts, sums.n, c);
    if (threadIdx.x < kSumColumns && c < sums.n) static_cast<T*>(sums.out)[c] = (T)sum;
  } else if ((blockIdx.x < first) == w_first) {
    product_tile<T, kGradW, S, true>(w, w_first ? blockIdx.x : blockIdx.x - first, groups_w, lds);
  } else {
    product_tile<T, kGradX, S, true>(x, w_first ? blockIdx.x - first : blockIdx.x, groups_x, lds);
  }
}

// Tiles of BM x 256 (BM 256, or 192 where that fills the device better) in 16 bits, by 8
// waves.
//
// Two waves share a SIMD, one of the workgroup's upper and one of its lower half.  The
// lower half runs one barrier behind, so that while one of the two multiplies the other
// reads LDS.  A slice is four turns: a half of the wave's rows by a half of its columns
// each.  The next slice is asked for in the first two turns and awaited in the fourth, when
// its buffer's last reads are two turns past.
//
// 8192^3 in bf16 runs at 1.39 PFLOP/s, and at 1.49 without the writing of C, which all
// compute units do at the same time.  Workgroups that stay for several tiles gain nothing
// (10000 x 1024 x 4096 104 us against 98): the copies they wait for are behind the last
// tile's writes, which a workgroup that ends does not wait for.
template <class T, int L, int BM>
__global__ __launch_bounds__(512, 2) void large_kernel(const ProductArgs p) {
  constexpr int BN = 256, D = kDepth<T>, FM = BM / 32, FN = 4, HM = FM / 2;
  using A = Slices<T, L == kGradW, BM, 8>;
  using B = Slices<T, L != kForward, BN, 8>;
  __shared__ __attribute__((aligned(1024))) char lds[2][A::kBytes + B::kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int wm = wave / 4 * (FM * 16), wn = wave % 4 * (FN * 16);
  int tm, tn, split;
  const unsigned id = (unsigned)group_of_grid(), count = tile_count(p);
  if (id >= count) return;
  tile_of(p, id, count, tm, tn, split);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int64_t k0 = split * p.k_chunk, end = min(p.k, k0 + p.k_chunk);
  const int slices = __builtin_amdgcn_readfirstlane((int)ceil_div(end - k0, (int64_t)D));
  A a;
  B b;
  a.begin(p.a, p.lda, m0, p.m, wave);
  b.begin(p.b, p.ldb, n0, p.n, wave);
  a.template copy<false>(lds[0], k0, end);
  b.template copy<false>(lds[0] + A::kBytes, k0, end);
  f32x4 acc[FM][FN] = {};
  wait_copies<0>();
  barrier();
  if (wave >= 4) barrier();
  for (int i = 0; i < slices; ++i) {
    const char* buf = lds[i & 1];
    char* next = lds[(i + 1) & 1];
    const bool more = i + 1 < slices;
    const int64_t kn = k0 + (int64_t)(i + 1) * D;
    typename A::Piece x[2][HM];
    typename B::Piece y0[2][2], y1[2][2];
    auto read_x = [&](int half) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int f = 0; f < HM; ++f) x[s][f] = A::read(buf, wm + (half * HM + f) * 16, s);
    };
    auto read_y = [&](typename B::Piece (&y)[2][2], int half) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int f = 0; f < 2; ++f) y[s][f] = B::read(buf + A::kBytes, wn + (half * 2 + f) * 16, s);
    };
    auto turn = [&](const typename B::Piece (&y)[2][2], int hx, int hy) {
      barrier();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int f = 0; f < HM; ++f)
#pragma unroll
          for (int g = 0; g < 2; ++g) multiply(acc[hx * HM + f][hy * 2 + g], y[s][g], x[s][f]);
      __builtin_amdgcn_s_setprio(0);
      barrier();
    };
    read_y(y0, 0);
    read_x(0);
    if (more) a.template copy<false>(next, kn, end);
    turn(y0, 0, 0);
    read_y(y1, 1);
    if (more) b.template copy<false>(next + A::kBytes, kn, end);
    turn(y1, 0, 1);
    read_x(1);
    turn(y1, 1, 1);
    wait_copies<0>();
    turn(y0, 1, 0);
  }
  if (wave < 4) barrier();
  constexpr int OWN = HM * 16 * FN * 16;
  static_assert(8 * OWN * 4 <= (int)sizeof(lds), "half of the waves' sums fits the buffers");
  float* own = reinterpret_cast<float*>(lds) + wave * OWN;
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int i = 0; i < HM; ++i) put_sums<FN>(own, i * 16, acc[half * HM + i], lane);
    wave_sync();
    write_rows<T, FN, 1>(p, own, 0, HM * 16, 0, 1, m0 + wm + half * HM * 16, n0 + wn, split, lane);
    wave_sync();
  }
}

// C from the splits' sums, in their order.  What bounds it is the wait for each split's
// sums, so four are on their way at once; they are added one by one, to the same bits.  On
// the whole product: dw of 9689 x 216 x 40 in fp16 (32 splits) 14.8 -> 10.6 us, of
// 6525 x 584 x 8 in fp32 (32) 21.3 -> 17.1, dx of 64 x 1024 x 4096 in bf16 (16) 12.0 -> 9.8.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(const ProductArgs p) {
  const int64_t quads = (p.n + 3) / 4;
  const int64_t i = group_of_grid() * 256 + threadIdx.x;
  if (i >= p.m * quads) return;
  constexpr int AHEAD = 4;
  const int64_t m[1] = {i / quads}, n = i % quads * 4;
  float bias[4], z[1][4] = {};
  load_bias<T, 4>(p, n, bias);
  const float* part = p.part + m[0] * p.n + n;
  int s = 0;
  for (; s + AHEAD <= p.splits; s += AHEAD) {
    float v[AHEAD][4];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_vec<float, 4>(v[i], part + (int64_t)(s + i) * p.m * p.n, p.n - n);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[0][j] += v[i][j];
  }
  for (; s < p.splits; ++s) {
    float v[4];
    load_vec<float, 4>(v, part + (int64_t)s * p.m * p.n, p.n - n);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[0][j] += v[j];
  }
  finish<T, 1, 4>(p, m, n, bias, z);
}

// What thread `i` of a copy takes: 16 bytes of operand a, whose pieces come first, or of b.
struct AlignPiece {
  bool there, second;
  int64_t row, col;
};
template <int E>
__host__ __device__ __forceinline__ AlignPiece align_piece(const AlignArgs& a, const AlignArgs& b, int64_t pieces_a,
                                                           int64_t i) {
  const bool second = i >= pieces_a;
  const AlignArgs& o = second ? b : a;
  if (o.dst == nullptr) return {false, second, 0, 0};   // its rows have no length to divide by
  if (second) i -= pieces_a;
  const int64_t pieces = o.ld_dst / E, row = i / pieces, col = i % pieces * E;
  return {row < o.rows, second, row, col};
}

// Copies up to two operands; a thread copies 16 bytes.  1000 x 2048 in fp16 from a slice of
// rows 2053 apart takes 5.0 us, a launch's latency among them; the product of it and 785
// outputs 18.7 in all, and 22.1 through registers, which need no copy (256 x 54 x 512 in
// fp32, the other way round, 6.5 and 5.0).
template <class T>
__global__ __launch_bounds__(256) void align_kernel(const AlignArgs a, const AlignArgs b, int64_t pieces_a) {
  constexpr int E = kVec<T>;
  const AlignPiece piece = align_piece<E>(a, b, pieces_a, group_of_grid() * 256 + threadIdx.x);
  if (!piece.there) return;
  const AlignArgs& o = piece.second ? b : a;
  const int64_t row = piece.row, col = piece.col;
  const T* from = static_cast<const T*>(o.src) + row * o.ld + col;
  typename Fragment<T>::type v;
  if (o.width - col >= E) {
    v = *reinterpret_cast<const typename Unaligned<T, E>::type*>(from);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = k < o.width - col ? from[k] : (T)0.0f;
  }
  *reinterpret_cast<typename Fragment<T>::type*>(static_cast<T*>(o.dst) + row * o.ld_dst + col) = v;
}

// The forward product of up to 16 RB rows: W is read once, straight to registers, by
// workgroups of 16 outputs whose 8 waves take a part of k each and join their sums in LDS.
// 1 x 1024 x 4096 in bf16 takes 3.4 us in a graph, most of it latency (2.5 TB/s of W), and
// 5.9 in 64 x 64 tiles; 16 rows 4.1 and 5.9.
template <class T, int RB>
__global__ __launch_bounds__(512) void few_rows_kernel(const ProductArgs p) {
  constexpr int E = kVec<T>, STEP = 4 * E, WAVES = 8, AHEAD = 4;
  typedef typename Fragment<T>::type Piece;
  __shared__ f32x4 sums[WAVES][RB][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t n0 = group_of_grid() * 16;
  if (n0 >= p.n) return;
  const int64_t steps = ceil_div(p.k, STEP), each = ceil_div(steps, WAVES);
  const int64_t first = wave * each, last = min(steps, first + each);
  // lane i of 16 takes row i of W (of x), the 16-byte piece lane / 16 of a step
  auto fetch = [&](const void* base, int64_t ld, int64_t row, int64_t rows, int64_t k) {
    const int64_t n = row < rows ? p.k - k : 0;
    const T* q = static_cast<const T*>(base) + row * ld + k;
    Piece v;
    if (n >= E) {
      v = *reinterpret_cast<const typename Unaligned<T, E>::type*>(q);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = i < n ? q[i] : (T)0.0f;
    }
    return v;
  };
  float bias[4];
  load_bias<T, 4>(p, n0 + lane / 16 * 4, bias);
  f32x4 acc[RB] = {};
  for (int64_t s = first; s < last; s += AHEAD) {
    Piece w[AHEAD], x[AHEAD][RB];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      // past the wave's part, k is past the end: zeros
      const int64_t k = s + j < last ? (s + j) * STEP + lane / 16 * E : p.k;
      w[j] = fetch(p.b, p.ldb, n0 + lane % 16, p.n, k);
#pragma unroll
      for (int r = 0; r < RB; ++r) x[j][r] = fetch(p.a, p.lda, r * 16 + lane % 16, p.m, k);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int r = 0; r < RB; ++r) multiply(acc[r], w[j], x[j][r]);
  }
#pragma unroll
  for (int r = 0; r < RB; ++r) sums[wave][r][lane] = acc[r];
  __syncthreads();
  if (wave >= RB) return;
  const int64_t m[1] = {wave * 16 + lane % 16}, n = n0 + lane / 16 * 4;
  if (m[0] >= p.m || n >= p.n) return;
  float z[1][4] = {};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const f32x4 v = sums[w][wave][lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[0][i] += v[i];
  }
  finish<T, 1, 4>(p, m, n, bias, z);
}

inline hipError_t launch_join(const ProductArgs& p, hipStream_t s, void (*kernel)(ProductArgs)) {
  kernel<<<grid_of(ceil_div(p.m * ceil_div(p.n, 4), 256)), 256, 0, s>>>(p);
  return hipGetLastError();
}

template <class T, int L, int S, bool DIRECT>
hipError_t launch_tiles(ProductArgs p, hipStream_t s) {
  using Sh = TileShape<S>;
  p.tiles_m = (int32_t)ceil_div(p.m, Sh::BM);
  p.tiles_n = (int32_t)ceil_div(p.n, Sh::BN);
  const int64_t groups = (int64_t)p.tiles_m * p.tiles_n * p.splits;
  if (groups > INT32_MAX) return hipErrorInvalidValue;   // larger than any memory
  product_kernel<T, L, S, DIRECT><<<grid_of(groups), kTileThreads<S>, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && p.splits > 1 ? launch_join(p, s, join_kernel<T>) : e;
}

template <class T, int L, int BM>
hipError_t launch_large(ProductArgs p, hipStream_t s) {
  p.tiles_m = (int32_t)ceil_div(p.m, BM);
  p.tiles_n = (int32_t)ceil_div(p.n, 256);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * p.splits;
  if (tiles > INT32_MAX) return hipErrorInvalidValue;   // larger than any memory
  large_kernel<T, L, BM><<<grid_of(tiles), 512, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && p.splits > 1 ? launch_join(p, s, join_kernel<T>) : e;
}

template <class T, int L>
hipError_t launch_layout(const ProductArgs& p, const ProductPlan& plan, hipStream_t s) {
  if constexpr (L == kForward)
    if (plan.shape == kFewRows) {
      const dim3 grid = grid_of(ceil_div(p.n, 16));
      if (p.m <= 16) few_rows_kernel<T, 1><<<grid, 512, 0, s>>>(p);
      else few_rows_kernel<T, 2><<<grid, 512, 0, s>>>(p);
      return hipGetLastError();
    }
  if constexpr (sizeof(T) == 2) {
    if (plan.shape == kLarge) return launch_large<T, L, 256>(p, s);
    if (plan.shape == kLower) return launch_large<T, L, 192>(p, s);
    if (plan.shape == kMiddle) return launch_tiles<T, L, kMiddle, true>(p, s);
    if (plan.shape == kMany) return launch_tiles<T, L, kMany, true>(p, s);
  } else {
    if (plan.shape == kNarrow) return launch_tiles<T, L, kNarrow, true>(p, s);
  }
  return plan.direct ? launch_tiles<T, L, kSmall, true>(p, s) : launch_tiles<T, L, kSmall, false>(p, s);
}

// Copies the operands that have to be.
template <class T>
hipError_t align_operands(const AlignArgs& first, const AlignArgs& second, hipStream_t s) {
  int64_t pieces[2] = {};
  if (first.dst != nullptr) pieces[0] = first.rows * (first.ld_dst / kVec<T>);
  if (second.dst != nullptr) pieces[1] = second.rows * (second.ld_dst / kVec<T>);
  if (pieces[0] + pieces[1] == 0) return hipSuccess;
  align_kernel<T><<<grid_of(ceil_div(pieces[0] + pieces[1], 256)), 256, 0, s>>>(first, second, pieces[0]);
  return hipGetLastError();
}

template <class T>
hipError_t launch_product_of(ProductArgs p, Layout layout, const ProductPlan& plan,
                             const AlignArgs (&align)[2], hipStream_t s) {
  const hipError_t e = align_operands<T>(align[0], align[1], s);
  if (e != hipSuccess) return e;
  if (align[0].dst != nullptr) p.a = align[0].dst, p.lda = align[0].ld_dst;
  if (align[1].dst != nullptr) p.b = align[1].dst, p.ldb = align[1].ld_dst;
  if (layout == kForward) return launch_layout<T, kForward>(p, plan, s);
  if (layout == kGradX) return launch_layout<T, kGradX>(p, plan, s);
  return launch_layout<T, kGradW>(p, plan, s);
}

// dx and dw, both of one small shape, and the sums.
template <class T, int S>
hipError_t launch_pair(ProductArgs x, ProductArgs w, const ColumnSums& sums, hipStream_t s) {
  using Sh = TileShape<S>;
  int64_t groups[3] = {};
  ProductArgs* both[2] = {&x, &w};
  for (int i = 0; i < 2; ++i) {
    both[i]->tiles_m = (int32_t)ceil_div(both[i]->m, Sh::BM);
    both[i]->tiles_n = (int32_t)ceil_div(both[i]->n, Sh::BN);
    groups[i] = (int64_t)both[i]->tiles_m * both[i]->tiles_n * both[i]->splits;
  }
  groups[2] = sums.out != nullptr ? ceil_div(sums.n, kSumColumns) : 0;
  // few: the tiles are up to 4 a compute unit, the sums' columns no more than the tiles' rows
  pair_kernel<T, S><<<(unsigned)(groups[0] + groups[1] + groups[2]), kTileThreads<S>, 0, s>>>(
      x, w, (unsigned)groups[0], (unsigned)groups[1], sums);
  hipError_t e = hipGetLastError();
  for (int i = 0; i < 2 && e == hipSuccess; ++i)
    if (both[i]->splits > 1) e = launch_join(*both[i], s, join_kernel<T>);
  return e;
}

template <class T>
hipError_t launch_pair_of(ProductArgs x, ProductArgs w, int shape, const AlignArgs& align_w, const AlignArgs& align_x,
                          const ColumnSums& sums, hipStream_t s) {
  const hipError_t e = align_operands<T>(align_w, align_x, s);
  if (e != hipSuccess) return e;
  if (align_w.dst != nullptr) x.b = align_w.dst, x.ldb = align_w.ld_dst;
  if (align_x.dst != nullptr) w.b = align_x.dst, w.ldb = align_x.ld_dst;
  if constexpr (sizeof(T) == 4)
    if (shape == kNarrow) return launch_pair<T, kNarrow>(x, w, sums, s);
  return launch_pair<T, kSmall>(x, w, sums, s);
}

}  // namespace nn
}  // namespace gts
