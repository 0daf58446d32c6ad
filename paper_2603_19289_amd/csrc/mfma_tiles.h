// One output tile of a matrix product on the matrix cores, for 16-bit operands that lie either way in memory:
//   C[m, n] = sum_k a(m, k) b(n, k),   acc in float, 16x16x32 instructions, K walked 64 at a time.
// An operand is "k-major" (the 64 values of a row of the tile are contiguous) or "i-major" (the tile's rows are contiguous for each k, as
// a weight matrix is for the gradient of its input, and both operands are for the gradient of a weight matrix).  Both kinds travel
// from global memory to LDS as they lie, 16 bytes a lane, without a register between; a k-major fragment is read as 16 bytes, an
// i-major one by two transposing reads of 8.  LDS is swizzled so that either read meets every bank once:
//   k-major: rows of 128 bytes, the 16-byte chunk c of row r at place c ^ (r / 2 % 8)  (16 rows of a fragment, one chunk each)
//   i-major: 32-byte granules, granule q of row k at place q ^ f(k)  (32 lanes read rows {0..3, 8..11} + 4 h of a fragment's 32)
// The next 64 columns are on their way into the other half of LDS while the matrix instructions work on this one.
#pragma once
#include <type_traits>

#include "train_common.h"

namespace moe_spec {

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(8))) short s16x8_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8v_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

struct Bf16 {
  static __device__ __forceinline__ f32x4_t mfma(s16x8_t a, s16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v_t, a), __builtin_bit_cast(bf16x8v_t, b), c, 0, 0, 0);
  }
};
struct F16 {
  static __device__ __forceinline__ f32x4_t mfma(s16x8_t a, s16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  }
};

constexpr int kTileK = 64;
__device__ const uint4 kZeroChunk = {0, 0, 0, 0};      // what lies outside a tile is read from here

using LdsPtr = __attribute__((address_space(3))) char *;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return uint32_t(reinterpret_cast<uintptr_t>((LdsPtr)p)); }

// 16 bytes a lane from global memory to LDS at base + 16 lane; base is the wavefront's.  Written as an instruction, since the compiler
// would wait for it before every later LDS read, whichever half that reads; it has no output register.  lds_loads_done() and a
// barrier come before the first read.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(base) : "memory");
}
__device__ __forceinline__ void lds_loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// An operand tile of ROWS x 64 (k-major) or 64 x ROWS (i-major) in LDS and the loads that fill it.
// WHOLE16: addresses, row strides and extents are multiples of 16 bytes: a chunk lies inside the matrix or outside of it.
template <int ROWS, bool IMAJOR, bool WHOLE16, int THREADS>
struct OperandTile {
  static constexpr int kBytes = ROWS * kTileK * 2, kChunks = ROWS * kTileK / 8, kEach = kChunks / THREADS;
  static_assert(kChunks % THREADS == 0 && THREADS % 64 == 0 && ROWS % 64 == 0, "whole chunks for every thread");
  const uint16_t *at[kEach];             // where this thread's chunks of the next step lie
  bool in[kEach];                        // i-major: whether those columns exist
  int64_t step;                          // elements from one step to the next
  int rows;                              // rows of the tile that exist (at least one)
  uint4 held[WHOLE16 ? 1 : kEach];

  static __device__ __forceinline__ int granule_swizzle(int k) {
    return ROWS >= 128 ? (k & 3) | (k >> 1 & 4) : (k >> 1 & 1) | (k >> 2 & 2);
  }
  // Row (k-major: of the tile, i-major: k) and first column of the chunk that goes to place c.
  static __device__ __forceinline__ int row_of(int c) { return IMAJOR ? c / (ROWS / 8) : c / 8; }
  static __device__ __forceinline__ int column_of(int c) {
    if constexpr (IMAJOR) {
      const int place = c % (ROWS / 8), k = c / (ROWS / 8);
      return (((place >> 1) ^ granule_swizzle(k)) << 4) | (place & 1) << 3;
    } else {
      return ((c % 8) ^ (c / 16 % 8)) * 8;
    }
  }
  // origin: the element (0, 0) of the tile; ld: elements between rows of memory.
  __device__ __forceinline__ void begin(const uint16_t *origin, int64_t ld, int rows_, int tid) {
    rows = rows_;
    step = IMAJOR ? ld * kTileK : kTileK;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int c = j * THREADS + tid, r = row_of(c), col = column_of(c);
      if constexpr (IMAJOR) {
        in[j] = col < rows;
        at[j] = origin + int64_t(r) * ld + col;
      } else {
        at[j] = origin + int64_t(min(r, rows - 1)) * ld + col;
      }
    }
  }
  // Asks for the next step; k_left: columns that are left (k-major), rows that are left (i-major).
  __device__ __forceinline__ void issue(uint32_t lds, int k_left, int tid) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int c = j * THREADS + tid;
      const int k = IMAJOR ? row_of(c) : column_of(c);
      if constexpr (WHOLE16) {
        const void *from = (k < k_left && (!IMAJOR || in[j])) ? static_cast<const void *>(at[j]) : &kZeroChunk;
        load_to_lds(from, __builtin_amdgcn_readfirstlane(lds + (c & ~63) * 16));
      } else {
        const int n = IMAJOR ? (k < k_left ? rows - column_of(c) : 0) : k_left - k;
        held[j] = uint4{0, 0, 0, 0};
        if (n >= 8) {
          held[j] = load_raw<uint4>(at[j]);
        } else if (n > 0) {
          uint16_t e[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < 7; ++i) if (i < n) e[i] = at[j][i];
          __builtin_memcpy(&held[j], e, 16);
        }
      }
      at[j] += step;
    }
  }
  // Puts what issue() asked for where it said.
  __device__ __forceinline__ void land(char *lds, int tid) {
    if constexpr (!WHOLE16) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) *reinterpret_cast<uint4 *>(lds + (j * THREADS + tid) * 16) = held[j];
    }
  }
  // Fragment of 16 rows from `row` on (a multiple of 16), columns 32 half .. + 31 of the step: lane (i, g) = (lane % 16, lane / 16)
  // gets row i, columns 8 g .. 8 g + 7.
  static __device__ __forceinline__ s16x8_t fragment(const char *lds, int row, int half, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (IMAJOR) {
      const int k = half * 32 + g * 8 + (i >> 2);
      const uint32_t at = lds_address(lds) + k * (ROWS * 2) + (((row >> 4) ^ granule_swizzle(k)) << 5) + (i & 3) * 8;
      using P = __attribute__((address_space(3))) s16x4_t *;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<P>(at));
      // four rows further on; their swizzle is the same where 128 or more rows need three bits, and otherwise differs in its second
      const int k4 = k + 4;
      const uint32_t at4 = lds_address(lds) + k4 * (ROWS * 2) + (((row >> 4) ^ granule_swizzle(k4)) << 5) + (i & 3) * 8;
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<P>(at4));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const s16x8_t *>(lds + (row + i) * 128 + (((half * 4 + g) ^ (i >> 1)) << 4));
    }
  }
};

// The product of a tile of BM x BN by WM x WN wavefronts.  acc[f][h][r] of lane (i, g): row 16 f + i, column 16 h + 4 g + r of the
// wavefront's part.
template <typename Type, int BM, int BN, int WM, int WN, bool A_IMAJOR, bool B_IMAJOR, bool WHOLE16>
struct TileProduct {
  static constexpr int kThreads = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
  using A = OperandTile<BM, A_IMAJOR, WHOLE16, kThreads>;
  using B = OperandTile<BN, B_IMAJOR, WHOLE16, kThreads>;
  static constexpr int kHalf = A::kBytes + B::kBytes, kLds = 2 * kHalf;
  f32x4_t acc[FM][FN];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[f][h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
  __device__ __forceinline__ void compute(const char *half, int wave, int lane) {
    const int row = wave / WN * (BM / WM), col = wave % WN * (BN / WN);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      s16x8_t a[FM], b[FN];
#pragma unroll
      for (int h = 0; h < FN; ++h) b[h] = B::fragment(half + A::kBytes, col + 16 * h, kk, lane);
#pragma unroll
      for (int f = 0; f < FM; ++f) a[f] = A::fragment(half, row + 16 * f, kk, lane);
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int h = 0; h < FN; ++h) acc[f][h] = Type::mfma(b[h], a[f], acc[f][h]);
    }
  }
  // a, b: the tile's first elements; K columns; rows and columns of the tile that exist.  Every thread of the workgroup calls it.
  __device__ __forceinline__ void run(char *lds, const uint16_t *a, int64_t lda, int a_rows, const uint16_t *b, int64_t ldb, int b_rows, int64_t K) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t base = lds_address(lds);
    clear();
    if (K <= 0) return;
    A ta;
    B tb;
    ta.begin(a, lda, a_rows, tid);
    tb.begin(b, ldb, b_rows, tid);
    const auto left = [](int64_t k) { return int(k < kTileK ? k : int64_t(kTileK)); };
    ta.issue(base, left(K), tid);
    tb.issue(base + A::kBytes, left(K), tid);
    ta.land(lds, tid);
    tb.land(lds + A::kBytes, tid);
    lds_loads_done();
    __syncthreads();
    int now = 0;
    for (int64_t k = K - kTileK;; k -= kTileK) {
      const int next = now ^ kHalf;
      if (k > 0) {
        ta.issue(base + next, left(k), tid);
        tb.issue(base + next + A::kBytes, left(k), tid);
      }
      compute(lds + now, wave, lane);
      if (k <= 0) break;
      ta.land(lds + next, tid);
      tb.land(lds + next + A::kBytes, tid);
      lds_loads_done();
      __syncthreads();
      now = next;
    }
  }
};

// Four values of one row of a result, of which the first n exist.
__device__ __forceinline__ void store4(uint16_t *p, f32x4_t v, int n) {
  const uint2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  if (n >= 4) {
    __builtin_memcpy(p, &w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < n) p[i] = uint16_t(i & 1 ? (i < 2 ? w.x : w.y) >> 16 : (i < 2 ? w.x : w.y));
  }
}
__device__ __forceinline__ void store4(float *p, f32x4_t v, int n) {
  if (n >= 4) {
    __builtin_memcpy(p, &v, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < n) p[i] = v[i];
  }
}

}  // namespace moe_spec
