// One output tile of a matrix product on the matrix cores, for operands of 16 bits or of float that lie either way in memory:
//   C[m, n] = sum_k a(m, k) b(n, k),   acc in float, 16x16x32 (16x16x4) instructions, K walked a step of 64 (or 32) at a time.
// An operand is "k-major" (a step's values of a row of the tile are contiguous) or "i-major" (the tile's rows are contiguous for each k, as
// a weight matrix is for the gradient of its input, and both operands are for the gradient of a weight matrix).  Both kinds travel
// from global memory to LDS as they lie, 16 bytes a lane, without a register between; a k-major fragment is read as 16 bytes, an
// i-major one by two transposing reads of 8 (float: four of 4, a row each).  LDS is swizzled so that either read meets every bank once:
//   k-major: rows of 128 bytes, the 16-byte chunk c of row r at place c ^ (r / 2 % 8)  (16 rows of a fragment, one chunk each); steps of 32:
//            rows of 64 bytes, place c ^ (r / 4 % 4)
//   i-major, float: the 16-byte chunk c of row k at place c ^ (k & 12)  (16 lanes a row, of rows four apart)
//   i-major: 32-byte granules, granule q of row k at place q ^ f(k)  (32 lanes read rows {0..3, 8..11} + 4 h of a fragment's 32)
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
  using Elem = uint16_t;
  static constexpr int kStep = 64, kWaves = 1;    // columns of a usual step; fewest wavefronts a SIMD
  static __device__ __forceinline__ f32x4_t mfma(s16x8_t a, s16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v_t, a), __builtin_bit_cast(bf16x8v_t, b), c, 0, 0, 0);
  }
};
struct F16 {
  using Elem = uint16_t;
  static constexpr int kStep = 64, kWaves = 1;
  static __device__ __forceinline__ f32x4_t mfma(s16x8_t a, s16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  }
};
// Sixteen columns: an operand's lane (i, g) holds columns 4 g .. 4 g + 3, one for each of four instructions.
struct F32 {
  using Elem = float;
  static constexpr int kStep = 32, kWaves = 6;   // wavefronts a SIMD: three workgroups of eight; 83 registers instead of 80 left two, 7 % slower
  static __device__ __forceinline__ f32x4_t mfma(s16x8_t a, s16x8_t b, f32x4_t c) {
    const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
};

using LdsPtr = __attribute__((address_space(3))) char *;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return uint32_t(reinterpret_cast<uintptr_t>((LdsPtr)p)); }

// 16 bytes a lane from memory to LDS at base + 16 lane (base is the wavefront's), through a buffer descriptor: what lies outside of its
// bounds arrives as zeros.  Written as an instruction, since the compiler would wait for it before every later LDS read, whichever
// half that reads; it has no output register.  lds_loads_done() and a barrier come before the first read.  Nor does the compiler keep a
// vector instruction's write of the descriptor (readfirstlane, a spilled word's readlane) five wait states away, as the hardware wants: the
// instructions in front of the load are as many, whatever is scheduled before them, and m0 wants one of its own.  A step's loads go two
// at a time, so that the second needs no more than that (256 x 256 orthogonalised: 79 us, each by itself 82; Muon of an estimator 156 and 159); those
// between a large tile's products by themselves (32768 rows, 32 of 5760 x 2880, transposed: 1088 us, two at a time 1110).
// m0 is reserved, so that nothing lives there for long; that it is named keeps other writes of it and their readers together.
typedef __attribute__((ext_vector_type(4))) uint32_t Buffer;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(Buffer from, uint32_t offset, uint32_t base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(from), "s"(base) : "memory", "m0");
}
// Two of them, the second APART bytes further on in LDS.
template <int APART>
__device__ __forceinline__ void load_two_to_lds(Buffer from, uint32_t first, uint32_t second, uint32_t base) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
               "s_add_u32 m0, %3, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               ::"v"(first), "v"(second), "s"(from), "s"(base), "n"(APART) : "memory", "m0", "scc");
}
#pragma clang diagnostic pop
// Until at most LEFT of this wavefront's loads are on their way.
template <int LEFT>
__device__ __forceinline__ void lds_loads_done() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }

constexpr uint32_t kOutside = 0xffffff00u;             // an offset that no descriptor here contains
constexpr int64_t kMostTileStride = 1 << 22;           // elements; 256 rows of 16 bits (128 of float) then stay below 2^32 bytes

// Sixteen bytes of a row by way of registers, of which the first n elements exist: asked for without a branch, which would hold up the next
// request, at an address that lies in the row (a chunk that is cut off is moved back to end with it, one that does not exist becomes `safe`),
// and put right when they are used.  Rows that are shorter than a chunk are read element by element.  8 experts of 1001 x 1501, 4000 rows: 41 to
// 47 us; with branches around the requests 64 to 86.
struct RowChunk {
  static __device__ __forceinline__ uint4 ask(const uint16_t *p, int n, const uint16_t *safe, bool narrow) {
    if (!narrow) return load_raw<uint4>(n >= 8 ? p : n > 0 ? p - (8 - n) : safe);
    uint16_t e[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i) if (i < n) e[i] = p[i];
    uint4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
  }
  static __device__ __forceinline__ uint4 use(uint4 v, int n, bool narrow) {
    if (narrow || n >= 8) return v;
    if (n <= 0) return uint4{0, 0, 0, 0};
    uint64_t lo = uint64_t(v.y) << 32 | v.x, hi = uint64_t(v.w) << 32 | v.z;
    const int s = (8 - n) * 16;
    lo = s >= 64 ? hi >> (s - 64) : lo >> s | hi << (64 - s);
    hi = s >= 64 ? 0 : hi >> s;
    return uint4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
  }
};

// An operand tile of ROWS x KS (k-major) or KS x ROWS (i-major) in LDS, and the loads that fill it.
// WHOLE16: straight to LDS.  Addresses, row strides and extents are multiples of 16 bytes (a chunk lies inside the matrix or outside of
// it), rows do not overlap and lie at most kMostTileStride apart.  Otherwise: through registers, any stride and alignment.
template <typename Elem, int ROWS, bool IMAJOR, bool WHOLE16, int THREADS, int KS>
struct OperandTile {
  static constexpr int kElem = sizeof(Elem), kOfChunk = 16 / kElem, kBytes = ROWS * KS * kElem, kChunks = kBytes / 16, kEach = kChunks / THREADS;
  static constexpr int kAcross = (IMAJOR ? ROWS : KS) / kOfChunk, kApart = THREADS / kAcross;      // chunks of a row; rows between a thread's chunks
  static_assert(kChunks % THREADS == 0 && THREADS % 128 == 0 && ROWS % 64 == 0 && (!IMAJOR || kApart % 16 == 0), "a thread's chunks lie in one column");
  static_assert(kElem == 2 || (WHOLE16 && KS == 32), "float: straight to LDS");

  static __device__ __forceinline__ int granule_swizzle(int k) {
    return ROWS >= 128 ? (k & 3) | (k >> 1 & 4) : (k >> 1 & 1) | (k >> 2 & 2);
  }
  // Row (k-major: of the tile, i-major: k) and first column of the chunk that goes to place c.
  static __device__ __forceinline__ int row_of(int c) { return c / kAcross; }
  static __device__ __forceinline__ int column_of(int c) {
    if constexpr (IMAJOR && kElem == 4) return ((c % kAcross) ^ (c / kAcross & 12)) * 4;
    else if constexpr (IMAJOR) return (((c % kAcross >> 1) ^ granule_swizzle(c / kAcross)) << 4) | (c & 1) << 3;
    else return (kAcross == 8 ? (c % 8) ^ (c / 16 % 8) : (c % 4) ^ (c / 16 % 4)) * kOfChunk;
  }

  Buffer from;                           // WHOLE16: the rest of the operand
  uint32_t offset, row_bytes;            // this thread's first chunk; between rows
  int64_t step;                          // from one step to the next, bytes or elements
  const Elem *at[WHOLE16 ? 1 : kEach], *safe;
  uint4 held[WHOLE16 ? 1 : kEach];
  int rows, column;                      // rows of the tile that exist (at least one); this thread's column
  int k_held;                            // columns or rows of memory of the step that is held
  bool narrow;

  // origin: the element (0, 0) of the tile; ld: elements between rows of memory; K columns in all.
  __device__ __forceinline__ void begin(const Elem *origin, int64_t ld, int rows_, int64_t K, int tid) {
    rows = rows_;
    narrow = (IMAJOR ? rows : K) < 8;
    safe = origin;
    column = column_of(tid);
    step = IMAJOR ? ld * KS : KS;
    if constexpr (WHOLE16) {
      const uint64_t p = reinterpret_cast<uint64_t>(origin);
      row_bytes = uint32_t(ld) * kElem;
      from[0] = __builtin_amdgcn_readfirstlane(uint32_t(p));
      from[1] = __builtin_amdgcn_readfirstlane(uint32_t(p >> 32));
      from[2] = __builtin_amdgcn_readfirstlane(uint32_t(rows) * row_bytes);
      from[3] = 0x00020000u;
      offset = IMAJOR && column >= rows ? kOutside : row_of(tid) * row_bytes + column * kElem;
      step *= kElem;
    } else {
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int r = row_of(tid) + j * kApart;
        at[j] = origin + int64_t(IMAJOR ? r : min(r, rows - 1)) * ld + column;
      }
    }
  }
  // Asks for the next step, of which k_left (at most KS) columns (k-major) or rows of memory (i-major) exist.
  __device__ __forceinline__ void issue(uint32_t lds, int k_left, int tid) {
    if constexpr (WHOLE16) {
      limit(k_left);
#pragma unroll
      for (int j = 0; j < kEach; j += kTogether) issue_chunks<kTogether>(lds, j, k_left, tid);
      advance();
    } else {
      k_held = k_left;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        held[j] = RowChunk::ask(at[j], elements(j, tid), safe, narrow);
        at[j] += step;
      }
    }
  }
  // The same in parts, straight to LDS: limit, one chunk or two after the other, advance.
  static constexpr int kTogether = kEach % 2 == 0 ? 2 : 1;
  __device__ __forceinline__ void limit(int k_left) {
    if constexpr (IMAJOR) from[2] = uint32_t(k_left) * row_bytes;
  }
  template <int N>
  __device__ __forceinline__ void issue_chunks(uint32_t lds, int j, int k_left, int tid) {
    const uint32_t mine = !IMAJOR && column >= k_left ? kOutside : offset, base = __builtin_amdgcn_readfirstlane(lds + (tid & ~63) * 16) + j * THREADS * 16;
    const auto place = [&](int i) { return i == 0 || mine != kOutside ? mine + i * kApart * row_bytes : kOutside; };
    if constexpr (N == 2) load_two_to_lds<THREADS * 16>(from, place(j), place(j + 1), base);
    else load_to_lds(from, place(j), base);
  }
  __device__ __forceinline__ void advance() {
    const uint64_t p = (uint64_t(from[1]) << 32 | from[0]) + uint64_t(step);
    from[0] = uint32_t(p);
    from[1] = uint32_t(p >> 32);
  }
  // How many elements of a thread's chunk j exist.
  __device__ __forceinline__ int elements(int j, int tid) const {
    return IMAJOR ? (row_of(tid) + j * kApart < k_held ? rows - column : 0) : k_held - column;
  }
  // Puts what issue() asked for where it said.
  __device__ __forceinline__ void land(char *lds, int tid) {
    if constexpr (!WHOLE16) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) *reinterpret_cast<uint4 *>(lds + (j * THREADS + tid) * 16) = RowChunk::use(held[j], elements(j, tid), narrow);
    }
  }
  // Fragment of 16 rows from `row` on (a multiple of 16), columns 32 half .. + 31 (float: 16 half .. + 15) of the step: lane (i, g) =
  // (lane % 16, lane / 16) gets row i, columns 8 g .. 8 g + 7 (4 g .. 4 g + 3).
  static __device__ __forceinline__ s16x8_t fragment(const char *lds, int row, int half, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (IMAJOR && kElem == 4) {
      const float *at = reinterpret_cast<const float *>(lds) + (half * 16 + 4 * g) * ROWS + ((row + i) ^ 16 * g);
      return __builtin_bit_cast(s16x8_t, f32x4_t{at[0], at[ROWS], at[2 * ROWS], at[3 * ROWS]});
    } else if constexpr (IMAJOR) {
      using P = __attribute__((address_space(3))) s16x4_t *;
      s16x4_t part[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = half * 32 + g * 8 + h * 4 + (i >> 2);
        part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<P>(lds_address(lds) + k * (ROWS * 2) + (((row >> 4) ^ granule_swizzle(k)) << 5) + (i & 3) * 8));
      }
      return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const s16x8_t *>(lds + (row + i) * (KS * kElem) + (KS * kElem == 128 ? ((half * 4 + g) ^ (i >> 1)) << 4 : (g ^ (i >> 2)) << 4));
    }
  }
};

// Products of float operands are summed 256 at a time (fewer in the kernels for few rows), and those sums added up, so that a long sum's roundings
// stay small: 4096 products leave 3.0e-7 of a result's norm, in one run 1.2e-6, 65536 4.1e-7 and 4.6e-6; for 1 % of the time.  Tiles of bfloat16 are
// summed in one run: an instruction adds 32 of them at once, and 65536 leave 8.2e-7 in a float result.
template <int FM, int FN>
struct RunOfSums {
  f32x4_t sum[FM][FN];
  int steps = 0;
  __device__ __forceinline__ RunOfSums() {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) sum[f][h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // Behind `more` columns' products.
  __device__ __forceinline__ void behind(f32x4_t (&acc)[FM][FN], int more) {
    if ((steps += more) < 256) return;
    steps = 0;
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) {
        sum[f][h] += acc[f][h];
        acc[f][h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      }
  }
  __device__ __forceinline__ void end(f32x4_t (&acc)[FM][FN]) const {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[f][h] += sum[f][h];
  }
};

// The product of a tile of BM x BN by WM x WN wavefronts.  acc[f][h][r] of lane (i, g): row 16 f + i, column 16 h + 4 g + r of the
// wavefront's part.
// STEPS: how many steps of KS columns are in LDS or on their way there.  8192 x 8192 x 2048, 256 x 256 tiles, k-major operands: two steps of 64
// 250 us, four of 32 266; i-major ones 280 and 268.
template <typename Type, int BM, int BN, int WM, int WN, bool A_IMAJOR, bool B_IMAJOR, bool WHOLE16, int STEPS = 2, int KS = Type::kStep>
struct TileProduct {
  static constexpr int kThreads = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
  using Elem = typename Type::Elem;
  using A = OperandTile<Elem, BM, A_IMAJOR, WHOLE16, kThreads, KS>;
  using B = OperandTile<Elem, BN, B_IMAJOR, WHOLE16, kThreads, KS>;
  static constexpr int kPart = A::kBytes + B::kBytes, kLds = STEPS * kPart;
  static_assert(STEPS >= 2 && (WHOLE16 || STEPS == 2) && (sizeof(Elem) == 2 || FM == 2), "");
  f32x4_t acc[FM][FN];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[f][h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // The operands of 32 columns: all of b, and half of a's rows.
  static constexpr int FH = FM / 2;
  static_assert(FM % 2 == 0, "two halves of rows");
  static __device__ __forceinline__ void read_a(s16x8_t (&v)[FH], const char *part, int kk, int upper, int row, int lane) {
#pragma unroll
    for (int f = 0; f < FH; ++f) v[f] = A::fragment(part, row + 16 * (upper * FH + f), kk, lane);
  }
  static __device__ __forceinline__ void read_b(s16x8_t (&v)[FN], const char *part, int kk, int col, int lane) {
#pragma unroll
    for (int h = 0; h < FN; ++h) v[h] = B::fragment(part + A::kBytes, col + 16 * h, kk, lane);
  }
  template <int UPPER>
  __device__ __forceinline__ void multiply(const s16x8_t (&a)[FH], const s16x8_t (&b)[FN]) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int f = 0; f < FH; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[UPPER * FH + f][h] = Type::mfma(b[h], a[f], acc[UPPER * FH + f][h]);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  }
  // The same for large tiles, where a wavefront's reads and loads, asked for at once, would hold up its products while the others' go first: a quarter
  // of them, between(f), behind each row of products.  256 x 256, 16 x 2048 rows of 2048 to 4096 columns: 494 -> 474 us, 1160 TFLOP/s; 65536 rows of
  // 128 experts, 1536 x 2048: 478 -> 450.  i-major operands are read ahead all the same (32768 rows, 32 of 5760 x 2880, transposed: 1095 us, between the
  // products 1120), and shorter runs
  // have no room for it (8 of 1024 x 4096 orthogonalised, mostly by 128 x 128: 795 us, with it 835).
  static constexpr bool kLong = FH >= 4, kReadAhead = B_IMAJOR;
  template <int UPPER, typename Between>
  __device__ __forceinline__ void multiply(const s16x8_t (&a)[FH], const s16x8_t (&b)[FN], Between between) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < FH; ++f) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[UPPER * FH + f][h] = Type::mfma(b[h], a[f], acc[UPPER * FH + f][h]);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      between(f);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  static __device__ __forceinline__ void read_a(s16x8_t (&v)[FH], int f, const char *part, int kk, int upper, int row, int lane) {
    v[f] = A::fragment(part, row + 16 * (upper * FH + f), kk, lane);
  }
  static __device__ __forceinline__ void read_b(s16x8_t (&v)[FN], int f, const char *part, int kk, int col, int lane) {
#pragma unroll
    for (int h = 0; h < FN; ++h) if (h * FH / FN == f) v[h] = B::fragment(part + A::kBytes, col + 16 * h, kk, lane);
  }
  // a, b: the tile's first elements; K columns; rows and columns of the tile that exist.  Every thread of the workgroup calls it.
  __device__ __forceinline__ void run(char *lds, const Elem *a, int64_t lda, int a_rows, const Elem *b, int64_t ldb, int b_rows, int64_t K) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = wave / WN * (BM / WM), col = wave % WN * (BN / WN);
    const uint32_t base = lds_address(lds);
    clear();
    if (K <= 0) return;
    A ta;
    B tb;
    ta.begin(a, lda, a_rows, K, tid);
    tb.begin(b, ldb, b_rows, K, tid);
    const auto issue = [&](int part, int64_t k) {                  // the step that has k columns left
      const int left = int(k < KS ? (k > 0 ? k : 0) : int64_t(KS));
      ta.issue(base + part, left, tid);
      tb.issue(base + part + A::kBytes, left, tid);
    };
    s16x8_t a0[FH], a1[FH], b0[FN], b1[FN];
    if constexpr (WHOLE16 && FM == 2) {
      // Small tiles, whose runs would be too short to cover a read: all that the next step needs is read while a step is multiplied.  Steps
      // behind the last are asked for and read too, as zeros.
#pragma unroll
      for (int i = 0; i < STEPS; ++i) issue(i * kPart, K - i * KS);
      s16x8_t va[2][2][FM], vb[2][2][FN];
      const auto read = [&](s16x8_t (&x)[2][FM], s16x8_t (&y)[2][FN], int part) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
          for (int h = 0; h < FN; ++h) y[kk][h] = B::fragment(lds + part + A::kBytes, col + 16 * h, kk, lane);
#pragma unroll
          for (int f = 0; f < FM; ++f) x[kk][f] = A::fragment(lds + part, row + 16 * f, kk, lane);
        }
      };
      lds_loads_done<(STEPS - 1) * (A::kEach + B::kEach)>();
      __syncthreads();
      read(va[0], vb[0], 0);
      int now = 0;
      RunOfSums<FM, FN> sums;
      for (int64_t k = K; k > 0; k -= 2 * KS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          lds_loads_done<(STEPS - 2) * (A::kEach + B::kEach)>();
          __syncthreads();                       // the next step is there, and this one has been read by all
          const int next = now + kPart == kLds ? 0 : now + kPart;
          read(va[i ^ 1], vb[i ^ 1], next);
          issue(now, k - (STEPS + i) * KS);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int f = 0; f < FM; ++f)
#pragma unroll
              for (int h = 0; h < FN; ++h) acc[f][h] = Type::mfma(vb[i][kk][h], va[i][kk][f], acc[f][h]);
          __builtin_amdgcn_sched_barrier(0);
          now = next;
        }
        if constexpr (sizeof(Elem) == 4) sums.behind(acc, 2 * KS);
      }
      if constexpr (sizeof(Elem) == 4) sums.end(acc);
      lds_loads_done<0>();                       // nothing may arrive once the workgroup has given its LDS back
    } else if constexpr (WHOLE16 && KS * sizeof(Elem) == 64) {
      // As below, with two runs a step.
#pragma unroll
      for (int i = 0; i < STEPS; ++i) issue(i * kPart, K - i * KS);
      lds_loads_done<(STEPS - 1) * (A::kEach + B::kEach)>();
      __syncthreads();
      read_b(b0, lds, 0, col, lane);
      read_a(a0, lds, 0, 0, row, lane);
      int now = 0;
      const auto step = [&](int64_t k, const s16x8_t (&b)[FN], s16x8_t (&b_next)[FN]) {
        read_a(a1, lds + now, 0, 1, row, lane);
        multiply<0>(a0, b);
        lds_loads_done<(STEPS - 2) * (A::kEach + B::kEach)>();
        __syncthreads();
        const int next = now + kPart == kLds ? 0 : now + kPart;
        read_b(b_next, lds + next, 0, col, lane);
        read_a(a0, lds + next, 0, 0, row, lane);
        multiply<1>(a1, b);
        issue(now, k - STEPS * KS);
        now = next;
      };
      for (int64_t k = K; k > 0; k -= 2 * KS) {
        step(k, b0, b1);
        step(k - KS, b1, b0);
      }
      lds_loads_done<0>();                       // nothing may arrive once the workgroup has given its LDS back
    } else if constexpr (WHOLE16) {
      // Large tiles: each step is four runs of products; what the next run needs is read while one goes on.  Before the last run all of a step has
      // been read, and its part of LDS gets the step that is STEPS further on.  Steps behind the last are asked for and read too, as zeros,
      // so that the loop has no branches.
#pragma unroll
      for (int i = 0; i < STEPS; ++i) issue(i * kPart, K - i * KS);
      lds_loads_done<(STEPS - 1) * (A::kEach + B::kEach)>();
      __syncthreads();
      read_b(b0, lds, 0, col, lane);
      read_a(a0, lds, 0, 0, row, lane);
      int now = 0;
      for (int64_t k = K; k > 0; k -= KS) {
        const int next = now + kPart == kLds ? 0 : now + kPart;
        const char *part = lds + now, *following = lds + next;
        const auto there = [] {
          lds_loads_done<(STEPS - 2) * (A::kEach + B::kEach)>();
          __syncthreads();
        };
        if constexpr (kLong) {
          multiply<0>(a0, b0, [&](int f) { read_a(a1, f, part, 0, 1, row, lane); });
          if constexpr (kReadAhead) read_b(b1, part, 1, col, lane);
          multiply<1>(a1, b0, [&](int f) {
            if constexpr (!kReadAhead) read_b(b1, f, part, 1, col, lane);
            read_a(a0, f, part, 1, 0, row, lane);
          });
          multiply<0>(a0, b1, [&](int f) { read_a(a1, f, part, 1, 1, row, lane); });
          there();
          if constexpr (kReadAhead) read_b(b0, following, 0, col, lane);
          const int64_t ahead = k - STEPS * KS;
          const int left = int(ahead < KS ? (ahead > 0 ? ahead : 0) : int64_t(KS));
          ta.limit(left);
          tb.limit(left);
          multiply<1>(a1, b1, [&](int f) {
            if constexpr (!kReadAhead) read_b(b0, f, following, 0, col, lane);
            read_a(a0, f, following, 0, 0, row, lane);
            constexpr int kAll = A::kEach + B::kEach;
#pragma unroll
            for (int j = 0; j < kAll; ++j) {
              if (j * FH / kAll != f) continue;
              if (j < A::kEach) ta.template issue_chunks<1>(base + now, j, left, tid);
              else tb.template issue_chunks<1>(base + now + A::kBytes, j - A::kEach, left, tid);
            }
          });
          ta.advance();
          tb.advance();
        } else {
          read_a(a1, part, 0, 1, row, lane);
          multiply<0>(a0, b0);
          read_b(b1, part, 1, col, lane);
          read_a(a0, part, 1, 0, row, lane);
          multiply<1>(a1, b0);
          read_a(a1, part, 1, 1, row, lane);
          multiply<0>(a0, b1);
          there();
          read_b(b0, following, 0, col, lane);
          read_a(a0, following, 0, 0, row, lane);
          multiply<1>(a1, b1);
          issue(now, k - STEPS * KS);
        }
        now = next;
      }
      lds_loads_done<0>();                       // nothing may arrive once the workgroup has given its LDS back
    } else {
      issue(0, K);
      int now = 0;
      for (int64_t k = K; k > 0; k -= KS, now ^= kPart) {
        ta.land(lds + now, tid);
        tb.land(lds + now + A::kBytes, tid);
        __syncthreads();                         // one a step: what is written next is the half that was read before the last one
        issue(now ^ kPart, k - KS);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          read_b(b0, lds + now, kk, col, lane);
          read_a(a0, lds + now, kk, 0, row, lane);
          read_a(a1, lds + now, kk, 1, row, lane);
          multiply<0>(a0, b0);
          multiply<1>(a1, b0);
        }
      }
    }
  }
};

// A wavefront's part of a 16-bit result in LDS, row by row, so that it leaves in rows of 16 bytes a lane instead of 8 bytes of 16 rows.
// The 16-byte chunk c of row r lies at place c ^ (r / 2 % chunks).  This way out has what bank conflicts there are: 1024 cycles a tile of 256 x 256,
// 347 of 128 x 128, whatever its sums' length (1 % of LDS cycles at 5760 columns, 11 % at 512).
template <int ROWS, int COLS>
struct ResultTile {
  static constexpr int kAcross = COLS / 8, kBytes = ROWS * COLS * 2, kEach = ROWS * kAcross / 64;
  static __device__ __forceinline__ int place(int row, int chunk) { return row * (COLS * 2) + ((chunk ^ (row >> 1 & (kAcross - 1))) << 4); }
  // Four columns from 16 h + 4 g on of row 16 f + i, as two words, from lane (i, g).
  static __device__ __forceinline__ void put(char *lds, int f, int h, uint2 v, int lane) {
    const int row = 16 * f + (lane & 15), col = 16 * h + 4 * (lane >> 4);
    *reinterpret_cast<uint2 *>(lds + place(row, col >> 3) + (col & 4) * 2) = v;
  }
  // What is put, or will be, at the same place.
  static __device__ __forceinline__ uint2 get(const char *lds, int f, int h, int lane) {
    const int row = 16 * f + (lane & 15), col = 16 * h + 4 * (lane >> 4);
    return *reinterpret_cast<const uint2 *>(lds + place(row, col >> 3) + (col & 4) * 2);
  }
  static __device__ __forceinline__ void set(char *lds, int row, int c, uint4 v) { *reinterpret_cast<uint4 *>(lds + place(row, c)) = v; }
  static __device__ __forceinline__ uint4 chunk(const char *lds, int row, int c) { return *reinterpret_cast<const uint4 *>(lds + place(row, c)); }
  // Eight rows from `row` on (a multiple of 8) of column `col` + lane % 16 (col a multiple of 16; row the same for 16 lanes).
  static __device__ __forceinline__ uint4 column(const char *lds, int row, int col, int lane) {
    using P = __attribute__((address_space(3))) s16x4_t *;
    const int j = lane & 15, c = col + 4 * (j & 3);
    uint2 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<P>(lds_address(lds) + place(row + 4 * h + (j >> 2), c >> 3) + (c & 4) * 2)));
    return uint4{v[0].x, v[0].y, v[1].x, v[1].y};
  }
};

// Sixteen bytes past the caches, to an address that has an element's alignment.
__device__ __forceinline__ void store_past(void *p, uint4 v) {
  typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(Words{v.x, v.y, v.z, v.w}, static_cast<Words *>(p));
}

// Up to eight 16-bit values at p, of which n exist.
__device__ __forceinline__ void store8(uint16_t *p, uint4 v, int n) {
  if (n >= 8) {
    __builtin_memcpy(p, &v, 16);
  } else {
    uint16_t e[8];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < 7; ++i) if (i < n) p[i] = e[i];
  }
}

// Four values of one row of a result, of which the first n exist.
__device__ __forceinline__ void store4(float *p, f32x4_t v, int n) {
  if (n >= 4) {
    __builtin_memcpy(p, &v, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < n) p[i] = v[i];
  }
}

}  // namespace moe_spec
