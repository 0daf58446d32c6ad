// Updates of matrices by the orthogonal factor of their momentum (Muon), many matrices in a few launches.
//   X_0 = U / |U|_F (turned so that it has at most as many rows as columns), then as often as asked
//   A = X X^T,  B = a I + b A + c A A,  X <- B X
// The iteration runs on the matrix cores with X, A and B in float16 and sums in float: with the usual coefficients |X| stays below 1.3 and every
// value of A and B below 15, so float16's range is enough (others are looked at before a call begins, iterates_within()).  The three are held 64-fold,
// so that the smallest values that count stay above float16's denormal ones.  Matrices that one workgroup takes have no float16 in them.
// Eleven bits do for A and B, and for the X that they are made of and that b A + c A A multiplies: roundings stay what they are beside the
// large values that they belong to, and A has next to nothing for small ones.  But a X brings small singular values up by a each time, and roundings of
// large ones with them: of a gradient that has two directions over noise of a hundredth five iterations would leave 3 %, ten of singular values
// 1 / i^2 23 %.  So what rounding takes from X is kept, 11 more bits, and a times it added to X' in the first iterations (rests()): 0.05 to 0.2 % whatever the
// spectrum.  For 48 matrices of 768 x 2048 that is 160 us of 2020, 8 of 1024 x 4096 35 of 845, one of 256 x 256 3 of 82: 2 bytes a value
// left by the launch that brings X, taken up and left by B X (165 us; 193 with it, 168 where it is only taken up).
// Three products an iteration, each one launch over all matrices of a call; a matrix that the framework holds upright is laid on its side
// on the way in and stood up on the way out.
#include <math.h>

#include "mfma_tiles.h"

namespace moe_spec {
namespace {

constexpr int kMuonBlock = 256, kPerMuonLaunch = 24, kSliceValues = 4096, kTurn = 64;
constexpr float kHeld = 64.0f;

// A stack of matrices of one size.
struct MuonStack {
  uint16_t *x[2], *a, *b;        // workspace: iterates [count, m, ld_n], A and B [count, m, ld_m]
  uint16_t *rest;                // and what rounding took from the iterate, as it, kRest-fold
  double *partial;               // [count, slices] sums of squares
  float *p;
  const void *grad;
  float *momentum;
  void *out;                     // bf16 copy of p, or what orthogonalise returns
  int64_t grad_stride, grad_matrix, out_stride, out_matrix;
  int64_t count;
  int rows, cols, m, n, ld_m, ld_n, slices, slice_rows;
};
// Settings of a call, and the stacks of a launch: up to N of them.  One stack by itself needs no search and has a dependent read of the
// argument block fewer, up to four have a short one: up to 0.9 us a launch (17 launches; one matrix of 256 x 256: 94 -> 78 us, three: 162 -> 154).
struct MuonSettings {
  float mu, decay, rate, scale, ca, cb, cc;
  const float *scale_dev;
  uint32_t total;                        // workgroups that have a tile
  int nesterov, which;
  int rests;                             // whether X_0 leaves its rests
};
template <int N>
struct MuonArgs : MuonSettings {
  MuonStack t[N];
  uint32_t first[N];                     // a stack's first workgroup
};
static_assert(sizeof(MuonArgs<kPerMuonLaunch>) <= 4096, "an argument block");

template <int N>
__device__ __forceinline__ int stack_of(const uint32_t (&first)[N], uint32_t workgroup) {
  if constexpr (N == 1) return 0;
  int which = -1;
#pragma unroll
  for (int i = 0; i < N; ++i) which += first[i] <= workgroup;
  return which;
}

// The gradient and the momentum of a chunk of eight values, where there is one.
template <typename GT>
struct Chunk {
  Run<GT, 8> g;
  Run<float, 8> m;
  int row, col, n;                       // n: how many exist (at most eight count), none or less: no chunk
  __device__ __forceinline__ int64_t at(const MuonStack &t, int64_t matrix) const { return (matrix * t.rows + row) * t.cols + col; }
  __device__ __forceinline__ void load(const MuonStack &t, int64_t matrix) {
    if (n <= 0) return;
    g.load(static_cast<const GT *>(t.grad) + matrix * t.grad_matrix + row * t.grad_stride + col, n);
    if (t.momentum) m.load(t.momentum + at(t, matrix), n);
  }
  // What is orthogonalised: the gradient, or the momentum (which is up to date) with the gradient in it.
  __device__ __forceinline__ void direction(const MuonSettings &a, const MuonStack &t, float scale, float (&u)[8]) const {
#pragma clang fp contract(off)
    g.get(u);
    if (!t.momentum) return;
    float v[8];
    m.get(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = a.nesterov ? u[j] * scale + v[j] * a.mu : v[j];
  }
};

// A workgroup's part of a matrix that is gone through as it lies: whole rows, kAhead chunks a thread at a time.  Parts of 4096 values in two rounds of
// loads at once stream at 4.4 (momentum) and 4.8 TB/s (X_0) over 75 M values and start small matrices on more compute units; parts of
// 16384 at 4.0 and 4.7, with one chunk at a time 4.7 and 4.5.
constexpr int kAhead = 2;
struct Slice {
  int64_t matrix;
  int row0, chunks, across;
  __device__ __forceinline__ Slice(const MuonStack &t, uint32_t at) {
    matrix = at / uint32_t(t.slices);
    const int slice = at % uint32_t(t.slices);
    across = (t.cols + 7) / 8;
    row0 = slice * t.slice_rows;
    chunks = min(t.slice_rows, t.rows - row0) * across;
  }
  template <typename C>
  __device__ __forceinline__ void place(C &c, int i, int cols) const {
    const int r = i / across;
    c.row = row0 + r;
    c.col = (i - r * across) * 8;
    c.n = i < chunks ? cols - c.col : 0;
  }
};

// Momentum and sums of squares, a slice of a matrix's rows a workgroup.
template <typename GT, int N>
__global__ __launch_bounds__(kMuonBlock) void muon_begin_kernel(const MuonArgs<N> a) {
#pragma clang fp contract(off)
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const uint32_t at = blockIdx.x - a.first[which];
  const Slice slice(t, at);
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  double sum = 0.0;
  for (int i = threadIdx.x; i < slice.chunks; i += kAhead * kMuonBlock) {
    Chunk<GT> c[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      slice.place(c[q], i + q * kMuonBlock, t.cols);
      c[q].load(t, slice.matrix);
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (c[q].n <= 0) continue;
      float u[8];
      c[q].g.get(u);
      if (t.momentum) {
        float m[8];
        c[q].m.get(m);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float g = u[j] * scale;
          m[j] = m[j] * a.mu + g;
          u[j] = a.nesterov ? g + m[j] * a.mu : m[j];
        }
        store_run<float, 8>(t.momentum + c[q].at(t, slice.matrix), m, c[q].n);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) if (j < c[q].n) sum += double(u[j]) * double(u[j]);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  __shared__ double part[kMuonBlock / 64];
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) t.partial[at] = (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ __forceinline__ uint16_t to_f16(float v) { return __builtin_bit_cast(uint16_t, _Float16(v)); }
__device__ __forceinline__ float from_f16(uint16_t v) { return float(__builtin_bit_cast(_Float16, v)); }
// What rounding v to float16, h, takes from it, at most half a step: kRest-fold it is as large as v at most.
constexpr float kRest = 2048.0f;
__device__ __forceinline__ uint16_t rest_of(float v, uint16_t h) { return to_f16((v - from_f16(h)) * kRest); }

// What makes X_0, or 64 X_0, of a matrix's values: they are taken times 2^shift, which alone could leave float's range where they are tiny, and then
// times factor: zero where the matrix has only zeros, NaN where it holds what is not finite.
struct Normaliser {
  float factor;
  int shift;
  __device__ __forceinline__ float scaled(float u) const { return factor > 0.0f ? ldexpf(u, shift) * factor : factor == 0.0f ? 0.0f : NAN; }
};
// From a matrix's sum of squares.
__device__ __forceinline__ Normaliser normaliser(double sum, float held) {
  if (!(sum < double(INFINITY))) return {NAN, 0};
  if (!(sum > 0.0)) return {0.0f, 0};
  int exponent;
  const double part = frexp(sqrt(sum), &exponent);
  return {float(double(held) / part), -exponent};
}
__device__ __forceinline__ Normaliser normaliser(const MuonStack &t, int64_t matrix) {
  const int lane = threadIdx.x & 63;
  double sum = 0.0;
  for (int i = lane; i < t.slices; i += 64) sum += t.partial[matrix * t.slices + i];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  return normaliser(sum, kHeld);
}

// X_0 as float16.  A matrix that is not upright as it lies; an upright one is laid on its side, tiles of 64 x 64 through LDS, whose columns are read
// value by value: two thirds of the LDS cycles are bank conflicts, behind a memory that is at 5.2 TB/s meanwhile.
struct Turn {
  int64_t matrix;
  int row0, col0;
  __device__ __forceinline__ Turn(const MuonStack &t, uint32_t at) {
    const uint32_t across = (t.cols + kTurn - 1) / kTurn, down = (t.rows + kTurn - 1) / kTurn;
    matrix = at / (across * down);
    const int q = at % (across * down);
    row0 = q / int(across) * kTurn;
    col0 = q % int(across) * kTurn;
  }
};

template <typename GT, int N>
__global__ __launch_bounds__(kMuonBlock) void muon_normalise_kernel(const MuonArgs<N> a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTurn][kTurn + 8], rests[kTurn][kTurn + 8];
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const uint32_t at = blockIdx.x - a.first[which];
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  // eight values of X and their rests, zeros behind a row's last
  struct Held { uint4 x, rest; };
  const auto held = [&](const Normaliser &normal, const Chunk<GT> &c) {
    uint16_t e[8], r[8];
    float u[8];
    if (c.n > 0) c.direction(a, t, scale, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = j < c.n ? normal.scaled(u[j]) : 0.0f;
      e[j] = to_f16(v);
      r[j] = rest_of(v, e[j]);
    }
    Held v;
    __builtin_memcpy(&v.x, e, 16);
    __builtin_memcpy(&v.rest, r, 16);
    return v;
  };
  if (t.rows <= t.cols) {
    const Slice slice(t, at);
    const Normaliser normal = normaliser(t, slice.matrix);
    const int64_t begin = slice.matrix * t.m * t.ld_n;
    for (int i = threadIdx.x; i < slice.chunks; i += kAhead * kMuonBlock) {
      Chunk<GT> c[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        slice.place(c[q], i + q * kMuonBlock, t.cols);
        c[q].load(t, slice.matrix);
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (c[q].n <= 0) continue;
        const Held v = held(normal, c[q]);
        const int64_t to = begin + int64_t(c[q].row) * t.ld_n + c[q].col;
        *reinterpret_cast<uint4 *>(t.x[0] + to) = v.x;
        if (a.rests) *reinterpret_cast<uint4 *>(t.rest + to) = v.rest;
      }
    }
    return;
  }
  const Turn turn(t, at);
  const Normaliser normal = normaliser(t, turn.matrix);
  const int64_t begin = turn.matrix * t.m * t.ld_n;
  Chunk<GT> c[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int i = threadIdx.x + q * kMuonBlock;
    c[q].row = turn.row0 + i / (kTurn / 8);
    c[q].col = turn.col0 + i % (kTurn / 8) * 8;
    c[q].n = c[q].row < t.rows ? t.cols - c[q].col : 0;
    c[q].load(t, turn.matrix);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const Held v = held(normal, c[q]);
    const int r = c[q].row - turn.row0, across = c[q].col - turn.col0;
    *reinterpret_cast<uint4 *>(&tile[r][across]) = v.x;
    *reinterpret_cast<uint4 *>(&rests[r][across]) = v.rest;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int i = threadIdx.x + q * kMuonBlock, across = i / (kTurn / 8), r = i % (kTurn / 8) * 8;      // a column of the matrix is a row of X
    if (turn.col0 + across >= t.cols || turn.row0 + r >= t.ld_n) continue;
    uint16_t e[8];
    const int64_t to = begin + int64_t(turn.col0 + across) * t.ld_n + turn.row0 + r;
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = tile[r + j][across];
    __builtin_memcpy(t.x[0] + to, e, 16);
    if (!a.rests) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = rests[r + j][across];
    __builtin_memcpy(t.rest + to, e, 16);
  }
}

// The result of eight values: p <- p decay - rate o and its copy, or o itself.
struct Result {
  Run<float, 8> p;
  uint4 x;
  int row, col, n;
  __device__ __forceinline__ int64_t at(const MuonStack &t, int64_t matrix) const { return (matrix * t.rows + row) * t.cols + col; }
  __device__ __forceinline__ void load(const MuonStack &t, int64_t matrix) {
    if (n > 0 && t.p) p.load(t.p + at(t, matrix), n);
  }
  __device__ __forceinline__ void store(const MuonSettings &a, const MuonStack &t, int64_t matrix) const {
    uint16_t e[8];
    __builtin_memcpy(e, &x, 16);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = from_f16(e[j]) * (1.0f / kHeld);
    store(a, t, matrix, v);
  }
  __device__ __forceinline__ void store(const MuonSettings &a, const MuonStack &t, int64_t matrix, float (&v)[8]) const {
#pragma clang fp contract(off)
    if (n <= 0) return;
    if (t.p) {
      float old[8];
      p.get(old);
      const float rate = a.rate * sqrtf(float(t.n));
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = old[j] * a.decay - v[j] * rate;
      store_run<float, 8>(t.p + at(t, matrix), v, n);
    }
    if (t.out) store_run<uint16_t, 8>(static_cast<uint16_t *>(t.out) + matrix * t.out_matrix + row * t.out_stride + col, v, n);
  }
};

// One product for every matrix.  SQUARE: A = X X^T; POLYNOMIAL: B = a I + b A + c A A; APPLY: X' = B X; RESULT: the last of those,
// which goes to the parameters and copies instead; APPLY_TAKE and APPLY_PASS: B X and a times the rests of X, the second with rests of its own, in the
// place of those that it took up.  A and B are symmetric: of them only tiles on and below the diagonal are worked out, and written
// to both places.
enum MuonProduct { SQUARE, POLYNOMIAL, APPLY, RESULT, APPLY_TAKE, APPLY_PASS };

template <int TILE, int WM, int WN, int STEPS, MuonProduct KIND, int N>
__global__ __launch_bounds__(WM *WN * 64) void muon_product_kernel(const MuonArgs<N> a) {
#pragma clang fp contract(off)                   // a matrix gets the same bits in every launch's company
  constexpr bool SYMMETRIC = KIND == SQUARE || KIND == POLYNOMIAL, TAKE = KIND == APPLY_TAKE || KIND == APPLY_PASS, PASS = KIND == APPLY_PASS;
  using P = TileProduct<F16, TILE, TILE, WM, WN, false, !SYMMETRIC, true, STEPS>;
  using R = ResultTile<TILE / WM, TILE / WN>;
  __shared__ __attribute__((aligned(16))) char lds[P::kLds];
  const uint32_t share = (a.total + 7) / 8, logical = blockIdx.x % 8 * share + blockIdx.x / 8;      // a die gets a run of tiles
  if (blockIdx.x / 8 >= share || logical >= a.total) return;
  const int which = stack_of(a.first, logical);
  const MuonStack &t = a.t[which];
  const int cols = SYMMETRIC ? t.m : t.n, down = (t.m + TILE - 1) / TILE, across = (cols + TILE - 1) / TILE;
  const uint32_t at = logical - a.first[which], per = SYMMETRIC ? down * (down + 1) / 2 : down * across;
  const int64_t matrix = at / per;
  const int tile = at % per;
  int tile_row = tile / across, tile_col = tile % across;
  if constexpr (SYMMETRIC) {
    tile_row = int((sqrtf(8.0f * tile + 1.0f) - 1.0f) * 0.5f);
    while (tile_row * (tile_row + 1) / 2 > tile) --tile_row;
    while ((tile_row + 1) * (tile_row + 2) / 2 <= tile) ++tile_row;
    tile_row = __builtin_amdgcn_readfirstlane(tile_row);
    tile_col = tile - tile_row * (tile_row + 1) / 2;
  }
  const int row0 = tile_row * TILE, col0 = tile_col * TILE;
  const uint16_t *x = t.x[a.which] + matrix * t.m * t.ld_n, *ta = t.a + matrix * t.m * t.ld_m, *tb = t.b + matrix * t.m * t.ld_m;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int wave_row = row0 + wave / WN * (TILE / WM), wave_col = col0 + wave % WN * (TILE / WN);
  P p;
  // A's own values, which B takes too: small tiles ask for them before their products (one matrix of 256 x 256: 69.5 -> 67.5 us on the device,
  // three of an estimator 155 -> 151)
  constexpr bool EARLY = KIND == POLYNOMIAL && P::FM == 2;
  const auto own = [&](int f, int h) {
    const int row = wave_row + 16 * f + i, col = wave_col + 16 * h + 4 * g;
    uint2 v{0, 0};
    if (row < t.m && col < t.ld_m) v = *reinterpret_cast<const uint2 *>(ta + int64_t(row) * t.ld_m + col);
    return v;
  };
  uint2 early[EARLY ? P::FM : 1][EARLY ? P::FN : 1];
  if constexpr (EARLY) {
#pragma unroll
    for (int f = 0; f < P::FM; ++f)
#pragma unroll
      for (int h = 0; h < P::FN; ++h) early[f][h] = own(f, h);
  }
  const int ld = SYMMETRIC ? t.ld_m : t.ld_n;
  const auto chunk_at = [&](int q) {             // offset of a lane's chunk of eight, negative: there is none
    const int row = wave_row + (q * 64 + lane) / R::kAcross, col = wave_col + (q * 64 + lane) % R::kAcross * 8;
    return row < t.m && col < ld ? int64_t(row) * ld + col : int64_t(-1);
  };
  // The iterate's rests, which a alone multiplies (see above), two fragments' rows at a time: the first before the products, others while those
  // before them are worked on.
  constexpr int kParts = P::FM / 2, kOfPart = R::kEach / kParts;
  uint16_t *const rests = t.rest + matrix * t.m * t.ld_n;
  uint4 rest[TAKE ? 2 : 1][kOfPart];
  const auto ask_rests = [&](int part) {
#pragma unroll
    for (int j = 0; j < kOfPart; ++j) {
      const int64_t from = chunk_at(part * kOfPart + j);
      rest[part & 1][j] = from < 0 ? uint4{0, 0, 0, 0} : *reinterpret_cast<const uint4 *>(rests + from);
    }
  };
  if constexpr (TAKE) ask_rests(0);
  const int rows = min(TILE, t.m - row0), some = min(TILE, cols - col0), K = KIND == SQUARE ? t.n : t.m;
  if constexpr (KIND == SQUARE) p.run(lds, x + int64_t(row0) * t.ld_n, t.ld_n, rows, x + int64_t(col0) * t.ld_n, t.ld_n, some, K);
  if constexpr (KIND == POLYNOMIAL) p.run(lds, ta + int64_t(row0) * t.ld_m, t.ld_m, rows, ta + int64_t(col0) * t.ld_m, t.ld_m, some, K);
  if constexpr (!SYMMETRIC) p.run(lds, tb + int64_t(row0) * t.ld_m, t.ld_m, rows, x + col0, t.ld_n, some, K);
  uint16_t *out = !SYMMETRIC ? t.x[a.which ^ 1] + matrix * t.m * t.ld_n : (KIND == SQUARE ? t.a : t.b) + matrix * t.m * t.ld_m;
  char *mine = lds + wave * R::kBytes;
  __syncthreads();                               // the operands have been read by all
  const auto leave = [&](uint16_t *to, int from, int until) {
#pragma unroll
    for (int q = from; q < until; ++q) {
      const int64_t at = chunk_at(q);
      if (at >= 0) *reinterpret_cast<uint4 *>(to + at) = R::chunk(mine, (q * 64 + lane) / R::kAcross, (q * 64 + lane) % R::kAcross);
    }
  };
  if constexpr (TAKE) {
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
#pragma unroll
      for (int j = 0; j < kOfPart; ++j) {
        const int q = part * kOfPart + j;
        R::set(mine, (q * 64 + lane) / R::kAcross, (q * 64 + lane) % R::kAcross, rest[part & 1][j]);
      }
      if (part + 1 < kParts) ask_rests(part + 1);
#pragma unroll
      for (int f = 2 * part; f < 2 * part + 2; ++f)
#pragma unroll
        for (int h = 0; h < P::FN; ++h) {        // a lane's values go where its rests were
          const uint2 of_x = R::get(mine, f, h, lane);
          uint16_t e[4];
          __builtin_memcpy(e, &of_x, 8);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = __builtin_fmaf(from_f16(e[r]), a.ca * (1.0f / kRest), p.acc[f][h][r] * (1.0f / kHeld));
            e[r] = to_f16(v);
            p.acc[f][h][r] = v - from_f16(e[r]);
          }
          uint2 w;
          __builtin_memcpy(&w, e, 8);
          R::put(mine, f, h, w, lane);
        }
      leave(out, part * kOfPart, (part + 1) * kOfPart);
      if constexpr (PASS) {
#pragma unroll
        for (int f = 2 * part; f < 2 * part + 2; ++f)
#pragma unroll
          for (int h = 0; h < P::FN; ++h) {
            uint16_t e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) e[r] = to_f16(p.acc[f][h][r] * kRest);
            uint2 w;
            __builtin_memcpy(&w, e, 8);
            R::put(mine, f, h, w, lane);
          }
        leave(rests, part * kOfPart, (part + 1) * kOfPart);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return;
  }
#pragma unroll
  for (int f = 0; f < P::FM; ++f) {
#pragma unroll
    for (int h = 0; h < P::FN; ++h) {
      const int row = wave_row + 16 * f + i, col = wave_col + 16 * h + 4 * g;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = p.acc[f][h][r] * (1.0f / kHeld);
      if constexpr (KIND == POLYNOMIAL) {
        const uint2 of_a = EARLY ? early[EARLY ? f : 0][EARLY ? h : 0] : own(f, h);
        uint16_t e[4];
        __builtin_memcpy(e, &of_a, 8);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = a.cb * from_f16(e[r]) + a.cc * v[r] + (col + r == row ? a.ca * kHeld : 0.0f);
      }
      uint16_t e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = col + r < cols && row < t.m ? to_f16(v[r]) : uint16_t(0);     // what fills up a row is zero
      uint2 w;
      __builtin_memcpy(&w, e, 8);
      R::put(mine, f, h, w, lane);
    }
  }
  if constexpr (KIND == RESULT) {
    // as many chunks at once as a lane has registers for
    constexpr int kGroup = R::kEach < 4 ? R::kEach : 4;
    const bool upright = t.rows > t.cols;        // a column of X is a row of the matrix
#pragma unroll
    for (int from = 0; from < R::kEach; from += kGroup) {
      Result result[kGroup];
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        const int q = from + j;
        constexpr int kDown = TILE / WM / 32;    // runs of 32 rows of X
        const int r = upright ? q % kDown * 32 + 8 * g : (q * 64 + lane) / R::kAcross;
        const int c = upright ? q / kDown * 16 : (q * 64 + lane) % R::kAcross * 8;
        result[j].row = upright ? wave_col + c + i : wave_row + r;
        result[j].col = upright ? wave_row + r : wave_col + c;
        result[j].n = result[j].row < t.rows ? t.cols - result[j].col : 0;
        result[j].load(t, matrix);
        result[j].x = upright ? R::column(mine, r, c, lane) : R::chunk(mine, r, c / 8);
      }
#pragma unroll
      for (int j = 0; j < kGroup; ++j) result[j].store(a, t, matrix);
    }
    return;
  }
  leave(out, 0, R::kEach);
  if constexpr (SYMMETRIC) {
    if (tile_row == tile_col) return;
#pragma unroll
    for (int r = 0; r < TILE / WM; r += 32)
#pragma unroll
      for (int c = 0; c < TILE / WN; c += 16) {
        const uint4 v = R::column(mine, r + 8 * g, c, lane);
        const int row = wave_col + c + i, col = wave_row + r + 8 * g;
        if (row < cols && col < ld) *reinterpret_cast<uint4 *>(out + int64_t(row) * ld + col) = v;
      }
  }
}

// ---- small matrices ----------------------------------------------------------------------------------------------
// All of a step for a matrix that fits into LDS, in one workgroup and in float throughout: momentum, norm, the iteration by 16x16x4
// instructions, result.  Up to 64 rows once it lies on its side.  X, A and B have rows of four times an odd number of floats, so that a fragment's
// sixteen rows of four columns lie in banks of their own; rows and columns that fill them up are zeros and stay so.  is_small()
// says which.
constexpr int kSmallBlock = 1024, kSmallWaves = kSmallBlock / 64, kSmallRows = 64, kSmallFloats = 24576;       // of X
constexpr int kSmallLd = 68, kSmallPartial = 16 * 256;
inline __host__ __device__ int small_ld(int n) { return (n + 3) / 8 * 8 + 4; }        // the next four times an odd number

template <typename GT, int N>
__global__ __launch_bounds__(kSmallBlock) void muon_small_kernel(const MuonArgs<N> a, int iterations) {
#pragma clang fp contract(off)
  __shared__ float x[kSmallFloats], sa[kSmallRows * kSmallLd], sb[kSmallRows * kSmallLd], part[kSmallPartial];
  __shared__ double sums[kSmallWaves];
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const int64_t matrix = blockIdx.x - a.first[which];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const int ld = small_ld(t.n), high = (t.m + 15) / 16, strips = (t.n + 15) / 16, across = (t.cols + 7) / 8, chunks = t.rows * across;
  const bool upright = t.rows > t.cols;
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  for (int q = tid; q < high * 16 * ld; q += kSmallBlock) x[q] = 0.0f;
  __syncthreads();
  double sum = 0.0;
  for (int q = tid; q < chunks; q += kSmallBlock) {
    Chunk<GT> c;
    c.row = q / across;
    c.col = (q - c.row * across) * 8;
    c.n = t.cols - c.col;
    c.load(t, matrix);
    float u[8];
    c.g.get(u);
    if (t.momentum) {
      float m[8];
      c.m.get(m);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = u[j] * scale;
        m[j] = m[j] * a.mu + v;
        u[j] = a.nesterov ? v + m[j] * a.mu : m[j];
      }
      store_run<float, 8>(t.momentum + c.at(t, matrix), m, c.n);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= c.n) continue;
      sum += double(u[j]) * double(u[j]);
      x[upright ? (c.col + j) * ld + c.row : c.row * ld + c.col + j] = u[j];
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) sum += sums[w];
  const Normaliser normal = normaliser(sum, 1.0f);
  for (int q = tid; q < high * 16 * ld; q += kSmallBlock) x[q] = normal.scaled(x[q]);
  __syncthreads();

  const int tiles = high * (high + 1) / 2, slices = kSmallWaves / tiles, steps = (t.n + 3) / 4, per = (steps + slices - 1) / slices;
  // tile number -> its row and column, on and below the diagonal
  const auto tile_row = [](int tile) { return tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3; };
  for (int it = 0; it < iterations; ++it) {
    if (wave < tiles * slices) {                 // A = X X^T, a slice of the columns a wavefront
      const int tile = wave % tiles, slice = wave / tiles, r = tile_row(tile), c = tile - r * (r + 1) / 2;
      f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
      const int from = slice * per, to = min(from + per, steps);
      const float *xr = x + (16 * r + i) * ld + g, *xc = x + (16 * c + i) * ld + g;
      for (int k = from; k < to; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(xr[4 * k], xc[4 * k], acc, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) part[(slice * tiles + tile) * 256 + (4 * g + q) * 16 + i] = acc[q];
    }
    __syncthreads();
    for (int q = tid; q < tiles * 256; q += kSmallBlock) {
      const int tile = q / 256, r = tile_row(tile), c = tile - r * (r + 1) / 2, row = 16 * r + q % 256 / 16, col = 16 * c + q % 16;
      float v = 0.0f;
      for (int s = 0; s < slices; ++s) v += part[s * tiles * 256 + q];
      sa[row * kSmallLd + col] = v;
      if (r != c) sa[col * kSmallLd + row] = v;
    }
    __syncthreads();
    for (int tile = wave; tile < tiles; tile += kSmallWaves) {        // B = a I + b A + c A A
      const int r = tile_row(tile), c = tile - r * (r + 1) / 2;
      f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
      const float *ar = sa + (16 * r + i) * kSmallLd + g, *ac = sa + (16 * c + i) * kSmallLd + g;
      for (int k = 0; k < 4 * high; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(ar[4 * k], ac[4 * k], acc, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 16 * r + 4 * g + q, col = 16 * c + i;
        const float v = a.cb * sa[row * kSmallLd + col] + a.cc * acc[q] + (row == col && row < t.m ? a.ca : 0.0f);
        sb[row * kSmallLd + col] = v;
        if (r != c) sb[col * kSmallLd + row] = v;
      }
    }
    __syncthreads();
    for (int strip = wave; strip < strips; strip += kSmallWaves) {    // X = B X, sixteen columns a wavefront, in place
      float v[16];
      const bool in = 16 * strip + i < ld;
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = k < 4 * high && in ? x[(4 * k + g) * ld + 16 * strip + i] : 0.0f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (r >= high) continue;
        f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < 4 * high) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(sb[(16 * r + i) * kSmallLd + 4 * k + g], v[k], acc, 0, 0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) if (in) x[(16 * r + 4 * g + q) * ld + 16 * strip + i] = acc[q];
      }
    }
    __syncthreads();
  }

  for (int q = tid; q < chunks; q += kSmallBlock) {
    Result r;
    r.row = q / across;
    r.col = (q - r.row * across) * 8;
    r.n = t.cols - r.col;
    r.load(t, matrix);
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = j < r.n ? x[upright ? (r.col + j) * ld + r.row : r.row * ld + r.col + j] : 0.0f;
    r.store(a, t, matrix, o);
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------
inline int round8(int n) { return (n + 7) / 8 * 8; }
inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Whether a matrix is one workgroup's: it fits into LDS, and its products (16 rows squared times columns) are few enough for one compute unit.  In
// microseconds, with one workgroup and with launches over many: 8 x 8 15 and 50, 16 x 1500 55 and 78, 32 x 700 55 and 66, 48 x 400 60 and 62,
// 64 x 192 53 and 56, 64 x 256 65 and 56.
inline bool is_small(const MuonStack &t) {
  const int high = (t.m + 15) / 16;
  return t.m <= kSmallRows && high * 16 * small_ld(t.n) <= kSmallFloats && high * high * t.n <= 3600;
}

// Sizes of a stack and the workspace that it takes.
size_t shape(MuonStack &t, int64_t count, int rows, int cols) {
  t.count = count;
  t.rows = rows;
  t.cols = cols;
  t.m = rows < cols ? rows : cols;
  t.n = rows < cols ? cols : rows;
  t.ld_m = round8(t.m);
  t.ld_n = round8(t.n);
  t.slice_rows = cols >= kSliceValues ? 1 : kSliceValues / cols;
  if (t.slice_rows > rows) t.slice_rows = rows;
  t.slices = (rows + t.slice_rows - 1) / t.slice_rows;
  if (is_small(t)) return 0;
  return 3 * round256(size_t(count) * t.m * t.ld_n * 2) + 2 * round256(size_t(count) * t.m * t.ld_m * 2) + round256(size_t(count) * t.slices * 8);
}
char *place(MuonStack &t, char *at) {
  const size_t x = round256(size_t(t.count) * t.m * t.ld_n * 2), a = round256(size_t(t.count) * t.m * t.ld_m * 2);
  t.x[0] = reinterpret_cast<uint16_t *>(at);
  t.x[1] = reinterpret_cast<uint16_t *>(at + x);
  t.rest = reinterpret_cast<uint16_t *>(at + 2 * x);
  t.a = reinterpret_cast<uint16_t *>(at + 3 * x);
  t.b = reinterpret_cast<uint16_t *>(at + 3 * x + a);
  t.partial = reinterpret_cast<double *>(at + 3 * x + 2 * a);
  return at + 3 * x + 2 * a + round256(size_t(t.count) * t.slices * 8);
}

const char *iteration_fault(const double *c, int iterations) {
  if (iterations < 1 || iterations > 64) return "iterations must be between 1 and 64";
  for (int i = 0; i < 3; ++i) if (!(fabs(c[i]) <= 16.0)) return "coefficients must lie between -16 and 16";
  return nullptr;
}

// Whether X, A and B stay within `most` for every matrix.  An iteration takes each singular value s to s q(s^2), q(t) = a + b t + c t^2, of which it
// makes A's eigenvalues s^2 and B's q(s^2), and no value of a matrix is larger than its largest singular value.  They begin in [0, 1] and after
// an iteration fill [0, top] with top the largest |s q(s^2)| there: at the end or where the slope a + 3 b t + 5 c t^2 is zero; q has its own at an
// end or at -b / 2c.  Roundings may take top further, by `slack` of it each time.
bool iterates_within(double most, double slack, const double *coefficients, int iterations) {
  const double a = coefficients[0], b = coefficients[1], c = coefficients[2];
  const auto q = [=](double t) { return fabs(a + t * (b + t * c)); };
  double flat[2] = {-1.0, -1.0};                         // t where the slope is zero, negative: none
  if (const double d = 9.0 * b * b - 20.0 * a * c; d >= 0.0) {
    const double r = -0.5 * (3.0 * b + copysign(sqrt(d), b));
    if (c != 0.0) flat[0] = r / (5.0 * c);
    if (r != 0.0) flat[1] = a / r;
  }
  double top = 1.0;
  for (int i = 0; i < iterations; ++i) {
    top *= 1.0 + slack;
    const double end = top * top;
    double largest = fmax(q(0.0), q(end)), next = top * q(end);
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < end) largest = fmax(largest, q(-b / (2.0 * c)));
    for (const double t : flat) if (t > 0.0 && t < end) next = fmax(next, sqrt(t) * q(t));
    if (!(end <= most && largest <= most && next <= most)) return false;
    top = next;
  }
  return true;
}
// 65504 is what float16 holds, and X, A and B are held 64-fold: 1023.  A 64th is 32 roundings of float16; those of a matrix, each
// another way, come to about 2 in any one direction.  Of a matrix of one workgroup A A in float has to stay in range, with 64 of float's roundings.
const char *range_fault(const MuonStack &t, const double *coefficients, int iterations) {
  if (is_small(t)) return iterates_within(double(int64_t(1) << 60), 64.0 / (1 << 24), coefficients, iterations) ? nullptr : "coefficients that take iterates out of float's range";
  return iterates_within(1000.0, 1.0 / 64, coefficients, iterations) ? nullptr : "coefficients that take iterates beyond 1000, which matrices of more than one workgroup cannot hold";
}

// Where each stack's workgroups begin in a launch, and how many there are.
template <int N, typename Count>
void firsts(MuonArgs<N> &a, int n, Count workgroups, unsigned &grid) {
  grid = 0;
  for (int i = 0; i < N; ++i) {
    a.first[i] = i < n ? grid : UINT32_MAX;
    if (i < n) grid += unsigned(workgroups(a.t[i]));
  }
}

inline int64_t tiles(int64_t n, int tile) { return (n + tile - 1) / tile; }
inline int64_t begin_blocks(const MuonStack &t) { return t.count * t.slices; }
// Of the launch that brings X.
inline int64_t turn_blocks(const MuonStack &t) {
  return t.rows <= t.cols ? begin_blocks(t) : t.count * tiles(t.rows, kTurn) * tiles(t.cols, kTurn);
}
inline int64_t square_blocks(const MuonStack &t, int tile) { return t.count * tiles(t.m, tile) * (tiles(t.m, tile) + 1) / 2; }
inline int64_t apply_blocks(const MuonStack &t, int tile) { return t.count * tiles(t.m, tile) * tiles(t.n, tile); }
// Most of them, of any launch over the stack.
inline int64_t most_blocks(const MuonStack &t) {
  if (is_small(t)) return t.count * (kSmallBlock / kMuonBlock);
  const int64_t b = begin_blocks(t), u = turn_blocks(t), p = apply_blocks(t, 64), s = square_blocks(t, 64);
  const int64_t x = b > u ? b : u, y = p > s ? p : s;
  return x > y ? x : y;
}
constexpr int64_t kMostMuonBlocks = (int64_t(1) << 32) / kMuonBlock - 1;

// One product over n stacks.  256 tiles of 256 x 256 are a round of what the compute units hold, and so are 512 of 128 x 128; they take about 1 : 0.62 of the
// time, and two rounds of 64 x 64, 1024 tiles, 0.6 (256 x 256 tiles reach 1050 TFLOP/s, 128 x 128 820, 64 x 64 420): the tile that is done first.  The last product,
// whose workgroups then read and write parameters, has two of them a compute unit, so that one's products cover another's traffic: 48 matrices of
// 768 x 2048 1791 us (before rests), with 256 x 256 tiles there 1810, with a launch for the parameters 1807 (one matrix of 256 x 256: 78 and 80).
template <MuonProduct KIND, int N>
hipError_t run_product(MuonArgs<N> &a, int n, hipStream_t s) {
  int tile = KIND == RESULT ? 128 : 256, best = tile;
  double least = INFINITY;
  const auto blocks = [&](const MuonStack &t) { return KIND == SQUARE || KIND == POLYNOMIAL ? square_blocks(t, tile) : apply_blocks(t, tile); };
  for (; tile >= 64; tile /= 2) {
    firsts(a, n, blocks, a.total);
    const double time = tile == 256 ? (a.total + 255) / 256 : tile == 128 ? 0.62 * ((a.total + 511) / 512) : 0.6 * ((a.total + 1023) / 1024);
    if (time < least) best = tile, least = time;
  }
  tile = best;
  firsts(a, n, blocks, a.total);
  const unsigned grid = (a.total + 7) / 8 * 8;
  if constexpr (KIND != RESULT)
    if (tile == 256) return launch(muon_product_kernel<256, 2, 4, 2, KIND, N>, grid, 512, s, a);
  if (tile == 128) return launch(muon_product_kernel<128, 2, 4, 2, KIND, N>, grid, 512, s, a);
  return launch(muon_product_kernel<64, 2, 2, 4, KIND, N>, grid, 256, s, a);
}

// Why a stack cannot be taken, or null.
const char *stack_fault(int64_t count, int64_t rows, int64_t cols) {
  if (count < 0 || rows < 0 || cols < 0) return "a negative size";
  if (rows > MOE_SPEC_TRAIN_MAX_FEATURES || cols > MOE_SPEC_TRAIN_MAX_FEATURES) return "more than 65536 rows or columns";
  if (count == 0 || rows == 0 || cols == 0) return nullptr;
  if (count > MOE_SPEC_MUON_MAX_ELEMENTS / (rows * cols)) return "more than 2^32 values";
  MuonStack t;
  shape(t, count, int(rows), int(cols));
  return most_blocks(t) > kMostMuonBlocks ? "more matrices than one launch can take" : nullptr;
}

// How many iterations take rests up: those after which what they save still grows, and not the last, whose launch has the parameters to move.  Five
// iterations of two directions over noise, of singular values 1 / i^2, and of a random matrix: with rests in 0 of them 2.9, 2.0 and 0.13 % off, 2 0.27, 0.34
// and 0.11, 3 0.12, 0.14 and 0.12, 4 0.07, 0.09 and 0.14.  Ten: 0 8, 23 and 0.24 %, 7 0.16, 0.12 and 0.31, 9 0.19, 0.14 and 0.33.
inline int rests(int iterations) { return iterations < 5 ? iterations - 1 : iterations < 9 ? iterations - 2 : 7; }

// All launches for up to N stacks; a's scalars are set.  Stops at the first that fails.
template <int N>
hipError_t run_launches(MuonArgs<N> &a, int n, int iterations, bool grad_bf16, hipStream_t s) {
  unsigned grid;
  hipError_t e;
  firsts(a, n, begin_blocks, grid);
  e = grad_bf16 ? launch(muon_begin_kernel<uint16_t, N>, grid, kMuonBlock, s, a) : launch(muon_begin_kernel<float, N>, grid, kMuonBlock, s, a);
  if (e != hipSuccess) return e;
  const int with_rest = rests(iterations);
  a.rests = with_rest > 0;
  firsts(a, n, turn_blocks, grid);
  e = grad_bf16 ? launch(muon_normalise_kernel<uint16_t, N>, grid, kMuonBlock, s, a) : launch(muon_normalise_kernel<float, N>, grid, kMuonBlock, s, a);
  for (int i = 0; i < iterations && e == hipSuccess; ++i) {
    a.which = i & 1;
    e = run_product<SQUARE>(a, n, s);
    if (e == hipSuccess) e = run_product<POLYNOMIAL>(a, n, s);
    if (e != hipSuccess) break;
    e = i + 1 < with_rest ? run_product<APPLY_PASS>(a, n, s) : i < with_rest ? run_product<APPLY_TAKE>(a, n, s)
        : i + 1 < iterations ? run_product<APPLY>(a, n, s) : run_product<RESULT>(a, n, s);
  }
  return e;
}

template <int N>
hipError_t run_small(const MuonArgs<kPerMuonLaunch> &a, int n, int iterations, bool grad_bf16, hipStream_t s) {
  MuonArgs<N> few{};
  static_cast<MuonSettings &>(few) = a;
  for (int i = 0; i < n; ++i) few.t[i] = a.t[i];
  unsigned grid;
  firsts(few, n, [](const MuonStack &t) { return t.count; }, grid);
  void *args[] = {&few, &iterations};
  const void *kernel = grad_bf16 ? reinterpret_cast<const void *>(muon_small_kernel<uint16_t, N>) : reinterpret_cast<const void *>(muon_small_kernel<float, N>);
  return hipLaunchKernel(kernel, dim3(grid), dim3(kSmallBlock), args, 0, s);
}

template <int N>
hipError_t run_few(const MuonArgs<kPerMuonLaunch> &a, int n, int iterations, bool grad_bf16, hipStream_t s) {
  MuonArgs<N> few{};
  static_cast<MuonSettings &>(few) = a;
  for (int i = 0; i < n; ++i) few.t[i] = a.t[i];
  return run_launches(few, n, iterations, grad_bf16, s);
}
hipError_t run_stacks(MuonArgs<kPerMuonLaunch> &a, int n, int iterations, bool grad_bf16, bool small, hipStream_t s) {
  if (small) return n == 1 ? run_small<1>(a, n, iterations, grad_bf16, s) : run_small<kPerMuonLaunch>(a, n, iterations, grad_bf16, s);
  if (n == 1) return run_few<1>(a, n, iterations, grad_bf16, s);
  if (n <= 4) return run_few<4>(a, n, iterations, grad_bf16, s);
  return run_launches(a, n, iterations, grad_bf16, s);
}

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" size_t moe_spec_muon_workspace_bytes(const moe_spec_muon_tensor *tensors, int n_tensors) {
  if (n_tensors < 1 || n_tensors > MOE_SPEC_TRAIN_MAX_TENSORS || !tensors) return 0;
  size_t need = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const moe_spec_muon_tensor &m = tensors[i];
    if (stack_fault(m.count, m.rows, m.cols)) return 0;
    MuonStack t;
    if (m.count && m.rows && m.cols) need += shape(t, m.count, m.rows, m.cols);
  }
  return need;
}

extern "C" int moe_spec_muon_step(void *stream, const moe_spec_muon_tensor *tensors, int n_tensors, const moe_spec_muon_config *cfg,
                                  void *workspace, size_t workspace_bytes) {
  if (!cfg) return train_fail(MOE_SPEC_EINVAL, "muon_step: cfg is null");
  if (n_tensors < 0 || n_tensors > MOE_SPEC_TRAIN_MAX_TENSORS) return train_fail(MOE_SPEC_EINVAL, "muon_step: a number of tensors out of range");
  if (n_tensors && !tensors) return train_fail(MOE_SPEC_EINVAL, "muon_step: tensors is null");
  if (!known_type(cfg->grad_dtype)) return train_fail(MOE_SPEC_EINVAL, "muon_step: unknown grad_dtype %d", cfg->grad_dtype);
  if (!(cfg->momentum >= 0.0 && cfg->momentum < 1.0)) return train_fail(MOE_SPEC_EINVAL, "muon_step: momentum must be at least 0 and below 1");
  if (!(cfg->lr == cfg->lr) || !(cfg->weight_decay >= 0.0) || !(cfg->update_rms >= 0.0))
    return train_fail(MOE_SPEC_EINVAL, "muon_step: weight_decay or update_rms is negative, or one of them or lr is no number");
  if (const char *why = iteration_fault(cfg->coefficients, cfg->iterations)) return train_fail(MOE_SPEC_EINVAL, "muon_step: %s", why);
  if (misaligned(cfg->grad_scale_dev, 4)) return train_fail(MOE_SPEC_EINVAL, "muon_step: grad_scale_dev is not aligned to its type");
  for (int i = 0; i < n_tensors; ++i) {
    const moe_spec_muon_tensor &m = tensors[i];
    if (const char *why = stack_fault(m.count, m.rows, m.cols)) return train_fail(MOE_SPEC_EINVAL, "muon_step: tensor %d has %s", i, why);
    if (m.count == 0 || m.rows == 0 || m.cols == 0) continue;
    if (!m.p || !m.grad || !m.m) return train_fail(MOE_SPEC_EINVAL, "muon_step: tensor %d has a null pointer", i);
    if (misaligned(m.p, 4) || misaligned(m.m, 4) || misaligned(m.grad, size_of(cfg->grad_dtype)) || misaligned(m.copy, 2))
      return train_fail(MOE_SPEC_EINVAL, "muon_step: tensor %d has a pointer that is not aligned to its type", i);
    if (m.copy_stride != 0 && (m.copy_stride < int64_t(m.rows) * m.cols || m.copy_stride > int64_t(1) << 40))
      return train_fail(MOE_SPEC_EINVAL, "muon_step: tensor %d has a copy_stride below a matrix or above 2^40", i);
  }
  bool any = false, seen[2] = {false, false};
  for (int i = 0; i < n_tensors; ++i) {
    const moe_spec_muon_tensor &m = tensors[i];
    if (m.count == 0 || m.rows == 0 || m.cols == 0) continue;
    any = true;
    MuonStack t;
    shape(t, m.count, m.rows, m.cols);
    if (seen[is_small(t)]) continue;                     // the same for all of a kind
    seen[is_small(t)] = true;
    if (const char *why = range_fault(t, cfg->coefficients, cfg->iterations)) return train_fail(MOE_SPEC_EINVAL, "muon_step: tensor %d: %s", i, why);
  }
  const size_t need = moe_spec_muon_workspace_bytes(tensors, n_tensors);
  if (need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need))
    return train_fail(MOE_SPEC_EINVAL, "muon_step: the workspace is null, not aligned to 16 bytes or smaller than %zu bytes", need);
  if (!any) return MOE_SPEC_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "muon_step: %s", hipGetErrorString(on.error()));
  MuonArgs<kPerMuonLaunch> a{};
  a.mu = float(cfg->momentum);
  a.decay = float(1.0 - cfg->lr * cfg->weight_decay);
  a.rate = float(cfg->lr * cfg->update_rms);
  a.scale = float(cfg->grad_scale);
  a.scale_dev = cfg->grad_scale_dev;
  a.ca = float(cfg->coefficients[0]);
  a.cb = float(cfg->coefficients[1]);
  a.cc = float(cfg->coefficients[2]);
  a.nesterov = cfg->nesterov != 0;
  const bool bf16 = cfg->grad_dtype == MOE_SPEC_BF16;
  char *at = static_cast<char *>(workspace);
  hipError_t e = hipSuccess;
  for (int small = 0; small < 2; ++small) {              // large matrices, then those that fit into a workgroup
    int n = 0;
    int64_t blocks = 0;
    for (int i = 0; i < n_tensors && e == hipSuccess; ++i) {
      const moe_spec_muon_tensor &m = tensors[i];
      if (m.count == 0 || m.rows == 0 || m.cols == 0) continue;
      MuonStack t{};
      shape(t, m.count, m.rows, m.cols);
      if (is_small(t) != bool(small)) continue;
      if (n == kPerMuonLaunch || (n && blocks + most_blocks(t) > kMostMuonBlocks)) {
        e = run_stacks(a, n, cfg->iterations, bf16, small, s);
        n = 0;
        blocks = 0;
      }
      if (!small) at = place(t, at);
      t.p = m.p;
      t.grad = m.grad;
      t.momentum = m.m;
      t.out = m.copy;
      t.grad_stride = t.out_stride = m.cols;
      t.grad_matrix = int64_t(m.rows) * m.cols;
      t.out_matrix = m.copy_stride ? m.copy_stride : t.grad_matrix;
      a.t[n++] = t;
      blocks += most_blocks(t);
    }
    if (e == hipSuccess && n) e = run_stacks(a, n, cfg->iterations, bf16, small, s);
  }
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "muon_step: %s", hipGetErrorString(e));
}

extern "C" size_t moe_spec_orthogonalise_workspace_bytes(int64_t count, int rows, int cols) {
  MuonStack t;
  if (stack_fault(count, rows, cols) || count == 0 || rows == 0 || cols == 0) return 0;
  return shape(t, count, rows, cols);
}

extern "C" int moe_spec_orthogonalise(void *stream, int dtype, const void *g, int64_t g_matrix_stride, int64_t g_stride, int64_t count, int rows,
                                      int cols, const double *coefficients, int iterations, void *out, int64_t out_matrix_stride,
                                      int64_t out_stride, void *workspace, size_t workspace_bytes) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: unknown dtype %d", dtype);
  if (const char *why = stack_fault(count, rows, cols)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: %s", why);
  if (!coefficients) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: coefficients is null");
  if (const char *why = iteration_fault(coefficients, iterations)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: %s", why);
  if (count == 0 || rows == 0 || cols == 0) return MOE_SPEC_OK;
  if (const char *why = matrix_fault(g, g_stride, rows, cols, size_of(dtype), false)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: g %s", why);
  if (const char *why = matrix_fault(out, out_stride, rows, cols, 2, true)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: out %s", why);
  if (rows == 1) g_stride = out_stride = cols;
  const int64_t most = int64_t(1) << 40;
  if (count > 1 && (g_matrix_stride < 0 || g_matrix_stride > most)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: g's matrix stride must be between 0 and 2^40");
  if (count > 1 && (out_matrix_stride < (rows - 1) * out_stride + cols || out_matrix_stride > most))
    return train_fail(MOE_SPEC_EINVAL, "orthogonalise: out's matrix stride is below a matrix or above 2^40");
  if (out == g) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: out must not be g");
  MuonArgs<kPerMuonLaunch> a{};
  MuonStack &t = a.t[0];
  const size_t need = shape(t, count, rows, cols);
  if (const char *why = range_fault(t, coefficients, iterations)) return train_fail(MOE_SPEC_EINVAL, "orthogonalise: %s", why);
  if (need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need))
    return train_fail(MOE_SPEC_EINVAL, "orthogonalise: the workspace is null, not aligned to 16 bytes or smaller than %zu bytes", need);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "orthogonalise: %s", hipGetErrorString(on.error()));
  if (need) place(t, static_cast<char *>(workspace));
  t.grad = g;
  t.grad_stride = g_stride;
  t.grad_matrix = count > 1 ? g_matrix_stride : 0;
  t.out = out;
  t.out_stride = out_stride;
  t.out_matrix = count > 1 ? out_matrix_stride : 0;
  a.scale = 1.0f;
  a.ca = float(coefficients[0]);
  a.cb = float(coefficients[1]);
  a.cc = float(coefficients[2]);
  const hipError_t e = run_stacks(a, 1, iterations, dtype == MOE_SPEC_BF16, is_small(t), s);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "orthogonalise: %s", hipGetErrorString(e));
}
