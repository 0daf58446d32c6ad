// Updates of matrices by the orthogonal factor of their momentum (Muon), many matrices in a few launches.
//   X_0 = U / |U|_F (turned so that it has at most as many rows as columns), then as often as asked
//   A = X X^T,  B = a I + b A + c A A,  X <- B X
// The iteration runs on the matrix cores with X, A and B in float16 and sums in float: |X| stays below 1.3 and every value of A and B below 15,
// so float16's range is enough, and its 11 bits are what a bfloat16 result can show (0.1 % of the result after five iterations; bfloat16
// iterates are off by 1 %).  The three are held 64-fold, so that the smallest values that count stay above float16's denormal ones.
// Three products an iteration, each one launch over all matrices of a call; a matrix that the framework holds upright is laid on its side
// on the way in and stood up on the way out.
#include <math.h>

#include "mfma_tiles.h"

namespace moe_spec {
namespace {

constexpr int kMuonBlock = 256, kPerMuonLaunch = 24, kSliceValues = 16384, kTurn = 64;
constexpr float kHeld = 64.0f;

// A stack of matrices of one size.
struct MuonStack {
  uint16_t *x[2], *a, *b;        // workspace: iterates [count, m, ld_n], A and B [count, m, ld_m]
  double *partial;               // [count, slices] sums of squares
  float *p;
  const void *grad;
  float *momentum;
  void *out;                     // bf16 copy of p, or what orthogonalise returns
  int64_t grad_stride, grad_matrix, out_stride, out_matrix;
  int64_t count;
  int rows, cols, m, n, ld_m, ld_n, slices, slice_rows;
};
struct MuonArgs {
  MuonStack t[kPerMuonLaunch];
  uint32_t first[kPerMuonLaunch];        // a stack's first workgroup
  float mu, decay, rate, scale, ca, cb, cc;
  const float *scale_dev;
  uint32_t total;                        // workgroups that have a tile
  int nesterov, which;
};
static_assert(sizeof(MuonArgs) <= 4096, "an argument block");

__device__ __forceinline__ int stack_of(const uint32_t (&first)[kPerMuonLaunch], uint32_t workgroup) {
  int which = -1;
#pragma unroll
  for (int i = 0; i < kPerMuonLaunch; ++i) which += first[i] <= workgroup;
  return which;
}

// Eight values of a gradient.
template <typename GT>
__device__ __forceinline__ void gradient8(const MuonStack &t, int64_t matrix, int row, int c, int n, float (&g)[8]) {
  Run<GT, 8> r;
  r.load(static_cast<const GT *>(t.grad) + matrix * t.grad_matrix + row * t.grad_stride + c, n);
  r.get(g);
}

// What is orthogonalised: the gradient, or the momentum with the gradient in it.  STEP: the momentum has been updated already.
template <typename GT>
__device__ __forceinline__ void direction8(const MuonArgs &a, const MuonStack &t, float scale, int64_t matrix, int row, int c, int n, float (&u)[8]) {
#pragma clang fp contract(off)
  gradient8<GT>(t, matrix, row, c, n, u);
  if (!t.momentum) return;
  Run<float, 8> rm;
  float m[8];
  rm.load(t.momentum + matrix * t.rows * t.cols + int64_t(row) * t.cols + c, n);
  rm.get(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = a.nesterov ? u[i] * scale + m[i] * a.mu : m[i];
}

// Momentum and sums of squares, a slice of a matrix's rows a workgroup.
template <typename GT>
__global__ __launch_bounds__(kMuonBlock) void muon_begin_kernel(const MuonArgs a) {
#pragma clang fp contract(off)
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const uint32_t at = blockIdx.x - a.first[which];
  const int64_t matrix = at / t.slices;
  const int slice = at % t.slices, row0 = slice * t.slice_rows, rows = min(t.slice_rows, t.rows - row0), across = (t.cols + 7) / 8;
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  double sum = 0.0;
  for (int i = threadIdx.x; i < rows * across; i += kMuonBlock) {
    const int row = row0 + i / across, c = i % across * 8, n = t.cols - c;
    float u[8];
    gradient8<GT>(t, matrix, row, c, n, u);
    if (t.momentum) {
      float *m_at = t.momentum + matrix * t.rows * t.cols + int64_t(row) * t.cols + c;
      Run<float, 8> rm;
      float m[8];
      rm.load(m_at, n);
      rm.get(m);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = u[j] * scale;
        m[j] = m[j] * a.mu + g;
        u[j] = a.nesterov ? g + m[j] * a.mu : m[j];
      }
      store_run<float, 8>(m_at, m, n);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j < n) sum += double(u[j]) * double(u[j]);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  __shared__ double part[kMuonBlock / 64];
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) t.partial[matrix * t.slices + slice] = (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ __forceinline__ uint16_t to_f16(float v) { return __builtin_bit_cast(uint16_t, _Float16(v)); }
__device__ __forceinline__ float from_f16(uint16_t v) { return float(__builtin_bit_cast(_Float16, v)); }

// What makes 64 X_0 of a matrix's values: they are taken times 2^shift, which alone could leave float's range where they are tiny, and then
// times factor: zero where the matrix has only zeros, NaN where it holds what is not finite.
struct Normaliser {
  float factor;
  int shift;
  __device__ __forceinline__ uint16_t operator()(float u) const {
    return factor > 0.0f ? to_f16(ldexpf(u, shift) * factor) : factor == 0.0f ? uint16_t(0) : uint16_t(0x7e00);
  }
};
__device__ __forceinline__ Normaliser normaliser(const MuonStack &t, int64_t matrix) {
  const int lane = threadIdx.x & 63;
  double sum = 0.0;
  for (int i = lane; i < t.slices; i += 64) sum += t.partial[matrix * t.slices + i];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  if (!(sum < double(INFINITY))) return {NAN, 0};
  if (!(sum > 0.0)) return {0.0f, 0};
  int exponent;
  const double part = frexp(sqrt(sum), &exponent);
  return {float(double(kHeld) / part), -exponent};
}

// X_0 as float16, laid on its side where the matrix is upright: tiles of 64 x 64 then go through LDS.
template <typename GT>
__global__ __launch_bounds__(kMuonBlock) void muon_normalise_kernel(const MuonArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTurn][kTurn + 8];
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const int across = (t.cols + kTurn - 1) / kTurn, down = (t.rows + kTurn - 1) / kTurn;
  const uint32_t at = blockIdx.x - a.first[which];
  const int64_t matrix = at / uint32_t(across * down);
  const int q = at % uint32_t(across * down), row0 = q / across * kTurn, col0 = q % across * kTurn;
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  const Normaliser normal = normaliser(t, matrix);
  const bool upright = t.rows > t.cols;
  uint16_t *x = t.x[0] + matrix * t.m * t.ld_n;
#pragma unroll
  for (int i = threadIdx.x; i < kTurn * kTurn / 8; i += kMuonBlock) {
    const int r = i / (kTurn / 8), c = i % (kTurn / 8) * 8, row = row0 + r, col = col0 + c;
    float u[8];
    uint16_t e[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < t.rows && col < t.cols) {
      direction8<GT>(a, t, scale, matrix, row, col, t.cols - col, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = col + j < t.cols ? normal(u[j]) : uint16_t(0);
    }
    if (upright) __builtin_memcpy(&tile[r][c], e, 16);
    else if (row < t.rows && col < t.ld_n) __builtin_memcpy(x + int64_t(row) * t.ld_n + col, e, 16);
  }
  if (!upright) return;
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x; i < kTurn * kTurn / 8; i += kMuonBlock) {
    const int c = i / (kTurn / 8), r = i % (kTurn / 8) * 8;              // a column of the matrix is a row of X
    if (col0 + c >= t.cols || row0 + r >= t.ld_n) continue;
    uint16_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = tile[r + j][c];
    __builtin_memcpy(x + int64_t(col0 + c) * t.ld_n + row0 + r, e, 16);
  }
}

// The result: p <- p decay - rate o and its copy, or o itself.
template <typename OT>
__device__ __forceinline__ void finish8(const MuonArgs &a, const MuonStack &t, int64_t matrix, int row, int c, int n, const float (&o)[8]) {
#pragma clang fp contract(off)
  if (t.p) {
    float *p_at = t.p + matrix * t.rows * t.cols + int64_t(row) * t.cols + c;
    Run<float, 8> rp;
    float p[8];
    rp.load(p_at, n);
    rp.get(p);
    const float rate = a.rate * sqrtf(float(t.n));
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = p[j] * a.decay - o[j] * rate;
    store_run<float, 8>(p_at, p, n);
    if (t.out) store_run<OT, 8>(static_cast<OT *>(t.out) + matrix * t.out_matrix + row * t.out_stride + c, p, n);
  } else {
    store_run<OT, 8>(static_cast<OT *>(t.out) + matrix * t.out_matrix + row * t.out_stride + c, o, n);
  }
}

template <typename OT>
__global__ __launch_bounds__(kMuonBlock) void muon_finish_kernel(const MuonArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTurn][kTurn + 8];
  const int which = stack_of(a.first, blockIdx.x);
  const MuonStack &t = a.t[which];
  const int across = (t.cols + kTurn - 1) / kTurn, down = (t.rows + kTurn - 1) / kTurn;
  const uint32_t at = blockIdx.x - a.first[which];
  const int64_t matrix = at / uint32_t(across * down);
  const int q = at % uint32_t(across * down), row0 = q / across * kTurn, col0 = q % across * kTurn;
  const bool upright = t.rows > t.cols;
  const uint16_t *x = t.x[a.which] + matrix * t.m * t.ld_n;
  if (upright) {
#pragma unroll
    for (int i = threadIdx.x; i < kTurn * kTurn / 8; i += kMuonBlock) {
      const int c = i / (kTurn / 8), r = i % (kTurn / 8) * 8;
      uint4 v = {0, 0, 0, 0};
      if (col0 + c < t.cols && row0 + r < t.ld_n) v = load_raw<uint4>(x + int64_t(col0 + c) * t.ld_n + row0 + r);
      uint16_t e[8];
      __builtin_memcpy(e, &v, 16);
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[r + j][c] = e[j];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = threadIdx.x; i < kTurn * kTurn / 8; i += kMuonBlock) {
    const int r = i / (kTurn / 8), c = i % (kTurn / 8) * 8, row = row0 + r, col = col0 + c;
    if (row >= t.rows || col >= t.cols) continue;
    uint16_t e[8];
    if (upright) __builtin_memcpy(e, &tile[r][c], 16);
    else __builtin_memcpy(e, x + int64_t(row) * t.ld_n + col, 16);
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = from_f16(e[j]) * (1.0f / kHeld);
    finish8<OT>(a, t, matrix, row, col, t.cols - col, o);
  }
}

// One product for every matrix.  SQUARE: A = X X^T; POLYNOMIAL: B = a I + b A + c A A; APPLY: X' = B X.  A and B are symmetric: of them
// only tiles on and below the diagonal are worked out, and written to both places.
enum MuonProduct { SQUARE, POLYNOMIAL, APPLY };

template <int TILE, int WM, int WN, MuonProduct KIND>
__global__ __launch_bounds__(WM *WN * 64) void muon_product_kernel(const MuonArgs a) {
  constexpr bool SYMMETRIC = KIND != APPLY;
  using P = TileProduct<F16, TILE, TILE, WM, WN, false, KIND == APPLY, true>;
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
  P p;
  const int rows = min(TILE, t.m - row0), some = min(TILE, cols - col0);
  // X may have rows of 65536 values and A of as many: the strides that a tile takes at most
  if constexpr (KIND == SQUARE) p.run(lds, x + int64_t(row0) * t.ld_n, t.ld_n, rows, x + int64_t(col0) * t.ld_n, t.ld_n, some, t.n);
  if constexpr (KIND == POLYNOMIAL) p.run(lds, ta + int64_t(row0) * t.ld_m, t.ld_m, rows, ta + int64_t(col0) * t.ld_m, t.ld_m, some, t.m);
  if constexpr (KIND == APPLY) p.run(lds, tb + int64_t(row0) * t.ld_m, t.ld_m, rows, x + col0, t.ld_n, some, t.m);
  const int ld = SYMMETRIC ? t.ld_m : t.ld_n;
  uint16_t *out = KIND == APPLY ? t.x[a.which ^ 1] + matrix * t.m * t.ld_n : (KIND == SQUARE ? t.a : t.b) + matrix * t.m * t.ld_m;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int wave_row = row0 + wave / WN * (TILE / WM), wave_col = col0 + wave % WN * (TILE / WN);
  char *mine = lds + wave * R::kBytes;
  __syncthreads();                               // the operands have been read by all
#pragma unroll
  for (int f = 0; f < P::FM; ++f) {
#pragma unroll
    for (int h = 0; h < P::FN; ++h) {
      const int row = wave_row + 16 * f + i, col = wave_col + 16 * h + 4 * g;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = p.acc[f][h][r] * (1.0f / kHeld);
      if constexpr (KIND == POLYNOMIAL) {
        uint16_t e[4] = {0, 0, 0, 0};
        if (row < t.m && col < ld) __builtin_memcpy(e, ta + int64_t(row) * ld + col, 8);
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
#pragma unroll
  for (int q = 0; q < R::kEach; ++q) {
    const int r = (q * 64 + lane) / R::kAcross, c = (q * 64 + lane) % R::kAcross, row = wave_row + r, col = wave_col + 8 * c;
    if (row < t.m && col < ld) *reinterpret_cast<uint4 *>(out + int64_t(row) * ld + col) = R::chunk(mine, r, c);
  }
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

// ---- host ----------------------------------------------------------------------------------------------------------
inline int round8(int n) { return (n + 7) / 8 * 8; }
inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

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
  return 2 * round256(size_t(count) * t.m * t.ld_n * 2) + 2 * round256(size_t(count) * t.m * t.ld_m * 2) + round256(size_t(count) * t.slices * 8);
}
char *place(MuonStack &t, char *at) {
  const size_t x = round256(size_t(t.count) * t.m * t.ld_n * 2), a = round256(size_t(t.count) * t.m * t.ld_m * 2);
  t.x[0] = reinterpret_cast<uint16_t *>(at);
  t.x[1] = reinterpret_cast<uint16_t *>(at + x);
  t.a = reinterpret_cast<uint16_t *>(at + 2 * x);
  t.b = reinterpret_cast<uint16_t *>(at + 2 * x + a);
  t.partial = reinterpret_cast<double *>(at + 2 * x + 2 * a);
  return at + 2 * x + 2 * a + round256(size_t(t.count) * t.slices * 8);
}

const char *iteration_fault(const double *c, int iterations) {
  if (iterations < 1 || iterations > 64) return "iterations must be between 1 and 64";
  for (int i = 0; i < 3; ++i) if (!(fabs(c[i]) <= 16.0)) return "coefficients must lie between -16 and 16";
  return nullptr;
}

// All launches for up to kPerMuonLaunch stacks; a's scalars are set.  Stops at the first that fails.
template <typename Count>
void firsts(MuonArgs &a, int n, Count workgroups, unsigned &grid) {
  grid = 0;
  for (int i = 0; i < kPerMuonLaunch; ++i) {
    a.first[i] = i < n ? grid : UINT32_MAX;
    if (i < n) grid += unsigned(workgroups(a.t[i]));
  }
}

inline int64_t tiles(int64_t n, int tile) { return (n + tile - 1) / tile; }
inline int64_t begin_blocks(const MuonStack &t) { return t.count * t.slices; }
inline int64_t turn_blocks(const MuonStack &t) { return t.count * tiles(t.rows, kTurn) * tiles(t.cols, kTurn); }
inline int64_t square_blocks(const MuonStack &t, int tile) { return t.count * tiles(t.m, tile) * (tiles(t.m, tile) + 1) / 2; }
inline int64_t apply_blocks(const MuonStack &t, int tile) { return t.count * tiles(t.m, tile) * tiles(t.n, tile); }
// Most of them, of any launch over the stack.
inline int64_t most_blocks(const MuonStack &t) {
  const int64_t b = begin_blocks(t), u = turn_blocks(t);
  return b > u ? b : u;                                 // products have no more: their smallest tiles are as large
}
constexpr int64_t kMostMuonBlocks = (int64_t(1) << 32) / kMuonBlock - 1;

// One product over n stacks, in the largest tiles of which there are as many as compute units.
template <MuonProduct KIND>
hipError_t run_product(MuonArgs &a, int n, hipStream_t s) {
  int tile = 256;
  const auto blocks = [&](const MuonStack &t) { return KIND == APPLY ? apply_blocks(t, tile) : square_blocks(t, tile); };
  for (;; tile /= 2) {
    firsts(a, n, blocks, a.total);
    if (tile == 64 || a.total >= 256) break;
  }
  const unsigned grid = (a.total + 7) / 8 * 8;
  if (tile == 256) return launch(muon_product_kernel<256, 2, 4, KIND>, grid, 512, s, a);
  if (tile == 128) return launch(muon_product_kernel<128, 2, 4, KIND>, grid, 512, s, a);
  return launch(muon_product_kernel<64, 2, 2, KIND>, grid, 256, s, a);
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

hipError_t run_stacks(MuonArgs &a, int n, int iterations, bool grad_bf16, bool out_bf16, hipStream_t s) {
  unsigned grid;
  hipError_t e;
  firsts(a, n, begin_blocks, grid);
  e = grad_bf16 ? launch(muon_begin_kernel<uint16_t>, grid, kMuonBlock, s, a) : launch(muon_begin_kernel<float>, grid, kMuonBlock, s, a);
  if (e != hipSuccess) return e;
  firsts(a, n, turn_blocks, grid);
  e = grad_bf16 ? launch(muon_normalise_kernel<uint16_t>, grid, kMuonBlock, s, a) : launch(muon_normalise_kernel<float>, grid, kMuonBlock, s, a);
  for (int i = 0; i < iterations && e == hipSuccess; ++i) {
    a.which = i & 1;
    e = run_product<SQUARE>(a, n, s);
    if (e == hipSuccess) e = run_product<POLYNOMIAL>(a, n, s);
    if (e == hipSuccess) e = run_product<APPLY>(a, n, s);
  }
  if (e != hipSuccess) return e;
  a.which = iterations & 1;
  firsts(a, n, turn_blocks, grid);
  return out_bf16 ? launch(muon_finish_kernel<uint16_t>, grid, kMuonBlock, s, a) : launch(muon_finish_kernel<float>, grid, kMuonBlock, s, a);
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
  }
  const size_t need = moe_spec_muon_workspace_bytes(tensors, n_tensors);
  if (need == 0) return MOE_SPEC_OK;
  if (!workspace || misaligned(workspace, 16) || workspace_bytes < need)
    return train_fail(MOE_SPEC_EINVAL, "muon_step: the workspace is null, not aligned to 16 bytes or smaller than %zu bytes", need);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "muon_step: %s", hipGetErrorString(on.error()));
  MuonArgs a{};
  a.mu = float(cfg->momentum);
  a.decay = float(1.0 - cfg->lr * cfg->weight_decay);
  a.rate = float(cfg->lr * cfg->update_rms);
  a.scale = float(cfg->grad_scale);
  a.scale_dev = cfg->grad_scale_dev;
  a.ca = float(cfg->coefficients[0]);
  a.cb = float(cfg->coefficients[1]);
  a.cc = float(cfg->coefficients[2]);
  a.nesterov = cfg->nesterov != 0;
  char *at = static_cast<char *>(workspace);
  int n = 0;
  int64_t blocks = 0;
  hipError_t e = hipSuccess;
  for (int i = 0; i < n_tensors && e == hipSuccess; ++i) {
    const moe_spec_muon_tensor &m = tensors[i];
    if (m.count == 0 || m.rows == 0 || m.cols == 0) continue;
    MuonStack t{};
    shape(t, m.count, m.rows, m.cols);
    if (n == kPerMuonLaunch || (n && blocks + most_blocks(t) > kMostMuonBlocks)) {
      e = run_stacks(a, n, cfg->iterations, cfg->grad_dtype == MOE_SPEC_BF16, true, s);
      n = 0;
      blocks = 0;
    }
    at = place(t, at);
    t.p = m.p;
    t.grad = m.grad;
    t.momentum = m.m;
    t.out = m.copy;
    t.grad_stride = t.out_stride = m.cols;
    t.grad_matrix = t.out_matrix = int64_t(m.rows) * m.cols;
    a.t[n++] = t;
    blocks += most_blocks(t);
  }
  if (e == hipSuccess && n) e = run_stacks(a, n, cfg->iterations, cfg->grad_dtype == MOE_SPEC_BF16, true, s);
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
  MuonArgs a{};
  MuonStack &t = a.t[0];
  const size_t need = shape(t, count, rows, cols);
  if (!workspace || misaligned(workspace, 16) || workspace_bytes < need)
    return train_fail(MOE_SPEC_EINVAL, "orthogonalise: the workspace is null, not aligned to 16 bytes or smaller than %zu bytes", need);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "orthogonalise: %s", hipGetErrorString(on.error()));
  place(t, static_cast<char *>(workspace));
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
  const hipError_t e = run_stacks(a, 1, iterations, dtype == MOE_SPEC_BF16, true, s);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "orthogonalise: %s", hipGetErrorString(e));
}
