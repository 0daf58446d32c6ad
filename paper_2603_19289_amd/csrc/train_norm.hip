// LayerNorm over rows, forward and backward (paper: Appendix A, the estimator's last step before its head).
//   y = (x - mean) * rstd * gain + bias
//   w = dy * gain, h = (x - mean) * rstd:  dx = rstd * (w - mean(w) - h * mean(w h)),  dgain = sum_rows dy h,  dbias = sum_rows dy
// Both are bound by memory: x is read once and y written once, dy and x read once and dx written once.  A row stays in
// registers between its loads and its stores, so the variance is taken about the mean that is already known (no sums of
// squares that cancel).  Means are sums times 1 / cols, rounded to float: one rounding more than a division.
//
// Lanes: a row has as many as there are 16-byte chunks in it, a power of two up to 64 (several rows share a wavefront), and
// beyond one chunk each up to 16 values a lane in up to eight wavefronts.  16 values keep the gains, the backward pass's two
// running column sums and a row in flight in registers at two to four wavefronts per SIMD.
#include "train_common.h"

namespace moe_spec {
namespace {

// Wavefronts of a launch, which walk over the rows: 16 a compute unit forward (32 of the shapes with one chunk a lane), 8
// backward, where each workgroup's column sums are written and read once more and fewer of them cost less.  Measured, TB/s:
// forward 32768 x 2048 bf16 with 8 / 16 / 20 / 32 wavefronts a compute unit 4.7 / 6.3 / 6.0 / 5.8, 65536 x 512 with 16 / 32
// 5.2 / 5.8; backward 16387 x 4096 bf16 with 4 / 6 / 8 / 10 / 12 3.7 / 4.9 / 5.2 / 4.8 / 4.7.
constexpr int kForwardWaves = 4096, kBackwardWaves = 2048, kMaxBlocks = 512;

struct NormForwardArgs {
  const void *x;
  const float *gain, *bias;
  void *y;
  float *mean, *rstd;
  int64_t x_stride, y_stride, rows;
  int cols;
  float eps, inv_cols;
};

struct NormBackwardArgs {
  const void *dy, *x;
  const float *mean, *rstd, *gain;
  void *dx;
  float *dgain, *dbias;
  float *partial;                       // [blocks][2][ld], or null
  int64_t dy_stride, x_stride, dx_stride, rows;
  int cols, ld, blocks;
  float inv_cols;
};

// Row shape: LANES lanes with C chunks of V values each; chunk c of a lane begins at column (c * LANES + lane) * V.
template <typename WT, int LANES, int C>
struct Shape {
  static constexpr int V = Packed<WT>::N, kLanes = LANES, kChunks = C, kGroup = LANES < kWave ? LANES : kWave;
  static constexpr int kWavesPerRow = LANES <= kWave ? 1 : LANES / kWave;
  static constexpr int kBlock = LANES <= kWave ? 256 : LANES, kRows = kBlock / LANES;   // workgroup of the forward pass
  static constexpr int kBlock2 = LANES <= kWave || LANES > 256 ? 512 : 256, kRows2 = kBlock2 / LANES;   // and of the backward pass
};

// Sums over a row's lanes of N values at once.  Rows of several wavefronts meet in LDS, in one of two places by turns: a
// wavefront writes a place again only behind the barrier of the sum in between, which the others reach after they have read.
template <int N, int GROUP, int WAVES, int BLOCK>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*place)[N * BLOCK / kWave], int &turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = group_sum<GROUP>(v[i]);
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x / kWave;
    float *at = place[turn];
    turn ^= 1;
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[wave * N + i] = v[i];
    }
    __syncthreads();
    at += wave / WAVES * WAVES * N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += at[w * N + i];
      v[i] = s;
    }
  }
}

// Where a lane's chunk lies in its row.
template <int V, bool RAGGED>
struct Place {
  int col, count, skip;                 // first column; values that exist; those of them that are the neighbour's
  bool used;
  __device__ __forceinline__ Place(int index, int cols) {
    col = index * V;
    used = col < cols;
    count = V;
    skip = 0;
    if constexpr (RAGGED) {
      if (cols < V) count = cols;
      else if (used && col + V > cols) {
        skip = col + V - cols;
        col = cols - V;
      }
    }
  }
  __device__ __forceinline__ bool mine(int i) const { return !RAGGED || (i >= skip && i < count); }
};

template <int V, bool RAGGED>
__device__ __forceinline__ void load_columns(const float *p, const Place<V, RAGGED> &at, float none, float (&f)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = none;
  if (!p || !at.used) return;
  Run<float, V> r;
  r.load(p + at.col, at.count, none);
  r.get(f);
}

template <typename WT, int LANES, int C, bool RAGGED>
__global__ __launch_bounds__((Shape<WT, LANES, C>::kBlock)) void norm_forward_kernel(const NormForwardArgs a) {
  using S = Shape<WT, LANES, C>;
  constexpr int V = S::V;
  __shared__ float place[2][S::kBlock / kWave];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  int turn = 0;
  float gain[C][V], bias[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Place<V, RAGGED> at(c * LANES + lane, a.cols);
    load_columns(a.gain, at, 1.0f, gain[c]);
    load_columns(a.bias, at, 0.0f, bias[c]);
  }
  const int64_t step = int64_t(gridDim.x) * S::kRows;
  Run<WT, V> next[C];
  auto fetch = [&](int64_t row) {
    const WT *x = static_cast<const WT *>(a.x) + row * a.x_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
      next[c].clear();
      if (row < a.rows && at.used) next[c].load(x + at.col, at.count);
    }
  };
  int64_t row = int64_t(blockIdx.x) * S::kRows + slot;
  fetch(row);
  for (int64_t first = int64_t(blockIdx.x) * S::kRows; first < a.rows; first += step, row += step) {
    float f[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) next[c].get(f[c]);
    fetch(row + step);                  // the next row is on its way while this one is worked on
    float sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[0] += at.mine(i) ? f[c][i] : 0.0f;
    }
    row_sums<1, S::kGroup, S::kWavesPerRow, S::kBlock>(sum, place, turn);
    const float mean = sum[0] * a.inv_cols;
    float sq[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        f[c][i] -= mean;
        if (at.used && at.mine(i)) sq[0] += f[c][i] * f[c][i];
      }
    }
    row_sums<1, S::kGroup, S::kWavesPerRow, S::kBlock>(sq, place, turn);
    const float rstd = 1.0f / sqrtf(sq[0] * a.inv_cols + a.eps);
    if (row < a.rows) {
      WT *y = static_cast<WT *>(a.y) + row * a.y_stride;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<V, RAGGED> at(c * LANES + lane, a.cols);
        if (at.used) {
#pragma unroll
          for (int i = 0; i < V; ++i) f[c][i] = f[c][i] * rstd * gain[c][i] + bias[c][i];
          store_run<WT, V>(y + at.col, f[c], at.count);
        }
      }
      if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

// Column sums of few rows: sixteen columns a workgroup, the rows over its threads, straight from dy and x.  These workgroups run
// beside those that form dx, in the same launch.
constexpr int kDirectCols = 16;
template <typename WT, int BLOCK>
__device__ __forceinline__ void direct_columns(const NormBackwardArgs &a, int index) {
  constexpr int kSlices = BLOCK / kDirectCols;
  __shared__ float part[2][kSlices][kDirectCols + 1];
  const int lane = threadIdx.x % kDirectCols, slice = threadIdx.x / kDirectCols;
  const int col = index * kDirectCols + lane, from = col < a.cols ? col : a.cols - 1;
  float dgain = 0.0f, dbias = 0.0f;
#pragma unroll 8
  for (int64_t row = slice; row < a.rows; row += kSlices) {
    const float x = to_float(static_cast<const WT *>(a.x)[row * a.x_stride + from]);
    const float dy = to_float(static_cast<const WT *>(a.dy)[row * a.dy_stride + from]);
    dgain += dy * ((x - a.mean[row]) * a.rstd[row]);
    dbias += dy;
  }
  part[0][slice][lane] = dgain;
  part[1][slice][lane] = dbias;
  __syncthreads();
  if (threadIdx.x < 2 * kDirectCols) {
    const int which = threadIdx.x / kDirectCols;
    float *out = which ? a.dbias : a.dgain;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSlices; ++i) sum += part[which][i][lane];
    if (out && col < a.cols) out[col] = float(sum);
  }
}

// One row after the other as above; the column sums of a workgroup's rows stay in registers and go out once, to its place in
// the workspace, where norm_columns_kernel adds up the workgroups'.  No atomics: the order of the sums is fixed.
template <typename WT, int LANES, int C, bool RAGGED>
__global__ __launch_bounds__((Shape<WT, LANES, C>::kBlock2)) void norm_backward_kernel(const NormBackwardArgs a) {
  using S = Shape<WT, LANES, C>;
  constexpr int V = S::V;
  __shared__ float place[2][2 * S::kBlock2 / kWave];
  if (int(blockIdx.x) >= a.blocks) {
    direct_columns<WT, S::kBlock2>(a, blockIdx.x - a.blocks);
    return;
  }
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  int turn = 0;
  float gain[C][V], dgain[C][V], dbias[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_columns(a.gain, Place<V, RAGGED>(c * LANES + lane, a.cols), 1.0f, gain[c]);
#pragma unroll
    for (int i = 0; i < V; ++i) dgain[c][i] = dbias[c][i] = 0.0f;
  }
  const int64_t step = int64_t(a.blocks) * S::kRows2;
  Run<WT, V> next_x[C], next_dy[C];
  float next_mean, next_rstd;
  auto fetch = [&](int64_t row) {
    const WT *x = static_cast<const WT *>(a.x) + row * a.x_stride;
    const WT *dy = static_cast<const WT *>(a.dy) + row * a.dy_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
      next_x[c].clear();
      next_dy[c].clear();
      if (row < a.rows && at.used) {
        next_x[c].load(x + at.col, at.count);
        next_dy[c].load(dy + at.col, at.count);
      }
    }
    next_mean = row < a.rows ? a.mean[row] : 0.0f;
    next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
  };
  int64_t row = int64_t(blockIdx.x) * S::kRows2 + slot;
  fetch(row);
  for (int64_t first = int64_t(blockIdx.x) * S::kRows2; first < a.rows; first += step, row += step) {
    float h[C][V], w[C][V], sums[2] = {0.0f, 0.0f};
    const float mean = next_mean, rstd = next_rstd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      next_x[c].get(h[c]);
      next_dy[c].get(w[c]);
    }
    fetch(row + step);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
      const float centre = at.used ? mean : 0.0f;      // behind the last column h is zero, not mean * rstd, which may be infinite
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float dy = w[c][i];       // zero behind the last column and the last row
        h[c][i] = (h[c][i] - centre) * rstd;
        dgain[c][i] += dy * h[c][i];
        dbias[c][i] += dy;
        w[c][i] = dy * gain[c][i];
        sums[0] += at.mine(i) ? w[c][i] : 0.0f;
        sums[1] += at.mine(i) ? w[c][i] * h[c][i] : 0.0f;
      }
    }
    row_sums<2, S::kGroup, S::kWavesPerRow, S::kBlock2>(sums, place, turn);
    const float c1 = sums[0] * a.inv_cols, c2 = sums[1] * a.inv_cols;
    if (a.dx && row < a.rows) {
      WT *dx = static_cast<WT *>(a.dx) + row * a.dx_stride;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<V, RAGGED> at(c * LANES + lane, a.cols);
        if (at.used) {
#pragma unroll
          for (int i = 0; i < V; ++i) w[c][i] = rstd * (w[c][i] - c1 - h[c][i] * c2);
          store_run<WT, V>(dx + at.col, w[c], at.count);
        }
      }
    }
  }
  if (!a.partial) return;
  // rows of one wavefront first, then the wavefronts'
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      for (int m = LANES; m < kWave; m <<= 1) {
        dgain[c][i] += __shfl_xor(dgain[c][i], m);
        dbias[c][i] += __shfl_xor(dbias[c][i], m);
      }
    }
  float *out = a.partial + size_t(blockIdx.x) * 2 * a.ld;
  constexpr int kParts = S::kBlock2 / (LANES < kWave ? kWave : LANES);
  if constexpr (kParts == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<V, RAGGED> at(c * LANES + lane, a.cols);
      if (at.used) {                    // ends within ld; a length below V leaves room for V
        store_run<float, V>(out + at.col, dgain[c], V);
        store_run<float, V>(out + a.ld + at.col, dbias[c], V);
      }
    }
    return;
  }
  // then the rows of the workgroup, one of the two sums after the other
  __shared__ float sums[kParts][LANES * C * V];
  const int part = threadIdx.x / (LANES < kWave ? kWave : LANES);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();
    if (threadIdx.x % kWave < LANES) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<V, RAGGED> at(c * LANES + lane, a.cols);
        if (!at.used) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) sums[part][at.col + i] = which ? dbias[c][i] : dgain[c][i];
      }
    }
    __syncthreads();
    for (int col = threadIdx.x; col < a.ld; col += S::kBlock2) {
      float s = 0.0f;
      if (col < a.cols) {
#pragma unroll
        for (int k = 0; k < kParts; ++k) s += sums[k][col];
      }
      out[which * a.ld + col] = s;
    }
  }
}

// Adds up what the workgroups left: 32 columns a workgroup, the workgroups' rows over 32 threads, in double.
constexpr int kSlices = 32;
__global__ __launch_bounds__(32 * kSlices) void norm_columns_kernel(const NormBackwardArgs a) {
  __shared__ double part[kSlices][33];
  const int at = blockIdx.x * 32 + threadIdx.x % 32, slice = threadIdx.x / 32;
  double s = 0.0;
  if (at < 2 * a.ld) {
#pragma unroll 8
    for (int b = slice; b < a.blocks; b += kSlices) s += double(a.partial[size_t(b) * 2 * a.ld + at]);
  }
  part[slice][threadIdx.x % 32] = s;
  __syncthreads();
  if (slice == 0 && at < 2 * a.ld) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSlices; ++i) sum += part[i][threadIdx.x];
    const int which = at >= a.ld, col = which ? at - a.ld : at;
    float *out = which ? a.dbias : a.dgain;
    if (out && col < a.cols) out[col] = float(sum);
  }
}

int blocks_for(int64_t rows, int rows_per_block, int most) {
  const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
  return int(need < most ? need : most);
}

// Calls f with the row shape for a number of columns, by the rule at the top.
template <typename WT, typename F>
auto with_shape(int cols, F f) {
  constexpr int V = Packed<WT>::N, C16 = 16 / V;
  const int chunks = (cols + V - 1) / V;
  if (chunks <= 8) return f(Shape<WT, 8, 1>());
  if (chunks <= 16) return f(Shape<WT, 16, 1>());
  if (chunks <= 32) return f(Shape<WT, 32, 1>());
  if (chunks <= 64) return f(Shape<WT, 64, 1>());
  if (cols <= 1024) return f(Shape<WT, 64, C16>());
  if (cols <= 2048) return f(Shape<WT, 128, C16>());
  if (cols <= 4096) return f(Shape<WT, 256, C16>());
  return f(Shape<WT, 512, C16>());
}

template <typename WT>
hipError_t forward(hipStream_t stream, NormForwardArgs &a) {
  return with_shape<WT>(a.cols, [&](auto shape) {
    using S = decltype(shape);
    const int blocks = blocks_for(a.rows, S::kRows, (S::kChunks == 1 ? 2 : 1) * kForwardWaves * kWave / S::kBlock);
    if (a.cols % S::V) return launch(norm_forward_kernel<WT, S::kLanes, S::kChunks, true>, blocks, S::kBlock, stream, a);
    return launch(norm_forward_kernel<WT, S::kLanes, S::kChunks, false>, blocks, S::kBlock, stream, a);
  });
}

// Few rows: the column sums are formed beside dx, from dy and x once more, which then come out of a cache.  Measured in us, beside dx /
// in a launch of its own, bf16: 16 x 512 2.3 / 4.8, 256 x 512 2.8 / 5.2, 512 x 2048 6.0 / 8.8, 512 x 8192 18.4 / 18.8, 1024 x 64 4.2 / 5.7,
// 1024 x 2048 9.8 / 13.2, 1024 x 4096 15.1 / 18.1, 1024 x 8192 32 / 20, 2048 x 64 6.4 / 5.7, 2048 x 512 12.0 / 6.1.  float32 reads twice as much:
// 16 x 512 2.7 / 5.5, 256 x 512 2.9 / 5.7, 512 x 2048 6.5 / 10.1, 1024 x 1024 8.2 / 8.0, 1024 x 2048 11.2 / 14.5, but 1024 x 4096 19.1 / 16.5 and
// 512 x 8192 21.4 / 17.0: between 2 M and 4 M values the rule costs it up to a quarter.
bool columns_beside(int64_t rows, int cols) { return rows <= 1024 && rows * cols <= (4 << 20); }

template <typename WT>
hipError_t backward(hipStream_t stream, NormBackwardArgs &a) {
  const bool direct = (a.dgain || a.dbias) && !a.partial;
  return with_shape<WT>(a.cols, [&](auto shape) {
    using S = decltype(shape);
    a.blocks = blocks_for(a.rows, S::kRows2, kBackwardWaves * kWave / S::kBlock2);
    const unsigned grid = a.blocks + (direct ? (a.cols + kDirectCols - 1) / kDirectCols : 0);
    const hipError_t e = a.cols % S::V ? launch(norm_backward_kernel<WT, S::kLanes, S::kChunks, true>, grid, S::kBlock2, stream, a)
                                       : launch(norm_backward_kernel<WT, S::kLanes, S::kChunks, false>, grid, S::kBlock2, stream, a);
    if (e != hipSuccess) return e;
    if (!a.partial) return hipSuccess;
    return launch(norm_columns_kernel, (2 * a.ld + 31) / 32, 32 * kSlices, stream, a);
  });
}

static_assert(kBackwardWaves * kWave / 256 <= kMaxBlocks, "the workspace has room for the shape with the most workgroups");
int padded(int cols) { return (cols + 7) / 8 * 8; }

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" int moe_spec_layernorm_forward(void *stream, int dtype, const void *x, int64_t x_stride, int64_t rows, int cols,
                                          const float *gain, const float *bias, float eps, void *y, int64_t y_stride,
                                          float *mean, float *rstd) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: unknown dtype %d", dtype);
  if (rows < 0 || rows > MOE_SPEC_TRAIN_MAX_ROWS) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: rows out of range");
  if (cols < 1 || cols > MOE_SPEC_TRAIN_MAX_COLS) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: cols must be 1 to %d", MOE_SPEC_TRAIN_MAX_COLS);
  if (!(eps >= 0.0f)) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: eps must not be negative");
  const int elem = size_of(dtype);
  if (const char *why = matrix_fault(x, x_stride, rows, cols, elem, false)) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: x %s", why);
  if (const char *why = matrix_fault(y, y_stride, rows, cols, elem, true)) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: y %s", why);
  if (x == y && x_stride != y_stride && rows > 1) return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: in place the strides must be equal");
  if (misaligned(gain, 4) || misaligned(bias, 4) || misaligned(mean, 4) || misaligned(rstd, 4))
    return train_fail(MOE_SPEC_EINVAL, "layernorm_forward: gain, bias, mean and rstd must be aligned to 4 bytes");
  if (rows == 0) return MOE_SPEC_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "layernorm_forward: %s", hipGetErrorString(on.error()));
  NormForwardArgs a = {x, gain, bias, y, mean, rstd, x_stride, y_stride, rows, cols, eps, 1.0f / float(cols)};
  const hipError_t e = dtype == MOE_SPEC_BF16 ? forward<uint16_t>(s, a) : forward<float>(s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "layernorm_forward: %s", hipGetErrorString(e));
}

extern "C" size_t moe_spec_layernorm_backward_workspace_bytes(int64_t rows, int cols) {
  if (rows < 0 || rows > MOE_SPEC_TRAIN_MAX_ROWS || cols < 1 || cols > MOE_SPEC_TRAIN_MAX_COLS) return 0;
  if (columns_beside(rows, cols)) return 0;
  return size_t(blocks_for(rows, 1, kMaxBlocks)) * 2 * padded(cols) * sizeof(float);
}

extern "C" int moe_spec_layernorm_backward(void *stream, int dtype, const void *dy, int64_t dy_stride, const void *x,
                                           int64_t x_stride, int64_t rows, int cols, const float *mean, const float *rstd,
                                           const float *gain, void *dx, int64_t dx_stride, float *dgain, float *dbias,
                                           void *workspace, size_t workspace_bytes) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: unknown dtype %d", dtype);
  if (rows < 0 || rows > MOE_SPEC_TRAIN_MAX_ROWS) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: rows out of range");
  if (cols < 1 || cols > MOE_SPEC_TRAIN_MAX_COLS) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: cols must be 1 to %d", MOE_SPEC_TRAIN_MAX_COLS);
  const int elem = size_of(dtype);
  if (const char *why = matrix_fault(dy, dy_stride, rows, cols, elem, false)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: dy %s", why);
  if (const char *why = matrix_fault(x, x_stride, rows, cols, elem, false)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: x %s", why);
  if (dx) {
    if (const char *why = matrix_fault(dx, dx_stride, rows, cols, elem, true)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: dx %s", why);
    if (rows && (dx == x || dx == dy)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: dx must not be x or dy");
  }
  if (rows && (!mean || !rstd)) return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: mean or rstd is null");
  if (misaligned(gain, 4) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dgain, 4) || misaligned(dbias, 4))
    return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: gain, mean, rstd, dgain and dbias must be aligned to 4 bytes");
  const bool columns = dgain || dbias;
  const size_t need = moe_spec_layernorm_backward_workspace_bytes(rows, cols);
  if (columns && need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need))
    return train_fail(MOE_SPEC_EINVAL, "layernorm_backward: the workspace must be 16-byte aligned and have %zu bytes", need);
  if ((rows == 0 && !columns) || (!dx && !columns)) return MOE_SPEC_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "layernorm_backward: %s", hipGetErrorString(on.error()));
  NormBackwardArgs a = {dy, x, mean, rstd, gain, dx, dgain, dbias, nullptr, dy_stride, x_stride, dx_stride, rows, cols,
                        padded(cols), 0, 1.0f / float(cols)};
  if (columns) {
    if (need) a.partial = static_cast<float *>(workspace);
    if (rows == 0) {                    // nothing to add up: the column kernel writes zeros
      const hipError_t e = launch(norm_columns_kernel, (2 * a.ld + 31) / 32, 32 * kSlices, s, a);
      return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "layernorm_backward: %s", hipGetErrorString(e));
    }
  }
  const hipError_t e = dtype == MOE_SPEC_BF16 ? backward<uint16_t>(s, a) : backward<float>(s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "layernorm_backward: %s", hipGetErrorString(e));
}
