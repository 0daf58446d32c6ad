// LayerNorm over rows, forward and backward (paper: Appendix A, the estimator's last step before its head).
//   y = (x - mean) * rstd * gain + bias
//   w = dy * gain, h = (x - mean) * rstd:  dx = rstd * (w - mean(w) - h * mean(w h)),  dgain = sum_rows dy h,  dbias = sum_rows dy
// Both are bound by memory: x is read once and y written once, dy and x read once and dx written once.  A row stays in
// registers between its loads and its stores, so the variance is taken about the mean that is already known (no sums of
// squares that cancel).
//
// Lanes: a row has as many as there are 16-byte chunks in it, a power of two up to 64 (several rows share a wavefront), and
// beyond one chunk each up to 16 values a lane in up to eight wavefronts.  16 values keep the gains, the backward pass's two
// running column sums and a row in flight in registers at two to four wavefronts per SIMD.
#include "train_common.h"

namespace moe_spec {
namespace {

constexpr int kMaxBlocks = 1024;        // workgroups of a launch: four or more per compute unit

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
  static constexpr int V = Packed<WT>::N, kLanes = LANES, kChunks = C;
  static constexpr int kBlock = LANES <= kWave ? 256 : LANES, kRows = kBlock / LANES, kGroup = LANES < kWave ? LANES : kWave;
  static constexpr int kWavesPerRow = LANES <= kWave ? 1 : LANES / kWave;
};

// Sums over a row's lanes of N values at once.  Rows of several wavefronts meet in LDS, in one of two places by turns: a
// wavefront writes a place again only behind the barrier of the sum in between, which the others reach after they have read.
template <int N, int GROUP, int WAVES>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*place)[N * WAVES], int &turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = group_sum<GROUP>(v[i]);
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x / kWave;
    float *at = place[turn];
    turn ^= 1;
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * WAVES + wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += at[i * WAVES + w];
      v[i] = s;
    }
  }
}

template <int V>
__device__ __forceinline__ void load_columns(const float *p, int col, int cols, float none, float (&f)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = none;
  if (!p) return;
  Run<float, V> r;
  r.clear();
  if (col < cols) r.load(p + col, cols - col, none);
  r.get(f);
}

template <typename WT, int LANES, int C>
__global__ __launch_bounds__((Shape<WT, LANES, C>::kBlock)) void norm_forward_kernel(const NormForwardArgs a) {
  using S = Shape<WT, LANES, C>;
  constexpr int V = S::V;
  __shared__ float place[2][S::kWavesPerRow];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  int turn = 0;
  float gain[C][V], bias[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * LANES + lane) * V;
    load_columns<V>(a.gain, col, a.cols, 1.0f, gain[c]);
    load_columns<V>(a.bias, col, a.cols, 0.0f, bias[c]);
  }
  const int64_t step = int64_t(gridDim.x) * S::kRows;
  Run<WT, V> next[C];
  auto fetch = [&](int64_t row) {
    const WT *x = static_cast<const WT *>(a.x) + row * a.x_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * LANES + lane) * V;
      next[c].clear();
      if (row < a.rows && col < a.cols) next[c].load(x + col, a.cols - col);
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
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) sum[0] += f[c][i];
    row_sums<1, S::kGroup, S::kWavesPerRow>(sum, place, turn);
    const float mean = sum[0] * a.inv_cols;
    float sq[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int left = a.cols - (c * LANES + lane) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        f[c][i] -= mean;
        if (i < left) sq[0] += f[c][i] * f[c][i];
      }
    }
    row_sums<1, S::kGroup, S::kWavesPerRow>(sq, place, turn);
    const float rstd = 1.0f / sqrtf(sq[0] * a.inv_cols + a.eps);
    if (row < a.rows) {
      WT *y = static_cast<WT *>(a.y) + row * a.y_stride;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * LANES + lane) * V;
        if (col < a.cols) {
#pragma unroll
          for (int i = 0; i < V; ++i) f[c][i] = f[c][i] * rstd * gain[c][i] + bias[c][i];
          store_run<WT, V>(y + col, f[c], a.cols - col);
        }
      }
      if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

// One row after the other as above; the column sums of a workgroup's rows stay in registers and go out once, to its place in
// the workspace, where norm_columns_kernel adds up the workgroups'.  No atomics: the order of the sums is fixed.
template <typename WT, int LANES, int C>
__global__ __launch_bounds__((Shape<WT, LANES, C>::kBlock)) void norm_backward_kernel(const NormBackwardArgs a) {
  using S = Shape<WT, LANES, C>;
  constexpr int V = S::V;
  __shared__ float place[2][2 * S::kWavesPerRow];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  int turn = 0;
  float gain[C][V], dgain[C][V], dbias[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_columns<V>(a.gain, (c * LANES + lane) * V, a.cols, 1.0f, gain[c]);
#pragma unroll
    for (int i = 0; i < V; ++i) dgain[c][i] = dbias[c][i] = 0.0f;
  }
  const int64_t step = int64_t(gridDim.x) * S::kRows;
  Run<WT, V> next_x[C], next_dy[C];
  float next_mean, next_rstd;
  auto fetch = [&](int64_t row) {
    const WT *x = static_cast<const WT *>(a.x) + row * a.x_stride;
    const WT *dy = static_cast<const WT *>(a.dy) + row * a.dy_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * LANES + lane) * V;
      next_x[c].clear();
      next_dy[c].clear();
      if (row < a.rows && col < a.cols) {
        next_x[c].load(x + col, a.cols - col);
        next_dy[c].load(dy + col, a.cols - col);
      }
    }
    next_mean = row < a.rows ? a.mean[row] : 0.0f;
    next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
  };
  int64_t row = int64_t(blockIdx.x) * S::kRows + slot;
  fetch(row);
  for (int64_t first = int64_t(blockIdx.x) * S::kRows; first < a.rows; first += step, row += step) {
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
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float dy = w[c][i];       // zero behind the last column and the last row
        h[c][i] = (h[c][i] - mean) * rstd;
        dgain[c][i] += dy * h[c][i];
        dbias[c][i] += dy;
        w[c][i] = dy * gain[c][i];
        sums[0] += w[c][i];
        sums[1] += w[c][i] * h[c][i];
      }
    }
    row_sums<2, S::kGroup, S::kWavesPerRow>(sums, place, turn);
    const float c1 = sums[0] * a.inv_cols, c2 = sums[1] * a.inv_cols;
    if (a.dx && row < a.rows) {
      WT *dx = static_cast<WT *>(a.dx) + row * a.dx_stride;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * LANES + lane) * V;
        if (col < a.cols) {
#pragma unroll
          for (int i = 0; i < V; ++i) w[c][i] = rstd * (w[c][i] - c1 - h[c][i] * c2);
          store_run<WT, V>(dx + col, w[c], a.cols - col);
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
  if constexpr (LANES <= kWave) {
    constexpr int W = 256 / kWave, N = LANES * C * V;
    __shared__ float sums[W][2][N];
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave < LANES) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sums[wave][0][(c * LANES + lane) * V + i] = dgain[c][i];
          sums[wave][1][(c * LANES + lane) * V + i] = dbias[c][i];
        }
    }
    __syncthreads();
    for (int at = threadIdx.x; at < 2 * a.ld; at += 256) {
      const int which = at >= a.ld, col = which ? at - a.ld : at;
      float s = 0.0f;
      if (col < a.cols) {
#pragma unroll
        for (int v = 0; v < W; ++v) s += sums[v][which][col];
      }
      out[at] = s;
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * LANES + lane) * V;
      if (col < a.cols) {               // a lane's columns end within ld, which is a multiple of eight
        store_run<float, V>(out + col, dgain[c], V);
        store_run<float, V>(out + a.ld + col, dbias[c], V);
      }
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
#pragma unroll 4
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

int blocks_for(int64_t rows, int rows_per_block) {
  const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
  return int(need < kMaxBlocks ? need : kMaxBlocks);
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
    return launch(norm_forward_kernel<WT, S::kLanes, S::kChunks>, blocks_for(a.rows, S::kRows), S::kBlock, stream, a);
  });
}

template <typename WT>
hipError_t backward(hipStream_t stream, NormBackwardArgs &a) {
  return with_shape<WT>(a.cols, [&](auto shape) {
    using S = decltype(shape);
    a.blocks = blocks_for(a.rows, S::kRows);
    if (a.blocks) {
      const hipError_t e = launch(norm_backward_kernel<WT, S::kLanes, S::kChunks>, a.blocks, S::kBlock, stream, a);
      if (e != hipSuccess) return e;
    }
    if (!a.partial) return hipSuccess;
    return launch(norm_columns_kernel, (2 * a.ld + 31) / 32, 32 * kSlices, stream, a);
  });
}

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
  return size_t(blocks_for(rows, 1)) * 2 * padded(cols) * sizeof(float);
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
    a.partial = static_cast<float *>(workspace);
    if (rows == 0) {                    // nothing to add up: the column kernel writes zeros
      const hipError_t e = launch(norm_columns_kernel, (2 * a.ld + 31) / 32, 32 * kSlices, s, a);
      return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "layernorm_backward: %s", hipGetErrorString(e));
    }
  }
  const hipError_t e = dtype == MOE_SPEC_BF16 ? backward<uint16_t>(s, a) : backward<float>(s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "layernorm_backward: %s", hipGetErrorString(e));
}
