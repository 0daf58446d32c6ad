// The experts' gated activation, with a weight for each row (the gate of that choice: the down projection is linear, so weighting its input
// weights its output):
//   h = w silu(g) u;   dg = w dh u s (1 + g (1 - s)),  du = w dh g s,  dw = sum over the row of dh g s u;   s = 1 / (1 + exp(-g))
// Bound by memory: three values are moved for one in the forward pass, five in the backward pass.  A row has 8, 64 or 256 threads by its
// length, eight values each at a time, and sums what its weight's gradient needs on the way.
#include "train_common.h"

namespace moe_spec {
namespace {

struct GatedArgs {
  const void *a, *dh;
  void *out;                    // h, or da
  const float *weight;
  float *dweight;
  int64_t a_stride, dh_stride, out_stride, rows;
  int cols;
};

constexpr int kGatedBlock = 256;

// 1 / (1 + exp(-g)).  With bfloat16 the hardware's 2^x and reciprocal: their errors and that of the exponent's rounding, which grows with it, come to
// (2 |g| + 6) 2^-24 of the result, 2^-16 at |g| = 88, where it is next to zero, against the 2^-9 of what goes in and out; with float the
// library's exponential and a division.
template <typename WT> __device__ __forceinline__ float sigmoid(float g);
template <> __device__ __forceinline__ float sigmoid<uint16_t>(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
template <> __device__ __forceinline__ float sigmoid<float>(float g) { return 1.0f / (1.0f + expf(-g)); }

template <typename WT, int LANES, bool BACKWARD>
__global__ __launch_bounds__(kGatedBlock) void gated_kernel(const GatedArgs a) {
  constexpr int kRows = kGatedBlock / LANES;
  const int lane = threadIdx.x % LANES;
  __shared__ float part[kGatedBlock / 64];
  for (int64_t first = int64_t(blockIdx.x) * kRows; first < a.rows; first += int64_t(gridDim.x) * kRows) {
    const int64_t row = first + threadIdx.x / LANES;
    const bool there = row < a.rows;
    float sum = 0.0f;
    if (there) {
      const WT *gate = static_cast<const WT *>(a.a) + row * a.a_stride, *up = gate + a.cols;
      const WT *dh = BACKWARD ? static_cast<const WT *>(a.dh) + row * a.dh_stride : nullptr;
      WT *out = static_cast<WT *>(a.out) + row * a.out_stride;
      const float weight = a.weight ? a.weight[row] : 1.0f;
      for (int c = lane * 8; c < a.cols; c += LANES * 8) {
        const int n = a.cols - c;
        Run<WT, 8> rg, ru, rd;
        rg.load(gate + c, n);
        ru.load(up + c, n);
        if constexpr (BACKWARD) rd.load(dh + c, n);
        float g[8], u[8], d[8], x[8], y[8];
        rg.get(g);
        ru.get(u);
        if constexpr (BACKWARD) rd.get(d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float s = sigmoid<WT>(g[i]), act = g[i] * s;
          if constexpr (BACKWARD) {
            const float wd = d[i] * weight;
            if (i < n) sum += d[i] * act * u[i];
            x[i] = wd * u[i] * s * (1.0f + g[i] * (1.0f - s));
            y[i] = wd * act;
          } else {
            x[i] = act * u[i] * weight;
          }
        }
        store_run<WT, 8>(out + c, x, n);
        if constexpr (BACKWARD) store_run<WT, 8>(out + a.cols + c, y, n);
      }
    }
    if constexpr (BACKWARD) {
      if (a.dweight) {                          // the same for the whole workgroup
        sum = group_sum<(LANES < 64 ? LANES : 64)>(sum);
        if constexpr (LANES > 64) {
          if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
          __syncthreads();
          sum = (part[0] + part[1]) + (part[2] + part[3]);
          __syncthreads();
        }
        if (there && lane == 0) a.dweight[row] = sum;
      }
    }
  }
}

// Lanes by a row's chunks of eight: 8 up to 16 chunks, 64 up to 256, a whole workgroup beyond.
template <typename WT, bool BACKWARD>
hipError_t go_gated(GatedArgs &a, hipStream_t s) {
  const int chunks = (a.cols + 7) / 8, lanes = chunks <= 16 ? 8 : chunks <= 256 ? 64 : 256;
  const int64_t blocks = (a.rows + kGatedBlock / lanes - 1) / (kGatedBlock / lanes);
  const unsigned grid = unsigned(blocks < 65536 ? blocks : 65536);
  if (lanes == 8) return launch(gated_kernel<WT, 8, BACKWARD>, grid, kGatedBlock, s, a);
  if (lanes == 64) return launch(gated_kernel<WT, 64, BACKWARD>, grid, kGatedBlock, s, a);
  return launch(gated_kernel<WT, 256, BACKWARD>, grid, kGatedBlock, s, a);
}

// Checks and launch of either direction; dh null: forward.
int gated(const char *name, bool backward, void *stream, int dtype, const void *dh, int64_t dh_stride, const void *a, int64_t a_stride,
          int64_t rows, int cols, const float *weight, void *out, int64_t out_stride, float *dweight) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "%s: unknown dtype %d", name, dtype);
  if (rows < 0 || rows > MOE_SPEC_TRAIN_MAX_ROWS) return train_fail(MOE_SPEC_EINVAL, "%s: rows must be between 0 and 2^31 - 1", name);
  if (cols < 1 || cols > MOE_SPEC_TRAIN_MAX_FEATURES) return train_fail(MOE_SPEC_EINVAL, "%s: cols must be between 1 and 65536", name);
  const int elem = size_of(dtype), out_cols = backward ? 2 * cols : cols;
  if (const char *why = matrix_fault(a, a_stride, rows, 2 * cols, elem, false)) return train_fail(MOE_SPEC_EINVAL, "%s: a %s", name, why);
  if (const char *why = backward ? matrix_fault(dh, dh_stride, rows, cols, elem, false) : nullptr) return train_fail(MOE_SPEC_EINVAL, "%s: dh %s", name, why);
  if (const char *why = matrix_fault(out, out_stride, rows, out_cols, elem, true)) return train_fail(MOE_SPEC_EINVAL, "%s: %s %s", name, backward ? "da" : "h", why);
  if (misaligned(weight, 4) || misaligned(dweight, 4)) return train_fail(MOE_SPEC_EINVAL, "%s: weight or dweight is not aligned to its elements", name);
  if (rows && (out == a || (backward && out == dh))) return train_fail(MOE_SPEC_EINVAL, "%s: %s must not be an input", name, backward ? "da" : "h");
  if (rows == 0) return MOE_SPEC_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "%s: %s", name, hipGetErrorString(on.error()));
  GatedArgs args{a, dh, out, weight, dweight, a_stride, dh_stride, out_stride, rows, cols};
  const bool bf16 = dtype == MOE_SPEC_BF16;
  const hipError_t e = backward ? (bf16 ? go_gated<uint16_t, true>(args, s) : go_gated<float, true>(args, s))
                                : (bf16 ? go_gated<uint16_t, false>(args, s) : go_gated<float, false>(args, s));
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "%s: %s", name, hipGetErrorString(e));
}

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" int moe_spec_swiglu_forward(void *stream, int dtype, const void *a, int64_t a_stride, int64_t rows, int cols, const float *weight,
                                       void *h, int64_t h_stride) {
  return gated("swiglu_forward", false, stream, dtype, nullptr, 0, a, a_stride, rows, cols, weight, h, h_stride, nullptr);
}

extern "C" int moe_spec_swiglu_backward(void *stream, int dtype, const void *dh, int64_t dh_stride, const void *a, int64_t a_stride, int64_t rows,
                                        int cols, const float *weight, void *da, int64_t da_stride, float *dweight) {
  return gated("swiglu_backward", true, stream, dtype, dh, dh_stride, a, a_stride, rows, cols, weight, da, da_stride, dweight);
}
