// Losses over rows of router logits, each with its gradient in the same pass over the logits.
//
// Distillation (paper: Appendix A), p and q the softmax of the teacher's and of the student's row, n the valid rows:
//   loss = 1/n sum_t sum_e p (log p - log q),  d loss / d student = (q - p) / (n tau)
//   sum_e p (log p - log q) = sum_e p (a_e - b_e) - log A + log B  with a, b the logits less their maxima, A = sum exp a, ...
// Balance, c_e the choices of expert e and f_e = c_e / (n k):
//   loss = coef E sum_e f_e 1/n sum_t p_te = coef E / n sum_t inner_t  with inner_t = sum_e f_e p_te, the very sum that the
//   gradient needs:  d loss / d z_te = coef E / n p_te (f_e - inner_t).  So no per-expert sum of probabilities is formed.
//
// Bound by memory: logits are read once, gradients written once; the gradient's factors (n, f) come first, from the mask and
// the ids, which are a few per cent of the bytes.  A row lies in the registers of a group of 1 to 32 lanes, eight
// values each.  Exponentials go through the hardware's 2^x (a unit in its last place).  Its argument, x log2 e with x a logit less
// the row's largest over tau, has four roundings: the difference, log2 e, its quotient by tau and their product.  They move exp(x) by up to
// 4 |x| 2^-24 relative, so by at most 4 * 0.37 * 2^-24 of the row's largest term.  One reciprocal and one logarithm a row are the
// hardware's too (a unit in the last place).  Row results are added up in double.
#include "train_common.h"

#include <type_traits>

namespace moe_spec {
namespace {

// Workgroups that walk over the rows, 24 wavefronts a compute unit: 131072 rows of 128 experts with 16 / 24 / 32 / 64 of them 27.7 / 27.4 /
// 28.9 / 30.5 us (distillation).  512 threads rather than 256: half as many workgroups add up what was counted (balance 24.1 -> 23.3 us).
constexpr int kLossBlock = 512, kLossBlocks = 768, kVals = 8, kFinishBlock = 256;
constexpr int kCountBlock = 512, kCountBlocks = 128;
// Rows that one workgroup deals with in so many rounds take one launch.  A round is some 2 us of one compute unit's arithmetic, the
// two launches saved some 2.5 us each: 301 rows of 32 experts, two rounds 5.2 us, 200 rows of 128 experts, four rounds 12.3 us, in
// launches 7.7.
constexpr int kOneBlock = 1024, kOneBlockRounds = 2;
constexpr float kLog2E = 1.442695040888963f, kLn2 = 0.693147180559945f;

struct LossArgs {
  const void *z, *teacher;              // z: the student's logits, or the router's
  void *grad;
  const uint8_t *valid;
  const uint8_t *mask;                  // valid, or without one any byte that can be read, with a stride of 0: loads need no condition
  const int32_t *ids;
  int32_t *counts;
  float *loss;
  int *counted;                         // [kCountBlocks][padded_bins]: choices of each expert, then valid rows
  double *partial;                      // [blocks]
  int64_t z_stride, teacher_stride, grad_stride, ids_stride, mask_stride, rows;
  int experts, bins, top_k, blocks;     // bins: experts, or 0 where no choices are counted
  int count_blocks;                     // workgroups that count
  float inv_tau, to_log2, coef;         // to_log2: log2 e / tau
};

template <typename WT> __device__ __forceinline__ WT lowest();            // minus infinity
template <> __device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <> __device__ __forceinline__ uint16_t lowest<uint16_t>() { return 0xff80; }

struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// Adds the choices of the valid rows from `row` on, `step` apart, to hist, and the number of those rows to hist[bins].  A thread
// takes two rows at a time, whose loads go out together: without a condition (behind the end: the last row's), so that none is
// waited for before the others are out.  (Loads behind conditions: 10.7 us for 131072 rows x 8 choices, these 6.7.)  More
// workgroups count faster, and the loss kernel's add up what more of them left: the balance loss of 131072 rows takes 27.9 us with 32 of
// 1024 threads, 23.3 with 64, 22.9 with 128, 22.4 with 128 of 512 threads, 22.6 with 256.  The launch takes 5 us for 4.3 MB, of which a
// bare launch is some 2; what the other 3 are is not known (not contention: counters for groups of lanes changed nothing).
template <int UNITS>                    // four choices each
__device__ __forceinline__ int count_rows(const LossArgs &a, int64_t row, int64_t step, int *hist) {
  constexpr int kAhead = 2;
  int live = 0;
  for (; row < a.rows; row += kAhead * step) {
    int e[kAhead][4 * UNITS + 1], alive[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t at = row + u * step < a.rows ? row + u * step : a.rows - 1;
      alive[u] = a.mask[at * a.mask_stride];
      if constexpr (UNITS > 0) {
        const int32_t *ids = a.ids + at * a.ids_stride;
        if (a.top_k == 4 * UNITS) {
          __builtin_memcpy(e[u], ids, 16 * UNITS);
        } else {
#pragma unroll
          for (int j = 0; j < 4 * UNITS; ++j) e[u][j] = ids[j < a.top_k ? j : 0];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (row + u * step >= a.rows || (a.valid && !alive[u])) continue;
      ++live;
#pragma unroll
      for (int j = 0; j < 4 * UNITS; ++j)
        if (j < a.top_k && e[u][j] >= 0 && e[u][j] < a.bins) atomicAdd(&hist[e[u][j]], 1);
    }
  }
  return live;
}
__device__ __forceinline__ void count_rows(const LossArgs &a, int64_t first, int64_t step, int *hist) {
  int live;
  if (!a.bins) live = count_rows<0>(a, first, step, hist);
  else if (a.top_k <= 4) live = count_rows<1>(a, first, step, hist);
  else if (a.top_k <= 8) live = count_rows<2>(a, first, step, hist);
  else live = count_rows<4>(a, first, step, hist);
  for (int m = 1; m < kWave; m <<= 1) live += __shfl_xor(live, m);
  if (threadIdx.x % kWave == 0) atomicAdd(&hist[a.bins], live);
}

// The choices of each expert and the number of valid rows, as many as 16-byte loads take.
constexpr __host__ __device__ int padded_bins(int bins) { return (bins + 1 + 3) / 4 * 4; }

// Valid rows and their choices, a share of the rows for each workgroup.
__global__ __launch_bounds__(kCountBlock) void loss_count_kernel(const LossArgs a) {
  __shared__ int hist[padded_bins(MOE_SPEC_MAX_EXPERTS)];
  for (int i = threadIdx.x; i < padded_bins(a.bins); i += kCountBlock) hist[i] = 0;
  __syncthreads();
  count_rows(a, int64_t(blockIdx.x) * kCountBlock + threadIdx.x, int64_t(gridDim.x) * kCountBlock, hist);
  __syncthreads();
  for (int i = threadIdx.x; i < padded_bins(a.bins); i += kCountBlock) a.counted[blockIdx.x * padded_bins(a.bins) + i] = hist[i];
}

// Sum over the workgroup of one double per thread, in every thread.
template <int BLOCK>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[BLOCK / kWave];
  v = wave_sum(v);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < BLOCK / kWave; ++i) s += part[i];
  return s;
}

// ST: the logits' type; TT: the teacher's (void: balance loss); G lanes per row.  One workgroup of kOneBlock threads does it all:
// it counts for itself and writes the loss.
template <typename ST, typename TT, int G, int BLOCK>
__global__ __launch_bounds__(BLOCK) void loss_kernel(const LossArgs a) {
  constexpr bool kDistill = !__is_same(TT, void);
  using Teacher = std::conditional_t<kDistill, TT, float>;
  constexpr int kRows = BLOCK / G;
  const int lane = threadIdx.x % G, slot = threadIdx.x / G;
  // a lane's columns: [col + skip, col + count); the last lane's eight are moved back to end with the row, so that they are one load
  int col = lane * kVals, skip = 0, count = col < a.experts ? (a.experts < kVals ? a.experts : kVals) : 0;
  if (a.experts >= kVals && count && col + kVals > a.experts) {
    skip = col + kVals - a.experts;
    col = a.experts - kVals;
  }
  Run<ST, kVals> next_z;
  Run<Teacher, kVals> next_t;
  const int64_t step = int64_t(gridDim.x) * kRows, row0 = int64_t(blockIdx.x) * kRows + slot;
  const ST *from_z = static_cast<const ST *>(a.z) + row0 * a.z_stride + col;
  const Teacher *from_t = static_cast<const Teacher *>(a.teacher) + row0 * a.teacher_stride + col;
  ST *to = static_cast<ST *>(a.grad) + row0 * a.grad_stride + col;
  auto mask = [&](int64_t row) { return int(a.mask[(row < a.rows ? row : a.rows - 1) * a.mask_stride]); };
  auto fetch = [&](bool live) {         // the next of the rows, which lie a step apart
    if (a.experts >= kVals) {           // eight values or, of rows that do not count, none
      next_z.load_if(live && count, from_z, lowest<ST>());
      if constexpr (kDistill) next_t.load_if(live && count, from_t, lowest<Teacher>());
    } else {
      next_z.load(from_z, live ? count : 0, lowest<ST>());
      if constexpr (kDistill) next_t.load(from_t, live ? count : 0, lowest<Teacher>());
    }
    from_z += step * a.z_stride;
    if constexpr (kDistill) from_t += step * a.teacher_stride;
  };
  double sum = 0.0;
  int64_t row = row0;
  int ahead = mask(row + step);
  bool live = row < a.rows && (mask(row) || !a.valid);
  fetch(live);

  __shared__ int total[padded_bins(MOE_SPEC_MAX_EXPERTS)];
  const bool counting = a.bins || a.valid;
  if (counting) {                       // the valid rows and the choices, counted here or added up over what was counted
    for (int i = threadIdx.x; i < padded_bins(a.bins); i += BLOCK) total[i] = 0;
    __syncthreads();
    if constexpr (BLOCK == kOneBlock) {
      count_rows(a, threadIdx.x, BLOCK, total);
    } else {                            // four bins a load, the counting workgroups' rows over the threads
      const int quads = padded_bins(a.bins) / 4, wide = quads > 64 ? 128 : quads > 32 ? 64 : quads > 8 ? 32 : 8;
      const int q = threadIdx.x % wide, rows = BLOCK / wide;
      const int4 *from = reinterpret_cast<const int4 *>(a.counted) + (q < quads ? q : 0);
      int4 sum = {0, 0, 0, 0};
#pragma unroll 8
      for (int b = threadIdx.x / wide; b < a.count_blocks; b += rows) {
        const int4 v = from[b * quads];
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
      }
      if (q < quads) {
        atomicAdd(&total[4 * q], sum.x);
        atomicAdd(&total[4 * q + 1], sum.y);
        atomicAdd(&total[4 * q + 2], sum.z);
        atomicAdd(&total[4 * q + 3], sum.w);
      }
    }
    __syncthreads();
    if (!kDistill && blockIdx.x == 0) {
      for (int i = threadIdx.x; i < a.bins; i += BLOCK) a.counts[i] = total[i];
    }
  }
  const float n = counting ? float(total[a.bins]) : float(a.rows);
  const float share = n > 0.0f ? 1.0f / n : 0.0f;
  float f[kVals];
  float scale;
  if constexpr (kDistill) {
    scale = share * a.inv_tau;
  } else {
    scale = a.coef * float(a.experts) * share;
#pragma unroll
    for (int i = 0; i < kVals; ++i) f[i] = i < count ? float(total[col + i]) * (share / float(a.top_k)) : 0.0f;
  }

  for (int64_t first = int64_t(blockIdx.x) * kRows; first < a.rows; first += step, row += step) {
    float z[kVals], t[kVals], grad[kVals];
    next_z.get(z);
    if constexpr (kDistill) next_t.get(t);
    if (a.experts % kVals) {
#pragma unroll
      for (int i = 0; i < kVals - 1; ++i) {
        if (i >= skip) continue;
        z[i] = -INFINITY;
        if constexpr (kDistill) t[i] = -INFINITY;
      }
    }
    const bool counts = live;
    live = row + step < a.rows && (ahead || !a.valid);
    fetch(live);
    ahead = mask(row + 2 * step);
#pragma unroll
    for (int i = 0; i < kVals; ++i) grad[i] = 0.0f;
    if (__any(counts)) {                // padding lies together: whole wavefronts pass by
      float result;
      if constexpr (kDistill) {
        float top_z = -INFINITY, top_t = -INFINITY;
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
          top_z = fmaxf(top_z, z[i]);
          top_t = fmaxf(top_t, t[i]);
        }
        top_z = group_reduce<G>(top_z, Max());
        top_t = group_reduce<G>(top_t, Max());
        if (top_z == -INFINITY) top_z = 0.0f;
        if (top_t == -INFINITY) top_t = 0.0f;
        float sum_z = 0.0f, sum_t = 0.0f, cross = 0.0f, apart = 0.0f, p[kVals];
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
          z[i] -= top_z;
          t[i] -= top_t;
          sum_z += grad[i] = __builtin_amdgcn_exp2f(z[i] * a.to_log2);
          sum_t += p[i] = __builtin_amdgcn_exp2f(t[i] * a.to_log2);
        }
        sum_z = group_sum<G>(sum_z);
        sum_t = group_sum<G>(sum_t);
        const bool empty = sum_z == 0.0f;                                  // the student's row is masked out whole
        const float inv_t = sum_t == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum_t), over_z = empty ? 0.0f : __builtin_amdgcn_rcpf(sum_z) * scale;
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
          p[i] *= inv_t;
          cross += p[i] == 0.0f ? 0.0f : p[i] * (t[i] - z[i]);             // 0 log 0 = 0
          apart = fmaxf(apart, t[i] - z[i]);                               // both minus infinity: NaN, which fmaxf passes over
          grad[i] = grad[i] * over_z - p[i] * scale;
        }
        if (apart == INFINITY) cross = INFINITY;                           // the student's alone is, however small p is
        cross = group_sum<G>(cross);
        result = cross * a.inv_tau + kLn2 * ((empty ? 0.0f : __builtin_amdgcn_logf(sum_z)) - __builtin_amdgcn_logf(sum_t));
        if (sum_t == 0.0f || !counts) {                                    // nothing to teach, the teacher's row is masked out whole
          result = 0.0f;
#pragma unroll
          for (int i = 0; i < kVals; ++i) grad[i] = 0.0f;
        }
      } else {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kVals; ++i) top = fmaxf(top, z[i]);
        top = group_reduce<G>(top, Max());
        if (top == -INFINITY) top = 0.0f;
        float total_e = 0.0f, inner = 0.0f;
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
          z[i] = __builtin_amdgcn_exp2f((z[i] - top) * a.to_log2);
          total_e += z[i];
          inner += z[i] * f[i];
        }
        total_e = group_sum<G>(total_e);
        inner = group_sum<G>(inner);
        const float inv = total_e == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(total_e), over = inv * scale;
        result = inner * inv;           // a row that does not count holds minus infinities: zeros from here on
#pragma unroll
        for (int i = 0; i < kVals; ++i) grad[i] = z[i] * ((f[i] - result) * over);
      }
      if (lane == 0) sum += double(result);
    }
    if (a.grad && row < a.rows && count) {
      if (!skip) {
        store_run<ST, kVals>(to, grad, count);
      } else {
#pragma unroll
        for (int i = 1; i < kVals; ++i) if (i >= skip) to[i] = from_float<ST>(grad[i]);
      }
    }
    to += step * a.grad_stride;
  }
  sum = block_sum<BLOCK>(sum) * double(kDistill ? share : scale);
  if (threadIdx.x == 0) {
    if (BLOCK == kOneBlock) *a.loss = float(sum);
    else a.partial[blockIdx.x] = sum;
  }
}

__global__ __launch_bounds__(kFinishBlock) void loss_finish_kernel(const LossArgs a) {
  double s = 0.0;
#pragma unroll
  for (int i = threadIdx.x; i < kLossBlocks; i += kFinishBlock) s += i < a.blocks ? a.partial[i] : 0.0;
  s = block_sum<kFinishBlock>(s);
  if (threadIdx.x == 0) *a.loss = float(s);
}

// No rows: a loss of zero, no choices.
__global__ void loss_none_kernel(const LossArgs a) {
  if (threadIdx.x == 0) *a.loss = 0.0f;
  if (a.counts && int(threadIdx.x) < a.experts) a.counts[threadIdx.x] = 0;
}

int lanes_for(int experts) {
  int g = 1;
  while (g * kVals < experts) g *= 2;
  return g;
}
bool in_one_block(int64_t rows, int experts) { return rows * lanes_for(experts) <= int64_t(kOneBlock) * kOneBlockRounds; }

template <typename ST, typename TT, int G>
hipError_t run_loss(hipStream_t stream, LossArgs &a) {
  if (in_one_block(a.rows, a.experts)) return launch(loss_kernel<ST, TT, G, kOneBlock>, 1, kOneBlock, stream, a);
  const int64_t need = (a.rows + kLossBlock / G - 1) / (kLossBlock / G);
  a.blocks = int(need < kLossBlocks ? need : kLossBlocks);
  hipError_t e = hipSuccess;
  if (a.bins || a.valid) {
    const int64_t need = (a.rows + 2 * kCountBlock - 1) / (2 * kCountBlock);
    a.count_blocks = int(need < kCountBlocks ? need : kCountBlocks);
    e = launch(loss_count_kernel, a.count_blocks, kCountBlock, stream, a);
  }
  if (e == hipSuccess) e = launch(loss_kernel<ST, TT, G, kLossBlock>, a.blocks, kLossBlock, stream, a);
  if (e == hipSuccess) e = launch(loss_finish_kernel, 1, kFinishBlock, stream, a);
  return e;
}

template <typename ST, typename TT>
hipError_t run_loss(hipStream_t stream, LossArgs &a) {
  a.mask = a.valid ? a.valid : static_cast<const uint8_t *>(a.z);
  a.mask_stride = a.valid ? 1 : 0;
  if (a.rows == 0) return launch(loss_none_kernel, 1, MOE_SPEC_MAX_EXPERTS, stream, a);
  switch (lanes_for(a.experts)) {
    case 1: return run_loss<ST, TT, 1>(stream, a);
    case 2: return run_loss<ST, TT, 2>(stream, a);
    case 4: return run_loss<ST, TT, 4>(stream, a);
    case 8: return run_loss<ST, TT, 8>(stream, a);
    case 16: return run_loss<ST, TT, 16>(stream, a);
    default: return run_loss<ST, TT, 32>(stream, a);
  }
}

size_t partial_bytes() { return kLossBlocks * sizeof(double); }
size_t counted_bytes(int bins) { return size_t(kCountBlocks) * padded_bins(bins) * sizeof(int); }

bool sizes_fit(int64_t rows, int experts) {
  return rows >= 0 && rows <= MOE_SPEC_TRAIN_MAX_ROWS && experts >= 1 && experts <= MOE_SPEC_MAX_EXPERTS;
}

const char *grad_fault(const void *grad, int64_t grad_stride, const void *z, int64_t z_stride, int64_t rows, int cols, int elem) {
  if (!grad) return nullptr;
  if (const char *why = matrix_fault(grad, grad_stride, rows, cols, elem, true)) return why;
  if (grad == z && grad_stride != z_stride && rows > 1) return "has another stride than the logits it overwrites";
  return nullptr;
}

const char *workspace_fault(const void *workspace, size_t bytes, size_t need) {
  if (need == 0) return nullptr;
  if (!workspace || misaligned(workspace, 16)) return "must be given and aligned to 16 bytes";
  return bytes < need ? "is too small" : nullptr;
}

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" size_t moe_spec_distill_loss_workspace_bytes(int64_t rows, int n_experts) {
  return sizes_fit(rows, n_experts) && !in_one_block(rows, n_experts) ? partial_bytes() + counted_bytes(0) : 0;
}

extern "C" size_t moe_spec_balance_loss_workspace_bytes(int64_t rows, int n_experts, int top_k) {
  if (!sizes_fit(rows, n_experts) || top_k < 1 || top_k > MOE_SPEC_MAX_TOP_K) return 0;
  return in_one_block(rows, n_experts) ? 0 : partial_bytes() + counted_bytes(n_experts);
}

extern "C" int moe_spec_distill_loss(void *stream, int student_dtype, const void *student, int64_t student_stride,
                                     int teacher_dtype, const void *teacher, int64_t teacher_stride, int64_t rows,
                                     int n_experts, float temperature, const uint8_t *valid, float *loss, void *grad,
                                     int64_t grad_stride, void *workspace, size_t workspace_bytes) {
  if (!known_type(student_dtype) || !known_type(teacher_dtype)) return train_fail(MOE_SPEC_EINVAL, "distill_loss: unknown dtype");
  if (!sizes_fit(rows, n_experts)) return train_fail(MOE_SPEC_EINVAL, "distill_loss: rows or n_experts out of range");
  const float to_log2 = kLog2E / temperature;
  if (!(temperature > 0.0f) || !(1.0f / temperature > 0.0f) || !(to_log2 < INFINITY))
    return train_fail(MOE_SPEC_EINVAL, "distill_loss: temperature must be positive and finite, and so 1.5 times its reciprocal");
  if (const char *why = matrix_fault(student, student_stride, rows, n_experts, size_of(student_dtype), false))
    return train_fail(MOE_SPEC_EINVAL, "distill_loss: student %s", why);
  if (const char *why = matrix_fault(teacher, teacher_stride, rows, n_experts, size_of(teacher_dtype), false))
    return train_fail(MOE_SPEC_EINVAL, "distill_loss: teacher %s", why);
  if (const char *why = grad_fault(grad, grad_stride, student, student_stride, rows, n_experts, size_of(student_dtype)))
    return train_fail(MOE_SPEC_EINVAL, "distill_loss: grad %s", why);
  if (grad && grad == teacher) return train_fail(MOE_SPEC_EINVAL, "distill_loss: grad must not be the teacher");
  if (!loss || misaligned(loss, 4)) return train_fail(MOE_SPEC_EINVAL, "distill_loss: loss is null or not aligned to 4 bytes");
  if (const char *why = workspace_fault(workspace, workspace_bytes, moe_spec_distill_loss_workspace_bytes(rows, n_experts)))
    return train_fail(MOE_SPEC_EINVAL, "distill_loss: the workspace %s", why);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "distill_loss: %s", hipGetErrorString(on.error()));
  LossArgs a = {};
  a.z = student; a.teacher = teacher; a.grad = grad; a.valid = valid; a.loss = loss;
  a.z_stride = student_stride; a.teacher_stride = teacher_stride; a.grad_stride = grad_stride; a.rows = rows;
  a.experts = n_experts; a.inv_tau = 1.0f / temperature; a.to_log2 = to_log2;
  a.partial = static_cast<double *>(workspace);
  if (workspace) a.counted = reinterpret_cast<int *>(static_cast<char *>(workspace) + partial_bytes());
  hipError_t e;
  if (student_dtype == MOE_SPEC_BF16)
    e = teacher_dtype == MOE_SPEC_BF16 ? run_loss<uint16_t, uint16_t>(s, a) : run_loss<uint16_t, float>(s, a);
  else
    e = teacher_dtype == MOE_SPEC_BF16 ? run_loss<float, uint16_t>(s, a) : run_loss<float, float>(s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "distill_loss: %s", hipGetErrorString(e));
}

extern "C" int moe_spec_balance_loss(void *stream, int dtype, const void *logits, int64_t logits_stride, int64_t rows,
                                     int n_experts, const int32_t *ids, int64_t ids_stride, int top_k, float coef,
                                     const uint8_t *valid, float *loss, int32_t *counts, void *grad, int64_t grad_stride,
                                     void *workspace, size_t workspace_bytes) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "balance_loss: unknown dtype %d", dtype);
  if (!sizes_fit(rows, n_experts)) return train_fail(MOE_SPEC_EINVAL, "balance_loss: rows or n_experts out of range");
  if (top_k < 1 || top_k > MOE_SPEC_MAX_TOP_K || rows * top_k > INT32_MAX)
    return train_fail(MOE_SPEC_EINVAL, "balance_loss: top_k must be 1 to %d and rows * top_k below 2^31", MOE_SPEC_MAX_TOP_K);
  if (!(fabsf(coef) < INFINITY)) return train_fail(MOE_SPEC_EINVAL, "balance_loss: coef is not finite");
  if (const char *why = matrix_fault(logits, logits_stride, rows, n_experts, size_of(dtype), false))
    return train_fail(MOE_SPEC_EINVAL, "balance_loss: logits %s", why);
  if (const char *why = matrix_fault(ids, ids_stride, rows, top_k, 4, false)) return train_fail(MOE_SPEC_EINVAL, "balance_loss: ids %s", why);
  if (const char *why = grad_fault(grad, grad_stride, logits, logits_stride, rows, n_experts, size_of(dtype)))
    return train_fail(MOE_SPEC_EINVAL, "balance_loss: grad %s", why);
  if (!loss || misaligned(loss, 4) || !counts || misaligned(counts, 4))
    return train_fail(MOE_SPEC_EINVAL, "balance_loss: loss or counts is null or not aligned to 4 bytes");
  if (const char *why = workspace_fault(workspace, workspace_bytes, moe_spec_balance_loss_workspace_bytes(rows, n_experts, top_k)))
    return train_fail(MOE_SPEC_EINVAL, "balance_loss: the workspace %s", why);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "balance_loss: %s", hipGetErrorString(on.error()));
  LossArgs a = {};
  a.z = logits; a.grad = grad; a.valid = valid; a.ids = ids; a.loss = loss; a.counts = counts;
  a.z_stride = logits_stride; a.grad_stride = grad_stride; a.ids_stride = ids_stride; a.rows = rows;
  a.experts = a.bins = n_experts; a.top_k = top_k; a.coef = coef; a.inv_tau = 1.0f; a.to_log2 = kLog2E;
  a.partial = static_cast<double *>(workspace);
  if (workspace) a.counted = reinterpret_cast<int *>(static_cast<char *>(workspace) + partial_bytes());
  const hipError_t e = dtype == MOE_SPEC_BF16 ? run_loss<uint16_t, void>(s, a) : run_loss<float, void>(s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "balance_loss: %s", hipGetErrorString(e));
}
