// What the training operators share: argument checks and launches on the host, rows of values in registers on the device.
#pragma once
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include "../../include/moe_spec_train.h"
#include "device_utils.h"

namespace moe_spec {

// ---- host ---------------------------------------------------------------------------------------------------
int train_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));   // keeps the text, returns the code

// Makes the stream's device the current one for the launches of a call.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(hipStream_t stream) {
    int dev = 0;
    err_ = hipGetDevice(&before_);
    if (err_ == hipSuccess && stream) err_ = hipStreamGetDevice(stream, &dev);
    if (err_ == hipSuccess && stream && dev != before_) {
      err_ = hipSetDevice(dev);
      changed_ = err_ == hipSuccess;
    }
  }
  ~OnDeviceOf() { if (changed_) (void)hipSetDevice(before_); }
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool changed_ = false;
  hipError_t err_;
};

// One kernel of one argument block.  The status is the launch's own, not what another call left behind.
template <typename Args>
hipError_t launch(void (*kernel)(Args), unsigned grid, unsigned block, hipStream_t stream, Args &args) {
  void *ptrs[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3(grid), dim3(block), ptrs, 0, stream);
}

inline bool known_type(int dtype) { return dtype == MOE_SPEC_F32 || dtype == MOE_SPEC_BF16; }
inline int size_of(int dtype) { return dtype == MOE_SPEC_F32 ? 4 : 2; }
inline bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// Why a matrix argument cannot be used, or null.
inline const char *matrix_fault(const void *p, int64_t stride, int64_t rows, int cols, int elem, bool output) {
  if (rows == 0) return nullptr;
  if (!p) return "is null";
  if (misaligned(p, elem)) return "is not aligned to its elements";
  if (rows == 1) return nullptr;
  if (stride < (output ? cols : 0)) return output ? "has a row stride below its row length" : "has a negative row stride";
  if (stride > (int64_t(1) << 31)) return "has a row stride above 2^31";
  return nullptr;
}

// ---- device -------------------------------------------------------------------------------------------------
// Sixteen bytes from or to an address that has only its elements' alignment: global memory takes such accesses whole.
template <typename Raw>
__device__ __forceinline__ Raw load_raw(const void *p) {
  Raw r;
  __builtin_memcpy(&r, p, sizeof(Raw));
  return r;
}

typedef __attribute__((ext_vector_type(2))) float float2_t;
// Two floats as two bfloat16 in a word, to nearest even; a NaN stays one.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const float2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}
__device__ __forceinline__ uint16_t to_bf16(float x) { return uint16_t(pack_bf16(x, 0.0f)); }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }
template <typename WT> __device__ __forceinline__ WT from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float x) { return to_bf16(x); }

// N values at p[0 .. N), of which the first n exist (the rest are `fill`); N a multiple of what 16 bytes hold.
template <typename WT, int N>
struct Run {
  static constexpr int V = Packed<WT>::N, R = N / V;
  using Raw = typename Packed<WT>::Raw;
  Raw raw[R];
  __device__ __forceinline__ void load(const WT *p, int n, WT fill = WT(0)) {
    if (n >= N) {
#pragma unroll
      for (int r = 0; r < R; ++r) raw[r] = load_raw<Raw>(p + r * V);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        WT e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = r * V + i < n ? p[r * V + i] : fill;
        __builtin_memcpy(&raw[r], e, sizeof(Raw));
      }
    }
  }
  // All N of them, or `fill` where there are none: nothing that is loaded is looked at here.
  __device__ __forceinline__ void load_if(bool there, const WT *p, WT fill) {
    WT e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fill;
#pragma unroll
    for (int r = 0; r < R; ++r) __builtin_memcpy(&raw[r], e, sizeof(Raw));
    if (there) {
#pragma unroll
      for (int r = 0; r < R; ++r) raw[r] = load_raw<Raw>(p + r * V);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = Raw{};
  }
  __device__ __forceinline__ void get(float (&f)[N]) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float e[V];
      Packed<WT>::unpack(raw[r], e);
#pragma unroll
      for (int i = 0; i < V; ++i) f[r * V + i] = e[i];
    }
  }
};

template <typename WT, int N>
__device__ __forceinline__ void store_run(WT *p, const float (&f)[N], int n) {
  static_assert(N % 4 == 0, "");
  if constexpr (sizeof(WT) == 4) {
    if (n >= N) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const float4 v = {f[i], f[i + 1], f[i + 2], f[i + 3]};
        __builtin_memcpy(p + i, &v, 16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) if (i < n) p[i] = f[i];
    }
  } else {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    if (n >= N) {
      if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N / 2; i += 4) {
          const uint4 v = {w[i], w[i + 1], w[i + 2], w[i + 3]};
          __builtin_memcpy(p + 2 * i, &v, 16);
        }
      } else {
        const uint2 v = {w[0], w[1]};
        __builtin_memcpy(p, &v, 8);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) if (i < n) p[i] = uint16_t(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    }
  }
}

// What lane and lane ^ 16, or lane ^ 32, hold, combined, in both.
template <typename Op>
__device__ __forceinline__ float across16(float v, Op op) {
  const auto both = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  return op(__int_as_float(int(both[0])), __int_as_float(int(both[1])));
}
template <typename Op>
__device__ __forceinline__ float across32(float v, Op op) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return op(__int_as_float(int(both[0])), __int_as_float(int(both[1])));
}

// A value combined over aligned groups of G lanes (G a power of two up to 64); every lane of a group gets it.  All lanes
// of the wavefront take part.  The order of the operands is the same in every lane of a group only up to commutation, which
// sums and maxima do not see.
template <int G, typename Op>
__device__ __forceinline__ float group_reduce(float v, Op op) {
  if constexpr (G >= 2) v = op(v, dpp_move<0xB1>(v));
  if constexpr (G >= 4) v = op(v, dpp_move<0x4E>(v));
  if constexpr (G >= 8) v = op(v, dpp_move<0x141>(v));
  if constexpr (G >= 16) v = op(v, dpp_move<0x140>(v));
  if constexpr (G >= 32) v = across16(v, op);
  if constexpr (G >= 64) v = across32(v, op);
  return v;
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
template <int G> __device__ __forceinline__ float group_sum(float v) { return group_reduce<G>(v, Add()); }

}  // namespace moe_spec
