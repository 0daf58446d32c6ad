// AdamW over many tensors in as few launches as their pointers fit into.
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Bound by memory: 24 bytes an element and the gradient with 32-bit moments, 12 with 8-bit ones.  75 M elements, bf16 gradients and
// copies: 393 us, 5.4 TB/s, what a large copy reaches, and 243 us, 5.0 TB/s: 96 vector instructions an element with 8-bit moments, whose
// issue is four fifths of that time.  Eight elements a thread, 2048 a workgroup; which tensor a workgroup works on it finds in the
// launch's argument block, so that nothing has to be copied to the device first and a captured launch carries its tensors with
// it: 40 of them, 3 KB of the 4 KB that an argument block may have (55 would fit; not compared).
//
// 8-bit moments: a run of 128 elements lies in 16 lanes, whose largest magnitude four exchanges find.  With X its biased
// exponent, |m| 2^(14-X) is a float whose upper bits are the code (exponent fields 0 to 14, denormals included); adding 16
// random bits below the last one that is kept rounds up with the probability of what is cut off.  One rounding an operation
// (no contraction), IEEE division and root: parameters, moments and codes are those of the formulas in float, bit for bit.
#include "train_common.h"
#include "train_rules.h"

#include <math.h>

namespace moe_spec {
namespace {

constexpr uint32_t kOdd1 = 0x9E3779B1u, kOdd2 = 0x85EBCA77u;
static_assert(MOE_SPEC_MOMENT_BLOCK == 16 * kAdamVals, "a run of a moment block is a row of 16 lanes");

struct AdamConsts {
  float beta1, rest1, beta2, rest2, decay, alpha, root_scale, eps;
  uint32_t key;
};

struct AdamArgs {
  moe_spec_adamw_tensor t[kPerLaunch];
  uint32_t first[kPerLaunch];           // a tensor's first workgroup; behind the last tensor none that there is
  uint32_t place[kPerLaunch];           // a tensor's place in the call
  AdamConsts c;                         // valid if step_dev is null, but for what does not depend on the step
  double lr, beta1, beta2;
  const int64_t *step_dev;
  const float *scale_dev;
  float scale;
  uint32_t seed;
};
static_assert(sizeof(AdamArgs) <= 4096, "an argument block");

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * kOdd1;
  x = (x ^ (x >> 15)) * kOdd2;
  return x ^ (x >> 16);
}

// b^t by squaring, in double.
__device__ __forceinline__ double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b) if (t & 1) r *= b;
  return r;
}

// The tensor of this workgroup: the last that has begun.  Scalar work on the argument block, which is read at once.
__device__ __forceinline__ int tensor_of(const uint32_t (&first)[kPerLaunch]) {
  int which = -1;
#pragma unroll
  for (int i = 0; i < kPerLaunch; ++i) which += first[i] <= blockIdx.x;
  return which;
}

// Eight codes in two words; n of them exist.
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int n) {
  uint2 w = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) (i < 4 ? w.x : w.y) |= uint32_t(p[i]) << (8 * (i & 3));
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 w, int n) {
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) p[i] = uint8_t((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

// Values of eight first moments' codes: they are e4m3 codes with another bias, which the hardware converts two at a time.
// A power of two times it is exact, or rounded once where the value is denormal.
__device__ __forceinline__ void first_moments(uint2 w, int exponent, float (&f)[8]) {
  const float unit = ldexpf(1.0f, exponent - 134);      // 2^(X - 14) and the 2^-120 between the biases
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int word = int(i ? w.y : w.x);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(word, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
    f[4 * i] = lo[0] * unit;
    f[4 * i + 1] = lo[1] * unit;
    f[4 * i + 2] = hi[0] * unit;
    f[4 * i + 3] = hi[1] * unit;
  }
}
__device__ __forceinline__ bool has_last_code(uint32_t w) { return ((~w - 0x01010101u) & w & 0x80808080u) != 0; }
__device__ __forceinline__ void second_moments(uint2 w, int exponent, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t word = i < 4 ? w.x : w.y;
    const int up = 19 - 8 * (i & 3);                    // the code's bits go where a float's exponent and mantissa are
    f[i] = ldexpf(__uint_as_float((up > 0 ? word << up : word >> -up) & 0x07f80000u), exponent - 14);
  }
  if (has_last_code(w.x) || has_last_code(w.y)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (((i < 4 ? w.x : w.y) >> (8 * (i & 3)) & 0xff) == 0xff) f[i] = NAN;
  }
}

// Codes of eight values and the exponent of their run of 128, that is of 16 lanes' values.  random: 32 bits each, of which first
// moments take the upper half and second moments the lower one.
template <bool FIRST>
__device__ __forceinline__ uint2 encode(const float (&x)[8], const uint32_t (&random)[8], int &exponent) {
  constexpr uint32_t kInfinity = 0x7f800000u;
  constexpr int kDrop = FIRST ? 20 : 19;                // mantissa bits that go
  float y[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = x[i];
    top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  }
  const bool odd = __any(top >= kInfinity);             // seldom: an infinity or NaN somewhere, which gets its code at the end
  if (odd) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((__float_as_uint(x[i]) & 0x7fffffffu) >= kInfinity) y[i] = 0.0f;
      top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
    }
  }
  top = __float_as_uint(group_reduce<16>(__uint_as_float(top), [](float a, float b) { return fmaxf(a, b); }));
  exponent = int(top >> 23);
  uint2 w = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // fields stay below 15, so the random bits never carry into the sign
    const uint32_t bits = __float_as_uint(ldexpf(y[i], 14 - exponent)), low = FIRST ? (random[i] >> 12 & 0xffff0u) | 8u : (random[i] << 3 & 0x7fff8u) | 4u;
    const uint32_t up = bits + low;
    uint32_t code;
    if constexpr (FIRST) code = (up >> 20 & 0x7fu) | (up >> 24 & 0x80u);
    else code = max(up >> kDrop, min(__float_as_uint(y[i]), 1u));          // what is not zero does not become it
    (i < 4 ? w.x : w.y) |= code << (8 * (i & 3));
  }
  if (odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((__float_as_uint(x[i]) & 0x7fffffffu) < kInfinity) continue;
      uint32_t &word = i < 4 ? w.x : w.y;
      const uint32_t code = FIRST ? 0x7fu : 0xffu;
      word = (word & ~(0xffu << (8 * (i & 3)))) | code << (8 * (i & 3));
    }
  }
  return w;
}

// Eight elements of a thread.  WHOLE: all of the workgroup's elements exist, and its loads go out together.
template <typename GT, bool EIGHT, bool WHOLE>
__device__ __forceinline__ void adamw_elements(const moe_spec_adamw_tensor &t, const AdamConsts &c, float scale, uint32_t place, int64_t at, int n) {
#pragma clang fp contract(off)
  if constexpr (WHOLE) n = 8;
  const int64_t block = at / MOE_SPEC_MOMENT_BLOCK;
  Run<float, 8> rp, rm, rv;
  Run<GT, 8> rg;
  uint2 cm, cv;
  int em = 0, ev = 0;
  rp.load(t.p + at, n);
  rg.load(static_cast<const GT *>(t.grad) + at, n);
  if constexpr (EIGHT) {
    if constexpr (WHOLE) {
      cm = load_raw<uint2>(static_cast<const uint8_t *>(t.m) + at);
      cv = load_raw<uint2>(static_cast<const uint8_t *>(t.v) + at);
      em = t.m_exp[block];
      ev = t.v_exp[block];
    } else {
      cm = load_codes(static_cast<const uint8_t *>(t.m) + at, n);
      cv = load_codes(static_cast<const uint8_t *>(t.v) + at, n);
      if (n) em = t.m_exp[block], ev = t.v_exp[block];
    }
  } else {
    rm.load(static_cast<const float *>(t.m) + at, n);
    rv.load(static_cast<const float *>(t.v) + at, n);
  }
  float p[8], g[8], m[8], v[8];
  if constexpr (EIGHT) {
    first_moments(cm, em, m);
    second_moments(cv, ev, v);
  } else {
    rm.get(m);
    rv.get(v);
  }
  rp.get(p);
  rg.get(g);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float gi = g[i] * scale;
    m[i] = m[i] * c.beta1 + gi * c.rest1;
    v[i] = v[i] * c.beta2 + (gi * gi) * c.rest2;
    const float root = sqrtf(v[i]) * c.root_scale + c.eps;
    p[i] = p[i] * c.decay - (m[i] / root) * c.alpha;
  }
  store_run<float, 8>(t.p + at, p, n);
  if (t.copy) store_run<uint16_t, 8>(static_cast<uint16_t *>(t.copy) + at, p, n);
  if constexpr (EIGHT) {
    const uint32_t key1 = mix(c.key + kOdd2 * (place + 1)), key2 = mix(key1 ^ kOdd1);
    uint32_t random[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t x = uint32_t(at) + i + key1;
      x = (x ^ (x >> 16)) * kOdd1;
      x = ((x ^ (x >> 15)) + key2) * kOdd2;
      random[i] = x ^ (x >> 16);
    }
    cm = encode<true>(m, random, em);
    cv = encode<false>(v, random, ev);
    if constexpr (WHOLE) {
      __builtin_memcpy(static_cast<uint8_t *>(t.m) + at, &cm, 8);
      __builtin_memcpy(static_cast<uint8_t *>(t.v) + at, &cv, 8);
    } else {
      store_codes(static_cast<uint8_t *>(t.m) + at, cm, n);
      store_codes(static_cast<uint8_t *>(t.v) + at, cv, n);
    }
    if (n && threadIdx.x % 16 == 0) {
      t.m_exp[block] = uint8_t(em);
      t.v_exp[block] = uint8_t(ev);
    }
  } else {
    store_run<float, 8>(static_cast<float *>(t.m) + at, m, n);
    store_run<float, 8>(static_cast<float *>(t.v) + at, v, n);
  }
}

// 32-bit moments: four wavefronts per SIMD leave the compiler the registers to ask for everything at once (2.2 M elements 14.0 ->
// 13.4 us, 75 M 397 -> 392); 8-bit ones need eight of them for the arithmetic (15.9 us with the reading of the moments, 16.6 with four).
template <typename GT, bool EIGHT>
__global__ __launch_bounds__(kAdamBlock) __attribute__((amdgpu_waves_per_eu(EIGHT ? 8 : 4, EIGHT ? 8 : 4))) void adamw_kernel(const AdamArgs a) {
  __shared__ AdamConsts shared;
  const int which = tensor_of(a.first);
  const moe_spec_adamw_tensor t = a.t[which];
  AdamConsts c = a.c;
  if (a.step_dev) {                     // what depends on the step, by one thread
    if (threadIdx.x == 0) {
      const int64_t step = *a.step_dev > 1 ? *a.step_dev : 1;
      c.alpha = float(a.lr / (1.0 - power(a.beta1, step)));
      c.root_scale = float(1.0 / sqrt(1.0 - power(a.beta2, step)));
      c.key = mix(a.seed + kOdd1 * uint32_t(step));
      shared = c;
    }
    __syncthreads();
    c = shared;
  }
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  const int64_t begin = int64_t(blockIdx.x - a.first[which]) * kAdamChunk, at = begin + threadIdx.x * kAdamVals;
  if (begin + kAdamChunk <= t.n) {
    adamw_elements<GT, EIGHT, true>(t, c, scale, a.place[which], at, 8);
  } else {
    const int n = int(t.n - at < kAdamVals ? (t.n - at > 0 ? t.n - at : 0) : kAdamVals);
    adamw_elements<GT, EIGHT, false>(t, c, scale, a.place[which], at, n);
  }
}

struct MomentTensor {
  const uint8_t *m, *v, *m_exp, *v_exp;
  void *m_out, *v_out;
  int64_t n;
};
struct MomentArgs {
  MomentTensor t[kPerLaunch];
  uint32_t first[kPerLaunch];
};
static_assert(sizeof(MomentArgs) <= 4096, "an argument block");

template <typename OT>
__global__ __launch_bounds__(kAdamBlock) void moments_kernel(const MomentArgs a) {
  const int which = tensor_of(a.first);
  const MomentTensor t = a.t[which];
  const int64_t at = int64_t(blockIdx.x - a.first[which]) * kAdamChunk + threadIdx.x * kAdamVals, block = at / MOE_SPEC_MOMENT_BLOCK;
  const int n = int(t.n - at < kAdamVals ? t.n - at : kAdamVals);
  if (n <= 0) return;
  float m[8], v[8];
  if (n == kAdamVals && t.m_out && t.v_out) {
    const uint2 cm = load_raw<uint2>(t.m + at), cv = load_raw<uint2>(t.v + at);
    const int em = t.m_exp[block], ev = t.v_exp[block];
    first_moments(cm, em, m);
    store_run<OT, 8>(static_cast<OT *>(t.m_out) + at, m, 8);
    second_moments(cv, ev, v);
    store_run<OT, 8>(static_cast<OT *>(t.v_out) + at, v, 8);
    return;
  }
  if (t.m_out) {
    first_moments(load_codes(t.m + at, n), t.m_exp[block], m);
    store_run<OT, 8>(static_cast<OT *>(t.m_out) + at, m, n);
  }
  if (t.v_out) {
    second_moments(load_codes(t.v + at, n), t.v_exp[block], v);
    store_run<OT, 8>(static_cast<OT *>(t.v_out) + at, v, n);
  }
}

// Closes the list of a launch's first workgroups.
void no_more(uint32_t (&first)[kPerLaunch], int count) {
  for (int i = count; i < kPerLaunch; ++i) first[i] = UINT32_MAX;
}

const char *count_fault(const moe_spec_adamw_tensor *t, int n) {
  if (n < 0 || n > MOE_SPEC_TRAIN_MAX_TENSORS) return "a number of tensors out of range";
  if (n && !t) return "tensors is null";
  for (int i = 0; i < n; ++i) if (t[i].n < 0 || t[i].n > MOE_SPEC_ADAMW_MAX_ELEMENTS) return "a tensor's n is out of range";
  return nullptr;
}

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" int moe_spec_adamw_step(void *stream, const moe_spec_adamw_tensor *tensors, int n_tensors,
                                   const moe_spec_adamw_config *cfg) {
  if (!cfg) return train_fail(MOE_SPEC_EINVAL, "adamw_step: cfg is null");
  if (const char *why = count_fault(tensors, n_tensors)) return train_fail(MOE_SPEC_EINVAL, "adamw_step: %s", why);
  const bool eight = cfg->moments == MOE_SPEC_MOMENTS_8BIT;
  if (!eight && cfg->moments != MOE_SPEC_MOMENTS_32BIT) return train_fail(MOE_SPEC_EINVAL, "adamw_step: unknown moments %d", cfg->moments);
  if (!known_type(cfg->grad_dtype)) return train_fail(MOE_SPEC_EINVAL, "adamw_step: unknown grad_dtype %d", cfg->grad_dtype);
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
    return train_fail(MOE_SPEC_EINVAL, "adamw_step: beta1 and beta2 must be at least 0 and below 1");
  if (!(cfg->eps >= 0.0) || !(cfg->lr == cfg->lr) || !(cfg->weight_decay >= 0.0))
    return train_fail(MOE_SPEC_EINVAL, "adamw_step: eps or weight_decay is negative, or one of them or lr is no number");
  if (!cfg->step_dev && cfg->step < 1) return train_fail(MOE_SPEC_EINVAL, "adamw_step: step must be 1 or more");
  if (misaligned(cfg->step_dev, 8) || misaligned(cfg->grad_scale_dev, 4))
    return train_fail(MOE_SPEC_EINVAL, "adamw_step: step_dev or grad_scale_dev is not aligned to its type");
  for (int i = 0; i < n_tensors; ++i) {
    const moe_spec_adamw_tensor &t = tensors[i];
    if (t.n == 0) continue;
    if (!t.p || !t.grad || !t.m || !t.v || (eight && (!t.m_exp || !t.v_exp)))
      return train_fail(MOE_SPEC_EINVAL, "adamw_step: tensor %d has a null pointer", i);
    if (misaligned(t.p, 4) || misaligned(t.grad, size_of(cfg->grad_dtype)) || misaligned(t.copy, 2) ||
        (!eight && (misaligned(t.m, 4) || misaligned(t.v, 4))))
      return train_fail(MOE_SPEC_EINVAL, "adamw_step: tensor %d has a pointer that is not aligned to its type", i);
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "adamw_step: %s", hipGetErrorString(on.error()));
  AdamArgs a;
  a.c.beta1 = float(cfg->beta1);
  a.c.rest1 = float(1.0 - cfg->beta1);
  a.c.beta2 = float(cfg->beta2);
  a.c.rest2 = float(1.0 - cfg->beta2);
  a.c.decay = float(1.0 - cfg->lr * cfg->weight_decay);
  a.c.eps = float(cfg->eps);
  a.c.alpha = a.c.root_scale = 0.0f;
  a.c.key = 0;
  if (!cfg->step_dev) {
    a.c.alpha = float(cfg->lr / (1.0 - pow(cfg->beta1, double(cfg->step))));
    a.c.root_scale = float(1.0 / sqrt(1.0 - pow(cfg->beta2, double(cfg->step))));
    a.c.key = mix(cfg->seed + kOdd1 * uint32_t(cfg->step));
  }
  a.lr = cfg->lr; a.beta1 = cfg->beta1; a.beta2 = cfg->beta2;
  a.step_dev = cfg->step_dev; a.scale_dev = cfg->grad_scale_dev; a.scale = float(cfg->grad_scale);
  a.seed = cfg->seed;
  const bool bf16 = cfg->grad_dtype == MOE_SPEC_BF16;
  const hipError_t e = in_launches(tensors, n_tensors, [&](int slot, int i, uint32_t first) {
    a.t[slot] = tensors[i];
    a.place[slot] = uint32_t(i);
    a.first[slot] = first;
  }, [&](int count, unsigned blocks) {
    no_more(a.first, count);
    if (eight) return bf16 ? launch(adamw_kernel<uint16_t, true>, blocks, kAdamBlock, s, a) : launch(adamw_kernel<float, true>, blocks, kAdamBlock, s, a);
    return bf16 ? launch(adamw_kernel<uint16_t, false>, blocks, kAdamBlock, s, a) : launch(adamw_kernel<float, false>, blocks, kAdamBlock, s, a);
  });
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "adamw_step: %s", hipGetErrorString(e));
}

extern "C" int moe_spec_adamw_read_moments(void *stream, const moe_spec_adamw_tensor *tensors, int n_tensors, int out_dtype,
                                           void *const *m_out, void *const *v_out) {
  if (const char *why = count_fault(tensors, n_tensors)) return train_fail(MOE_SPEC_EINVAL, "adamw_read_moments: %s", why);
  if (!known_type(out_dtype)) return train_fail(MOE_SPEC_EINVAL, "adamw_read_moments: unknown out_dtype %d", out_dtype);
  if (n_tensors == 0 || (!m_out && !v_out)) return MOE_SPEC_OK;
  for (int i = 0; i < n_tensors; ++i) {
    const moe_spec_adamw_tensor &t = tensors[i];
    if (t.n == 0) continue;
    if ((m_out && (!m_out[i] || !t.m || !t.m_exp)) || (v_out && (!v_out[i] || !t.v || !t.v_exp)))
      return train_fail(MOE_SPEC_EINVAL, "adamw_read_moments: tensor %d has a null pointer", i);
    if ((m_out && misaligned(m_out[i], size_of(out_dtype))) || (v_out && misaligned(v_out[i], size_of(out_dtype))))
      return train_fail(MOE_SPEC_EINVAL, "adamw_read_moments: an output of tensor %d is not aligned to its type", i);
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  if (on.error() != hipSuccess) return train_fail(MOE_SPEC_EHIP, "adamw_read_moments: %s", hipGetErrorString(on.error()));
  MomentArgs a;
  const hipError_t e = in_launches(tensors, n_tensors, [&](int slot, int i, uint32_t first) {
    const moe_spec_adamw_tensor &t = tensors[i];
    a.t[slot] = {static_cast<const uint8_t *>(t.m), static_cast<const uint8_t *>(t.v), t.m_exp, t.v_exp,
                 m_out ? m_out[i] : nullptr, v_out ? v_out[i] : nullptr, t.n};
    a.first[slot] = first;
  }, [&](int count, unsigned blocks) {
    no_more(a.first, count);
    return out_dtype == MOE_SPEC_BF16 ? launch(moments_kernel<uint16_t>, blocks, kAdamBlock, s, a) : launch(moments_kernel<float>, blocks, kAdamBlock, s, a);
  });
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "adamw_read_moments: %s", hipGetErrorString(e));
}
