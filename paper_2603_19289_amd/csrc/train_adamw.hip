// AdamW over many tensors in as few launches as their pointers fit into.
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Bound by memory: 24 bytes an element and the gradient with 32-bit moments, 12 with 8-bit ones.  Eight elements a thread,
// 2048 a workgroup; which tensor a workgroup works on it finds in the launch's argument block, so that nothing has to be
// copied to the device first and a captured launch carries its tensors with it.
//
// 8-bit moments: a run of 128 elements lies in 16 lanes, whose largest magnitude four exchanges find.  With X its biased
// exponent, |m| 2^(14-X) is a float whose upper bits are the code (exponent fields 0 to 14, denormals included); adding 16
// random bits below the last one that is kept rounds up with the probability of what is cut off.  One rounding an operation
// (no contraction), IEEE division and root, so that the codes are those of the formulas in float.
#include "train_common.h"

#include <math.h>

namespace moe_spec {
namespace {

constexpr int kAdamBlock = 256, kAdamVals = 8, kAdamChunk = kAdamBlock * kAdamVals, kPerLaunch = 40;
constexpr uint32_t kOdd1 = 0x9E3779B1u, kOdd2 = 0x85EBCA77u;
static_assert(kPerLaunch < kWave, "a wavefront looks through the table of a launch");
static_assert(MOE_SPEC_MOMENT_BLOCK == 16 * kAdamVals, "a run of a moment block is a row of 16 lanes");

struct AdamConsts {
  float beta1, rest1, beta2, rest2, decay, alpha, root_scale, eps;
  uint32_t key;
};

struct AdamArgs {
  moe_spec_adamw_tensor t[kPerLaunch];
  uint32_t first[kPerLaunch];           // a tensor's first workgroup
  uint32_t place[kPerLaunch];           // a tensor's place in the call
  int count;
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

// The tensor of this workgroup and its first element there.
__device__ __forceinline__ int tensor_of(const uint32_t *first, int count) {
  const int lane = threadIdx.x % kWave;
  const bool begun = lane < count && first[lane] <= blockIdx.x;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(begun)) - 1);
}

__device__ __forceinline__ float decode(uint32_t size, int drop, int exponent) { return ldexpf(__uint_as_float(size << drop), exponent - 14); }

// Eight codes in two words.
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int n) {
  uint2 w = {0, 0};
  if (n >= 8) return load_raw<uint2>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) (i < 4 ? w.x : w.y) |= uint32_t(p[i]) << (8 * (i & 3));
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 w, int n) {
  if (n >= 8) { __builtin_memcpy(p, &w, 8); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) p[i] = uint8_t((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}
__device__ __forceinline__ uint32_t code_at(const uint2 &w, int i) { return ((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 0xff; }

// The value of a first moment's code, or of a second one's.
__device__ __forceinline__ float first_moment(uint32_t code, int exponent) {
  const float size = (code & 0x7f) == 0x7f ? NAN : decode(code & 0x7f, 20, exponent);
  return code & 0x80 ? -size : size;
}
__device__ __forceinline__ float second_moment(uint32_t code, int exponent) {
  return code == 0xff ? NAN : decode(code, 19, exponent);
}

// Codes of eight values and the exponent of their run of 128; `noise`: 16 random bits each.
template <int DROP>
__device__ __forceinline__ uint2 encode(const float (&x)[8], const uint32_t (&noise)[8], int &exponent) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float size = fabsf(x[i]);
    top = fmaxf(top, size < INFINITY ? size : 0.0f);
  }
  top = group_reduce<16>(top, [](float a, float b) { return fmaxf(a, b); });
  exponent = int(__float_as_uint(top) >> 23);
  uint2 w = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float size = fabsf(x[i]);
    uint32_t code = (__float_as_uint(ldexpf(size, 14 - exponent)) + (noise[i] << (DROP - 16)) + (1u << (DROP - 17))) >> DROP;
    if (!(size < INFINITY)) code = DROP == 20 ? 0x7f : 0xff;
    if constexpr (DROP == 20) code |= (__float_as_uint(x[i]) >> 31) << 7;
    else if (size > 0.0f && code == 0) code = 1;
    (i < 4 ? w.x : w.y) |= code << (8 * (i & 3));
  }
  return w;
}

template <typename GT, bool EIGHT>
__global__ __launch_bounds__(kAdamBlock) void adamw_kernel(const AdamArgs a) {
#pragma clang fp contract(off)
  __shared__ AdamConsts shared;
  AdamConsts c = a.c;
  if (a.step_dev) {                     // what depends on the step, by one thread
    if (threadIdx.x == 0) {
      const int64_t t = *a.step_dev;
      c.alpha = float(a.lr / (1.0 - power(a.beta1, t)));
      c.root_scale = float(1.0 / sqrt(1.0 - power(a.beta2, t)));
      c.key = mix(a.seed + kOdd1 * uint32_t(t));
      shared = c;
    }
    __syncthreads();
    c = shared;
  }
  const float scale = a.scale_dev ? a.scale * *a.scale_dev : a.scale;
  const int which = tensor_of(a.first, a.count);
  const moe_spec_adamw_tensor &t = a.t[which];
  const int64_t at = int64_t(blockIdx.x - a.first[which]) * kAdamChunk + threadIdx.x * kAdamVals;
  const int n = int(t.n - at < kAdamVals ? (t.n - at > 0 ? t.n - at : 0) : kAdamVals);
  Run<float, 8> rp;
  Run<GT, 8> rg;
  rp.load(t.p + at, n);
  rg.load(static_cast<const GT *>(t.grad) + at, n);
  float p[8], g[8], m[8], v[8];
  if constexpr (EIGHT) {
    const uint2 cm = load_codes(static_cast<const uint8_t *>(t.m) + at, n), cv = load_codes(static_cast<const uint8_t *>(t.v) + at, n);
    const int em = n ? t.m_exp[at / MOE_SPEC_MOMENT_BLOCK] : 0, ev = n ? t.v_exp[at / MOE_SPEC_MOMENT_BLOCK] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = first_moment(code_at(cm, i), em);
      v[i] = second_moment(code_at(cv, i), ev);
    }
  } else {
    Run<float, 8> r;
    r.load(static_cast<const float *>(t.m) + at, n);
    r.get(m);
    r.load(static_cast<const float *>(t.v) + at, n);
    r.get(v);
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
    const uint32_t key1 = mix(c.key + kOdd2 * (a.place[which] + 1)), key2 = mix(key1 ^ kOdd1);
    uint32_t up_m[8], up_v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t x = uint32_t(at) + i + key1;
      x = (x ^ (x >> 16)) * kOdd1;
      x = ((x ^ (x >> 15)) + key2) * kOdd2;
      x ^= x >> 16;
      up_m[i] = x >> 16;
      up_v[i] = x & 0xffff;
    }
    int em, ev;
    const uint2 cm = encode<20>(m, up_m, em), cv = encode<19>(v, up_v, ev);
    store_codes(static_cast<uint8_t *>(t.m) + at, cm, n);
    store_codes(static_cast<uint8_t *>(t.v) + at, cv, n);
    if (n && threadIdx.x % 16 == 0) {
      t.m_exp[at / MOE_SPEC_MOMENT_BLOCK] = uint8_t(em);
      t.v_exp[at / MOE_SPEC_MOMENT_BLOCK] = uint8_t(ev);
    }
  } else {
    store_run<float, 8>(static_cast<float *>(t.m) + at, m, n);
    store_run<float, 8>(static_cast<float *>(t.v) + at, v, n);
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
  int count;
};
static_assert(sizeof(MomentArgs) <= 4096, "an argument block");

template <typename OT>
__global__ __launch_bounds__(kAdamBlock) void moments_kernel(const MomentArgs a) {
  const int which = tensor_of(a.first, a.count);
  const MomentTensor &t = a.t[which];
  const int64_t at = int64_t(blockIdx.x - a.first[which]) * kAdamChunk + threadIdx.x * kAdamVals;
  const int n = int(t.n - at < kAdamVals ? t.n - at : kAdamVals);
  if (n <= 0) return;
  float f[8];
  if (t.m_out) {
    const uint2 w = load_codes(t.m + at, n);
    const int e = t.m_exp[at / MOE_SPEC_MOMENT_BLOCK];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = first_moment(code_at(w, i), e);
    store_run<OT, 8>(static_cast<OT *>(t.m_out) + at, f, n);
  }
  if (t.v_out) {
    const uint2 w = load_codes(t.v + at, n);
    const int e = t.v_exp[at / MOE_SPEC_MOMENT_BLOCK];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = second_moment(code_at(w, i), e);
    store_run<OT, 8>(static_cast<OT *>(t.v_out) + at, f, n);
  }
}

// Deals the tensors to launches: as many as an argument block holds and as workgroups fit a grid.  `put` fills in one.
template <typename Args, typename Put, typename Go>
hipError_t in_launches(const moe_spec_adamw_tensor *tensors, int n_tensors, Args &a, Put put, Go go) {
  constexpr int64_t kMostBlocks = 1 << 30;
  int64_t blocks = 0;
  a.count = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const int64_t need = (tensors[i].n + kAdamChunk - 1) / kAdamChunk;
    if (need == 0) continue;
    if (a.count == kPerLaunch || (a.count && blocks + need > kMostBlocks)) {
      const hipError_t e = go(unsigned(blocks));
      if (e != hipSuccess) return e;
      a.count = 0;
      blocks = 0;
    }
    a.first[a.count] = uint32_t(blocks);
    put(a.count++, i);
    blocks += need;
  }
  return a.count ? go(unsigned(blocks)) : hipSuccess;
}

const char *count_fault(const moe_spec_adamw_tensor *t, int n) {
  if (n < 0 || n > MOE_SPEC_TRAIN_MAX_TENSORS) return "a number of tensors out of range";
  if (n && !t) return "tensors is null";
  for (int i = 0; i < n; ++i) if (t[i].n < 0 || t[i].n > (int64_t(1) << 40)) return "a tensor's n is out of range";
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
  const hipError_t e = in_launches(tensors, n_tensors, a, [&](int slot, int i) { a.t[slot] = tensors[i]; a.place[slot] = uint32_t(i); }, [&](unsigned blocks) {
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
  const hipError_t e = in_launches(tensors, n_tensors, a, [&](int slot, int i) {
    const moe_spec_adamw_tensor &t = tensors[i];
    a.t[slot] = {static_cast<const uint8_t *>(t.m), static_cast<const uint8_t *>(t.v), t.m_exp, t.v_exp,
                 m_out ? m_out[i] : nullptr, v_out ? v_out[i] : nullptr, t.n};
  }, [&](unsigned blocks) {
    return out_dtype == MOE_SPEC_BF16 ? launch(moments_kernel<uint16_t>, blocks, kAdamBlock, s, a) : launch(moments_kernel<float>, blocks, kAdamBlock, s, a);
  });
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "adamw_read_moments: %s", hipGetErrorString(e));
}
