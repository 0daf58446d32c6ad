// One output tile of a float32 matrix product on the matrix cores (16x16x4 instructions, float throughout), with the interface
// of mfma_tiles.h, for operands of any stride and alignment; those of whole 16-byte chunks take the tiles there (4096 rows, 8 experts of 1024 x 2048:
// 168 us, these 201).  K is walked 32 at a time; a tile goes through registers into LDS, where rows are padded so that the one value a
// lane needs per instruction lies in a bank of its own: k-major rows of 36 floats, i-major ones of ROWS + 16.
#pragma once
#include "mfma_tiles.h"

namespace moe_spec {

template <int ROWS, bool IMAJOR, int THREADS>
struct OperandTileF32 {
  static constexpr int kStep = 32, kPitch = IMAJOR ? ROWS + 16 : kStep + 4, kFloats = IMAJOR ? kStep * kPitch : ROWS * kPitch;
  static constexpr int kChunks = ROWS * kStep / 4, kEach = kChunks / THREADS, kAcross = IMAJOR ? ROWS / 4 : kStep / 4;
  static_assert(kChunks % THREADS == 0, "whole chunks for every thread");
  const float *at[kEach];
  int64_t step;
  int rows;
  float4 held[kEach];

  // Every second step from the step `first` on.
  __device__ __forceinline__ void begin(const float *origin, int64_t ld, int rows_, int tid, int first) {
    rows = rows_;
    step = (IMAJOR ? ld * kStep : kStep) * 2;
    origin += first * (step / 2);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int c = j * THREADS + tid, r = c / kAcross, col = c % kAcross * 4;
      at[j] = origin + int64_t(IMAJOR ? r : min(r, rows - 1)) * ld + col;
    }
  }
  __device__ __forceinline__ void issue(int k_left, int tid) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int c = j * THREADS + tid, r = c / kAcross, col = c % kAcross * 4;
      const int n = IMAJOR ? (r < k_left ? rows - col : 0) : k_left - col;
      if (n >= 4) {
        held[j] = load_raw<float4>(at[j]);
      } else {
        held[j].x = n > 0 ? at[j][0] : 0.0f;
        held[j].y = n > 1 ? at[j][1] : 0.0f;
        held[j].z = n > 2 ? at[j][2] : 0.0f;
        held[j].w = 0.0f;
      }
      at[j] += step;
    }
  }
  __device__ __forceinline__ void land(float *lds, int tid) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int c = j * THREADS + tid;
      *reinterpret_cast<float4 *>(lds + c / kAcross * kPitch + c % kAcross * 4) = held[j];
    }
  }
  // Lane (i, g): row `row` + i, column k + g.
  static __device__ __forceinline__ float value(const float *lds, int row, int k, int lane) {
    const int i = row + (lane & 15), c = k + (lane >> 4);
    return IMAJOR ? lds[c * kPitch + i] : lds[i * kPitch + c];
  }
};

template <int BM, int BN, int WM, int WN, bool A_IMAJOR, bool B_IMAJOR>
struct TileProductF32 {
  static constexpr int kThreads = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
  using A = OperandTileF32<BM, A_IMAJOR, kThreads>;
  using B = OperandTileF32<BN, B_IMAJOR, kThreads>;
  static constexpr int kPart = A::kFloats + B::kFloats, kLds = 2 * kPart * 4;
  f32x4_t acc[FM][FN];

  __device__ __forceinline__ void run(char *lds_bytes, const float *a, int64_t lda, int a_rows, const float *b, int64_t ldb, int b_rows, int64_t K) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = wave / WN * (BM / WM), col = wave % WN * (BN / WN);
    float *lds = reinterpret_cast<float *>(lds_bytes);
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) acc[f][h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (K <= 0) return;
    // two steps are on their way in registers, one is in LDS while another goes there: one barrier a step
    A ta[2];
    B tb[2];
    const auto left = [](int64_t k) { return int(k < A::kStep ? (k > 0 ? k : 0) : int64_t(A::kStep)); };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ta[i].begin(a, lda, a_rows, tid, i);
      tb[i].begin(b, ldb, b_rows, tid, i);
      ta[i].issue(left(K - i * A::kStep), tid);
      tb[i].issue(left(K - i * A::kStep), tid);
    }
    const auto step = [&](int64_t k, A &now_a, B &now_b, float *part) {
      now_a.land(part, tid);
      now_b.land(part + A::kFloats, tid);
      __syncthreads();
      now_a.issue(left(k - 2 * A::kStep), tid);
      now_b.issue(left(k - 2 * A::kStep), tid);
#pragma unroll
      for (int kk = 0; kk < A::kStep; kk += 4) {
        float va[FM], vb[FN];
#pragma unroll
        for (int f = 0; f < FM; ++f) va[f] = A::value(part, row + 16 * f, kk, lane);
#pragma unroll
        for (int h = 0; h < FN; ++h) vb[h] = B::value(part + A::kFloats, col + 16 * h, kk, lane);
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int h = 0; h < FN; ++h) acc[f][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(vb[h], va[f], acc[f][h], 0, 0, 0);
      }
    };
    RunOfSums<FM, FN> sums;
    for (int64_t k = K; k > 0; k -= 2 * A::kStep) {
      step(k, ta[0], tb[0], lds);
      if (k > A::kStep) step(k - A::kStep, ta[1], tb[1], lds + kPart);
      sums.behind(acc, 2 * A::kStep);
    }
    sums.end(acc);
  }
};

}  // namespace moe_spec
