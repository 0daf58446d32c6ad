// How the tensors of an AdamW call are dealt to launches.  Plain C++, so that it can be swept on the CPU.
#pragma once
#include <stdint.h>

#include "../../include/moe_spec_train.h"

namespace moe_spec {

constexpr int kAdamBlock = 256, kAdamVals = 8, kAdamChunk = kAdamBlock * kAdamVals, kPerLaunch = 40;
constexpr int64_t kAdamMostBlocks = (int64_t(1) << 32) / kAdamBlock - 1;        // a grid has fewer than 2^32 threads
static_assert(kAdamMostBlocks * kAdamChunk == MOE_SPEC_ADAMW_MAX_ELEMENTS, "a tensor fits a launch");

// As many tensors a launch as an argument block holds and as workgroups fit a grid; tensors without elements have no place.
// put(slot, tensor, first workgroup) fills one in, go(tensors, workgroups) launches and returns 0 or what ends the call.
template <typename Put, typename Go>
auto in_launches(const moe_spec_adamw_tensor *tensors, int n_tensors, Put put, Go go) -> decltype(go(0, 0u)) {
  using Status = decltype(go(0, 0u));
  int64_t blocks = 0;
  int count = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const int64_t need = (tensors[i].n + kAdamChunk - 1) / kAdamChunk;
    if (need == 0) continue;
    if (count == kPerLaunch || (count && blocks + need > kAdamMostBlocks)) {
      const Status e = go(count, unsigned(blocks));
      if (e != Status(0)) return e;
      count = 0;
      blocks = 0;
    }
    put(count++, i, uint32_t(blocks));
    blocks += need;
  }
  return count ? go(count, unsigned(blocks)) : Status(0);
}

}  // namespace moe_spec
