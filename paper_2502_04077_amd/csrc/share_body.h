// Device code that the kernels on rows behind a shared beginning have in common.
#pragma once

#include "cache_body.h"
#include "share_internal.h"

namespace ap {
namespace {

// The pieces that the attention over an instance's beginning left of its row `rest` of q: piece p is number x + kPrefillRows * p, p < y.
__device__ __forceinline__ int2 ahead_of(const Beginnings& b, int inst, int rest) {
  return b.start[inst] == 0 ? make_int2(0, 0) : b.row[(size_t)b.plan.pos[inst] * b.rows + rest];
}

}  // namespace
}  // namespace ap
