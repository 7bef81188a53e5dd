// Device code that the kernels on rows behind a shared beginning have in common.
#pragma once

#include "cache_body.h"
#include "share_internal.h"

namespace ap {
namespace {

// The pieces that the attention over an instance's beginning left of its row `rest` of q: piece p is number row + kPrefillRows * p.
struct Ahead { int row, parts; };
__device__ __forceinline__ Ahead ahead_of(const Beginnings& b, int inst, int rest) {
  if (b.start[inst] == 0) return {0, 0};
  const int4 group = b.plan.inst[inst];
  const int k = b.units[group.x], r = (b.plan.pos[inst] - group.y) * b.rows + rest;
  if (k == 0) return {0, 0};
  const unsigned long long u = b.before[group.x] + (unsigned long long)(r / kPrefillRows) * k, per = *b.per;
  const int w0 = (int)(u / per);
  return {group.y * b.rows + r + kPrefillRows * w0, (int)((u + k - 1) / per) - w0 + 1};
}

}  // namespace
}  // namespace ap
