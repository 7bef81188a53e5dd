// Device code that the kernels on caches with lengths of their own share.
#pragma once

#include "attention_body.h"
#include "cache_internal.h"

namespace ap {
namespace {

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Where row j of instance i lies, in rows of K and V.  Table entries outside the pool are clamped into it, as in the other calls.
__device__ __forceinline__ size_t row_at(const CacheRows& r, int i, int j) {
  if (r.table == nullptr) return (size_t)i * r.t_cap + j;
  const int page = clamped(r.table[(size_t)i * r.nb_cap + (j >> r.lb)], 0, r.n_phys - 1);
  return ((size_t)page << r.lb) + (j & ((1 << r.lb) - 1));
}
// The same for a row that is written: false where the table names no page of the pool.
__device__ __forceinline__ bool row_to_write(const CacheRows& r, int i, int j, size_t* at) {
  if (r.table == nullptr) { *at = (size_t)i * r.t_cap + j; return true; }
  const int page = r.table[(size_t)i * r.nb_cap + (j >> r.lb)];
  *at = ((size_t)page << r.lb) + (j & ((1 << r.lb) - 1));
  return page >= 0 && page < r.n_phys;
}

// Bytes of a 16-byte piece are moved whatever their type.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

}  // namespace
}  // namespace ap
