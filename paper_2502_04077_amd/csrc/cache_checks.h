// Argument checks that the calls on caches with lengths of their own share.
#pragma once

#include "cache_internal.h"

#define AP_REQUIRE_PTR(p)                                                       \
  do {                                                                          \
    if ((p) == nullptr) return AP_ERR_ARG;                                      \
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return AP_ERR_ALIGN;       \
  } while (0)
#define AP_OPTIONAL_PTR(p)                                                      \
  do {                                                                          \
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return AP_ERR_ALIGN;       \
  } while (0)

namespace ap {

static inline CacheRows rows_of(const Shape& s, const int32_t* len) {
  CacheRows r;
  r.table = s.table; r.len = len;
  r.n_inst = s.n_inst; r.t_cap = s.t_cap; r.nb_cap = s.nb_cap; r.n_phys = s.n_phys;
  r.lb = 0;
  while ((1 << r.lb) < s.b) ++r.lb;
  return r;
}

// Query rows are numbered in 32 bits within an instance.
static inline bool q_cap_ok(const Shape& s, int32_t q_cap) { return q_cap >= 1 && q_cap <= (1 << 30) / s.g; }

// A launch has less than 2^32 threads.
static inline bool fits(long long threads) { return threads < (1ll << 32); }
// Chunks that a prefill takes: 256 threads for 128 rows of q.
static inline bool chunk_ok(const Shape& s, int32_t q_cap) {
  return q_cap_ok(s, q_cap) && fits(((long long)q_cap * s.g + 127) / 128 * 256 * s.n_inst);
}
// A window of t_cap rows and more shows all of them; so sums of positions and windows stay in 32 bits.
static inline int seen_window(const Shape& s, int32_t window) { return window >= s.t_cap ? 0 : window; }
static inline int seen_first(const Shape& s, int32_t n_first) { return n_first < s.t_cap ? n_first : s.t_cap; }

}  // namespace ap
