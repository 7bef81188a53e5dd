// C entry points of the calls on caches whose instances have lengths of their own: argument checks, workspace, launches.
#include "cache_internal.h"

namespace ap {

CacheWs cache_decode_ws(const Shape& s, bool weights) {
  CacheWs w;
  size_t o = 0;
  auto take = [&o](size_t bytes) { const size_t at = o; o += (bytes + 15) / 16 * 16; return at; };
  w.before = take(((size_t)s.n_inst + 1) * 8);
  w.whole = take((size_t)s.n_inst * s.g * 2 * 4);
  w.part_ml = take((size_t)2 * kCacheDecodeWgs * s.g * 2 * 4);
  w.part_acc = take((size_t)2 * kCacheDecodeWgs * s.g * s.d * 4);
  w.tickets = take((size_t)kCacheDecodeWgs * kTicketStride * 8);
  w.logits = take(weights ? (size_t)s.n_inst * s.g * s.t_cap * 4 : 0);
  w.total = o;
  return w;
}
CacheQWs cache_prefill_ws(const Shape& s, int q_cap, bool weights) {
  CacheQWs w;
  size_t o = 0;
  auto take = [&o](size_t bytes) { const size_t at = o; o += (bytes + 15) / 16 * 16; return at; };
  w.stat = take(weights ? (size_t)s.n_inst * cache_stat_rows(s, q_cap) * 2 * 4 : 0);
  // (chunks x instances x tiles, whatever the window: more than one chunk only below kColumnWgs workgroups)
  w.sums = take(weights ? (size_t)(2 * kColumnWgs) * kPrefillRows * 4 : 0);
  // Rows of q in splits, for any q_cap up to this one: a workgroup's 128 each, and not more than all rows in the most splits.
  long long part = (long long)kSplitWgs * kPrefillRows;
  if (part > (long long)kMostSplits * s.n_inst * q_cap * s.g) part = (long long)kMostSplits * s.n_inst * q_cap * s.g;
  if (s.n_inst > kSplitWgs / 2) part = 0;
  w.part_ml = take((size_t)part * 2 * 4);
  w.part_o = take((size_t)part * s.d * 4);
  w.total = o;
  return w;
}

}  // namespace ap

using ap::CacheRows;
using ap::Shape;

#define AP_REQUIRE_PTR(p)                                                       \
  do {                                                                          \
    if ((p) == nullptr) return AP_ERR_ARG;                                      \
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return AP_ERR_ALIGN;       \
  } while (0)
#define AP_OPTIONAL_PTR(p)                                                      \
  do {                                                                          \
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return AP_ERR_ALIGN;       \
  } while (0)

static CacheRows rows_of(const Shape& s, const int32_t* len) {
  CacheRows r;
  r.table = s.table; r.len = len;
  r.n_inst = s.n_inst; r.t_cap = s.t_cap; r.nb_cap = s.nb_cap; r.n_phys = s.n_phys;
  r.lb = 0;
  while ((1 << r.lb) < s.b) ++r.lb;
  return r;
}

// Query rows are numbered in 32 bits within an instance.
static bool q_cap_ok(const Shape& s, int32_t q_cap) { return q_cap >= 1 && q_cap <= (1 << 30) / s.g; }

// A launch has less than 2^32 threads.
static bool fits(long long threads) { return threads < (1ll << 32); }
// Chunks that a prefill takes: 256 threads for 128 rows of q.
static bool chunk_ok(const Shape& s, int32_t q_cap) {
  return q_cap_ok(s, q_cap) && fits(((long long)q_cap * s.g + 127) / 128 * 256 * s.n_inst);
}
// A window of t_cap rows and more shows all of them; so sums of positions and windows stay in 32 bits.
static int seen_window(const Shape& s, int32_t window) { return window >= s.t_cap ? 0 : window; }
static int seen_first(const Shape& s, int32_t n_first) { return n_first < s.t_cap ? n_first : s.t_cap; }

extern "C" {

size_t ap_cache_workspace_bytes(const ap_ctx* ctx, int32_t q_cap, int32_t weights) {
  if (ctx == nullptr || q_cap < 0 || (q_cap > 0 && !chunk_ok(ctx->s, q_cap))) return 0;
  const size_t decode = ap::cache_decode_ws(ctx->s, weights != 0).total;
  const size_t prefill = q_cap > 0 ? ap::cache_prefill_ws(ctx->s, q_cap, weights != 0).total : 0;
  return decode > prefill ? decode : prefill;
}

int ap_cache_append(ap_ctx* ctx, const void* k_new, const void* v_new, const int32_t* n_new, int32_t q_cap, const int32_t* len, void* K,
                    void* V, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(k_new); AP_REQUIRE_PTR(v_new); AP_OPTIONAL_PTR(n_new); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V);
  const Shape& s = ctx->s;
  if (!q_cap_ok(s, q_cap) || !fits((long long)s.n_inst * q_cap * (s.d / 4))) return AP_ERR_RANGE;
  return ap::launch_cache_append(s, rows_of(s, len), k_new, v_new, n_new, q_cap, K, V, static_cast<hipStream_t>(stream)) == hipSuccess
             ? AP_OK : AP_ERR_HIP;
}

int ap_cache_decode(ap_ctx* ctx, const void* q, const void* K, const void* V, const int32_t* len, int32_t window, int32_t n_first,
                    float* out, float* acc, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(q); AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(out); AP_OPTIONAL_PTR(acc);
  AP_REQUIRE_PTR(ws);
  if (window < 0 || n_first < 0) return AP_ERR_ARG;
  const Shape& s = ctx->s;
  const ap::CacheWs w = ap::cache_decode_ws(s, acc != nullptr);
  char* base = static_cast<char*>(ws);
  ap::DecodeArgs a;
  a.r = rows_of(s, len);
  a.q = q; a.K = K; a.V = V; a.window = seen_window(s, window); a.n_first = seen_first(s, n_first); a.out = out; a.acc = acc;
  a.before = reinterpret_cast<unsigned long long*>(base + w.before);
  a.whole = reinterpret_cast<float*>(base + w.whole);
  a.part_ml = reinterpret_cast<float*>(base + w.part_ml);
  a.part_acc = reinterpret_cast<float*>(base + w.part_acc);
  a.tickets = reinterpret_cast<unsigned long long*>(base + w.tickets);
  a.nonce = 0;            // (the launcher draws it)
  a.logits = reinterpret_cast<float*>(base + w.logits);
  return ap::launch_cache_decode(s, a, static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_cache_prefill(ap_ctx* ctx, const void* q, const int32_t* n_q, int32_t q_cap, const void* K, const void* V, const int32_t* len,
                     int32_t window, int32_t n_first, void* out, float* acc, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(q); AP_OPTIONAL_PTR(n_q); AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(out);
  AP_OPTIONAL_PTR(acc); AP_REQUIRE_PTR(ws);
  if (window < 0 || n_first < 0) return AP_ERR_ARG;
  const Shape& s = ctx->s;
  if (!chunk_ok(s, q_cap)) return AP_ERR_RANGE;
  const ap::CacheQWs w = ap::cache_prefill_ws(s, q_cap, acc != nullptr);
  char* base = static_cast<char*>(ws);
  ap::PrefillArgs a;
  a.r = rows_of(s, len);
  a.q = q; a.K = K; a.V = V; a.n_q = n_q; a.q_cap = q_cap; a.window = seen_window(s, window); a.n_first = seen_first(s, n_first); a.out = out; a.acc = acc;
  a.stat = reinterpret_cast<float*>(base + w.stat);
  a.sums = reinterpret_cast<float*>(base + w.sums);
  a.part_ml = reinterpret_cast<float*>(base + w.part_ml);
  a.part_o = reinterpret_cast<float*>(base + w.part_o);
  return ap::launch_cache_prefill(s, a, static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_cache_evict(ap_ctx* ctx, void* K, void* V, const float* acc, const int32_t* len, int32_t budget, int32_t n_first, int32_t n_last,
                   float* acc_out, int32_t* len_out, int32_t* kept, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(acc); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(acc_out); AP_REQUIRE_PTR(len_out);
  AP_REQUIRE_PTR(kept);
  const Shape& s = ctx->s;
  if (n_first < 0 || n_last < 0 || budget < 1 || n_first > budget || n_last > budget - n_first) return AP_ERR_ARG;
  if (budget > s.t_cap) return AP_ERR_RANGE;
  return ap::launch_cache_evict(s, rows_of(s, len), K, V, acc, budget, n_first, n_last, acc_out, len_out, kept,
                                static_cast<hipStream_t>(stream)) == hipSuccess
             ? AP_OK : AP_ERR_HIP;
}

}  // extern "C"
