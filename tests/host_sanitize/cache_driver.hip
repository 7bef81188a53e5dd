// The calls on caches with lengths of their own, on the host: csrc/cache_api.hip beside csrc/api.hip under the sanitizers, with stubs in the
// place of the kernel launchers, which check what they are handed: every piece of the workspace lies inside the bytes that
// ap_cache_workspace_bytes names, none over another, whatever the sizes.
#define main api_main
#include "driver.hip"
#undef main

#include <algorithm>
#include <climits>

#include "cache_internal.h"

static size_t ws_bytes = 0;                                // of the workspace that the next call is handed, at address 1 << 20
static const char* const ws = reinterpret_cast<const char*>(1 << 20);
static int launched = 0;

struct Piece { const void* at; size_t bytes; };
static void check_pieces(std::vector<Piece> p) {
  std::sort(p.begin(), p.end(), [](const Piece& a, const Piece& b) { return a.at < b.at || (a.at == b.at && a.bytes < b.bytes); });
  const char* end = ws;
  for (const Piece& x : p) {
    CHECK(reinterpret_cast<uintptr_t>(x.at) % 16 == 0 && static_cast<const char*>(x.at) >= end);
    end = static_cast<const char*>(x.at) + x.bytes;
  }
  CHECK(end <= ws + ws_bytes);
}

namespace ap {
hipError_t launch_cache_append(const Shape&, const CacheRows& r, const void*, const void*, const int32_t*, int q_cap, void*, void*, hipStream_t) {
  CHECK(r.n_inst >= 1 && q_cap >= 1);
  ++launched;
  return hipErrorUnknown;
}
hipError_t launch_cache_decode(const Shape& s, const DecodeArgs& a, hipStream_t) {
  const size_t n = s.n_inst, heads = n * s.g;
  check_pieces({{a.before, (n + 1) * 8}, {a.whole, heads * 8}, {a.part_ml, (size_t)2 * kCacheDecodeWgs * s.g * 8},
                {a.part_acc, (size_t)2 * kCacheDecodeWgs * s.g * s.d * 4}, {a.tickets, (size_t)kCacheDecodeWgs * kTicketStride * 8},
                {a.logits, a.acc != nullptr ? heads * s.t_cap * 4 : 0}});
  CHECK(a.window >= 0 && a.window < s.t_cap && a.n_first >= 0 && a.n_first <= s.t_cap && (1 << a.r.lb) == s.b);
  ++launched;
  return hipErrorUnknown;
}
hipError_t launch_cache_prefill(const Shape& s, const PrefillArgs& a, hipStream_t) {
  // Splits as they come at most: as many as leave kSplitWgs workgroups.
  const size_t rows = (size_t)a.q_cap * s.g, wgs = (rows + kPrefillRows - 1) / kPrefillRows * s.n_inst;
  const size_t splits = std::min<size_t>(kSplitWgs / wgs, kMostSplits), part = splits > 1 ? splits * s.n_inst * rows : 0;
  const bool weights = a.acc != nullptr;
  check_pieces({{a.stat, weights ? (size_t)s.n_inst * cache_stat_rows(s, a.q_cap) * 8 : 0}, {a.sums, weights ? (size_t)2 * kColumnWgs * kPrefillRows * 4 : 0},
                {a.part_ml, part * 8}, {a.part_o, part * s.d * 4}});
  CHECK(a.window >= 0 && a.window < s.t_cap && a.n_first >= 0 && a.n_first <= s.t_cap);
  ++launched;
  return hipErrorUnknown;
}
hipError_t launch_cache_evict(const Shape& s, const CacheRows&, void*, void*, const float*, int budget, int n_first, int n_last, float*, int32_t*, int32_t*, hipStream_t) {
  CHECK(budget >= 1 && budget <= s.t_cap && n_first >= 0 && n_last >= 0 && n_first + n_last <= budget);
  ++launched;
  return hipErrorUnknown;
}
}  // namespace ap

int main() {
  void* ok = reinterpret_cast<void*>(4096);
  float* fok = static_cast<float*>(ok);
  int32_t* iok = static_cast<int32_t*>(ok);
  for (int n_inst : {1, 2, 63, 256, 257, 2048, 65535})
    for (int g : {1, 4, 8})
      for (int d : {64, 128})
        for (int t_cap : {64, 4096, 131072}) {
          ap_config c = base_cfg();
          c.n_inst = n_inst; c.g = g; c.head_dim = d; c.t_cap = t_cap; c.k_blocks = 4; c.n_sink = c.n_local = 1; c.kv_dtype = d == 64 ? AP_F32 : AP_BF16;
          ap_ctx* ctx = nullptr;
          CHECK(ap_create(&c, &ctx) == AP_OK && ctx != nullptr);
          if (ctx == nullptr) continue;
          for (int weights = 0; weights < 2; ++weights) {
            float* acc = weights ? fok : nullptr;
            void* at = const_cast<char*>(ws);
            ws_bytes = ap_cache_workspace_bytes(ctx, 0, weights);
            CHECK(ws_bytes > 0);
            for (int window : {0, 1, t_cap - 1, t_cap, INT_MAX})
              CHECK(ap_cache_decode(ctx, ok, ok, ok, iok, window, window, fok, acc, at, nullptr) == AP_ERR_HIP);
            for (int q_cap : {1, 2, 31, 33, 128, 1000, 8192, 1 << 20, 1 << 27, (1 << 30) / g, INT_MAX}) {
              ws_bytes = ap_cache_workspace_bytes(ctx, q_cap, weights);
              // what is sized for chunks of q_cap holds for shorter ones and for decode, with weights also for calls without
              for (int q : {q_cap, q_cap - 1, q_cap / 2, q_cap / 9, 1}) {
                if (q < 1) continue;
                const int rc = ap_cache_prefill(ctx, ok, iok, q, ok, ok, iok, 0, INT_MAX, ok, acc, at, nullptr);
                CHECK(ws_bytes > 0 ? rc == AP_ERR_HIP : q < q_cap || rc == AP_ERR_RANGE);
                if (ws_bytes == 0) break;
                CHECK(ap_cache_prefill(ctx, ok, nullptr, q, ok, ok, iok, 5, 0, ok, nullptr, at, nullptr) == AP_ERR_HIP);
              }
              if (ws_bytes > 0) CHECK(ap_cache_decode(ctx, ok, ok, ok, iok, 0, 0, fok, acc, at, nullptr) == AP_ERR_HIP);
              const int rc = ap_cache_append(ctx, ok, ok, iok, q_cap, iok, ok, ok, nullptr);
              CHECK(rc == AP_ERR_HIP || rc == AP_ERR_RANGE);
            }
          }
          CHECK(ap_cache_evict(ctx, ok, ok, fok, iok, t_cap, t_cap / 2, t_cap / 2, fok, iok, iok, nullptr) == AP_ERR_HIP);
          const int before = launched;
          CHECK(ap_cache_evict(ctx, ok, ok, fok, iok, t_cap + 1, 0, 0, fok, iok, iok, nullptr) == AP_ERR_RANGE);
          CHECK(ap_cache_evict(ctx, ok, ok, fok, iok, 5, INT_MAX, INT_MAX, fok, iok, iok, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_decode(ctx, ok, ok, ok, iok, -1, 0, fok, fok, ok, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_decode(ctx, ok, ok, ok, iok, 0, 0, fok, reinterpret_cast<float*>(4100), ok, nullptr) == AP_ERR_ALIGN);
          CHECK(ap_cache_prefill(ctx, ok, iok, INT_MIN, ok, ok, iok, 0, 0, ok, fok, ok, nullptr) == AP_ERR_RANGE);
          CHECK(ap_cache_prefill(ctx, ok, iok, 1, ok, ok, iok, 0, INT_MIN, ok, fok, ok, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_append(ctx, ok, nullptr, iok, 1, iok, ok, ok, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_workspace_bytes(ctx, -1, 0) == 0 && ap_cache_workspace_bytes(nullptr, 1, 1) == 0);
          CHECK(launched == before);
          CHECK(ap_destroy(ctx) == AP_OK);
        }
  std::printf(failures ? "cache driver: %d checks failed\n" : "cache driver: all checks passed\n", failures);
  return failures ? 1 : 0;
}
