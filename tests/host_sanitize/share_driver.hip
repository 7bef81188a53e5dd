// The calls on pages and on beginnings in common, on the host: csrc/share_api.hip beside csrc/cache_api.hip and csrc/api.hip under the sanitizers,
// with stubs in the place of the kernel launchers, which check what they are handed: every piece of a workspace, a plan or a state lies inside the
// bytes that its size query names, none over another, whatever the sizes.
#define main api_main
#include "driver.hip"
#undef main

#include <algorithm>
#include <climits>

#include "share_internal.h"

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

static size_t state_words = 0;
static int32_t* const state_at = reinterpret_cast<int32_t*>(1 << 24);

static void check_pool(const ap::Pages& p) {
  CHECK(p.refs == state_at && p.seg == state_at + p.n_pages && (size_t)p.n_pages + p.segments == state_words);
  CHECK((long long)p.segments * ap::kSegment >= p.n_pages && (long long)(p.segments - 1) * ap::kSegment < p.n_pages);
  CHECK(p.n_inst >= 1 && p.n_pages >= 1 && p.nb_cap << p.lb >= p.t_cap && p.row_pieces >= 8);
}
static void check_ws(const ap::Pages& p, char* at, const ap::PagesWs& w) {
  const size_t n = p.n_inst, pages = p.n_pages;
  check_pieces({{at + w.head, 16}, {at + w.need, n * 4}, {at + w.before, n * 4}, {at + w.length, n * 4}, {at + w.staged, n * p.nb_cap * 4},
                {at + w.picked, pages * 4}, {at + w.taken, (size_t)p.segments * 4}, {at + w.from, pages * 4}, {at + w.rank, pages * 4}});
  ++launched;
}
namespace ap {
// Of the calls on caches a prefill alone is reached.
hipError_t launch_cache_append(const Shape&, const CacheRows&, const void*, const void*, const int32_t*, int, void*, void*, hipStream_t) { CHECK(!"append"); return hipErrorUnknown; }
hipError_t launch_cache_decode(const Shape&, const DecodeArgs&, hipStream_t) { CHECK(!"decode"); return hipErrorUnknown; }
hipError_t launch_cache_evict(const Shape&, const CacheRows&, void*, void*, const float*, int, int, int, float*, int32_t*, int32_t*, hipStream_t) { CHECK(!"evict"); return hipErrorUnknown; }
hipError_t launch_cache_prefill(const Shape& s, const PrefillArgs& a, hipStream_t) {
  const size_t rows = (size_t)a.q_cap * s.g, wgs = (rows + kPrefillRows - 1) / kPrefillRows * s.n_inst;
  const size_t splits = std::min<size_t>(kSplitWgs / wgs, kMostSplits), part = splits > 1 ? splits * s.n_inst * rows : 0;
  CHECK(a.acc == nullptr);
  check_pieces({{a.part_ml, part * 8}, {a.part_o, part * s.d * 4}});
  ++launched;
  return hipErrorUnknown;
}
hipError_t launch_pages_count(const Pages& p, hipStream_t) { check_pool(p); ++launched; return hipErrorUnknown; }
hipError_t launch_pages_resize(const ResizeArgs& a, hipStream_t) { check_pool(a.p); check_ws(a.p, a.ws, a.w); CHECK(a.q_cap >= 0); return hipErrorUnknown; }
hipError_t launch_pages_fork(const ForkArgs& a, hipStream_t) { check_pool(a.p); check_ws(a.p, a.ws, a.w); return hipErrorUnknown; }
hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t) { check_pool(a.p); check_ws(a.p, a.ws, a.w); return hipErrorUnknown; }
hipError_t launch_pages_copy(const void*, const void*, int, const int32_t*, void*, void*, int, const int32_t*, int, int, hipStream_t) {
  CHECK(!"pageable memory was taken");
  return hipErrorUnknown;
}
static void check_plan(const Shape& s, const SharePlan& p) {
  const size_t n = s.n_inst;
  check_pieces({{p.inst, n * 16}, {p.groups, n * 16}, {p.count, 16}, {p.pos, n / 4 * 16}});
  CHECK(reinterpret_cast<const char*>(p.member + n) <= reinterpret_cast<const char*>(p.inst) + ap::share_plan_bytes(s) && p.member == p.pos + n);
}
hipError_t launch_cache_share(const Shape& s, const int32_t*, const int32_t*, const SharePlan& p, hipStream_t) {
  ws_bytes = ap::share_plan_bytes(s);
  check_plan(s, p);
  ++launched;
  return hipErrorUnknown;
}
hipError_t launch_cache_shared(const Shape& s, const SharedArgs& a, bool decode, hipStream_t) {
  const size_t n = s.n_inst, rows = (size_t)2 * n * a.q_cap * s.g, pieces = shared_pieces(s, a.q_cap);
  CHECK(pieces < (size_t)1 << 31 && (size_t)a.narrow0 == shared_narrow0(s, a.q_cap) && a.rows == a.q_cap * s.g && 1 << a.lg == s.g);
  // The last pieces that a workgroup and a wave can leave.
  CHECK(rows + (size_t)kPrefillRows * (kShareWgs - 1) < (size_t)a.narrow0 && a.narrow0 + rows + (size_t)kNarrowRows * (4 * kShareWgs - 1) < pieces);
  CHECK(!decode || (a.q_cap == 1 && a.n_q == nullptr));
  check_pieces({{a.begun, n * 4}, {a.behind, n * 4}, {a.row, rows * 8}, {a.ml, pieces * 8}, {a.o, pieces * s.d * 4}});
  CHECK(a.window >= 0 && a.window < s.t_cap && a.n_first >= 0 && a.n_first <= s.t_cap);
  ++launched;
  return hipErrorUnknown;
}
}  // namespace ap

int main() {
  void* ok = reinterpret_cast<void*>(4096);
  float* fok = static_cast<float*>(ok);
  int32_t* iok = static_cast<int32_t*>(ok);
  char* at = const_cast<char*>(ws);
  int32_t* iat = reinterpret_cast<int32_t*>(at);
  for (int n_inst : {1, 2, 3, 63, 257, 2048, 65535})
    for (int g : {1, 2, 4, 8})
      for (int d : {64, 128})
        for (int t_cap : {64, 4096, 131072}) {
          ap_config c = base_cfg();
          c.n_inst = n_inst; c.g = g; c.head_dim = d; c.t_cap = t_cap; c.k_blocks = 4; c.n_sink = c.n_local = 1; c.kv_dtype = d == 64 ? AP_F32 : AP_BF16;
          ap_ctx* ctx = nullptr;
          CHECK(ap_create(&c, &ctx) == AP_OK && ctx != nullptr);
          if (ctx == nullptr) continue;
          for (int n_pages : {1, 2, 1023, 1024, 1025, 1 << 20, (1 << 30) - 1, 1 << 30}) {
            state_words = ap_pages_state_bytes(ctx, n_pages) / 4;
            ws_bytes = ap_pages_workspace_bytes(ctx, n_pages);
            CHECK(state_words > 0 && ws_bytes > 0);
            CHECK(ap_pages_count(ctx, iok, n_pages, state_at, nullptr) == AP_ERR_HIP);
            for (int q_cap : {0, 1, 77, INT_MAX})
              CHECK(ap_pages_resize(ctx, ok, ok, iok, n_pages, state_at, iok, q_cap == 1 ? nullptr : iok, q_cap, iok, at, nullptr) == AP_ERR_HIP);
            CHECK(ap_pages_fork(ctx, ok, ok, iok, n_pages, state_at, iok, iok, iok, iok, at, nullptr) == AP_ERR_HIP);
            CHECK(ap_pages_compact(ctx, ok, ok, iok, n_pages, state_at, iok, at, nullptr) == AP_ERR_HIP);
          }
          for (int n_pages : {0, -1, INT_MIN, (1 << 30) + 1, INT_MAX}) {
            CHECK(ap_pages_state_bytes(ctx, n_pages) == 0 && ap_pages_workspace_bytes(ctx, n_pages) == 0);
            CHECK(ap_pages_count(ctx, iok, n_pages, state_at, nullptr) == AP_ERR_RANGE);
            CHECK(ap_pages_copy(ctx, ok, ok, n_pages, nullptr, ok, ok, 5, nullptr, 1, nullptr) == AP_ERR_RANGE);
            CHECK(ap_pages_copy(ctx, ok, ok, 5, nullptr, ok, ok, n_pages, nullptr, 1, nullptr) == AP_ERR_RANGE);
          }
          CHECK(ap_pages_copy(ctx, ok, ok, 5, nullptr, ok, ok, 5, nullptr, 0, nullptr) == AP_OK);
          CHECK(ap_pages_copy(ctx, ok, ok, 5, nullptr, ok, ok, 5, nullptr, INT_MIN, nullptr) == AP_ERR_RANGE);
          static char page[64];
          char* pageable = page + (16 - reinterpret_cast<uintptr_t>(page) % 16) % 16;
          CHECK(ap_pages_copy(ctx, pageable, pageable, 5, nullptr, pageable, pageable, 5, nullptr, 1, nullptr) == AP_ERR_ARG);

          CHECK(ap_cache_share_bytes(ctx) > 0);
          CHECK(ap_cache_share(ctx, iok, iok, at, nullptr) == AP_ERR_HIP);
          ws_bytes = ap_cache_shared_workspace_bytes(ctx, 0);
          CHECK(ws_bytes > 0);
          for (int window : {0, 1, t_cap - 1, t_cap, INT_MAX})
            CHECK(ap_cache_decode_shared(ctx, ok, ok, ok, iok, iok, window, window, fok, at, nullptr) == AP_ERR_HIP);
          for (int q_cap : {1, 2, 7, 8, 9, 15, 16, 31, 32, 33, 64, 65, 128, 1000, 8192, 1 << 20, 1 << 27, (1 << 30) / g, INT_MAX}) {
            ws_bytes = ap_cache_shared_workspace_bytes(ctx, q_cap);
            for (int q : {q_cap, q_cap - 1, q_cap / 2, q_cap / 9, 64 / g, 32 / g, 3, 2, 1}) {
              if (q < 1 || q > q_cap) continue;
              const int rc = ap_cache_prefill_shared(ctx, ok, iok, q, ok, ok, iok, iok, 0, INT_MAX, ok, at, nullptr);
              CHECK(ws_bytes > 0 ? rc == AP_ERR_HIP : q < q_cap || rc == AP_ERR_RANGE);
              if (ws_bytes == 0) break;
              CHECK(ap_cache_prefill_shared(ctx, ok, nullptr, q, ok, ok, iok, iok, 5, 0, ok, at, nullptr) == AP_ERR_HIP);
            }
            if (ws_bytes > 0) CHECK(ap_cache_decode_shared(ctx, ok, ok, ok, iok, iok, 0, 0, fok, at, nullptr) == AP_ERR_HIP);
          }
          const int before = launched;
          CHECK(ap_cache_decode_shared(ctx, ok, ok, ok, iok, iok, -1, 0, fok, at, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_decode_shared(ctx, ok, ok, ok, iok, iat + 1, 0, 0, fok, at, nullptr) == AP_ERR_ALIGN);
          CHECK(ap_cache_prefill_shared(ctx, ok, iok, INT_MIN, ok, ok, iok, iok, 0, 0, ok, at, nullptr) == AP_ERR_RANGE);
          CHECK(ap_cache_prefill_shared(ctx, ok, iok, 1, ok, ok, iok, iok, 0, INT_MIN, ok, at, nullptr) == AP_ERR_ARG);
          CHECK(ap_cache_share(ctx, iok, nullptr, at, nullptr) == AP_ERR_ARG);
          CHECK(ap_pages_resize(ctx, ok, ok, iok, 5, state_at, iok, iok, -1, iok, at, nullptr) == AP_ERR_RANGE);
          CHECK(ap_cache_shared_workspace_bytes(ctx, -1) == 0 && ap_cache_shared_workspace_bytes(nullptr, 1) == 0 && ap_cache_share_bytes(nullptr) == 0);
          CHECK(launched == before);
          CHECK(ap_destroy(ctx) == AP_OK);
        }
  std::printf(failures ? "share driver: %d checks failed\n" : "share driver: all checks passed\n", failures);
  return failures ? 1 : 0;
}
