// C entry points of the calls on pages and on shared beginnings: argument checks, workspace, launches.
#include "cache_checks.h"
#include "share_internal.h"

namespace ap {

PagesWs pages_ws(const Shape& s, int n_pages) {
  PagesWs w;
  size_t o = 0;
  auto take = [&o](size_t words) { const size_t at = o; o += (words * 4 + 15) / 16 * 16; return at; };
  w.head = take(4);
  w.need = take(s.n_inst);
  w.before = take(s.n_inst);
  w.length = take(s.n_inst);
  w.staged = take((size_t)s.n_inst * s.nb_cap);
  w.picked = take(n_pages);
  w.taken = take(page_segments(n_pages));
  w.from = take(n_pages);
  w.rank = take(n_pages);
  w.total = o;
  return w;
}

size_t share_plan_bytes(const Shape& s) { return ((size_t)s.n_inst * 10 * 4 + 16 + 15) / 16 * 16; }
SharePlan share_plan(const Shape& s, void* plan) {
  SharePlan p;
  p.inst = static_cast<int4*>(plan);
  p.groups = p.inst + s.n_inst;
  p.count = reinterpret_cast<int32_t*>(p.groups + s.n_inst);
  p.pos = p.count + 4;
  p.member = p.pos + s.n_inst;
  return p;
}

SharedWs shared_ws(const Shape& s, int q_cap) {
  SharedWs w;
  size_t o = 0;
  auto take = [&o](size_t bytes) { const size_t at = o; o += (bytes + 15) / 16 * 16; return at; };
  const size_t rows = (size_t)2 * s.n_inst * q_cap * s.g, pieces = shared_pieces(s, q_cap);
  w.begun = take((size_t)s.n_inst * 4);
  w.behind = take((size_t)s.n_inst * 4);
  w.row = take(rows * 8);
  w.low = take((size_t)s.n_inst * 4);
  w.sizes = take(shared_sources(s) * 16);
  w.totals = take(shared_sources(s) / 256 * 16);
  w.ml = take(pieces * 2 * 4);
  w.o = take(pieces * s.d * 4);
  w.total = o;
  return w;
}

}  // namespace ap

using ap::Shape;
using ap::fits;

// Pages of a pool are numbered in 32 bits, with room behind them.
static bool pool_ok(const Shape& s, int32_t n_pages) { return n_pages >= 1 && n_pages <= 1 << 30 && fits((long long)s.n_inst * 256); }

static ap::Pages pages_of(const Shape& s, void* K, void* V, int32_t* table, int32_t n_pages, int32_t* state) {
  ap::Pages p;
  p.table = table; p.refs = state; p.seg = state + n_pages;
  p.K = K; p.V = V;
  p.n_inst = s.n_inst; p.t_cap = s.t_cap; p.nb_cap = s.nb_cap; p.n_pages = n_pages;
  p.lb = 0;
  while ((1 << p.lb) < s.b) ++p.lb;
  p.segments = ap::page_segments(n_pages);
  p.row_pieces = s.d * (s.kv_dtype == AP_BF16 ? 2 : 4) / 16;
  return p;
}

// Chunks of so few rows of q that reading rows in common once is sooner than the prefill's tiles over every instance's own: an instance's rows are a
// wave's (kNarrowRows), and for fp32, where the prefill's product is slow, twice that.  Measured against the prefill, 8 KV heads, g = 4, d = 128, behind a
// beginning of 6000 tokens in pages that all share, by 8, 32, 48, 64, 128 rows of q: bf16, 16 sequences 29, 49, 55, 66, 100 us (the prefill 60, 62, 65, 66, 76), 128
// sequences 65, 172, 242, 319, 624 (356, 364, 375, 374, 412); fp32, 16 sequences 63, 174, 186, 237, 450 (378, 391, 396, 397, 414), 128 sequences 257, 1355, 1261, 1676, 3550
// (2974, 2993, 2998, 2998, 3038).  (bf16 chunks of 33 to 64 rows would be sooner by groups where many sequences share.)  And all rows are numbered in 32
// bits, and their pieces.
static bool few_rows(const Shape& s, int32_t q_cap) {
  return q_cap * s.g <= (s.kv_dtype == AP_BF16 ? 1 : 2) * ap::kNarrowRows && ap::shared_pieces(s, q_cap) < (size_t)1 << 31;
}
static hipError_t launch_shared(const Shape& s, const void* q, const int32_t* n_q, int32_t q_cap, const void* K, const void* V, const int32_t* len,
                                const void* plan, int32_t window, int32_t n_first, void* out, bool decode, void* ws, void* stream) {
  const ap::SharedWs w = ap::shared_ws(s, q_cap);
  char* base = static_cast<char*>(ws);
  ap::SharedArgs a;
  a.r = rows_of(s, len);
  a.q = q; a.K = K; a.V = V; a.n_q = n_q; a.q_cap = q_cap; a.rows = q_cap * s.g; a.narrow0 = (int)ap::shared_narrow0(s, q_cap);
  a.lg = 0;
  while ((1 << a.lg) < s.g) ++a.lg;
  a.window = seen_window(s, window); a.n_first = seen_first(s, n_first); a.out = out;
  a.plan = ap::share_plan(s, const_cast<void*>(plan));
  a.begun = reinterpret_cast<int32_t*>(base + w.begun);
  a.behind = reinterpret_cast<int32_t*>(base + w.behind);
  a.row = reinterpret_cast<int2*>(base + w.row);
  a.sized = 0;
  a.low = reinterpret_cast<int32_t*>(base + w.low);
  a.sizes = reinterpret_cast<unsigned long long*>(base + w.sizes);
  a.totals = reinterpret_cast<unsigned long long*>(base + w.totals);
  a.ml = reinterpret_cast<float*>(base + w.ml);
  a.o = reinterpret_cast<float*>(base + w.o);
  return ap::launch_cache_shared(s, a, decode, static_cast<hipStream_t>(stream));
}

// As in api.hip: memory that a kernel may read and write, on the device or pinned; pageable host memory would fault the GPU.
static bool reaches_device(const void* p) {
  hipPointerAttribute_t a;
  if (hipPointerGetAttributes(&a, p) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return a.type == hipMemoryTypeHost || a.type == hipMemoryTypeDevice || a.type == hipMemoryTypeManaged;
}

extern "C" {

size_t ap_pages_state_bytes(const ap_ctx* ctx, int32_t n_pages) {
  return ctx == nullptr || !pool_ok(ctx->s, n_pages) ? 0 : ((size_t)n_pages + ap::page_segments(n_pages)) * 4;
}
size_t ap_pages_workspace_bytes(const ap_ctx* ctx, int32_t n_pages) {
  return ctx == nullptr || !pool_ok(ctx->s, n_pages) ? 0 : ap::pages_ws(ctx->s, n_pages).total;
}

int ap_pages_count(ap_ctx* ctx, const int32_t* table, int32_t n_pages, int32_t* state, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(table); AP_REQUIRE_PTR(state);
  const Shape& s = ctx->s;
  if (!pool_ok(s, n_pages)) return AP_ERR_RANGE;
  return ap::launch_pages_count(pages_of(s, nullptr, nullptr, const_cast<int32_t*>(table), n_pages, state), static_cast<hipStream_t>(stream)) ==
                 hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_pages_resize(ap_ctx* ctx, void* K, void* V, int32_t* table, int32_t n_pages, int32_t* state, const int32_t* len, const int32_t* n_new,
                    int32_t q_cap, int32_t* info, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(table); AP_REQUIRE_PTR(state); AP_REQUIRE_PTR(len); AP_OPTIONAL_PTR(n_new);
  AP_REQUIRE_PTR(info); AP_REQUIRE_PTR(ws);
  const Shape& s = ctx->s;
  if (!pool_ok(s, n_pages) || q_cap < 0) return AP_ERR_RANGE;
  ap::ResizeArgs a;
  a.p = pages_of(s, K, V, table, n_pages, state);
  a.len = len; a.n_new = n_new; a.q_cap = q_cap; a.info = info; a.ws = static_cast<char*>(ws); a.w = ap::pages_ws(s, n_pages);
  return ap::launch_pages_resize(a, static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_pages_fork(ap_ctx* ctx, void* K, void* V, int32_t* table, int32_t n_pages, int32_t* state, const int32_t* parent, const int32_t* len,
                  int32_t* len_out, int32_t* info, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(table); AP_REQUIRE_PTR(state); AP_REQUIRE_PTR(parent); AP_REQUIRE_PTR(len);
  AP_REQUIRE_PTR(len_out); AP_REQUIRE_PTR(info); AP_REQUIRE_PTR(ws);
  const Shape& s = ctx->s;
  if (!pool_ok(s, n_pages)) return AP_ERR_RANGE;
  ap::ForkArgs a;
  a.p = pages_of(s, K, V, table, n_pages, state);
  a.parent = parent; a.len = len; a.len_out = len_out; a.info = info; a.ws = static_cast<char*>(ws); a.w = ap::pages_ws(s, n_pages);
  return ap::launch_pages_fork(a, static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_pages_compact(ap_ctx* ctx, void* K, void* V, int32_t* table, int32_t n_pages, int32_t* state, int32_t* info, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(table); AP_REQUIRE_PTR(state); AP_REQUIRE_PTR(info); AP_REQUIRE_PTR(ws);
  const Shape& s = ctx->s;
  if (!pool_ok(s, n_pages)) return AP_ERR_RANGE;
  ap::CompactArgs a;
  a.p = pages_of(s, K, V, table, n_pages, state);
  a.info = info; a.ws = static_cast<char*>(ws); a.w = ap::pages_ws(s, n_pages);
  return ap::launch_pages_compact(a, static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_pages_copy(ap_ctx* ctx, const void* K_src, const void* V_src, int32_t n_src, const int32_t* src, void* K_dst, void* V_dst, int32_t n_dst,
                  const int32_t* dst, int32_t n, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(K_src); AP_REQUIRE_PTR(V_src); AP_OPTIONAL_PTR(src); AP_REQUIRE_PTR(K_dst); AP_REQUIRE_PTR(V_dst); AP_OPTIONAL_PTR(dst);
  const Shape& s = ctx->s;
  if (!pool_ok(s, n_src) || !pool_ok(s, n_dst) || n < 0) return AP_ERR_RANGE;
  if (n == 0) return AP_OK;
  if (!reaches_device(K_src) || !reaches_device(V_src) || !reaches_device(K_dst) || !reaches_device(V_dst)) return AP_ERR_ARG;
  return ap::launch_pages_copy(K_src, V_src, n_src, src, K_dst, V_dst, n_dst, dst, n, s.b * s.d * (s.kv_dtype == AP_BF16 ? 2 : 4) / 16,
                               static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

size_t ap_cache_share_bytes(const ap_ctx* ctx) { return ctx == nullptr ? 0 : ap::share_plan_bytes(ctx->s); }

int ap_cache_share(ap_ctx* ctx, const int32_t* group, const int32_t* shared, void* plan, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(group); AP_REQUIRE_PTR(shared); AP_REQUIRE_PTR(plan);
  const Shape& s = ctx->s;
  return ap::launch_cache_share(s, group, shared, ap::share_plan(s, plan), static_cast<hipStream_t>(stream)) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

size_t ap_cache_shared_workspace_bytes(const ap_ctx* ctx, int32_t q_cap) {
  if (ctx == nullptr || q_cap < 0 || (q_cap > 0 && !chunk_ok(ctx->s, q_cap)) || !few_rows(ctx->s, 1)) return 0;
  const Shape& s = ctx->s;
  // Of any chunk up to q_cap: those of few rows read rows in common once, the others are a prefill's.
  int few = q_cap < ap::kPrefillRows ? q_cap : ap::kPrefillRows;
  while (few > 1 && !few_rows(s, few)) --few;
  const size_t shared = ap::shared_ws(s, few > 1 ? few : 1).total, prefill = q_cap > 0 ? ap::cache_prefill_ws(s, q_cap, false).total : 0;
  return shared > prefill ? shared : prefill;
}

int ap_cache_decode_shared(ap_ctx* ctx, const void* q, const void* K, const void* V, const int32_t* len, const void* plan, int32_t window,
                           int32_t n_first, float* out, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(q); AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(plan); AP_REQUIRE_PTR(out); AP_REQUIRE_PTR(ws);
  if (window < 0 || n_first < 0) return AP_ERR_ARG;
  const Shape& s = ctx->s;
  if (!few_rows(s, 1)) return AP_ERR_RANGE;
  return launch_shared(s, q, nullptr, 1, K, V, len, plan, window, n_first, out, true, ws, stream) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

int ap_cache_prefill_shared(ap_ctx* ctx, const void* q, const int32_t* n_q, int32_t q_cap, const void* K, const void* V, const int32_t* len,
                            const void* plan, int32_t window, int32_t n_first, void* out, void* ws, void* stream) {
  if (ctx == nullptr) return AP_ERR_ARG;
  AP_REQUIRE_PTR(q); AP_OPTIONAL_PTR(n_q); AP_REQUIRE_PTR(K); AP_REQUIRE_PTR(V); AP_REQUIRE_PTR(len); AP_REQUIRE_PTR(plan); AP_REQUIRE_PTR(out);
  AP_REQUIRE_PTR(ws);
  if (window < 0 || n_first < 0) return AP_ERR_ARG;
  const Shape& s = ctx->s;
  if (!chunk_ok(s, q_cap)) return AP_ERR_RANGE;
  if (!few_rows(s, q_cap)) return ap_cache_prefill(ctx, q, n_q, q_cap, K, V, len, window, n_first, out, nullptr, ws, stream);
  return launch_shared(s, q, n_q, q_cap, K, V, len, plan, window, n_first, out, false, ws, stream) == hipSuccess ? AP_OK : AP_ERR_HIP;
}

}  // extern "C"
