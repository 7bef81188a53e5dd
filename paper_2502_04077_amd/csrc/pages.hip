// Pages of a pool that instances share: taken and given back, forked, compacted, copied.
//
// refs[p] says how often the table names page p; p is free where that is 0.  seg holds the number of free pages among each 1024, so that workgroups know how
// many lie in front of their own segments, and whether there are enough, without reading through the counts; of its own segments a workgroup reads all counts, also of
// those without free pages, until enough are found.  Three steps, a launch each, as none can begin before the one before has ended
// everywhere: what every instance needs, which free pages it gets (the x-th need in the order of instances and blocks gets the x-th free
// page), and carrying it out.  The second step knows whether there are enough; if not, the third leaves all as it is.  Counts are whole numbers,
// so that the order of atomics does not show in any result.  Where there is little to do one workgroup takes all three steps (small).  Where the state does not belong to the
// table, what comes out is unspecified, but every page that is read or written lies in the pool.
//
// Latency bounds all but the copies: a resize of 32 instances takes 7.6 us (6 of them its one launch, trips to memory one after the other), one of 512 instances
// that give up 128 pages each 15 (3, 4 and 9 of three launches) and take them again 15 (3.5, 8 and 4), a fork of 32 instances 9.8, of 512 15.  Many instances and large pools
// are behind steps that go one after the other: 8064 instances 50 (resize) and 87 (fork), and a pool of 24 million pages in use but for its last hundred
// 223 us, as 64 workgroups read its counts; with the first hundred free 30.
#include "cache_body.h"
#include "share_internal.h"

namespace ap {
namespace {

constexpr int kThreads = 256, kWaves = 4;
// Workgroups that carry a resize out, each instance after instance: 512 instances that give up and take 128 pages each, and 2048 with 4 pages, by 128, 256,
// 512 and 4096 workgroups 16.9, 14.6, 14.8, 14.8 and 38, 29, 26.5, 32 us.
constexpr int kPickWgs = 64, kApplyWgs = 512;
constexpr int kEntries = 256;                              // of a table that a wave, or half of one, asks for together: one after the other is a trip to memory each
constexpr int kSmallThreads = 1024, kSmallSegments = 256, kSmallInstances = 32;

constexpr int kMostLacking = 0x7fffffff;                   // that info has room for

struct Head { int needed, lacking, live, moved; };

template <typename T> __device__ __forceinline__ T* at(char* ws, size_t offset) { return reinterpret_cast<T*>(ws + offset); }
__device__ __forceinline__ bool in_pool(const Pages& p, int page) { return (unsigned)page < (unsigned)p.n_pages; }
__device__ __forceinline__ int sum_int(int x) {            // over the wave's lanes
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ long long sum_long(long long x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ int lanes_before(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}
// An instance is a workgroup's, a wave's or, where one workgroup has them all, half a wave's: LANES of a wave, whose halves may go different ways.
template <int LANES> __device__ __forceinline__ unsigned long long ballot_of(bool x) {      // over the instance's lanes
  return __ballot(x) & (LANES == 64 ? ~0ull : 0xffffffffull << (threadIdx.x & 32));
}
// Adds to seg, of the page of every lane with `some`: an addition for each segment that lanes have, as additions to one word wait for each other.
__device__ __forceinline__ void add_by_segment(const Pages& p, bool some, int page, int by) {
  unsigned long long todo = __ballot(some);
  const int s = page / kSegment;
  while (todo != 0) {
    const int first = __ffsll(todo) - 1;
    const unsigned long long same = __ballot(some && s == __builtin_amdgcn_readlane(s, first)) & todo;
    if ((int)(threadIdx.x & 63) == first) atomicAdd(p.seg + s, by * __popcll(same));
    todo &= ~same;
  }
}
// Adds to the counts of U pages of every lane with `some`, which are asked for together: returns how many were `border` before.  seg follows.
template <int LANES, int U> __device__ __forceinline__ int change_pages(const Pages& p, const bool (&some)[U], const int (&page)[U], int by, int border) {
  int was[U], n = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) was[u] = some[u] ? atomicAdd(p.refs + page[u], by) : border - 1;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool crossed = some[u] && was[u] == border;
    add_by_segment(p, crossed, page[u], -by);
    n += __popcll(ballot_of<LANES>(crossed));
  }
  return n;
}
// One less entry that names the page: returns how many pages are free now.
template <int LANES, int U> __device__ __forceinline__ int drop_pages(const Pages& p, const bool (&some)[U], const int (&page)[U]) {
  return change_pages<LANES, U>(p, some, page, -1, 1);
}
// One more: returns how many pages are not free any longer (that were given up by others a moment ago).
template <int LANES, int U> __device__ __forceinline__ int name_pages(const Pages& p, const bool (&some)[U], const int (&page)[U]) {
  return change_pages<LANES, U>(p, some, page, 1, 0);
}
// Whether any lane has any of U.
template <int U> __device__ __forceinline__ bool any_of(const bool (&x)[U]) {
  bool y = false;
#pragma unroll
  for (int u = 0; u < U; ++u) y |= x[u];
  return __any(y);
}
// A workgroup's sum of what its waves freed, to info[0]; s_free is a word of LDS that was 0.
__device__ __forceinline__ void add_free(int freed, int* s_free, int32_t* info) {
  if ((threadIdx.x & 63) == 0 && freed != 0) atomicAdd(s_free, freed);
  __syncthreads();
  if (threadIdx.x == 0 && *s_free != 0) atomicAdd(info, *s_free);
}
// Number of this wave in the workgroup.
__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
// The first `rows` rows of K and V of a page, by `threads` threads: load() asks for kPieces pieces of each, store() puts them and all others.
struct RowCopy {
  static constexpr int kPieces = 4;
  u32x4 *K, *V;
  size_t src, dst;
  int n, tid, threads;
  u32x4 k[kPieces], v[kPieces];
  __device__ __forceinline__ RowCopy(const Pages& p, int from, int to, int rows, int tid_, int threads_) : tid(tid_), threads(threads_) {
    const size_t page = (size_t)p.row_pieces << p.lb;
    K = static_cast<u32x4*>(p.K); V = static_cast<u32x4*>(p.V);
    src = from * page; dst = to * page;
    n = rows * p.row_pieces;
  }
  __device__ __forceinline__ void load(int x0 = 0) {
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      const int x = x0 + tid + u * threads;
      if (x < n) {
        k[u] = K[src + x];
        v[u] = V[src + x];
      }
    }
  }
  __device__ __forceinline__ void store() {
    for (int x0 = 0; x0 < n; x0 += kPieces * threads) {
      if (x0 > 0) load(x0);
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int x = x0 + tid + u * threads;
        if (x < n) {
          K[dst + x] = k[u];
          V[dst + x] = v[u];
        }
      }
    }
  }
};

// Whole pages of K and V, one a workgroup at a time: page(x) says where from and where to, and whether at all.  The memory's rate bounds it, and what a
// call moves is not read again soon, so it goes past the caches: 2 x 130 MB of a pool of 4 GB 114 us (4.6 TB/s), with ordinary loads and stores 122;
// 2 x 170 MB of sequences set aside 137 (5.0) and 142.  Two or four pages of a thread under way change nothing.
struct Move { int src, dst; bool real; };
template <typename PAGE>
__device__ __forceinline__ void move_pages(const u32x4* K_src, const u32x4* V_src, u32x4* K_dst, u32x4* V_dst, int n, int page_pieces, PAGE page) {
  for (unsigned x = blockIdx.x; x < (unsigned)n; x += gridDim.x) {          // (up to 2^31 - 1, and a step behind)
    const Move m = page((int)x);
    if (!m.real) continue;
    const size_t src = (size_t)m.src * page_pieces, dst = (size_t)m.dst * page_pieces;
    for (int y = threadIdx.x; y < page_pieces; y += kThreads) {
      const u32x4 k = __builtin_nontemporal_load(K_src + src + y), v = __builtin_nontemporal_load(V_src + src + y);
      __builtin_nontemporal_store(k, K_dst + dst + y);
      __builtin_nontemporal_store(v, V_dst + dst + y);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- counting
__global__ __launch_bounds__(kThreads) void pages_clear_kernel(Pages p) {
  const long long x = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (x < p.n_pages) p.refs[x] = 0;
  if (x < p.segments) p.seg[x] = 0;
}
__global__ __launch_bounds__(kThreads) void pages_count_kernel(Pages p) {
  const size_t all = (size_t)p.n_inst * p.nb_cap;
  for (size_t x = (size_t)blockIdx.x * kThreads + threadIdx.x; x < all; x += (size_t)gridDim.x * kThreads)
    if (in_pool(p, p.table[x])) atomicAdd(p.refs + p.table[x], 1);
}
__global__ __launch_bounds__(kThreads) void pages_free_kernel(Pages p) {
  const int s = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (s >= p.segments) return;
  int n = 0;
  for (int x = lane; x < kSegment; x += 64) {
    const long long page = (long long)s * kSegment + x;
    n += page < p.n_pages && p.refs[page] <= 0;
  }
  n = sum_int(n);
  if (lane == 0) p.seg[s] = n;
}

// ---------------------------------------------------------------------------------------------------------------- needs
struct Rows { int length, kept, want, own; };              // rows; rows that are not to be written; blocks; first block that is
__device__ __forceinline__ Rows rows_of(const ResizeArgs& a, int i) {
  Rows r;
  r.length = clamped(a.len[i], 0, a.p.t_cap);
  const int n = a.n_new == nullptr ? a.q_cap : clamped(a.n_new[i], 0, a.q_cap);
  r.kept = n < r.length ? r.length - n : 0;
  r.want = (int)(((long long)r.length + (1 << a.p.lb) - 1) >> a.p.lb);
  r.own = n > 0 ? r.kept >> a.p.lb : r.want;
  return r;
}

// What an instance needs: pages, and (fork) the rows it has from now on.
struct Need { int pages, rows; };
// The blocks of instance i that need a page.
template <int LANES> __device__ __forceinline__ Need resize_need(const ResizeArgs& a, int i) {
  constexpr int U = kEntries / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const Rows r = rows_of(a, i);
  const int32_t* table = a.p.table + (size_t)i * a.p.nb_cap;
  int32_t* staged = at<int32_t>(a.ws, a.w.staged) + (size_t)i * a.p.nb_cap;
  int count = 0;
  for (int k0 = 0; k0 < r.want; k0 += kEntries) {
    int page[U];
    bool needs[U], asks[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + LANES * u + lane;
      page[u] = table[k < a.p.nb_cap ? k : a.p.nb_cap - 1];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + LANES * u + lane;
      needs[u] = k < r.want && !in_pool(a.p, page[u]);
      asks[u] = k < r.want && k >= r.own && !needs[u];
    }
    if (any_of(asks)) {                                    // of pages of its own, or shared?
      int refs[U];
#pragma unroll
      for (int u = 0; u < U; ++u) refs[u] = a.p.refs[asks[u] ? page[u] : 0];
#pragma unroll
      for (int u = 0; u < U; ++u) needs[u] |= asks[u] && refs[u] > 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned long long mask = ballot_of<LANES>(needs[u]);
      if (needs[u]) staged[count + lanes_before(mask)] = k0 + LANES * u + lane;
      count += __popcll(mask);
    }
  }
  return Need{count, 0};
}
// To the launches that follow.
__device__ __forceinline__ void hand_on(char* ws, const PagesWs& w, int i, Need need) {
  if ((threadIdx.x & 63) != 0) return;
  at<int32_t>(ws, w.need)[i] = need.pages;
  at<int32_t>(ws, w.length)[i] = need.rows;
}
__global__ __launch_bounds__(kThreads) void resize_need_kernel(ResizeArgs a) {
  const int i = blockIdx.x * kWaves + wave_of();
  if (i < a.p.n_inst) hand_on(a.ws, a.w, i, resize_need<64>(a, i));
}

// The new table of instance j, which goes on from instance p, and whether its last page is to be copied.  Rows: -1 if it stays as it is.
template <int LANES> __device__ __forceinline__ Need fork_need(const ForkArgs& a, int j) {
  constexpr int U = kEntries / LANES;
  const int lane = threadIdx.x & (LANES - 1), p = a.parent[j];
  const bool some = (unsigned)p < (unsigned)a.p.n_inst;
  if (!some || p == j) return Need{0, some ? -1 : 0};
  const int L = clamped(a.len[p], 0, a.p.t_cap), full = L >> a.p.lb, rest = L & ((1 << a.p.lb) - 1);
  bool heir = false;
  if (rest > 0 && a.parent[p] != p) {                      // the lowest that goes on from p takes its last page over
    heir = true;
    for (int x0 = 0; x0 < j && heir; x0 += kEntries) {
      int of[U];
#pragma unroll
      for (int u = 0; u < U; ++u) of[u] = a.parent[x0 + LANES * u + lane < j ? x0 + LANES * u + lane : 0];
      bool other = false;
#pragma unroll
      for (int u = 0; u < U; ++u) other |= x0 + LANES * u + lane < j && of[u] == p;
      heir = ballot_of<LANES>(other) == 0;
    }
  }
  const int32_t* table = a.p.table + (size_t)p * a.p.nb_cap;
  int32_t* staged = at<int32_t>(a.ws, a.w.staged) + (size_t)j * a.p.nb_cap;
  const int n = full + (rest > 0);
  for (int k0 = 0; k0 < n; k0 += kEntries) {
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + LANES * u + lane;
      page[u] = table[k < a.p.nb_cap ? k : a.p.nb_cap - 1];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + LANES * u + lane;
      if (k < n) staged[k] = page[u];
    }
  }
  return Need{rest > 0 && !heir && in_pool(a.p, table[full]), L};
}
__global__ __launch_bounds__(kThreads) void fork_need_kernel(ForkArgs a) {
  const int j = blockIdx.x * kWaves + wave_of();
  if (j < a.p.n_inst) hand_on(a.ws, a.w, j, fork_need<64>(a, j));
}

// ---------------------------------------------------------------------------------------------------------------- free pages
// The free pages of segments [s0, s1) are those from number `before` on; the first n of all are picked and in use from now on.  Called by a
// workgroup of NT threads; s_wave: a word of LDS for each of its waves.
template <int NT> __device__ __forceinline__ void pick_segments(const Pages& p, int s0, int s1, int before, int n, int32_t* picked, int32_t* taken, int* s_wave) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int s = s0; s < s1; ++s) {
    if (before >= n) {                                     // (no more are wanted)
      for (; s < s1; s += NT)
        if (s + tid < s1) taken[s + tid] = 0;
      return;
    }
    int mine[kSegment / NT], count = 0;
#pragma unroll
    for (int e = 0; e < kSegment / NT; ++e) {
      const long long page = (long long)s * kSegment + tid * (kSegment / NT) + e;
      mine[e] = before < n && page < p.n_pages && p.refs[page] <= 0;
      count += mine[e];
    }
    int upto = count;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int rank = before + upto - count, all = 0;
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) rank += s_wave[w];
      all += s_wave[w];
    }
#pragma unroll
    for (int e = 0; e < kSegment / NT; ++e)
      if (mine[e]) {
        if (rank >= 0 && rank < n) {
          const int page = s * kSegment + tid * (kSegment / NT) + e;
          picked[rank] = page;
          p.refs[page] = 1;
        }
        ++rank;
      }
    if (tid == 0) taken[s] = n - before < all ? (n > before ? n - before : 0) : all;
    before += all;
  }
}
template <int NT> __device__ __forceinline__ int sum_of(const int32_t* x, int n, int* s_wave) {     // by a workgroup
  int mine = 0;
  for (int k = threadIdx.x; k < n; k += NT) mine += x[k];
  mine = sum_int(mine);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = mine;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < NT / 64; ++w) all += s_wave[w];
  return all;
}

// What all instances need, by a workgroup: up to all entries of the table, which may be more than 32 bits hold.
__device__ __forceinline__ long long needed(const int32_t* need, int n, long long* s_wave) {
  long long mine = 0;
  for (int k = threadIdx.x; k < n; k += kThreads) mine += need[k];
  mine = sum_long(mine);
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = mine;
  __syncthreads();
  long long all = 0;
  for (int w = 0; w < kWaves; ++w) all += s_wave[w];
  return all;
}

// Picks the pages of the instances' needs: workgroup `which` of `wgs`; the one behind them sums up what the instances before each one need (sums that
// are asked for only where all of them are no more than the pool has pages).  info as if nothing were given up.
__global__ __launch_bounds__(kThreads) void pages_pick_kernel(Pages p, char* ws, PagesWs w, int32_t* info) {
  __shared__ int s_wave[kWaves];
  __shared__ long long s_needed[kWaves];
  const int which = blockIdx.x, wgs = gridDim.x - 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t* need = at<int32_t>(ws, w.need);
  if (which < wgs) {
    const long long all = needed(need, p.n_inst, s_needed);
    const int free = clamped(sum_of<kThreads>(p.seg, p.segments, s_wave), 0, p.n_pages), n = all <= free ? (int)all : 0;
    const int each = (p.segments + wgs - 1) / wgs;
    const int s0 = which * each, s1 = s0 + each < p.segments ? s0 + each : p.segments;
    if (s0 < s1) {
      const int before = s0 == 0 ? 0 : sum_of<kThreads>(p.seg, s0, s_wave);
      pick_segments<kThreads>(p, s0, s1, before, n, at<int32_t>(ws, w.picked), at<int32_t>(ws, w.taken), s_wave);
    }
    if (which == 0 && tid == 0) {
      const long long lacking = all - free;
      Head* head = at<Head>(ws, w.head);
      head->needed = n;
      head->lacking = lacking <= 0 ? 0 : (lacking < kMostLacking ? (int)lacking : kMostLacking);
      info[0] = free - n;
      info[1] = head->lacking;
    }
    return;
  }
  constexpr int U = 4;                                     // instances of a thread at a time
  unsigned done = 0;
  for (int i0 = 0; i0 < p.n_inst; i0 += U * kThreads) {
    unsigned x[U], mine = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + U * tid + u;
      x[u] = i < p.n_inst ? need[i] : 0;
      mine += x[u];
    }
    unsigned upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    unsigned ahead = done + upto - mine;
    for (int v = 0; v < kWaves; ++v) {
      if (v < wave) ahead += s_wave[v];
      done += s_wave[v];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + U * tid + u;
      if (i < p.n_inst) at<int32_t>(ws, w.before)[i] = ahead;
      ahead += x[u];
    }
  }
}
__device__ __forceinline__ void settle_segments(const Pages& p, const int32_t* taken) {
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < p.segments; s += gridDim.x * blockDim.x)
    if (taken[s] > 0) atomicAdd(p.seg + s, -taken[s]);
}

// ---------------------------------------------------------------------------------------------------------------- carrying it out
// Instance i's, by NT threads: a workgroup, or half a wave.  n pages are needed, `before` by the instances in front.  Returns how many pages are free now, a
// wave's (half's) own count.
template <int NT> __device__ __forceinline__ int resize_apply(const ResizeArgs& a, int i, int n, int before, int tid) {
  constexpr int LANES = NT < 64 ? NT : 64, U = NT < 64 ? kEntries / NT : 1;
  const Rows r = rows_of(a, i);
  int32_t* table = a.p.table + (size_t)i * a.p.nb_cap;
  const int32_t* staged = at<int32_t>(a.ws, a.w.staged) + (size_t)i * a.p.nb_cap;
  const int32_t* picked = at<int32_t>(a.ws, a.w.picked) + before;
  const int rest = r.kept & ((1 << a.p.lb) - 1);
  int freed = 0;
  if (n > 0 && rest > 0 && r.own < r.want) {
    // The first block that is written may have rows that stay, of a page that others keep.
    for (int x = 0; x < n && staged[x] <= r.own; ++x)
      if (staged[x] == r.own && in_pool(a.p, table[r.own]) && in_pool(a.p, picked[x])) {
        RowCopy copy(a.p, table[r.own], picked[x], rest, tid, NT);
        copy.load();
        copy.store();
      }
    if (NT > 64) __syncthreads();
  }
  for (int k0 = r.want; k0 < a.p.nb_cap; k0 += NT * U) {
    int page[U];
    bool named[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + NT * u + tid;
      page[u] = table[k < a.p.nb_cap ? k : a.p.nb_cap - 1];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + NT * u + tid;
      if (k >= a.p.nb_cap) page[u] = -1;
      named[u] = in_pool(a.p, page[u]);
      if (page[u] != -1) table[k] = -1;
    }
    if (any_of(named)) freed += drop_pages<LANES, U>(a.p, named, page);
  }
  for (int x0 = 0; x0 < n; x0 += NT) {
    const int x = x0 + tid, page = picked[x < n ? x : 0];
    const bool some = x < n && in_pool(a.p, page);
    const int k = staged[x < n ? x : 0], old[1] = {some ? table[k] : -1};
    const bool named[1] = {in_pool(a.p, old[0])};
    if (some) table[k] = page;
    if (any_of(named)) freed += drop_pages<LANES, 1>(a.p, named, old);
  }
  return freed;
}
__global__ __launch_bounds__(kThreads) void resize_apply_kernel(ResizeArgs a) {
  __shared__ int s_free;
  if (at<Head>(a.ws, a.w.head)->lacking > 0) return;
  if (threadIdx.x == 0) s_free = 0;
  __syncthreads();
  settle_segments(a.p, at<int32_t>(a.ws, a.w.taken));
  const int32_t *need = at<int32_t>(a.ws, a.w.need), *before = at<int32_t>(a.ws, a.w.before);
  int freed = 0;
  for (int i = blockIdx.x; i < a.p.n_inst; i += gridDim.x) freed += resize_apply<kThreads>(a, i, need[i], before[i], threadIdx.x);
  add_free(freed, &s_free, a.info);
}

// L: its rows from now on, -1: it stays as it is.
template <int NT> __device__ __forceinline__ int fork_apply(const ForkArgs& a, int j, int L, int need, int before, int tid) {
  constexpr int LANES = NT < 64 ? NT : 64, U = NT < 64 ? kEntries / NT : 2;
  if (L < 0) {
    if (tid == 0 && a.len_out != a.len) a.len_out[j] = a.len[j];
    return 0;
  }
  const int full = L >> a.p.lb, rest = L & ((1 << a.p.lb) - 1), n = full + (rest > 0);
  int32_t* table = a.p.table + (size_t)j * a.p.nb_cap;
  const int32_t* staged = at<int32_t>(a.ws, a.w.staged) + (size_t)j * a.p.nb_cap;
  int old[U], now[U];
  auto ask = [&](int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + NT * u + tid, x = k < a.p.nb_cap ? k : a.p.nb_cap - 1;
      old[u] = table[x];
      now[u] = staged[x];
    }
  };
  // The tables, then the rows that are copied and the counts: what a step needs is asked for together.
  const int page = need > 0 ? at<int32_t>(a.ws, a.w.picked)[before] : 0, last = need > 0 ? staged[full] : 0;
  ask(0);
  const bool copied = need > 0 && in_pool(a.p, page);
  RowCopy copy(a.p, last, page, copied ? rest : 0, tid, NT);
  copy.load();
  int freed = 0;
  for (int k0 = 0; k0 < a.p.nb_cap; k0 += NT * U) {
    bool changed[U], named[U], gone[U];
    if (k0 > 0) ask(k0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + NT * u + tid;
      const bool fresh = copied && k == full;
      now[u] = fresh ? page : (k < n ? now[u] : -1);
      changed[u] = k < a.p.nb_cap && now[u] != old[u];
      if (changed[u]) table[k] = now[u];
      named[u] = changed[u] && !fresh && in_pool(a.p, now[u]);
      gone[u] = changed[u] && in_pool(a.p, old[u]);
    }
    if (any_of(named)) freed -= name_pages<LANES, U>(a.p, named, now);
    if (any_of(gone)) freed += drop_pages<LANES, U>(a.p, gone, old);
  }
  copy.store();
  if (tid == 0) a.len_out[j] = L;
  return freed;
}
__global__ __launch_bounds__(kThreads) void fork_apply_kernel(ForkArgs a) {
  __shared__ int s_free;
  const bool lacking = at<Head>(a.ws, a.w.head)->lacking > 0;
  if (!lacking) settle_segments(a.p, at<int32_t>(a.ws, a.w.taken));
  if (threadIdx.x == 0) s_free = 0;
  __syncthreads();
  const int j = blockIdx.x, L = lacking ? -1 : at<int32_t>(a.ws, a.w.length)[j];
  add_free(fork_apply<kThreads>(a, j, L, at<int32_t>(a.ws, a.w.need)[j], at<int32_t>(a.ws, a.w.before)[j], threadIdx.x), &s_free, a.info);
}

// As pages_pick_kernel, by one workgroup for kSmallInstances instances and kSmallSegments segments at most: what is loaded is asked for together.
// need, before: in LDS.
__device__ __forceinline__ void pick_by_one(const Pages& p, char* ws, const PagesWs& w, const Need* need, int* before, int* info, int* s_wave) {
  __shared__ int s_needed, s_sums[kSmallSegments / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < kSmallSegments) {
    const int x = tid < p.n_inst ? need[tid].pages : 0, segment = sum_int(tid < p.segments ? p.seg[tid] : 0);
    if (lane == 0) s_sums[tid >> 6] = segment;
    if (tid < 64) {
      int upto = x;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      if (tid < p.n_inst) before[tid] = upto - x;
      if (lane == 63) s_needed = upto;
    }
  }
  __syncthreads();
  int free = 0;
#pragma unroll
  for (int v = 0; v < kSmallSegments / 64; ++v) free += s_sums[v];
  const int n = s_needed;
  free = clamped(free, 0, p.n_pages);
  pick_segments<kSmallThreads>(p, 0, p.segments, 0, n <= free ? n : 0, at<int32_t>(ws, w.picked), at<int32_t>(ws, w.taken), s_wave);
  if (tid == 0) {
    info[0] = n > free ? free : free - n;
    info[1] = n > free ? n - free : 0;
  }
}
// All of it by one workgroup, an instance half a wave at a time: a fork of 32 instances and a resize of them are one round of trips to memory each.
constexpr int kHalf = 32, kHalves = kSmallThreads / kHalf;
template <typename ARGS, typename NEED, typename APPLY> __device__ __forceinline__ void by_one(const ARGS& a, NEED need, APPLY apply) {
  __shared__ int s_wave[kSmallThreads / 64], s_free, s_info[2], s_before[kSmallInstances];
  __shared__ Need s_need[kSmallInstances];
  const int half = threadIdx.x / kHalf;
  if (threadIdx.x == 0) s_free = 0;
  for (int i = half; i < a.p.n_inst; i += kHalves) {
    const Need x = need(i);
    if (threadIdx.x % kHalf == 0) s_need[i] = x;
  }
  __syncthreads();
  pick_by_one(a.p, a.ws, a.w, s_need, s_before, s_info, s_wave);
  __syncthreads();
  const bool lacking = s_info[1] > 0;
  if (!lacking) settle_segments(a.p, at<int32_t>(a.ws, a.w.taken));
  int freed = 0;
  for (int i = half; i < a.p.n_inst; i += kHalves) freed += apply(i, s_need[i], s_before[i], lacking);
  if (threadIdx.x % kHalf == 0 && freed != 0) atomicAdd(&s_free, freed);
  __syncthreads();
  if (threadIdx.x == 0) {
    a.info[0] = s_info[0] + s_free;
    a.info[1] = s_info[1];
  }
}
__global__ __launch_bounds__(kSmallThreads) void resize_small_kernel(ResizeArgs a) {
  const int lane = threadIdx.x % kHalf;
  by_one(a, [&](int i) { return resize_need<kHalf>(a, i); }, [&](int i, Need need, int before, bool lacking) {
    return lacking ? 0 : resize_apply<kHalf>(a, i, need.pages, before, lane);
  });
}
__global__ __launch_bounds__(kSmallThreads) void fork_small_kernel(ForkArgs a) {
  const int lane = threadIdx.x % kHalf;
  by_one(a, [&](int j) { return fork_need<kHalf>(a, j); }, [&](int j, Need need, int before, bool lacking) {
    return fork_apply<kHalf>(a, j, lacking ? -1 : need.rows, need.pages, before, lane);
  });
}
// What one workgroup does sooner than three launches: few instances, tables that are looked through quickly, and few bytes that it may have to copy.
// Tables of 132 entries, captured and called one by one (where three launches are bound by the host): resize of 8, 32, 48, 64 instances 6.7 and 7.3, 9.2 and
// 9.5, 11.9 and 12.0, 14.5 and 14.7 us, by three launches 9.5 and 12.8; fork of 8, 32, 64 instances, pages of 8 KB (K and V), 9.1 and 9.2, 10.6 and 10.6, 16,
// by three launches 11.4 and 13.3.
bool small(const Pages& p, long long copied) {
  return p.n_inst <= kSmallInstances && (long long)p.n_inst * p.nb_cap <= 160 * kSmallInstances && p.segments <= kSmallSegments && copied <= 256 * 1024;
}

// ---------------------------------------------------------------------------------------------------------------- compaction
// The x-th page in use that lies at `live` (their number) or behind goes to the x-th free page in front.
__global__ __launch_bounds__(kThreads) void compact_list_kernel(CompactArgs a) {
  __shared__ int s_wave[kWaves];
  const Pages& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int live = p.n_pages - clamped(sum_of<kThreads>(p.seg, p.segments, s_wave), 0, p.n_pages);
  // Free pages in front: those of whole segments, and of the one that `live` lies in.
  const int sl = live / kSegment;
  int moved = sl > 0 ? sum_of<kThreads>(p.seg, sl, s_wave) : 0;
  {
    int x = 0;
    for (int page = sl * kSegment + tid; page < live; page += kThreads) x += p.refs[page] <= 0;
    x = sum_int(x);
    __syncthreads();
    if (lane == 0) s_wave[wave] = x;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) moved += s_wave[w];
    moved = clamped(moved, 0, live);
  }
  if (blockIdx.x == 0 && tid == 0) {
    Head* head = at<Head>(a.ws, a.w.head);
    head->live = live;
    head->moved = moved;
    a.info[0] = p.n_pages - live;
    a.info[1] = moved;
  }
  const int each = (p.segments + gridDim.x - 1) / gridDim.x;
  const int s0 = blockIdx.x * each, s1 = s0 + each < p.segments ? s0 + each : p.segments;
  if (s0 >= s1) return;
  int before = sum_of<kThreads>(p.seg, s0, s_wave);                  // free pages before
  for (int s = s0; s < s1; ++s) {
    int mine[kSegment / kThreads], count = 0;
#pragma unroll
    for (int e = 0; e < kSegment / kThreads; ++e) {
      const long long page = (long long)s * kSegment + tid * (kSegment / kThreads) + e;
      mine[e] = page < p.n_pages && p.refs[page] <= 0;
      count += mine[e];
    }
    int upto = count;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int rank = before + upto - count;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) rank += s_wave[w];
      before += s_wave[w];
    }
#pragma unroll
    for (int e = 0; e < kSegment / kThreads; ++e) {
      const long long page = (long long)s * kSegment + tid * (kSegment / kThreads) + e;
      if (page >= p.n_pages) continue;
      if (mine[e]) {
        if (page < live && rank >= 0 && rank < moved) at<int32_t>(a.ws, a.w.picked)[rank] = (int)page;
        ++rank;
      } else if (page >= live) {
        const int x = (int)page - rank - (live - moved);   // pages in use before it, without those in front
        if (x >= 0 && x < moved) at<int32_t>(a.ws, a.w.from)[x] = (int)page;
        at<int32_t>(a.ws, a.w.rank)[page] = x;
      }
    }
  }
}
__global__ __launch_bounds__(kThreads) void compact_move_kernel(CompactArgs a) {
  const Pages& p = a.p;
  const Head head = *at<Head>(a.ws, a.w.head);
  const int32_t *hole = at<int32_t>(a.ws, a.w.picked), *from = at<int32_t>(a.ws, a.w.from), *rank = at<int32_t>(a.ws, a.w.rank);
  const int tid = threadIdx.x;
  move_pages(static_cast<const u32x4*>(p.K), static_cast<const u32x4*>(p.V), static_cast<u32x4*>(p.K), static_cast<u32x4*>(p.V), head.moved,
             p.row_pieces << p.lb, [&](int x) { return Move{from[x], hole[x], in_pool(p, from[x]) && in_pool(p, hole[x])}; });
  for (int x = blockIdx.x * kThreads + tid; x < head.moved; x += gridDim.x * kThreads)
    if (in_pool(p, from[x]) && in_pool(p, hole[x])) {
      p.refs[hole[x]] = p.refs[from[x]];
      p.refs[from[x]] = 0;
    }
  const size_t all = (size_t)p.n_inst * p.nb_cap, step = (size_t)gridDim.x * kThreads;
  for (size_t x = (size_t)blockIdx.x * kThreads + tid; x < all; x += step) {
    const int page = p.table[x];
    if (!in_pool(p, page) || page < head.live) continue;
    const int y = rank[page];                              // (of a page that refs says is free, anything)
    if ((unsigned)y < (unsigned)head.moved && from[y] == page) p.table[x] = hole[y];
  }
  for (int s = blockIdx.x * kThreads + tid; s < p.segments; s += gridDim.x * kThreads) {
    const long long lo = (long long)s * kSegment, hi = lo + kSegment < p.n_pages ? lo + kSegment : p.n_pages;
    p.seg[s] = (int)(hi <= head.live ? 0 : hi - (lo > head.live ? lo : head.live));
  }
}

__global__ __launch_bounds__(kThreads) void pages_copy_kernel(const u32x4* K_src, const u32x4* V_src, int n_src, const int32_t* from, u32x4* K_dst,
                                                              u32x4* V_dst, int n_dst, const int32_t* to, int n, int page_pieces) {
  move_pages(K_src, V_src, K_dst, V_dst, n, page_pieces, [&](int x) {
    const int src = from == nullptr ? x : from[x], dst = to == nullptr ? x : to[x];
    return Move{src, dst, (unsigned)src < (unsigned)n_src && (unsigned)dst < (unsigned)n_dst};
  });
}

unsigned pick_wgs(const Pages& p) { return p.segments < kPickWgs ? p.segments : kPickWgs; }
unsigned per_wave(int n) { return ((unsigned)n + kWaves - 1) / kWaves; }

}  // namespace

hipError_t launch_pages_count(const Pages& p, hipStream_t st) {
  pages_clear_kernel<<<(unsigned)(((long long)p.n_pages + kThreads - 1) / kThreads), kThreads, 0, st>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t wgs = ((size_t)p.n_inst * p.nb_cap + kThreads - 1) / kThreads;
  pages_count_kernel<<<(unsigned)(wgs < 4096 ? wgs : 4096), kThreads, 0, st>>>(p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  pages_free_kernel<<<per_wave(p.segments), kThreads, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t launch_pages_resize(const ResizeArgs& a, hipStream_t st) {
  if (small(a.p, 0)) {                                     // (copies are rare here: where rows go back into shared pages)
    resize_small_kernel<<<1, kSmallThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  resize_need_kernel<<<per_wave(a.p.n_inst), kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_pick_kernel<<<pick_wgs(a.p) + 1, kThreads, 0, st>>>(a.p, a.ws, a.w, a.info);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  resize_apply_kernel<<<a.p.n_inst < kApplyWgs ? a.p.n_inst : kApplyWgs, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const ForkArgs& a, hipStream_t st) {
  if (small(a.p, (long long)a.p.n_inst * 32 * a.p.row_pieces << a.p.lb)) {
    fork_small_kernel<<<1, kSmallThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  fork_need_kernel<<<per_wave(a.p.n_inst), kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_pick_kernel<<<pick_wgs(a.p) + 1, kThreads, 0, st>>>(a.p, a.ws, a.w, a.info);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  fork_apply_kernel<<<a.p.n_inst, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t st) {
  compact_list_kernel<<<pick_wgs(a.p), kThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_move_kernel<<<2048, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const void* K_src, const void* V_src, int n_src, const int32_t* from, void* K_dst, void* V_dst, int n_dst,
                             const int32_t* to, int n, int page_pieces, hipStream_t st) {
  pages_copy_kernel<<<n < 4096 ? n : 4096, kThreads, 0, st>>>(static_cast<const u32x4*>(K_src), static_cast<const u32x4*>(V_src), n_src, from,
                                                              static_cast<u32x4*>(K_dst), static_cast<u32x4*>(V_dst), n_dst, to, n, page_pieces);
  return hipGetLastError();
}

}  // namespace ap
