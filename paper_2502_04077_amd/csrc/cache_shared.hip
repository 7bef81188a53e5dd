// Attention of one new token, or of few, per instance over a cache whose first rows the instance has in common with others.
//
// Rows in common are read once for all of a group: the members' queries are the rows of one product.  What lies behind them is every
// instance's own.  With a source of cache rows j (a group's beginning, or an instance's rows behind it), for every row x of q that belongs to it,
// at position p of its cache,
//
//   s_xj = q_x . K_j / sqrt(d),  m_x = max_j s_xj,  l_x = sum_j exp(s_xj - m_x),  o_x = sum_j exp(s_xj - m_x) V_j,   over the rows j that p sees;
//
// out_x = sum over its sources of exp(m_x - m) o_x / sum of exp(m_x - m) l_x, for m the largest m_x.
//
// A source's rows of q are in tiles of 128, its rows of K and V in tiles of 64 (fp32: 32); where a tile has no more than 32 rows of q, which is
// memory-bound, in groups of 32 (fp32, d = 128: 16).  The products of many rows of q, of all sources one after the other, are cut into equal shares, a workgroup each, and those of
// few rows into shares of a wave each: the one needs the matrix unit, the other the memory, and a CU has room for a workgroup of both.  Whoever has a
// share leaves (m, l, o) of every piece of it, and a second launch joins the pieces.
//
// 64 sequences of 40 to 2050 rows behind 8190 in common (8 KV heads, g = 4, d = 128, decode) take 53 us; their 172 MB are read in 24 at the rate of a large
// read.  Of the first launch's 46 us 6 go by until the shares are known (two trips to memory, sums over the sources, the sources of a share), 3 to 6 until a
// piece's first product (table, rows; members, lengths, queries), and the shares' ends lie 5 apart.  A tile of 64 rows takes a workgroup 3.3 us (128 rows of
// q, probabilities of 24 bits; the matrix unit), a group of 32 a wave 3 to 4 us: at d = 128 its part of LDS holds one group, whose K is sent for again when
// its scores are done and whose V when its second product is, so that every group waits for memory.  Over the launch the matrix unit is busy 25 % of the time, 36 % of the
// waves' time is spent waiting, and 210 MB come from memory, 4.6 TB/s.  In fp32 (16 sequences of 50 to 500 rows behind two beginnings of 4000, 36 us) 25 % and
// 42 %, 100 MB, 2.8 TB/s: bytes under way, one group of 16 rows a wave.
// Four samples of one prompt of 2041 rows take 18 us, which is this chain (4 us until the shares are known, 2.5 until the first product) and the second launch's.
#include "cache_tiles.h"
#include "share_internal.h"

namespace ap {
namespace {

// ---------------------------------------------------------------------------------------------------------------- the plan
// First member, place among the members, number of members and rows in common: every instance looks at all others.
__global__ __launch_bounds__(kThreads) void share_group_kernel(const int32_t* __restrict__ group, const int32_t* __restrict__ shared, int n,
                                                               int t_cap, SharePlan plan) {
  __shared__ __attribute__((aligned(16))) int s_group[kThreads], s_shared[kThreads];
  const int i = blockIdx.x * kThreads + threadIdx.x, mine = i < n ? group[i] : -1;
  int lead = n, rank = 0, count = 0, common = t_cap;
  for (int k0 = 0; k0 < n; k0 += kThreads) {
    __syncthreads();
    const int k = k0 + threadIdx.x;
    s_group[threadIdx.x] = k < n ? group[k] : -1;
    s_shared[threadIdx.x] = k < n ? shared[k] : 0;
    __syncthreads();
#pragma unroll 4
    for (int x = 0; x < kThreads; x += 4) {
      const int4 y = *reinterpret_cast<const int4*>(s_group + x), z = *reinterpret_cast<const int4*>(s_shared + x);
      const int gs[4] = {y.x, y.y, y.z, y.w}, rows[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool same = gs[e] == mine;
        lead = same && k0 + x + e < lead ? k0 + x + e : lead;
        rank += same && k0 + x + e < i;
        count += same;
        common = same && rows[e] < common ? rows[e] : common;
      }
    }
  }
  if (i >= n) return;
  const bool alone = mine < 0 || count < 2;
  plan.inst[i] = alone ? make_int4(i, 0, 1, 0) : make_int4(lead, rank, count, common > 0 ? common : 0);
}
// Groups one after the other, by their first member.
__global__ __launch_bounds__(kThreads) void share_place_kernel(int n, SharePlan plan) {
  __shared__ __attribute__((aligned(16))) int s_count[kThreads];
  const int i = blockIdx.x * kThreads + threadIdx.x;
  int4* inst = plan.inst;
  const int lead = i < n ? inst[i].x : 0, count = i < n ? inst[i].z : 1;
  int ahead = 0, groups = 0, all = 0;
  for (int k0 = 0; k0 < n; k0 += kThreads) {
    __syncthreads();
    const int k = k0 + threadIdx.x;
    s_count[threadIdx.x] = k < n && inst[k].x == k && inst[k].z > 1 ? inst[k].z : 0;
    __syncthreads();
#pragma unroll 4
    for (int x = 0; x < kThreads; x += 4) {
      const int4 y = *reinterpret_cast<const int4*>(s_count + x);
      const int c[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ahead += k0 + x + e < lead ? c[e] : 0;
        groups += k0 + x + e < lead && c[e] > 0;
        all += c[e] > 0;
      }
    }
  }
  if (i == 0) *plan.count = all;
  if (i >= n) return;
  if (count < 2) {
    plan.pos[i] = -1;
    return;
  }
  const int at = ahead + inst[i].y;                        // (nobody else reads or writes this word)
  inst[i].y = ahead;
  plan.pos[i] = at;
  plan.member[at] = i;
  if (lead == i) plan.groups[groups] = make_int4(i, ahead, count, inst[i].w);
}

// ---------------------------------------------------------------------------------------------------------------- sources
// Rows of the cache that a wave with few rows of q goes over at a time, as many as its part of LDS holds: 16 or 32.
template <typename T, int D> constexpr int kGroup = sizeof(T) == 4 && D == 128 ? 16 : 32;
constexpr int kSharedLds = 64 * 1024;       // two workgroups a CU
// What a share counts, in tenths of a microsecond: of a workgroup's time a tile of the cache, and what a tile of rows of q costs beside them; of a
// wave's time a group, and the same.  The least shares.  (As measured, and then varied by a third either way.  Of a wave's, in front and least, 40 and 60: a
// sequence of 150 rows 14.7 us, 4 samples of 2041 and more 18.3, 32 sequences of 110 to 400 19.3, drafts 42.1; 50 and 90: 16.0, 18.5, 20.7, 42.8; 40 and 45:
// 14.6, 19.3, 19.6, 42.1; 50 and 130: 19.1, 20.8, 23.4, 42.7.  A tile of the cache with probabilities of two parts, 24, 26, 28, 30: drafts 50.9, 48.6, 47.7, 48.6.)
template <typename T, bool EXACT> struct Counts {
  static constexpr int WIDE = sizeof(T) == 4 ? 84 : (EXACT ? 32 : 28), WIDE_FRONT = sizeof(T) == 4 ? 60 : 80, WIDE_LEAST = 120;
  static constexpr int NARROW = sizeof(T) == 4 ? 24 : 32, NARROW_FRONT = 40, NARROW_LEAST = sizeof(T) == 4 ? 50 : 60;
};

// Rows [a0, a1) of a cache, and the rows of q that they are for: of a group's members, one after the other, or of the instance alone (count 0).
struct Source {
  int inst, first, count;
  int x0, rows;          // number of its first row of q among all sources', and how many
  int p0;                // count 0: the position of the first query
  int a0, a1, p1, lo0, f;   // rows [a0, f) and [lo0, p1] are seen by one of them at least, f <= lo0; each may be empty
  __device__ __forceinline__ bool row(int j) const { return j >= a0 && j <= p1 && (j >= lo0 || j < f); }
  // Tiles of rows of q: those with many rows, and one with few at the end.
  // (rows >= 0, and so are the bounds but for p1: as unsigned numbers, division is a shift.)
  __device__ __forceinline__ unsigned last() const { return (unsigned)rows % kPrefillRows; }
  __device__ __forceinline__ unsigned wide() const { return (unsigned)rows / kPrefillRows + (last() > kNarrowRows); }
  __device__ __forceinline__ bool narrow() const { return last() - 1u < (unsigned)kNarrowRows; }
};
// The tiles of TT cache rows that it sees: ts from ta on, the others from tb.
struct Tiling {
  int ta, ts, tb, n;
  __device__ __forceinline__ int tile(int u) const { return u < ts ? ta + u : tb + (u - ts); }
};
template <int TT> __device__ __forceinline__ Tiling tiling_of(const Source& s) {
  Tiling t;
  t.ta = (unsigned)s.a0 / TT;
  const int end = ((unsigned)s.f + (TT - 1)) / TT, behind = ((unsigned)s.p1 + TT) / TT;
  t.ts = s.f > 0 ? end - t.ta : 0;
  t.tb = (unsigned)s.lo0 / TT;
  if (t.ts > 0 && t.tb < end) t.tb = end;
  t.n = s.a0 >= s.a1 || s.p1 < 0 || s.rows == 0 ? 0 : t.ts + (behind > t.tb ? behind - t.tb : 0);
  return t;
}
// What a tile of many rows of q counts, and the one with few.
template <typename C, int TT> __device__ __forceinline__ unsigned wide_size(const Source& s) {
  const int n = tiling_of<TT>(s).n;
  return n == 0 ? 0u : C::WIDE_FRONT + (unsigned)n * C::WIDE;
}
template <typename C, int TT> __device__ __forceinline__ unsigned narrow_size(const Source& s) {
  const int n = s.narrow() ? tiling_of<TT>(s).n : 0;
  return n == 0 ? 0u : C::NARROW_FRONT + (unsigned)n * C::NARROW;
}
__device__ __forceinline__ int queries(const SharedArgs& a, int i) { return a.n_q == nullptr ? a.q_cap : clamped(a.n_q[i], 0, a.q_cap); }
// What queries from position p_min on see of rows [a0, a1).
__device__ __forceinline__ void see(const SharedArgs& a, Source& s, int a0, int a1, int p_min) {
  s.a0 = a0;
  s.a1 = a1;
  s.p1 = a1 - 1;
  s.lo0 = a.window > 0 && p_min >= a.window ? p_min - a.window + 1 : 0;
  s.f = a.n_first < s.lo0 ? a.n_first : s.lo0;
  if (s.f > a1) s.f = a1;
  if (s.f <= a0) s.f = 0;
  if (s.lo0 < a0) s.lo0 = a0;
  if (s.lo0 > s.p1) {                                      // the first rows alone
    s.lo0 = s.f;
    s.p1 = s.f - 1;
  }
}
// A source that is the same for all lanes.
__device__ __forceinline__ Source uniform(Source s) {
  int* w = reinterpret_cast<int*>(&s);
#pragma unroll
  for (int k = 0; k < (int)(sizeof(Source) / 4); ++k) w[k] = __builtin_amdgcn_readfirstlane(w[k]);
  return s;
}
// The position of an instance's first query; past all others if it has none.
__device__ __forceinline__ int first_position(const SharedArgs& a, int i) {
  const int q = queries(a, i), own = clamped(a.r.len[i], 0, a.r.t_cap);
  return q > 0 ? own - q : 0x7fffffff;
}
// Sources in their order: the instances', then the groups'.  What has to be loaded for source x is asked for together.  s_low: by the first member, the
// lowest position of a query of the group (only with a window: members one after the other are two trips to memory each); a.low where sizes are in the workspace.
typedef const __attribute__((address_space(3))) int* LowestInLds;
__device__ __forceinline__ Source source_of(const SharedArgs& a, int x, LowestInLds s_low) {
  const int n = a.r.n_inst, i = x < n ? x : 0;
  const int4 line = *(x < n ? a.plan.inst + i : a.plan.groups + (x - n));
  const int m = queries(a, i), own = clamped(a.r.len[i], 0, a.r.t_cap);
  const bool several = line.z > 1 && (unsigned)line.x < (unsigned)n && line.y >= 0 && line.z <= n - line.y;
  const int lead = clamped(a.r.len[several ? line.x : i], 0, a.r.t_cap);
  const int S = several ? clamped(line.w, 0, lead) : 0;
  Source s;
  if (x >= n) {
    s.inst = line.x; s.first = line.y; s.count = line.z;
    s.rows = several ? line.z * a.rows : 0;
    s.x0 = (n + line.y) * a.rows;
    s.p0 = 0;
    int p = 0;
    if (S > 0 && a.window > 0) {
      if (a.sized) p = a.low[line.x];
      else p = s_low[line.x];
    }
    see(a, s, 0, S, p);
  } else {
    s.inst = i; s.first = 0; s.count = 0;
    s.rows = m << a.lg;
    s.x0 = i * a.rows;
    s.p0 = own - m;
    see(a, s, S, own, s.p0);
  }
  return s;
}

// ---------------------------------------------------------------------------------------------------------------- tiles of the cache
// RW consecutive rows that a wave fetches, which may lie in several pages of eight rows and more.  In the place of rows that the source does not see,
// which are not read, stands one that it does.  Wave-uniform, and looked up through the scalar cache: a vector load of the table's would wait for the
// rows under way (a tile that is seen in part then took some 8 us).
template <int RW> struct Fetch {
  static constexpr int RUNS = (RW + 7) / 8;
  const char *k, *v;                                       // row 0, as if all of them lay together
  long long run[RUNS];                                     // and what to add for every eight, in bytes
  long long other;                                         // the one that stands in, relative to row 0
  bool all;
  int j0;
};
template <int RW, int PIECES> __device__ __forceinline__ Fetch<RW> fetch_of(const SharedArgs& a, const TablePages& pages, const Source& s, int j0) {
  constexpr long long bytes = PIECES * 16;
  Fetch<RW> x;
  x.j0 = j0;
  x.all = j0 >= s.a0 && j0 + RW - 1 <= s.p1 && (j0 >= s.lo0 || j0 + RW <= s.f);
  const size_t at = pages.at(j0);
  x.k = static_cast<const char*>(a.K) + at * bytes;
  x.v = static_cast<const char*>(a.V) + at * bytes;
#pragma unroll
  for (int e = 0; e < Fetch<RW>::RUNS; ++e)
    x.run[e] = pages.table == nullptr || (8 * e) >> pages.lb == 0 ? 0 : ((long long)(pages.at(j0 + 8 * e) - at) - 8 * e) * bytes;
  x.other = 0;
  if (!x.all) {
    const int from = j0 < s.f ? s.a0 : s.lo0;
    int j = j0 > from ? j0 : from;
    if (j > s.p1) j = s.p1;
    x.other = ((long long)(pages.at(j & ~7) - at) + (j & 7)) * bytes;
  }
  return x;
}
// Sends them to LDS: the lane chooses the piece, so that it lies where the swizzle says.  r0: the first one's row of the tile.
template <int RW, typename F, bool IS_V, bool ONCE> __device__ __forceinline__ void send_rows(const Fetch<RW>& x, const Source& s, int r0, unsigned lds) {
  constexpr unsigned bytes = F::PIECES * 16;
  constexpr int LOADS = RW * F::PIECES / 64;
  const int lane = threadIdx.x & 63;
  const char* base = IS_V ? x.v : x.k;
  auto row = [&](int l) { return l * F::RPL + lane / F::PIECES; };
  auto piece = [&](int l) {
    const int place = lane % F::PIECES;
    return IS_V ? F::v_place(row(l), place) : F::k_place(r0 + row(l), place);
  };
  if (x.all) {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) to_lds<ONCE>(base + x.run[l * F::RPL / 8], row(l) * bytes + piece(l) * 16, lds + l * 1024);
  } else {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      const long long at = s.row(x.j0 + row(l)) ? x.run[l * F::RPL / 8] + row(l) * (long long)bytes : x.other;
      to_lds_from(base + at + piece(l) * 16, lds + l * 1024);
    }
  }
}
// A piece's tiles of the cache, one after the other.  The first is sent for where this is made, the others while the one before is worked off.
// All threads of the workgroup.
template <typename F> struct Tiles {
  const SharedArgs& a;
  const Source& s;
  const u32x4* s_tiles;
  int u_begin, u_end, wave;
  unsigned buffers;
  Tiling tiling;
  TablePages pages;
  Fetch<F::RW> next;
  __device__ __forceinline__ Tiles(const SharedArgs& a_, const Source& s_, int u0, int u1, const u32x4* lds) : a(a_), s(s_), s_tiles(lds), u_begin(u0), u_end(u1) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    buffers = lds_address(s_tiles);
    tiling = tiling_of<F::TT>(s);
    pages = pages_of(a.r, s.inst);
    next = fetch(u_begin);
    send(u_begin);
  }
  __device__ __forceinline__ Fetch<F::RW> fetch(int u) const {
    return fetch_of<F::RW, F::PIECES>(a, pages, s, tiling.tile(u) * F::TT + wave * F::RW);
  }
  __device__ __forceinline__ void send(int u) {            // tile u, whose rows are those of `next`
    const unsigned to = buffers + ((u % 2) * 2 * F::TILE + wave * F::LOADS * 64) * 16;
    send_rows<F::RW, F, false, false>(next, s, wave * F::RW, to);
    send_rows<F::RW, F, true, false>(next, s, wave * F::RW, to + F::TILE * 16);
    next = fetch(u + 1 < u_end ? u + 1 : u);               // a tile ahead: the table's latency
  }
  template <typename WORK> __device__ __forceinline__ void each(WORK work) {                // work(t0, K, V)
    for (int u = u_begin; u < u_end; ++u) {
      // This tile has landed; everybody is done with the buffer that is filled next.
      landed<0>();
      lds_read();
      __builtin_amdgcn_s_barrier();
      if (u + 1 < u_end) send(u + 1);
      const u32x4* Kt = s_tiles + (u % 2) * 2 * F::TILE;
      work(tiling.tile(u) * F::TT, Kt, Kt + F::TILE);
    }
  }
};

// ---------------------------------------------------------------------------------------------------------------- pieces
// A lane's row of q: row x of the source.
struct Query {
  int inst, p, lo;       // whose; its position, and the first row that its window shows
  bool real;             // or a row that is none: computed as another one, and not stored
  size_t row;            // of q
};
__device__ __forceinline__ Query query_of(const SharedArgs& a, const Source& s, int x) {
  Query q;
  int rest = x;
  q.real = x < s.rows;
  if (s.count > 0) {
    const int of = x / a.rows;
    rest = x - of * a.rows;
    q.inst = clamped(a.plan.member[s.first + (of < s.count ? of : 0)], 0, a.r.n_inst - 1);
    const int m = queries(a, q.inst), L = clamped(a.r.len[q.inst], 0, a.r.t_cap);
    q.real = q.real && rest < m << a.lg;
    if (!q.real) rest = 0;
    q.p = L - m + (rest >> a.lg);
  } else {
    if (!q.real) rest = 0;
    q.inst = s.inst;
    q.p = s.p0 + (rest >> a.lg);
  }
  q.lo = a.window > 0 && q.p >= a.window ? q.p - a.window + 1 : 0;
  q.row = (size_t)q.inst * a.rows + rest;
  return q;
}
__device__ __forceinline__ bool hidden(const SharedArgs& a, const Source& s, const Query& q, int j) {
  return (j < s.a0) | (j >= s.a1) | (j > q.p) | ((j < q.lo) & (j >= a.n_first));
}
// Whether every row of tile t0 is seen from all positions p_min .. p_max.
template <int TT> __device__ __forceinline__ bool all_seen(const SharedArgs& a, const Source& s, int t0, int p_min, int p_max) {
  return t0 >= s.a0 && t0 + TT <= s.a1 && t0 + TT - 1 <= p_min && (a.window <= 0 || t0 > p_max - a.window || t0 + TT <= a.n_first);
}
// The lowest and the highest position of the real ones of N lanes.
template <int N> __device__ __forceinline__ void positions(const Query& q, int* p_min, int* p_max) {
  int lo = q.real ? q.p : 0x7fffffff, hi = q.real ? q.p : -1;
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) {
    const int y = __shfl_xor(lo, o, 64), z = __shfl_xor(hi, o, 64);
    lo = y < lo ? y : lo;
    hi = z > hi ? z : hi;
  }
  *p_min = __builtin_amdgcn_readfirstlane(lo);
  *p_max = __builtin_amdgcn_readfirstlane(hi);
}
// A pair of probabilities as PARTS pairs of bf16 that add up to them: three have all of a probability's 24 bits.
template <int PARTS> __device__ __forceinline__ void in_parts(float x, float y, unsigned (&out)[PARTS]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int w = 0; w < PARTS; ++w) {
    bf16x2 z;
    z[0] = (__bf16)x;
    z[1] = (__bf16)y;
    out[w] = __builtin_bit_cast(unsigned, z);
    if (w + 1 < PARTS) {
      x -= __uint_as_float(out[w] << 16);
      y -= __uint_as_float(out[w] & 0xffff0000u);
    }
  }
}

// The product of product(), summed in four parts: fp32 sums of fewer terms round less.
template <int D> __device__ __forceinline__ float16v product_in_parts(const u32x4* X, const u32x4 (&b)[Form<float, D>::KS]) {
  using F = Form<float, D>;
  const int lane = threadIdx.x & 63, m = lane & 31, hb = lane >> 5;
  float16v c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) c[e][i] = 0.f;
#pragma unroll
  for (int k = 0; k < F::KS; ++k) {
    const u32x4 x = X[m * F::PIECES + F::k_place(m, 2 * k + hb)];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(b[k][e]), c[e], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) c[0][i] = (c[0][i] + c[1][i]) + (c[2][i] + c[3][i]);
  return c[0];
}

// Tile t of a source's rows of q, 32 a wave, over its tiles [u_begin, u_end) of the cache.  slot: of the tile's first row.
template <typename T, int D, bool EXACT>
__device__ __forceinline__ void wide_piece(const SharedArgs& a, const Source& s, int t, int u_begin, int u_end, size_t slot, const u32x4* s_tiles) {
  using F = Form<T, D>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hb = lane >> 5;
  Tiles<F> tiles(a, s, u_begin, u_end, s_tiles);
  const Query q = query_of(a, s, t * kPrefillRows + wave * 32 + n);
  int p_min, p_max;
  positions<32>(q, &p_min, &p_max);
  const bool idle = p_max < 0;                             // a wave without rows of q (or whose rows see nothing)
  u32x4 qf[F::KS];
#pragma unroll
  for (int k = 0; k < F::KS; ++k) qf[k] = static_cast<const u32x4*>(a.q)[q.row * F::PIECES + 2 * k + hb];
  float16v o[F::DB];
#pragma unroll
  for (int b = 0; b < F::DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  float m = -INFINITY, sum = 0.f;                          // the sum over this lane's half of the cache rows
  const float scale = kLog2E / sqrtf((float)D);
  // (From here on the compiler counts no load of its own as under way, and waits for none in the loop.)
#pragma unroll
  for (int k = 0; k < F::KS; ++k) asm volatile("" : "+v"(qf[k]));
  tiles.each([&](int t0, const u32x4* Kt, const u32x4* Vt) {
    if (idle) return;
    float16v c[F::TB];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int b = 0; b < F::TB; ++b) c[b] = product<T, D>(Kt, 32 * b, qf);
    } else {
      c[0] = product_in_parts<D>(Kt, qf);
    }
    // Scores that a query does not see become -inf.
    if (!all_seen<F::TT>(a, s, t0, p_min, p_max)) {
#pragma unroll
      for (int b = 0; b < F::TB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) c[b][i] = hidden(a, s, q, t0 + 32 * b + reg_row(i, hb)) ? -INFINITY : c[b][i];
    }
    float top = c[0][0];
#pragma unroll
    for (int b = 0; b < F::TB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, c[b][i]);
    top = max32(top);
    // The reference is a whole number in units of log2 (a change of it rounds nothing).  Exponents refer to 0 as long as nothing is seen, and where
    // it is far, as the scores are brought near then.
    const float ref = fmaxf(m, ceilf(top * scale));
    const bool far = is_far(ref);
    if (__any((ref != m) | far)) {
      const float shrink = ref == m ? 1.f : exp2_fast(m - ref);
      sum *= shrink;
#pragma unroll
      for (int b = 0; b < F::DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= shrink;
      m = ref;
      if (__any(far && m != -INFINITY)) {
#pragma unroll
        for (int b = 0; b < F::TB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) c[b][i] = far && m != -INFINITY ? brought_near(c[b][i], scale, m) : c[b][i];
      }
    }
    const float use = far ? 0.f : ref;
    float part[4] = {0.f, 0.f, 0.f, 0.f};                  // (sums of a tile first: long caches lose fewer digits so)
#pragma unroll
    for (int b = 0; b < F::TB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        c[b][i] = exp2_fast(__builtin_fmaf(c[b][i], scale, -use));
        part[i & 3] += c[b][i];
      }
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    if constexpr (sizeof(T) == 2) {
      // Where the output is rounded to bf16, probabilities keep 16 bits, else (EXACT) 24: two bf16 parts, or three.  Outputs of scores spread by 2 are off by
      // 0.0017 relative to the definition (root mean square), which is the rounding of the output; with one part 0.0023, drafts 47.7 -> 46.5 us.
      constexpr int PARTS = EXACT ? 3 : 2;
#pragma unroll
      for (int k = 0; k < F::TT / 16; ++k) {
        typedef unsigned u32x4p __attribute__((ext_vector_type(4)));
        u32x4p pb[PARTS];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          unsigned two[PARTS];
          in_parts<PARTS>(c[k / 2][8 * (k % 2) + 2 * e], c[k / 2][8 * (k % 2) + 2 * e + 1], two);
#pragma unroll
          for (int w = 0; w < PARTS; ++w) pb[w][e] = two[w];
        }
        // V^T of 16 cache rows: the transposing read gives lane (m, hb) column m of four rows; a lane of 16 points to the 8 bytes at
        // row lane / 4, columns 4 (lane % 4).
        const int i = lane & 15, r = 16 * k + 4 * hb + (i >> 2);
#pragma unroll
        for (int b = 0; b < F::DB; ++b) {
          const int col = 32 * b + 16 * ((lane >> 4) & 1) + 4 * (i & 3), piece = col / 8;
          bf16x8 va;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int rr = r + 8 * half;
            const char* at = reinterpret_cast<const char*>(Vt + rr * F::PIECES + F::v_place(rr, piece)) + (col % 8) * 2;
            const short4v w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at);
            const bf16x4 y = __builtin_bit_cast(bf16x4, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) va[4 * half + e] = y[e];
          }
#pragma unroll
          for (int w = PARTS - 1; w >= 0; --w) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, __builtin_bit_cast(bf16x8, pb[w]), o[b], 0, 0, 0);
        }
      }
    } else {
      const float* Vf = reinterpret_cast<const float*>(Vt);
#pragma unroll
      for (int b = 0; b < F::DB; ++b) {
        float16v y;                                        // of this tile alone, as the sums
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          y = __builtin_amdgcn_mfma_f32_32x32x2f32(Vf[reg_row(i, hb) * D + 32 * b + n], c[0][i], y, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] += y[i];
      }
    }
  });
  sum = sum32(sum);
  if (!q.real) return;
  slot += wave * 32 + n;
  if (hb == 0) {
    a.ml[slot * 2] = m;
    a.ml[slot * 2 + 1] = sum;
  }
#pragma unroll
  for (int b = 0; b < F::DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float4v y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = o[b][i + e];
      *reinterpret_cast<float4v*>(a.o + slot * D + 32 * b + reg_row(i, hb)) = y;
    }
}

// Waits until no more than FIRST loads and N for each of r later groups are under way, r < R or as if it were R - 1.
template <int N, int R, int FIRST = 0> __device__ __forceinline__ void landed_behind(int r) {
  if constexpr (R == 1) {
    landed<FIRST>();
  } else {
    if (r >= R - 1) landed<FIRST + N * (R - 1)>();
    else landed_behind<N, R - 1, FIRST>(r);
  }
}

// The last rows of q of a source, up to 16 RB, over its groups [u_begin, u_end) of 16 or 32 cache rows, by a wave: RING groups of K and V are on their way
// to LDS, past the registers.  A lane has, of each 16 rows of q, scores of row n and of four of each 16 cache rows, which are the second product's operand as
// they are, and sums of four of each 16 dims.  slot: of the first of the rows.  lds: RING groups.  Groups of 32 against two of 16 under way: drafts of 16
// sequences 45.8 -> 44.5 us, 42 sequences behind 6 prompts 61 -> 59, the 64 above 57.5 -> 56.
template <typename T, int D, bool EXACT, int RING, int RB>
__device__ __forceinline__ void narrow_piece(const SharedArgs& a, const Source& s, int u_begin, int u_end, size_t slot, const u32x4* lds) {
  using F = Form<T, D>;
  constexpr int G = kGroup<T, D>, XS = G / 16, KS = F::PIECES / 4, DB = D / 16, GROUP = G * F::PIECES, N = GROUP / 64;     // pieces of a group's K, or V, and loads
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4, count = u_end - u_begin;
  const Tiling tiling = tiling_of<G>(s);
  const TablePages pages = pages_of(a.r, s.inst);
  const unsigned ring = lds_address(lds);
  auto fetch = [&](int it) { return fetch_of<G, F::PIECES>(a, pages, s, tiling.tile(u_begin + (it < count ? it : count - 1)) * G); };
  auto at = [&](int it) { return (it % RING) * 2 * GROUP; };
  Fetch<G> next = fetch(0);
#pragma unroll
  for (int it = 0; it < RING; ++it)
    if (it < count) {
      send_rows<G, F, false, true>(next, s, 0, ring + at(it) * 16);
      send_rows<G, F, true, true>(next, s, 0, ring + (at(it) + GROUP) * 16);
      next = fetch(it + 1);
    }
  Query q[RB];
  int p_min = 0x7fffffff, p_max = -1;
  u32x4 qf[RB][KS];
  float4v o[RB][DB];
  float m[RB], sum[RB];                                    // the sums over this lane's rows
#pragma unroll
  for (int y = 0; y < RB; ++y) {
    q[y] = query_of(a, s, (int)(s.rows - s.last()) + 16 * y + n);
    int lo, hi;
    positions<16>(q[y], &lo, &hi);
    p_min = lo < p_min ? lo : p_min;
    p_max = hi > p_max ? hi : p_max;
#pragma unroll
    for (int l = 0; l < KS; ++l) qf[y][l] = static_cast<const u32x4*>(a.q)[q[y].row * F::PIECES + 4 * l + kg];
#pragma unroll
    for (int b = 0; b < DB; ++b) o[y][b] = float4v{0.f, 0.f, 0.f, 0.f};
    m[y] = -INFINITY;
    sum[y] = 0.f;
  }
  const float scale = kLog2E / sqrtf((float)D);
#pragma unroll
  for (int y = 0; y < RB; ++y)
#pragma unroll
    for (int l = 0; l < KS; ++l) asm volatile("" : "+v"(qf[y][l]));
  for (int it = 0; it < count; ++it) {
    const int t0 = tiling.tile(u_begin + it) * G, behind = count - 1 - it;           // groups that were sent for after this one, RING - 1 at most
    const u32x4 *Kt = lds + at(it), *Vt = Kt + GROUP;
    const bool more = it + RING < count;
    landed_behind<2 * N, RING, N>(behind);
    // Rows t0 + 16 x + 4 kg + r, of query n.  fp32 products go into four sums, whose roundings are smaller than those of one over all of d.
    constexpr int SUMS = sizeof(T) == 2 ? 1 : 4;
    float4v c[RB][XS];
#pragma unroll
    for (int x = 0; x < XS; ++x) {
      float4v sums[RB][SUMS];
#pragma unroll
      for (int y = 0; y < RB; ++y)
#pragma unroll
        for (int e = 0; e < SUMS; ++e) sums[y][e] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int l = 0; l < KS; ++l) {
        const u32x4 k = Kt[(16 * x + n) * F::PIECES + F::k_place(16 * x + n, 4 * l + kg)];
#pragma unroll
        for (int y = 0; y < RB; ++y) {
          if constexpr (sizeof(T) == 2) {
            sums[y][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[y][l]), sums[y][0], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sums[y][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(qf[y][l][e]), sums[y][e], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int y = 0; y < RB; ++y) {
        c[y][x] = sums[y][0];
        if constexpr (SUMS == 4) {
#pragma unroll
          for (int r = 0; r < 4; ++r) c[y][x][r] = (sums[y][0][r] + sums[y][1][r]) + (sums[y][2][r] + sums[y][3][r]);
        }
      }
    }
    if (more) {
      lds_read();
      send_rows<G, F, false, true>(next, s, 0, ring + at(it) * 16);
    }
    if (!all_seen<G>(a, s, t0, p_min, p_max)) {
#pragma unroll
      for (int y = 0; y < RB; ++y)
#pragma unroll
        for (int x = 0; x < XS; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) c[y][x][r] = hidden(a, s, q[y], t0 + 16 * x + 4 * kg + r) ? -INFINITY : c[y][x][r];
    }
#pragma unroll
    for (int y = 0; y < RB; ++y) {
      float top = c[y][0][0];
#pragma unroll
      for (int x = 0; x < XS; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, c[y][x][r]);
      top = max32(max16(top));
      const float ref = fmaxf(m[y], ceilf(top * scale));   // a whole number in units of log2, as above
      if (__any(ref != m[y])) {
        const float shrink = ref == m[y] ? 1.f : exp2_fast(m[y] - ref);
        sum[y] *= shrink;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[y][b][r] *= shrink;
        m[y] = ref;
      }
      const float use = m[y] == -INFINITY ? 0.f : m[y];
      float part[XS];
#pragma unroll
      for (int x = 0; x < XS; ++x) {
#pragma unroll
        for (int r = 0; r < 4; ++r) c[y][x][r] = exp2_of(c[y][x][r], scale, use);
        part[x] = (c[y][x][0] + c[y][x][1]) + (c[y][x][2] + c[y][x][3]);
      }
      if constexpr (XS == 2) part[0] += part[1];
      sum[y] += part[0];
    }
    // This group's V: behind it came the later groups, and the K that was just sent for.
    if (more) landed<2 * N * (RING - 1) + N>();
    else landed_behind<2 * N, RING>(behind);
    if constexpr (sizeof(T) == 2) {
      constexpr int PARTS = EXACT ? 3 : 2;
      typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int x = 0; x < XS; ++x) {
        short4v v[DB];
        const int r = 16 * x + 4 * kg + (n >> 2);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const int col = 16 * b + 4 * (n & 3);
          const char* from = reinterpret_cast<const char*>(Vt + r * F::PIECES + F::v_place(r, col / 8)) + (col % 8) * 2;
          v[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)from);
        }
#pragma unroll
        for (int y = 0; y < RB; ++y) {
          unsigned two[2][PARTS];
          in_parts<PARTS>(c[y][x][0], c[y][x][1], two[0]);
          in_parts<PARTS>(c[y][x][2], c[y][x][3], two[1]);
#pragma unroll
          for (int w = PARTS - 1; w >= 0; --w)
#pragma unroll
            for (int b = 0; b < DB; ++b)
              o[y][b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[b], __builtin_bit_cast(short4v, u32x2{two[0][w], two[1][w]}), o[y][b], 0, 0, 0);
        }
      }
    } else {
      const float* Vf = reinterpret_cast<const float*>(Vt);
#pragma unroll
      for (int x = 0; x < XS; ++x)
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = Vf[(16 * x + 4 * kg + r) * D + 16 * b + n];
#pragma unroll
            for (int y = 0; y < RB; ++y) o[y][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, c[y][x][r], o[y][b], 0, 0, 0);
          }
    }
    if (more) {
      lds_read();
      send_rows<G, F, true, true>(next, s, 0, ring + (at(it) + GROUP) * 16);
      next = fetch(it + RING + 1);
    }
  }
#pragma unroll
  for (int y = 0; y < RB; ++y) {
    sum[y] = sum32(sum16(sum[y]));
    if (!q[y].real) continue;
    const size_t to = slot + 16 * y + n;
    if (kg == 0) {
      a.ml[to * 2] = m[y];
      a.ml[to * 2 + 1] = sum[y];
    }
#pragma unroll
    for (int b = 0; b < DB; ++b) *reinterpret_cast<float4v*>(a.o + to * D + 16 * b + 4 * kg) = o[y][b];
  }
}

// A share of `all`, of which everybody has `per`.
struct Share {
  unsigned long long begin;
  unsigned left;
};
__device__ __forceinline__ Share share_of(unsigned long long all, unsigned per, int which) {
  Share s;
  s.begin = (unsigned long long)which * per;
  s.left = s.begin >= all ? 0 : (s.begin + per < all ? per : (unsigned)(all - s.begin));
  return s;
}
// What a sharer does of a tile of rows of q that counts `size`, from `r` on: `n` of it, which are its tiles [u_begin, u_end) of the cache.  A small one
// belongs to the share that it begins in.
struct Cut { unsigned n; bool skipped; int u_begin, u_end, parts; };
template <unsigned FRONT, unsigned EACH> __device__ __forceinline__ Cut cut_of(unsigned size, unsigned r, unsigned per, unsigned left, unsigned least) {
  Cut c;
  const unsigned small = per / 4 > least ? per / 4 : least;
  const bool whole = size <= small;
  c.n = __builtin_amdgcn_readfirstlane(whole || size - r < left ? size - r : left);
  c.skipped = whole && r > 0;
  c.u_begin = r <= FRONT ? 0 : (int)((r - FRONT + EACH - 1) / EACH);
  c.u_end = r + c.n <= FRONT ? 0 : (int)((r + c.n - FRONT + EACH - 1) / EACH);
  c.parts = c.n == size ? 1 : 1 + (int)((size - c.n + per - 1) / per);       // (asked for where r = 0)
  return c;
}

template <int N> struct Number { static constexpr int value = N; };

// Sources that a thread holds the sizes of.  Where there are more of them, launches of their own leave the sizes in the workspace, not every workgroup for
// itself: decode of 4096 caches, two behind each beginning of 17 rows, with a window 127 -> 59 us, of 3280 behind 656 of 65 rows 66 -> 29.
constexpr int kHeld = 6;
__host__ __device__ constexpr int places_of(int n_inst) { return n_inst + n_inst / 2; }           // (of groups there are half as many as instances at most)
__host__ __device__ constexpr int blocks_of(int n_inst) { return (places_of(n_inst) + kThreads - 1) / kThreads; }

// The groups' lowest positions, a wave each.
__global__ __launch_bounds__(kThreads) void share_low_kernel(SharedArgs a) {
  constexpr int U = 4;                                     // loads under way
  const int n = a.r.n_inst, lane = threadIdx.x & 63, groups = clamped(*a.plan.count, 0, n / 2);
  for (int g = blockIdx.x * kWaves + (threadIdx.x >> 6); g < groups; g += gridDim.x * kWaves) {
    const int4 line = a.plan.groups[g];
    const int count = line.y >= 0 && line.z <= n - line.y ? line.z : 0;
    int p = 0x7fffffff;
    for (int k0 = 0; k0 < count; k0 += 64 * U) {
      int i[U];
#pragma unroll
      for (int u = 0; u < U; ++u) i[u] = clamped(a.plan.member[line.y + (k0 + 64 * u + lane < count ? k0 + 64 * u + lane : 0)], 0, n - 1);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int y = first_position(a, i[u]);
        p = y < p ? y : p;
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const int y = __shfl_xor(p, o, 64);
      p = y < p ? y : p;
    }
    if (lane == 0) a.low[clamped(line.x, 0, n - 1)] = p;
  }
}
// The sources' sizes, as sums over those in front in a block of kThreads, and the blocks' sums.
template <typename T, int D, bool EXACT> __global__ __launch_bounds__(kThreads) void share_sizes_kernel(SharedArgs a) {
  using C = Counts<T, EXACT>;
  __shared__ unsigned long long s_wide[kWaves], s_narrow[kWaves];
  const int n = a.r.n_inst, places = places_of(n), sources = n + clamped(*a.plan.count, 0, n / 2);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = blockIdx.x * kThreads + threadIdx.x;
  const Source y = source_of(a, x < places ? x : 0, nullptr);
  const unsigned long long wide = x < sources ? (unsigned long long)wide_size<C, Form<T, D>::TT>(y) * y.wide() : 0;
  const unsigned long long narrow = x < sources ? narrow_size<C, kGroup<T, D>>(y) : 0;
  if (x < sources) (x < n ? a.behind + x : a.begun + clamped(y.inst, 0, n - 1))[0] = wide + narrow > 0;
  unsigned long long at_wide = wide, at_narrow = narrow;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long u = __shfl_up(at_wide, o, 64), v = __shfl_up(at_narrow, o, 64);
    if (lane >= o) {
      at_wide += u;
      at_narrow += v;
    }
  }
  if (lane == 63) {
    s_wide[wave] = at_wide;
    s_narrow[wave] = at_narrow;
  }
  __syncthreads();
  at_wide -= wide;
  at_narrow -= narrow;
  unsigned long long all_wide = 0, all_narrow = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) {
      at_wide += s_wide[w];
      at_narrow += s_narrow[w];
    }
    all_wide += s_wide[w];
    all_narrow += s_narrow[w];
  }
  a.sizes[2 * x] = at_wide;
  a.sizes[2 * x + 1] = at_narrow;
  if (threadIdx.x == 0) {
    a.totals[2 * blockIdx.x] = all_wide;
    a.totals[2 * blockIdx.x + 1] = all_narrow;
  }
}

template <typename T, int D, bool EXACT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void cache_shared_kernel(SharedArgs a) {
  using F = Form<T, D>;
  using C = Counts<T, EXACT>;
  constexpr int kListed = 16, GROUP = 2 * kGroup<T, D> * F::PIECES, RING = kSharedLds / 16 / (kWaves * GROUP);
  static_assert(RING >= 1 && 4 * F::TILE * 16 <= kSharedLds, "LDS");
  extern __shared__ __attribute__((aligned(16))) u32x4 s_tiles[];         // [2][K, V][TILE], or [wave][RING][K, V][group]
  __shared__ unsigned long long s_wide[kWaves], s_narrow[kWaves], s_from[1 + kWaves];
  __shared__ int s_first[1 + kWaves];                                     // of the workgroup's share, and of its waves'
  __shared__ Source s_source[1 + kWaves][kListed];                        // from there on
  __shared__ int s_low[kThreads * kHeld * 2 / 3];                         // (as many instances as there are where this is used)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  const int places = places_of(a.r.n_inst), groups = clamped(*a.plan.count, 0, a.r.n_inst / 2), sources = a.r.n_inst + groups;
  const LowestInLds lowest = (LowestInLds)s_low;
  if (a.window > 0 && !a.sized) {
    for (int i = tid; i < a.r.n_inst; i += kThreads) s_low[i] = 0x7fffffff;
    __syncthreads();
    for (int i0 = tid; i0 < a.r.n_inst; i0 += 2 * kThreads) {
      const int i1 = i0 + kThreads < a.r.n_inst ? i0 + kThreads : i0;
      const int4 y0 = a.plan.inst[i0], y1 = a.plan.inst[i1];
      const int p0 = first_position(a, i0), p1 = first_position(a, i1);
      if (y0.z > 1) atomicMin(s_low + clamped(y0.x, 0, a.r.n_inst - 1), p0);
      if (y1.z > 1) atomicMin(s_low + clamped(y1.x, 0, a.r.n_inst - 1), p1);
    }
    __syncthreads();
  }

  // All that there is to do: every thread sums up consecutive sources, or blocks of them.  (How many groups there are is asked for at the same time.)
  const int chunk = ((a.sized ? blocks_of(a.r.n_inst) : places) + kThreads - 1) / kThreads, i_begin = tid * chunk;
  unsigned long long wide[kHeld], narrow[kHeld], my_wide = 0, my_narrow = 0, all_wide = 0, all_narrow = 0, at = 0;
  unsigned per = 0;
  int wide_wgs = 0, narrow_wgs = kShareWgs;
  bool is_wide = false;
  // The waves' shares go round the workgroups, so that few of them are spread.
  auto number = [&](int w) { return w * narrow_wgs + (int)blockIdx.x - wide_wgs; };
  auto share = [&](int y) { return y == 0 ? share_of(all_wide, per, blockIdx.x) : share_of(all_narrow, per, number(y - 1)); };
  // The sizes of sources i_begin .. i_begin + M - 1, whose loads are under way together.
  auto look = [&](auto some) {
    constexpr int M = decltype(some)::value;
    Source s[M];
#pragma unroll
    for (int k = 0; k < M; ++k) s[k] = source_of(a, k < chunk && i_begin + k < places ? i_begin + k : 0, lowest);
#pragma unroll
    for (int k = 0; k < M; ++k) {
      const int x = i_begin + k;
      if (k >= chunk || x >= sources) continue;
      wide[k] = (unsigned long long)wide_size<C, F::TT>(s[k]) * s[k].wide();
      narrow[k] = narrow_size<C, kGroup<T, D>>(s[k]);
      // Which sources have pieces, for the join: the instances, and the groups by their first member.
      if ((unsigned)x % kShareWgs == blockIdx.x) {
        int32_t* has = x < a.r.n_inst ? a.behind + x : a.begun + clamped(s[k].inst, 0, a.r.n_inst - 1);
        *has = wide[k] + narrow[k] > 0;
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) wide[k] = narrow[k] = 0;
  if (a.sized) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (k < chunk && i_begin + k < blocks_of(a.r.n_inst)) {
        wide[k] = a.totals[2 * (i_begin + k)];
        narrow[k] = a.totals[2 * (i_begin + k) + 1];
      }
  } else if (chunk == 1) {
    look(Number<1>());
  } else if (chunk <= 3) {
    look(Number<3>());
  } else {
    look(Number<kHeld>());
  }
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    my_wide += wide[k];
    my_narrow += narrow[k];
  }
  {
    unsigned long long upto_wide = my_wide, upto_narrow = my_narrow;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned long long x = __shfl_up(upto_wide, o, 64), y = __shfl_up(upto_narrow, o, 64);
      if (lane >= o) {
        upto_wide += x;
        upto_narrow += y;
      }
    }
    if (lane == 63) {
      s_wide[wave] = upto_wide;
      s_narrow[wave] = upto_narrow;
    }
    if (tid <= kWaves) s_first[tid] = 0x7fffffff - kListed;          // (none)
    __syncthreads();
    unsigned long long at_wide = upto_wide - my_wide, at_narrow = upto_narrow - my_narrow;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) {
        at_wide += s_wide[w];
        at_narrow += s_narrow[w];
      }
      all_wide += s_wide[w];
      all_narrow += s_narrow[w];
    }
    // Workgroups for the one and for the other, by the time that both take.
    const float part = (float)all_wide / ((float)all_wide + (float)all_narrow / kWaves);    // (not a number where there is nothing to do)
    wide_wgs = all_wide == 0 ? 0 : (int)(part * (float)kShareWgs + 0.5f);
    if (all_wide > 0 && wide_wgs < 1) wide_wgs = 1;
    if (all_narrow > 0 && wide_wgs > kShareWgs - 1) wide_wgs = kShareWgs - 1;
    wide_wgs = __builtin_amdgcn_readfirstlane(wide_wgs);
    narrow_wgs = wide_wgs < kShareWgs ? kShareWgs - wide_wgs : 1;
    is_wide = (int)blockIdx.x < wide_wgs;
    at = is_wide ? at_wide : at_narrow;
    const unsigned sharers = is_wide ? wide_wgs : kWaves * narrow_wgs, least = is_wide ? C::WIDE_LEAST : C::NARROW_LEAST;
    const unsigned long long each = ((is_wide ? all_wide : all_narrow) + sharers - 1) / sharers;
    per = __builtin_amdgcn_readfirstlane(each < least ? least : (unsigned)each);
  }
  // Where shares begin, by the threads in whose sources they lie.
  {
    unsigned long long here = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) here += is_wide ? wide[k] : narrow[k];
#pragma unroll 1
    for (int y = is_wide ? 0 : 1; y <= (is_wide ? 0 : kWaves); ++y) {
      const Share s = share(y);
      if (s.left == 0 || s.begin < at || s.begin >= at + here) continue;
      unsigned long long to = at;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const unsigned long long n = is_wide ? wide[k] : narrow[k];
        if (to <= s.begin && s.begin < to + n) {
          s_first[y] = i_begin + k;
          s_from[y] = s.begin - to;
        }
        to += n;
      }
    }
  }
  __syncthreads();
  if (a.sized) {                                           // that was a block: now its sources
    int block[1 + kWaves];
    unsigned long long from[1 + kWaves], before[1 + kWaves], behind[1 + kWaves];
#pragma unroll
    for (int y = 0; y <= kWaves; ++y) {
      block[y] = s_first[y];
      from[y] = s_from[y];
      const bool some = block[y] < blocks_of(a.r.n_inst);
      const int x = (some ? block[y] : 0) * kThreads + tid, next = tid == kThreads - 1 ? x : x + 1;
      before[y] = a.sizes[2 * x + (y > 0)];
      behind[y] = tid == kThreads - 1 ? a.totals[2 * (some ? block[y] : 0) + (y > 0)] : a.sizes[2 * next + (y > 0)];
    }
    __syncthreads();
#pragma unroll
    for (int y = 0; y <= kWaves; ++y) {
      if (block[y] >= blocks_of(a.r.n_inst)) {
        if (tid == 0) s_first[y] = sources;
      } else if (before[y] <= from[y] && from[y] < behind[y]) {
        s_first[y] = block[y] * kThreads + tid;
        s_from[y] = from[y] - before[y];
      }
    }
    __syncthreads();
  }
  if (tid < (1 + kWaves) * kListed) {
    const int x = s_first[tid / kListed] + tid % kListed;
    s_source[tid / kListed][tid % kListed] = source_of(a, x < sources ? x : 0, lowest);
  }
  __syncthreads();

  if (is_wide) {                                           // the workgroup's share
    const int x_first = __builtin_amdgcn_readfirstlane(s_first[0]);
    const Share share0 = share(0);
    unsigned left = share0.left;
    unsigned long long from = x_first < sources ? s_from[0] : 0;
    for (int x = x_first; left > 0 && x < sources; ++x, from = 0) {
      const Source s = uniform(x - x_first < kListed ? s_source[0][x - x_first] : source_of(a, x, lowest));
      const unsigned size = wide_size<C, F::TT>(s);
      const unsigned long long end = (unsigned long long)size * s.wide();
      while (left > 0 && from < end) {
        const int t = __builtin_amdgcn_readfirstlane(end == size ? 0 : (int)(from / size));            // tile t of its rows of q
        const Cut c = cut_of<C::WIDE_FRONT, C::WIDE>(size, (unsigned)(from - (unsigned long long)t * size), per, left, C::WIDE_LEAST);
        const bool first = from == (unsigned long long)t * size;
        from += c.n;
        left -= c.n < left ? c.n : left;
        if (c.skipped) continue;
        const size_t x0 = (size_t)s.x0 + (size_t)t * kPrefillRows, slot = x0 + (size_t)kPrefillRows * blockIdx.x;
        const int rows = s.rows - t * kPrefillRows;
        __syncthreads();                                   // everybody is done with the piece before
        if (c.u_begin < c.u_end) {
          wide_piece<T, D, EXACT>(a, s, t, c.u_begin, c.u_end, slot, s_tiles);
        } else if (tid < rows && tid < kPrefillRows) {     // (what is in front alone)
          a.ml[(slot + tid) * 2] = -INFINITY;
          a.ml[(slot + tid) * 2 + 1] = 0.f;
        }
        if (first && tid < rows && tid < kPrefillRows) a.row[x0 + tid] = make_int2((int)slot + tid, c.parts);
      }
    }
    return;
  }

  // This wave's share.
  const int x_first = __builtin_amdgcn_readfirstlane(s_first[1 + wave]);
  const Share mine = share(1 + wave);
  unsigned left = __builtin_amdgcn_readfirstlane(mine.left), r = x_first < sources ? __builtin_amdgcn_readfirstlane((unsigned)s_from[1 + wave]) : 0;
  for (int x = x_first; left > 0 && x < sources; ++x, r = 0) {
    const Source s = uniform(x - x_first < kListed ? s_source[1 + wave][x - x_first] : source_of(a, x, lowest));
    const unsigned size = narrow_size<C, kGroup<T, D>>(s);
    if (size <= r) continue;
    const Cut c = cut_of<C::NARROW_FRONT, C::NARROW>(size, r, per, left, C::NARROW_LEAST);
    left -= c.n < left ? c.n : left;
    if (c.skipped) continue;
    const int rows = s.last(), row0 = s.rows - rows;
    const size_t x0 = (size_t)s.x0 + row0, slot = (size_t)a.narrow0 + x0 + (size_t)kNarrowRows * number(wave);
    if (c.u_begin < c.u_end) {
      if (rows <= 16) narrow_piece<T, D, EXACT, RING, 1>(a, s, c.u_begin, c.u_end, slot, s_tiles + wave * RING * GROUP);
      else narrow_piece<T, D, EXACT, RING, 2>(a, s, c.u_begin, c.u_end, slot, s_tiles + wave * RING * GROUP);
    } else if (lane < rows) {
      a.ml[(slot + lane) * 2] = -INFINITY;
      a.ml[(slot + lane) * 2 + 1] = 0.f;
    }
    if (r == 0 && lane < rows) a.row[x0 + lane] = make_int2((int)slot + lane, -c.parts);
  }
}

// A row of q over what it sees alone, as plain sums: D / 4 lanes have a row of the cache at a time, four dims each.  l: this lane's part of the sum of
// probabilities, o: of the output.  Ends where nothing but NaN can come of it, as of a q, a K or a V that is seen and holds no numbers: 64 sequences
// behind 8190 rows, one of them with such a q, take 30 us, as without it, with row 77 of K or V 84; gone over to the end 3000 and 4300.
template <typename T, int D> __device__ __forceinline__ void one_row(const SharedArgs& a, int inst, int row, float& l, float4v& o) {
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
  const int lane = threadIdx.x & 63, which = lane / LANES, col = lane % LANES * 4;
  const int p = clamped(a.r.len[inst], 0, a.r.t_cap) - queries(a, inst) + (row >> a.lg);
  const int lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0, f = a.n_first < lo ? a.n_first : lo;
  const TablePages pages = pages_of(a.r, inst);
  auto four = [&](const void* from, size_t r) {
    float4v x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) x[e] = (float)static_cast<const __bf16*>(from)[r * D + col + e];
      else x[e] = static_cast<const float*>(from)[r * D + col + e];
    }
    return x;
  };
  const float4v q = four(a.q, (size_t)inst * a.rows + row);
  const float scale = kLog2E / sqrtf((float)D);
  float m = -INFINITY;
  l = 0.f;
  o = float4v{0.f, 0.f, 0.f, 0.f};
  // Half of them go from the first row on, the others from the last one back: that is where rows without numbers lie, if anywhere.
  const int all = f + (p - lo + 1), from_first = (all + 1) / 2, mine = which % 2 == 0 ? from_first : all - from_first;
  for (int y = which / 2; y < mine; y += AT_ONCE / 2) {
    const int x = which % 2 == 0 ? y : all - 1 - y, j = x < f ? x : lo + (x - f);
    const size_t r = pages.at(j & ~7) + (j & 7);
    const float4v k = four(a.K, r), v = four(a.V, r);
    float s = (q[0] * k[0] + q[1] * k[1]) + (q[2] * k[2] + q[3] * k[3]);
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if (s == -INFINITY) continue;
    const float top = fmaxf(m, s), shrink = m == -INFINITY ? 0.f : exp2_fast((m - top) * scale), w = exp2_fast((s - top) * scale);
    l = l * shrink + w;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * shrink + w * v[e];
    m = top;
    const unsigned long long none = __ballot((l != l) | ((o[0] != o[0]) & (o[1] != o[1]) & (o[2] != o[2]) & (o[3] != o[3]))), row = (1ull << LANES) - 1;
    if (__any((none >> (which * LANES) & row) == row)) break;
  }
  const float top = wave_max(m), shrink = m == -INFINITY ? 0.f : exp2_fast((m - top) * scale);
  l = col == 0 ? l * shrink : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= shrink;
}

// Joins the pieces: a wave per row of q; D / 4 lanes have a piece at a time.  OUT: float, or the type of q.
template <typename T, int D, typename OUT> __global__ __launch_bounds__(kThreads) void cache_shared_join_kernel(SharedArgs a) {
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
  const long long at = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int inst = (int)(at / a.rows), row = (int)(at % a.rows), lane = threadIdx.x & 63;
  if (inst >= a.r.n_inst || row >= queries(a, inst) << a.lg) return;
  // (What may be there is asked for together with whether it is: every dependent load is a trip to memory.)
  const int4 line = a.plan.inst[inst];
  const int pos = clamped(a.plan.pos[inst], 0, a.r.n_inst - 1), behind = a.behind[inst];
  const int2 own_row = a.row[(size_t)inst * a.rows + row];
  const int begun = a.begun[clamped(line.x, 0, a.r.n_inst - 1)];
  const int2 first_row = a.row[((size_t)a.r.n_inst + pos) * a.rows + row];
  const int2 first = line.z > 1 && begun > 0 ? first_row : make_int2(0, 0), own = behind > 0 ? own_row : make_int2(0, 0);
  const int ahead = first.y < 0 ? -first.y : first.y, parts = ahead + (own.y < 0 ? -own.y : own.y);
  const int step = first.y < 0 ? kNarrowRows : kPrefillRows, own_step = own.y < 0 ? kNarrowRows : kPrefillRows;
  auto slot = [&](int p) { return p < ahead ? (size_t)first.x + (size_t)step * p : (size_t)own.x + (size_t)own_step * (p - ahead); };
  constexpr int kAhead = 8;                                // loads under way, of AT_ONCE pieces
  const int which = lane / LANES, col = lane % LANES * 4;
  float4v v[kAhead];
  auto load = [&](int p0) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int p = p0 + x * AT_ONCE + which;
      if (p < parts) v[x] = *reinterpret_cast<const float4v*>(a.o + slot(p) * D + col);
    }
  };
  load(0);
  float m = lane < parts ? a.ml[slot(lane) * 2] : -INFINITY, l = lane < parts ? a.ml[slot(lane) * 2 + 1] : 0.f, top = m;
  for (int p = lane + 64; p < parts; p += 64) top = fmaxf(top, a.ml[slot(p) * 2]);
  top = wave_max(top);
  const float use = top == -INFINITY ? 0.f : top;
  float4v o = {0.f, 0.f, 0.f, 0.f};
  float all = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 64) {
    if (p0 > 0) {
      m = p0 + lane < parts ? a.ml[slot(p0 + lane) * 2] : -INFINITY;
      l = p0 + lane < parts ? a.ml[slot(p0 + lane) * 2 + 1] : 0.f;
    }
    const float f = exp2_fast(m - use);                    // (0 behind the last piece)
    all += f * l;
    const int n = parts - p0 < 64 ? parts - p0 : 64;
    for (int x0 = 0; x0 < n; x0 += kAhead * AT_ONCE) {
      if (p0 + x0 > 0) load(p0 + x0);
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const float w = __shfl(f, x0 + x * AT_ONCE + which, 64);
        if (x0 + x * AT_ONCE + which < n && w != 0.f) {    // (a piece without tiles has left no sums)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += w * v[x][e];
        }
      }
    }
  }
  auto add_up = [&]() {
    all = wave_sum(all);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (LANES <= 16) o[e] = sum16(o[e]);
      o[e] = sum32(o[e]);
    }
  };
  add_up();
  // A row of the cache that no finite number is in makes NaN of every row of q that its tile is read for, also of those that do not see it: 0 x NaN.
  // Where a row is NaN it is computed again by itself.
  if (__any((all != all) | (o[0] != o[0]) | (o[1] != o[1]) | (o[2] != o[2]) | (o[3] != o[3]))) {
    one_row<T, D>(a, inst, row, all, o);
    add_up();
  }
  if (which > 0) return;
  OUT* out = static_cast<OUT*>(a.out) + ((size_t)inst * a.rows + row) * D + col;
  float4v y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = all == 0.f ? 0.f : o[e] / all;          // a query that sees nothing has a zero output
  if constexpr (sizeof(OUT) == 2) {
    bf16x4 z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = (__bf16)y[e];
    *reinterpret_cast<bf16x4*>(out) = z;
  } else {
    *reinterpret_cast<float4v*>(out) = y;
  }
}

template <typename T, int D, bool EXACT, typename OUT> hipError_t run(const SharedArgs& given, hipStream_t st) {
  hipError_t e;
  SharedArgs a = given;
  a.sized = places_of(a.r.n_inst) > kThreads * kHeld;
  if (a.sized && a.window > 0) {
    share_low_kernel<<<kShareWgs, kThreads, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.sized) {
    share_sizes_kernel<T, D, EXACT><<<blocks_of(a.r.n_inst), kThreads, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  cache_shared_kernel<T, D, EXACT><<<kShareWgs, kThreads, kSharedLds, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const unsigned wgs = (unsigned)(((long long)a.r.n_inst * a.rows + kWaves - 1) / kWaves);
  cache_shared_join_kernel<T, D, OUT><<<wgs, kThreads, 0, st>>>(a);
  return hipGetLastError();
}
template <typename T, int D> hipError_t run(const SharedArgs& a, bool decode, hipStream_t st) {
  if constexpr (sizeof(T) == 2) return decode ? run<T, D, true, float>(a, st) : run<T, D, false, T>(a, st);
  else return run<T, D, true, float>(a, st);
}

}  // namespace

hipError_t launch_cache_share(const Shape& s, const int32_t* group, const int32_t* shared, const SharePlan& plan, hipStream_t st) {
  const unsigned wgs = ((unsigned)s.n_inst + kThreads - 1) / kThreads;
  share_group_kernel<<<wgs, kThreads, 0, st>>>(group, shared, s.n_inst, s.t_cap, plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  share_place_kernel<<<wgs, kThreads, 0, st>>>(s.n_inst, plan);
  return hipGetLastError();
}

hipError_t launch_cache_shared(const Shape& s, const SharedArgs& a, bool decode, hipStream_t st) {
  if (s.kv_dtype == AP_BF16) return s.d == 128 ? run<bf16_t, 128>(a, decode, st) : run<bf16_t, 64>(a, decode, st);
  return s.d == 128 ? run<float, 128>(a, decode, st) : run<float, 64>(a, decode, st);
}

}  // namespace ap
