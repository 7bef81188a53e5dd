// Rows of caches with lengths of their own: new ones are appended, and caches beyond a budget lose those that gathered the least
// attention weight.
#include "cache_body.h"

namespace ap {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 8;        // 16-byte pieces that a thread holds at a time

// K[i][L - n + r] = k_new[i][r], V the same: a copy of 16-byte pieces, a thread each, whose bound is the memory's rate (chunks of 128
// instances, 220 MB read and written: 47 us among other calls, which a large copy at 5.2 TB/s would take 42 for; over and over on the same rows,
// which the last-level cache then has, 37).
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(CacheRows c, const u32x4* __restrict__ k_new,
                                                                      const u32x4* __restrict__ v_new, const int32_t* __restrict__ n_new,
                                                                      int q_cap, int pieces, u32x4* __restrict__ K, u32x4* __restrict__ V) {
  const long long at = (long long)blockIdx.x * kAppendThreads + threadIdx.x;
  const long long row = at / pieces;                       // of k_new
  const int i = (int)(row / q_cap), r = (int)(row % q_cap), piece = (int)(at % pieces);
  if (i >= c.n_inst) return;
  const int n = n_new == nullptr ? q_cap : clamped(n_new[i], 0, q_cap);
  const long long j = (long long)c.len[i] - n + r;
  size_t to;
  if (r >= n || j < 0 || j >= c.t_cap || !row_to_write(c, i, (int)j, &to)) return;
  K[to * pieces + piece] = k_new[at];
  V[to * pieces + piece] = v_new[at];
}

// Order of floats as order of whole numbers, above 0; -0 counts as +0, and comes back as +0.
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned u = __float_as_uint(x == 0.f ? 0.f : x);
  return (u & 0x80000000u) ? (u == ~0u ? 1u : ~u) : (u | 0x80000000u);
}
__device__ __forceinline__ float of_order(unsigned k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// One workgroup per instance: the rows that stay.  Which key the last of the middle rows has that do is found by digits: a histogram of the
// keys' uppermost 13 bits (256 threads: 11) in LDS, that is of steps of a sixteenth of a power of two, in which even weights that lie
// close together spread over some hundred words; then, as a rule, the few keys of one step are left, which one wave halves the range of
// until the count is met.  More than kFew keys in a step (equal ones, say) go through another histogram.  Then ballots
// give every row that stays its new place.  A thread has up to 64 rows in registers, four in a row next to its neighbours' four, so that
// caches of up to 65536 rows (256 threads: 16384) are read once, longer ones in rounds of as many, three times as a rule.
// Weights move along: a row's new place is never behind its old one, and a round's weights are all read before any is written, so acc_out
// may be acc.  Bound by the chain of its steps on one CU: 64 caches of 2 to 33 thousand rows 28 us, 256 of 1088 rows 13.5.
constexpr int kQuads = 16;                                 // quads of rows that a thread has in a round
constexpr int kFew = 2048;                                 // keys that a wave has in registers

// The key of the need-th largest of m keys, by one wave; `above`: how many are larger than it.
__device__ __forceinline__ unsigned nth_key(const unsigned* s, int m, int need, unsigned least, unsigned most, int* above) {
  const int lane = threadIdx.x & 63;
  unsigned k[kFew / 64];
#pragma unroll
  for (int x = 0; x < kFew / 64; ++x) k[x] = x * 64 + lane < m ? s[x * 64 + lane] : 0u;
  *above = 0;
  while (least < most) {
    const unsigned mid = least + (most - least) / 2 + ((most - least) & 1);
    int n = 0;
#pragma unroll
    for (int x = 0; x < kFew / 64; ++x)
      if (x * 64 < m) n += k[x] >= mid;
    n = (int)wave_sum((float)n);
    if (n >= need) least = mid;
    else { most = mid - 1; *above = n; }
    if (n == need) break;
  }
  return least;
}

template <int NT, bool LONG>
__global__ __launch_bounds__(NT) void evict_pick_kernel(CacheRows c, const float* acc, int budget, int n_first, int n_last, float* acc_out,
                                                        int32_t* len_out, int32_t* __restrict__ kept) {
  constexpr int NW = NT / 64, BITS = NT == 1024 ? 13 : 11, BINS = 1 << BITS, MINE = BINS / NT;
  __shared__ int s_hist[BINS];                             // ... and then the keys that are left
  __shared__ int s_wave[2][NW];
  __shared__ int s_found[4];
  static_assert(BINS >= kFew, "the keys that are left");
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int L = clamped(c.len[i], 0, c.t_cap);
  const float* w = acc + (size_t)i * c.t_cap;
  float* w_out = acc_out + (size_t)i * c.t_cap;
  kept += (size_t)i * budget;
  __syncthreads();                                         // everyone has the length before it may be overwritten
  if (L <= budget) {
    for (int j = tid; j < L; j += NT) {
      kept[j] = j;
      if (w_out != w) w_out[j] = w[j];
    }
    if (tid == 0) len_out[i] = L;
    return;
  }
  for (int j = tid; j < n_first; j += NT) {
    kept[j] = j;
    if (w_out != w) w_out[j] = w[j];
  }
  const int lo = n_first, hi = L - n_last;                 // the middle rows [lo, hi), of which `need` stay, fewer than there are
  const int need = budget - n_first - n_last;
  const int begin = lo & ~3, span = hi - begin;            // (rows of w are 16-byte aligned and a multiple of 8 long)
  const int quads = (span + 4 * NT - 1) / (4 * NT) < kQuads ? (span + 4 * NT - 1) / (4 * NT) : kQuads;
  const int per_wave = quads * 256, round = per_wave * NW;
  const bool rounds = LONG && span > round;
  unsigned key[kQuads][4];                                 // 0: no middle row
  auto row_of = [&](int r0, int q) { return r0 + wave * per_wave + q * 256 + lane * 4; };      // the quad's first
  auto load = [&](int r0) {
#pragma unroll
    for (int q = 0; q < kQuads; ++q)
      if (q < quads) {
        const int j = row_of(r0, q);
        float4v v = {0.f, 0.f, 0.f, 0.f};
        if (j < hi) v = *reinterpret_cast<const float4v*>(w + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) key[q][e] = j + e >= lo && j + e < hi ? order_of(v[e]) : 0u;
      }
  };
  if (need > 0) {
    load(begin);
    // The largest key that at least `need` rows reach lies in [least, least + 2^width - 1]; `reach` rows reach the least, `above` lie above
    // that range.
    unsigned least = 0;
    int width = 32, above = 0, reach = hi - lo;
    while (reach != need && width > 0 && (width == 32 || reach - above > kFew)) {
      const int shift = width > BITS ? width - BITS : 0;
      for (int x = tid; x < BINS; x += NT) s_hist[x] = 0;
      __syncthreads();
      for (int r0 = begin; r0 < hi; r0 += round) {
        if (rounds && (r0 > begin || width < 32)) load(r0);
#pragma unroll
        for (int q = 0; q < kQuads; ++q)
          if (q < quads) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned off = key[q][e] - least;
              if (key[q][e] != 0 && key[q][e] >= least && (width == 32 || (off >> width) == 0)) atomicAdd(&s_hist[off >> shift], 1);
            }
          }
        if (!rounds) break;
      }
      __syncthreads();
      // From the largest bin down, MINE a thread: the one in which the need is met.
      int h[MINE], mine = 0;
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        h[x] = s_hist[BINS - 1 - tid * MINE - x];
        mine += h[x];
      }
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      if (lane == 63) s_wave[0][wave] = upto;
      __syncthreads();
      int before = above + upto - mine;
      for (int v = 0; v < NW; ++v) before += v < wave ? s_wave[0][v] : 0;
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        if (before < need && need <= before + h[x]) {
          s_found[0] = BINS - 1 - tid * MINE - x;
          s_found[1] = before;
          s_found[2] = before + h[x];
        }
        before += h[x];
      }
      __syncthreads();
      least += (unsigned)s_found[0] << shift;
      above = s_found[1];
      reach = s_found[2];
      width = shift;
    }
    int ties = reach == need ? L : need - above;           // of the rows with the key `least` the first so many stay
    if (reach != need && width > 0) {                      // the keys that are left
      if (tid == 0) s_found[3] = 0;
      __syncthreads();
      for (int r0 = begin; r0 < hi; r0 += round) {
        if (rounds) load(r0);
#pragma unroll
        for (int q = 0; q < kQuads; ++q)
          if (q < quads) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key[q][e] >= least && ((key[q][e] - least) >> width) == 0 && key[q][e] != 0) s_hist[atomicAdd(&s_found[3], 1)] = (int)key[q][e];
          }
        if (!rounds) break;
      }
      __syncthreads();
      if (wave == 0) {
        int larger;
        const unsigned last = nth_key(reinterpret_cast<const unsigned*>(s_hist), reach - above, need - above, least, least + ((1u << width) - 1), &larger);
        if (lane == 0) {
          s_found[0] = (int)last;
          s_found[1] = above + larger;
        }
      }
      __syncthreads();
      least = (unsigned)s_found[0];
      ties = need - s_found[1];
    }
    // Middle rows with a larger key than `last` stay, and of those with this one the first `ties`.
    const unsigned last = least;
    int place = n_first, tied = 0;                         // of all rows before, in the rounds before
    int turn = 0;
    for (int r0 = begin; r0 < hi; r0 += round) {
      if (rounds) load(r0);
      int both = 0;                                        // larger ones, and equal ones in the upper half
#pragma unroll
      for (int q = 0; q < kQuads; ++q)
        if (q < quads) {
#pragma unroll
          for (int e = 0; e < 4; ++e) both += (key[q][e] > last ? 1 : 0) + (key[q][e] == last && last != 0 ? 1 << 8 : 0);
        }
      const int larger_here = (int)wave_sum((float)(both & 0xff)), equal_here = (int)wave_sum((float)(both >> 8));   // at most 4096 each
      int larger = place, equal = tied, all_larger = 0, all_equal = 0;
      int* s = s_wave[turn++ & 1];
      if (lane == 0) s[wave] = larger_here + (equal_here << 16);
      __syncthreads();                                     // ... and this round's weights have been read
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const int x = s[v];
        all_larger += x & 0xffff;
        all_equal += x >> 16;
        if (v < wave) { larger += x & 0xffff; equal += x >> 16; }
      }
#pragma unroll
      for (int q = 0; q < kQuads; ++q)
        if (q < quads) {
          unsigned long long b[4], t[4];
          int own_larger = larger, own_equal = equal;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            b[e] = __ballot(key[q][e] > last);
            t[e] = __ballot(key[q][e] == last && last != 0);
            own_larger = __builtin_amdgcn_mbcnt_hi((unsigned)(b[e] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)b[e], own_larger));
            own_equal = __builtin_amdgcn_mbcnt_hi((unsigned)(t[e] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)t[e], own_equal));
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool is_larger = key[q][e] > last, is_equal = key[q][e] == last && last != 0;
            if (is_larger || (is_equal && own_equal < ties)) {
              const int to = own_larger + (own_equal < ties ? own_equal : ties);
              kept[to] = row_of(r0, q) + e;
              w_out[to] = of_order(key[q][e]);
            }
            own_larger += is_larger;
            own_equal += is_equal;
            larger += __popcll(b[e]);
            equal += __popcll(t[e]);
          }
        }
      place += all_larger;
      tied += all_equal;
      if (!rounds) break;
    }
  }
  // The last rows, behind them; middle rows never reach the places that these are read from.
  for (int r0 = 0; r0 < n_last; r0 += NT) {
    const int r = r0 + tid;
    const float v = r < n_last ? w[hi + r] : 0.f;
    __syncthreads();
    if (r < n_last) {
      kept[budget - n_last + r] = hi + r;
      w_out[budget - n_last + r] = v;
    }
  }
  __syncthreads();
  for (int j = budget + tid; j < L; j += NT) w_out[j] = 0.f;
  if (tid == 0) len_out[i] = budget;
}

// Row kept[j] of K and V becomes row j, in place.  A workgroup owns a column of W * 16 bytes of an instance's K or V, so nobody else reads or
// writes what it moves, and goes through the rows in order: a row's new place is never behind its old one, so that rows still to come
// are not overwritten; within a round, all rows have arrived in registers before one is written.
template <int W>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(CacheRows c, u32x4* __restrict__ K, u32x4* __restrict__ V, int pieces,
                                                                  int budget, const int32_t* __restrict__ len_out,
                                                                  const int32_t* __restrict__ kept) {
  constexpr int RPL = kMoveThreads / W;                    // lanes a row, rows a load
  const int i = blockIdx.y, columns = pieces / W;
  u32x4* X = blockIdx.x < (unsigned)columns ? K : V;
  const int piece = (blockIdx.x % columns) * W + threadIdx.x % W, r = threadIdx.x / W;
  const int n = len_out[i];
  kept += (size_t)i * budget;
  // A round's rows: where they come from, and what they hold.  The next round's are looked up before this one's have arrived, and asked for
  // before this one's are written: what is still to come lies behind what is written.
  auto look = [&](int j0, int (&src)[kMoveLoads]) {
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l) {
      const int j = j0 + l * RPL + r;
      src[l] = j < n ? kept[j] : j;
    }
  };
  auto load = [&](int j0, const int (&src)[kMoveLoads], u32x4 (&x)[kMoveLoads]) {
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l)
      if (src[l] != j0 + l * RPL + r) x[l] = X[row_at(c, i, src[l]) * pieces + piece];
  };
  int src[kMoveLoads], next[kMoveLoads];
  u32x4 x[kMoveLoads], y[kMoveLoads];
  look(0, src);
  load(0, src, x);
  for (int j0 = 0; j0 < n; j0 += RPL * kMoveLoads) {
    const int j1 = j0 + RPL * kMoveLoads;
    if (j1 < n) look(j1, next);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                       // this round's rows have arrived, everywhere
    if (j1 < n) load(j1, next, y);
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l) {
      size_t to;
      if (src[l] != j0 + l * RPL + r && row_to_write(c, i, j0 + l * RPL + r, &to)) X[to * pieces + piece] = x[l];
    }
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l) {
      src[l] = next[l];
      x[l] = y[l];
    }
  }
}

}  // namespace

static int pieces_of(const Shape& s) { return s.d * (s.kv_dtype == AP_BF16 ? 2 : 4) / 16; }

hipError_t launch_cache_append(const Shape& s, const CacheRows& r, const void* k_new, const void* v_new, const int32_t* n_new, int q_cap,
                               void* K, void* V, hipStream_t st) {
  const int pieces = pieces_of(s);
  const long long all = (long long)s.n_inst * q_cap * pieces;
  cache_append_kernel<<<dim3((unsigned)((all + kAppendThreads - 1) / kAppendThreads)), kAppendThreads, 0, st>>>(
      r, static_cast<const u32x4*>(k_new), static_cast<const u32x4*>(v_new), n_new, q_cap, pieces, static_cast<u32x4*>(K),
      static_cast<u32x4*>(V));
  return hipGetLastError();
}

hipError_t launch_cache_evict(const Shape& s, const CacheRows& r, void* K, void* V, const float* acc, int budget, int n_first, int n_last,
                              float* acc_out, int32_t* len_out, int32_t* kept, hipStream_t st) {
  // Few rows are done sooner by few waves, which have less to tell each other in a step (32 instances of 500, 1088, 2000, 4000 rows down to
  // half of them, whole calls: by 256 threads 15.7, 21.0, 29.0, 43.7 us, by 1024 18.3, 23.0, 28.8, 40.9; 256 instances 23.1, 45.1, 82.9, 159
  // and 24.5, 46.4, 82.5, 157).  The lengths are on the device; what is known here is how many rows there can be.
  if (s.t_cap <= 2048)
    evict_pick_kernel<256, false><<<dim3(s.n_inst), 256, 0, st>>>(r, acc, budget, n_first, n_last, acc_out, len_out, kept);
  else if (s.t_cap <= 1024 * 4 * kQuads)
    evict_pick_kernel<1024, false><<<dim3(s.n_inst), 1024, 0, st>>>(r, acc, budget, n_first, n_last, acc_out, len_out, kept);
  else
    evict_pick_kernel<1024, true><<<dim3(s.n_inst), 1024, 0, st>>>(r, acc, budget, n_first, n_last, acc_out, len_out, kept);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pieces = pieces_of(s);
  // Columns of 128 bytes, a line of the caches, where that makes two workgroups a CU, which have too little under way otherwise; else of
  // 64.  (256 caches of 1088 rows down to 1024, whole calls: columns of 64 bytes 89 us, of 128 78, of 256 111; 64 caches after prompts, the
  // moves alone: of 64 bytes 20, of 128 28.)
  auto move = [&](auto kernel, int w) {
    kernel<<<dim3(2 * pieces / w, s.n_inst), kMoveThreads, 0, st>>>(r, static_cast<u32x4*>(K), static_cast<u32x4*>(V), pieces, budget, len_out, kept);
  };
  if (s.n_inst * (2 * pieces / 8) >= 512) move(evict_move_kernel<8>, 8);
  else move(evict_move_kernel<4>, 4);
  return hipGetLastError();
}

}  // namespace ap
