// Attention of one new token per instance over a cache of the instance's own length, the whole of it or a window and the first rows.
//
//   s_hj = q_h . K_j / sqrt(d),  m_h = max_j s_hj,  P_hj = exp(s_hj - m_h) / sum_j exp(s_hj - m_h),  out_h = sum_j P_hj V_j,
//   acc_j += sum_h P_hj,  over the rows j that the token at position L - 1 sees.
//
// Memory-bound: 2 d sizeof(T) bytes a row and 4 g d operations on them.  Lengths differ, so the rows are not dealt by instance: the rows
// seen by all instances, in groups of 16 and in the instances' order, are cut into equal shares, one a workgroup, and every
// workgroup finds out from the lengths where its share begins.  A workgroup that goes over a whole instance writes its output; the
// pieces of the others are joined by the last workgroup of the instance to be done.  With weights, which need the joined maximum and
// sum, a second launch joins and adds them.
//
// A wave goes over its groups with a running maximum and sum; two groups of K and V are on their way to LDS, past the registers and not
// kept in the caches, while one is worked off: q . K on the matrix unit, P . V with fp32 multiply-adds, as probabilities of fewer digits
// would show in the fp32 output.  Measured: 256 instances of 60 to 32790 rows (g = 4, d = 128, pages of 16; 785 MB) 149-157 us, 5.1 TB/s; 1024
// with a window of 4096 (g = 8; 2.1 GB) 353 us, 5.9 TB/s; 64 of 2000 to 16000 rows in fp32 (g = 4; 465 MB, a workgroup a CU) 82 us, 5.7 TB/s,
// d = 64 49 us, 4.8; with rows through registers and pages looked up by vector loads, which wait for
// the rows in flight, 246 and 639.  Where more instances than workgroups are all short, every wave takes whole ones: 2048 of 8 to 419 rows
// (g = 1, 111 MB) 38 us, by shares of a workgroup 61; of 16 to 56 (g = 2, d = 64) 18 and 40.
#include "cache_body.h"

namespace ap {
namespace {

constexpr int kThreads = 256, kWaves = 4, kGroup = 16;
constexpr int kLeastGroups = 8;      // least share of a workgroup: two passes a wave
constexpr int kShort = 64;           // groups of an instance that a wave goes over alone
constexpr unsigned long long kAlone = ~0ull;   // in the place of the number of groups: every instance was whole
constexpr int kLongShare = 64;       // share from which on a CU has several workgroups

// The rows that an instance's new token sees: [0, f) and [lo, L), f <= lo; in groups of 16 rows: gs groups from 0 on, the others from gb.
struct Seen {
  int L, lo, f, gs, gb, n;
  __device__ __forceinline__ int group(int u) const { return u < gs ? u : gb + (u - gs); }
  __device__ __forceinline__ bool row(int j) const { return j < L && (j >= lo || j < f); }
};
__device__ __forceinline__ Seen seen_of(int len, int t_cap, int window, int n_first) {
  Seen s;
  s.L = clamped(len, 0, t_cap);
  s.lo = window > 0 && s.L > window ? s.L - window : 0;
  s.f = n_first < s.lo ? n_first : s.lo;
  s.gs = (s.f + kGroup - 1) / kGroup;
  s.gb = s.lo / kGroup > s.gs ? s.lo / kGroup : s.gs;
  s.n = s.L == 0 ? 0 : s.gs + (s.L - 1) / kGroup - s.gb + 1;
  return s;
}

// Groups of a workgroup.  Up to kLongShare one workgroup a CU: what several gain in loads under way is less than what their pieces cost to
// join (8 instances of 8000 rows, g = 4, d = 128: 512 workgroups 22 us, 250 19; of 32000 rows 36 and 33; 16 of 32000 rows, from
// where on it does not matter, 53 and 51; 8 of 2041 rows by shares of 4, 8, 16: 13.5, 12.4, 13.4).
__device__ __forceinline__ unsigned long long share_of(unsigned long long groups, int wgs) {
  const unsigned long long one = (groups + 255) / 256, all = (groups + wgs - 1) / wgs;
  return one <= kLeastGroups ? kLeastGroups : (one <= kLongShare ? one : (all > kLongShare ? all : kLongShare));
}

// Scores below what 32 bits hold are -inf and weigh nothing.  Where a head has no others yet its maximum is -inf, which exponents do not refer to,
// and its sum 0, by which nothing is divided: the output is zero.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float over(float x, float sum) { return sum == 0.f ? 0.f : x / sum; }

template <typename T, int D, int G> struct Form {
  static constexpr int E = 16 / (int)sizeof(T);            // elements of a 16-byte piece
  static constexpr int PIECES = D / E;                     // pieces of a row = lanes that have a V row
  static constexpr int N = PIECES / 4;                     // pieces of a group's K (or V) per lane
  static constexpr int RPL = kWave / PIECES;               // V rows that a wave reads at a time
  static constexpr int TILE = kGroup * PIECES;             // pieces of a group's K (or V)
  static constexpr int QUERIES = (G * PIECES + kWave - 1) / kWave;     // loads of a wave for the queries
  static constexpr int WAVE = 4 * TILE + QUERIES * kWave;              // pieces of LDS of a wave: two groups of K and V, and the queries
  static constexpr int BUFFERS = kWaves * WAVE * 16;
  static constexpr int PER_CU = PIECES == 8 ? (G == 8 ? 3 : 4) : (PIECES == 16 ? 2 : 1);   // workgroups a CU, as LDS (G = 8: registers) has room for
  static constexpr int WGS = 256 * PER_CU;                 // the workgroups that 256 CUs hold at once
  static_assert((WGS + 4) * G * 4 + G * D * 4 <= BUFFERS && WGS < (1 << kTicketBits), "factors of the pieces, counts");
  static_assert(WGS <= kCacheDecodeWgs && PER_CU * (BUFFERS + 4096) <= 160 * 1024, "workspace, LDS");
  // Piece p of row r of a K group lies at place p ^ (r % PIECES): the operand layout reads a row per lane.
  __device__ static __forceinline__ int k_place(int r, int p) { return p ^ (r & (PIECES - 1)); }
};

// Where a group of 16 rows lies: its first and its second eight, in rows of K and V; and whether all 16 are seen.  Wave-uniform.
struct Place { size_t a, b; int t0; bool all; };
__device__ __forceinline__ Place place_of(const CacheRows& r, int inst, const Seen& s, int u) {
  Place p;
  p.t0 = __builtin_amdgcn_readfirstlane(s.group(u) * kGroup);
  p.a = rows_at(r, inst, p.t0);
  p.b = r.lb == 3 && r.table != nullptr ? rows_at(r, inst, p.t0 + 8) : p.a + 8;
  p.all = p.t0 + kGroup <= s.L && (p.t0 >= s.lo || p.t0 + kGroup <= s.f);
  return p;
}
// Sends the rows of a group of K (or V) to LDS.
template <typename F, bool IS_V> __device__ __forceinline__ void send(const void* X, const Place& p, const Seen& s, int lane, unsigned lds) {
  constexpr unsigned row = F::PIECES * 16;
  if (p.all && p.b == p.a + 8) {
    const char* base = static_cast<const char*>(X) + p.a * row;
#pragma unroll
    for (int l = 0; l < F::N; ++l) {
      const int x = l * kWave + lane, r = x / F::PIECES, place = x % F::PIECES;
      to_lds<true>(base, r * row + (IS_V ? place : F::k_place(r, place)) * 16, lds + l * 1024);
    }
  } else {
    // Rows that are not seen are not read: another row of the group, which is, stands in for them.
    const int other = (p.t0 < s.f ? p.t0 : (p.t0 > s.lo ? p.t0 : s.lo)) - p.t0;
#pragma unroll 1
    for (int l = 0; l < F::N; ++l) {
      const int x = l * kWave + lane, r = x / F::PIECES, place = x % F::PIECES;
      const int y = s.row(p.t0 + r) ? r : other;
      const size_t at = y < 8 ? p.a + y : p.b + (y - 8);
      to_lds_from(static_cast<const char*>(X) + at * row + (IS_V ? place : F::k_place(r, place)) * 16, lds + l * 1024);
    }
  }
}

// Called by every thread of a workgroup that has left its piece: true in the last of `parts` to get here.  The word, of a workspace that may
// hold anything, counts below the launch's number in its upper bits (as in take_ticket, but nobody sees to the number beforehand: many
// workgroups that do so at a time keep the first rows waiting): who finds another number there has counted for nothing and
// puts the number and a first count in the place of what it left, unless somebody was faster.  The last leaves zero.
__device__ __forceinline__ bool last_of(unsigned long long* word, unsigned long long nonce, int parts, int* s_last) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // this wave's share of the piece has reached memory
  __syncthreads();
  if (threadIdx.x == 0) {
    constexpr unsigned long long low = (1ull << kTicketBits) - 1;
    unsigned long long at = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (((at ^ nonce) >> kTicketBits) != 0) {
      ++at;
      for (;;) {
        if (__hip_atomic_compare_exchange_strong(word, &at, nonce | 1, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) {
          at = nonce;
          break;
        }
        if (((at ^ nonce) >> kTicketBits) == 0) {
          at = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          break;
        }
      }
    }
    const bool last = (int)(at & low) == parts - 1;
    if (last) end_tickets(word);
    *s_last = last;
  }
  __syncthreads();
  return *s_last != 0;
}

// Joins `parts` pieces, from that of workgroup w0 on, by one workgroup: maximum and 1 / sum of every head to s_m and s_inv, and, unless
// inst < 0, the output.  SHARED: the pieces were written by workgroups of the same launch.  s: `bytes` of LDS, the factors of the pieces in
// front, and behind them pieces, of which as many as there is room for are on their way at a time: one workgroup's loads are what this
// costs (64 pieces of g = 4, d = 128, 16 in registers at a time: 12 us).
template <int G, int D, bool SHARED>
__device__ __forceinline__ void join_pieces(const DecodeArgs& a, int inst, int w0, int parts, float* s, int bytes, float* s_m, float* s_inv) {
  constexpr int PP = G * D / 4, R = (G * D + kThreads - 1) / kThreads;              // 16-byte pieces of a part, outputs of a thread
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto read = [](const float* p) { return SHARED ? ld_shared_out(p) : *p; };
  auto slot = [&](int p) { return 2 * (size_t)(w0 + p) + (p == 0 ? 1 : 0); };      // the first is the last piece of its workgroup
  const int front = (parts * G + 3) / 4 * 4;               // floats
  float* s_parts = s + front;
  const int room = (bytes / 4 - front) / (G * D);          // parts
  const unsigned lds = lds_address(s_parts);
  auto send = [&](int p0) {
    const int n = parts - p0 < room ? parts - p0 : room;
    for (int x0 = wave * 64; x0 < n * PP; x0 += kThreads) {
      const int x = x0 + lane;
      if (x < n * PP) {
        const float* src = a.part_acc + slot(p0 + x / PP) * (G * D) + x % PP * 4;
        if constexpr (SHARED) shared_to_lds(src, lds + x0 * 16);
        else to_lds_from(src, lds + x0 * 16);
      }
    }
  };
  if (inst >= 0) send(0);
  constexpr int HEADS = (G + kWaves - 1) / kWaves;         // of a wave
  float m0[HEADS], l0[HEADS];                              // of the lane's first piece
#pragma unroll
  for (int x = 0; x < HEADS; ++x) {
    const int h = wave + x * kWaves;
    const bool have = h < G && lane < parts;
    m0[x] = have ? read(a.part_ml + (slot(lane) * G + h) * 2) : -INFINITY;
    l0[x] = have ? read(a.part_ml + (slot(lane) * G + h) * 2 + 1) : 0.f;
  }
#pragma unroll
  for (int x = 0; x < HEADS; ++x) {
    const int h = wave + x * kWaves;
    if (h >= G) break;
    float top = m0[x];
    for (int p = lane + 64; p < parts; p += 64) top = fmaxf(top, read(a.part_ml + (slot(p) * G + h) * 2));
    top = wave_max(top);
    const float use = reference(top);
    const float f0 = exp2_fast(m0[x] - use);
    if (lane < parts) s[lane * G + h] = f0;
    float all = f0 * l0[x];
    for (int p = lane + 64; p < parts; p += 64) {
      const float f = exp2_fast(read(a.part_ml + (slot(p) * G + h) * 2) - use);
      s[p * G + h] = f;
      all += f * read(a.part_ml + (slot(p) * G + h) * 2 + 1);
    }
    all = wave_sum(all);
    if (lane == 0) {
      s_m[h] = use;
      s_inv[h] = over(1.f, all);
    }
  }
  if (inst < 0) {
    __syncthreads();
    return;
  }
  float val[R];
#pragma unroll
  for (int r = 0; r < R; ++r) val[r] = 0.f;
  for (int p0 = 0; p0 < parts; p0 += room) {
    if (p0 > 0) {
      __syncthreads();
      send(p0);
    }
    landed<0>();
    __syncthreads();
    const int n = parts - p0 < room ? parts - p0 : room;
#pragma unroll 4
    for (int p = 0; p < n; ++p)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int x = r * kThreads + tid;
        if (x < G * D) val[r] += s[(p0 + p) * G + x / D] * s_parts[p * G * D + x];
      }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int x = r * kThreads + tid;
    if (x < G * D) a.out[(size_t)inst * G * D + x] = val[r] * s_inv[x / D];
  }
}

template <typename T, int D, int G, bool ACC>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(Form<T, D, G>::PER_CU))) void cache_decode_kernel(DecodeArgs a) {
  using F = Form<T, D, G>;
  extern __shared__ __attribute__((aligned(16))) u32x4 s_rows[];          // [wave]: [buffer][K, V][TILE], queries; at the end outputs, [G][D]
  __shared__ __attribute__((aligned(16))) float s_p[kWaves][kGroup][G];
  __shared__ float s_ml[kWaves][G][2];
  __shared__ unsigned long long s_wave[kWaves];
  __shared__ int s_first[kWaves], s_longest[kWaves], s_end, s_from, s_last;
  __shared__ float s_m[G], s_inv[G];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = lane & 15, kg = lane >> 4;

  // Where this workgroup's share begins: every thread sums the groups of consecutive instances.
  const int chunk = (a.r.n_inst + kThreads - 1) / kThreads;
  const int i_begin = tid * chunk < a.r.n_inst ? tid * chunk : a.r.n_inst;
  const int i_end = i_begin + chunk < a.r.n_inst ? i_begin + chunk : a.r.n_inst;
  unsigned long long mine = 0;
  int longest = 0;
#pragma unroll 4
  for (int i = i_begin; i < i_end; ++i) {
    const int n = seen_of(a.r.len[i], a.r.t_cap, a.window, a.n_first).n;
    mine += (unsigned)n;
    longest = n > longest ? n : longest;
  }
  unsigned long long upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long y = __shfl_up(upto, o, 64);
    if (lane >= o) upto += y;
  }
  if (a.r.n_inst > F::WGS) longest = (int)wave_max((float)(longest < kShort + 1 ? longest : kShort + 1));
  if (lane == 63) {
    s_wave[wave] = upto;
    s_longest[wave] = longest;
  }
  if (tid < kWaves) s_first[tid] = a.r.n_inst;
  if (tid == 0) s_end = 0;
  __syncthreads();
  unsigned long long groups = 0, ahead = upto - mine;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) ahead += s_wave[w];
    groups += s_wave[w];
    longest = s_longest[w] > longest ? s_longest[w] : longest;
  }
  // More instances than workgroups, all of them short: every wave takes whole instances, those that begin in its share, with no pieces and
  // nobody to wait for.
  const bool alone = __builtin_amdgcn_readfirstlane(a.r.n_inst > F::WGS && longest <= kShort);
  const unsigned long long per = alone ? kWaves * ((groups + kWaves * F::WGS - 1) / (kWaves * F::WGS)) : share_of(groups, F::WGS);
  const unsigned long long begin = (unsigned long long)blockIdx.x * per;
  const unsigned long long end = begin + per < groups ? begin + per : groups;
  // Empty instances have no share; their outputs are zero.
  for (int i = blockIdx.x; i < a.r.n_inst; i += F::WGS)
    if (a.r.len[i] <= 0)
      for (int x = tid; x < G * D; x += kThreads) a.out[(size_t)i * G * D + x] = 0.f;
  if (ACC && blockIdx.x == 0) {
    unsigned long long at = ahead;
    for (int i = i_begin; i < i_end; ++i) {
      a.before[i] = at;
      at += (unsigned)seen_of(a.r.len[i], a.r.t_cap, a.window, a.n_first).n;
    }
    if (tid == kThreads - 1) a.before[a.r.n_inst] = alone ? kAlone : groups;
  }
  if (begin >= end) return;
  const unsigned long long share = per / kWaves;           // alone: of a wave
  if (alone ? ahead < end && begin < ahead + mine : ahead <= begin && begin < ahead + mine) {
    unsigned long long at = ahead;
    for (int i = i_begin; i < i_end; ++i) {
      const unsigned n = (unsigned)seen_of(a.r.len[i], a.r.t_cap, a.window, a.n_first).n;
      if (alone) {
        if (n > 0 && at >= begin && at < end) {
          atomicMin(&s_first[(int)((at - begin) / share)], i);
          atomicMax(&s_end, i + 1);
        }
      } else if (begin < at + n) {
        s_first[0] = i;
        s_from = (int)(begin - at);
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  int inst = __builtin_amdgcn_readfirstlane(s_first[alone ? wave : 0]), from = alone ? 0 : __builtin_amdgcn_readfirstlane(s_from);
  unsigned long long left = end - begin, done = begin;      // groups to do, and the number of the next one
  int mine_to = 0;                                          // alone: the first instance behind this wave's
  if (alone) {
    mine_to = s_end;
    for (int w = kWaves - 1; w > wave; --w) mine_to = s_first[w] < mine_to ? s_first[w] : mine_to;
  }
  const int step = alone ? 1 : kWaves;

  const float scale = kLog2E / sqrtf((float)D);
  const u32x4* mine_rows = s_rows + wave * F::WAVE;
  const unsigned ring = lds_address(mine_rows);
  float* s_out = reinterpret_cast<float*>(s_rows);
  for (; alone ? left > 0 && inst < mine_to : left > 0; ++inst, from = 0) {
    const Seen s = seen_of(a.r.len[inst], a.r.t_cap, a.window, a.n_first);
    if (s.n <= from) continue;                             // an empty instance
    const int to = alone ? s.n : (unsigned long long)(s.n - from) <= left ? s.n : from + (int)left;
    if (!alone) left -= (unsigned)(to - from);
    const bool whole = from == 0 && to == s.n;
    // The other pieces: of the workgroups from w0 on.  The last of them to be done joins them; with weights a second launch does.
    int w0 = blockIdx.x, parts = 1;
    if (!ACC && !whole) {
      if (from > 0) w0 = (int)((done - (unsigned)from) / per);
      parts = (int)((done + (unsigned)(s.n - from) - 1) / per) - w0 + 1;
    }
    done += (unsigned)(to - from);
    unsigned long long* ticket = a.tickets + (size_t)w0 * kTicketStride;      // (an instance that begins in a workgroup and does not end there: one at most)

    // This wave's groups are from + wave, from + wave + 4, ...; two of them are on their way to LDS while one is worked off.
    const int mine_n = alone ? s.n : (to - from > wave ? (to - from - wave + kWaves - 1) / kWaves : 0);
    const int u0 = alone ? 0 : from + wave;
    Place next[2];                                         // of the groups behind the ones that were sent for
    if (mine_n > 0) {
#pragma unroll
      for (int x = 0; x < F::QUERIES; ++x) {
        const int piece = x * kWave + lane;
        to_lds<false>(static_cast<const u32x4*>(a.q) + (size_t)inst * G * F::PIECES, (piece < G * F::PIECES ? piece : 0) * 16,
                      ring + (4 * F::TILE + x * kWave) * 16);
      }
      const Place p = place_of(a.r, inst, s, u0), p1 = place_of(a.r, inst, s, mine_n > 1 ? u0 + step : u0);
      send<F, false>(a.K, p, s, lane, ring);
      send<F, true>(a.V, p, s, lane, ring + F::TILE * 16);
      if (mine_n > 1) {
        send<F, false>(a.K, p1, s, lane, ring + 2 * F::TILE * 16);
        send<F, true>(a.V, p1, s, lane, ring + 3 * F::TILE * 16);
      }
      next[0] = p; next[1] = p1;
    }
    // B operand of the products q . K: lane (head, kg) has piece 4 l + kg of the head's query; heads beyond g count for nothing.  The queries
    // were sent for first.
    u32x4 qf[F::N];
    if (mine_n > 1) landed<4 * F::N>(); else landed<2 * F::N>();
#pragma unroll
    for (int l = 0; l < F::N; ++l) {
      const u32x4 x = mine_rows[4 * F::TILE + (head % G) * F::PIECES + 4 * l + kg];
      qf[l] = x;
    }
    float m = -INFINITY, sum = 0.f;                        // of head `head`; the sum over this lane's rows
    float o[G][F::E];
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int e = 0; e < F::E; ++e) o[h][e] = 0.f;

    for (int it = 0; it < mine_n; ++it) {
      const Place here = next[0];
      next[0] = next[1];
      next[1] = place_of(a.r, inst, s, u0 + step * (it + 2 < mine_n ? it + 2 : it));
      const bool more = it + 2 < mine_n;
      const int t0 = here.t0;
      const unsigned slot = ring + (it & 1) * 2 * F::TILE * 16;
      const u32x4* Kt = mine_rows + (it & 1) * 2 * F::TILE;
      const u32x4* Vt = Kt + F::TILE;
      if (it + 1 < mine_n) landed<3 * F::N>(); else landed<F::N>();
      // Rows t0 + 4 kg + r of head `head`.  fp32 products go into four sums, whose roundings are smaller than those of one over all of d.
      constexpr int SUMS = sizeof(T) == 2 ? 1 : 4;
      float4v sums[SUMS];
#pragma unroll
      for (int x = 0; x < SUMS; ++x) sums[x] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int l = 0; l < F::N; ++l) {
        const u32x4 k = Kt[head * F::PIECES + F::k_place(head, 4 * l + kg)];
        if constexpr (sizeof(T) == 2) {
          sums[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[l]), sums[0], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sums[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(qf[l][e]), sums[e], 0, 0, 0);
        }
      }
      float4v c = sums[0];
      if constexpr (SUMS == 4) {
#pragma unroll
        for (int r = 0; r < 4; ++r) c[r] = (sums[0][r] + sums[1][r]) + (sums[2][r] + sums[3][r]);
      }
      if (more) {
        lds_read();
        send<F, false>(a.K, next[1], s, lane, slot);
      }
      if (!here.all) {
        const int j = t0 + 4 * kg;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!s.row(j + r)) c[r] = -INFINITY;
      }
      float top = fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3]));
      top = max32(max16(top));
      // The reference is a whole number in units of log2: changing it multiplies by a power of two and rounds nothing, and the exponent
      // is one fused multiply-add.
      const float ref = fmaxf(m, ceilf(top * scale));
      if (__any(ref != m)) {
        const float shrink = ref == m ? 1.f : exp2_fast(m - ref);
        sum *= shrink;
#pragma unroll
        for (int h = 0; h < G; ++h) {
          const float f = __shfl(shrink, h, 64);
#pragma unroll
          for (int e = 0; e < F::E; ++e) o[h][e] *= f;
        }
        m = ref;
      }
      const float use = reference(m);
      if (ACC && head < G && t0 + 4 * kg < a.r.t_cap) {    // (t_cap is a multiple of 8: four rows are within it or not)
        float4v z;
#pragma unroll
        for (int r = 0; r < 4; ++r) z[r] = c[r];
        *reinterpret_cast<float4v*>(a.logits + ((size_t)inst * G + head) * a.r.t_cap + t0 + 4 * kg) = z;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = exp2_of(c[r], scale, use);
        sum += p;
        if (head < G) s_p[wave][4 * kg + r][head] = p;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (more) landed<3 * F::N>();
      else if (it + 1 < mine_n) landed<2 * F::N>();
      else landed<0>();
#pragma unroll
      for (int l = 0; l < F::N; ++l) {
        float v[F::E];
        const u32x4 x = Vt[l * kWave + lane];              // piece lane % PIECES of row l * RPL + lane / PIECES
        unpack16(make_uint4(x.x, x.y, x.z, x.w), v, T{});
        const float* p = s_p[wave][l * F::RPL + lane / F::PIECES];
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int e = 0; e < F::E; ++e) o[h][e] = __builtin_fmaf(p[h], v[e], o[h][e]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (more) {
        lds_read();
        send<F, true>(a.V, next[1], s, lane, slot + F::TILE * 16);
      }
    }

    // The wave's lanes, then the workgroup's waves.
    sum = sum32(sum16(sum));
#pragma unroll
    for (int h = 0; h < G; ++h) {
#pragma unroll
      for (int e = 0; e < F::E; ++e) {
        if (F::PIECES <= 8) o[h][e] += dpp_move<0x128>(o[h][e]);          // row_ror:8
        if (F::PIECES <= 16) o[h][e] = sum16(o[h][e]);
        o[h][e] = sum32(o[h][e]);
      }
    }
    if (alone) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float all = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sum), h));
        if (lane < F::PIECES) {
          float* to_out = a.out + ((size_t)inst * G + h) * D + lane * F::E;
#pragma unroll
          for (int e = 0; e < F::E; ++e) to_out[e] = over(o[h][e], all);
        }
      }
      if (ACC && lane < G) {
        a.whole[((size_t)inst * G + lane) * 2] = m;
        a.whole[((size_t)inst * G + lane) * 2 + 1] = sum;
      }
      continue;
    }
    if (lane < F::PIECES) {
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int e = 0; e < F::E; ++e) s_out[wave * F::WAVE * 4 + h * D + lane * F::E + e] = o[h][e];
    }
    if (lane < G) {
      s_ml[wave][lane][0] = m;
      s_ml[wave][lane][1] = sum;
    }
    __syncthreads();
    const size_t slot = 2 * (size_t)blockIdx.x + (from == 0 ? 1 : 0);   // the piece an instance begins with is its workgroup's last
    for (int x = tid; x < G * D; x += kThreads) {
      const int h = x / D, e = x % D;
      float top = s_ml[0][h][0];
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_ml[w][h][0]);
      const float use = reference(top);
      float all = 0.f, val = 0.f;
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_fast(s_ml[w][h][0] - use);
        all += f * s_ml[w][h][1];
        val += f * s_out[w * F::WAVE * 4 + x];
      }
      if (whole) a.out[((size_t)inst * G + h) * D + e] = over(val, all);
      else st_shared_out<!ACC>(a.part_acc + (slot * G + h) * D + e, val);
      if (e == 0 && (ACC || !whole)) {
        float* ml = whole ? a.whole + ((size_t)inst * G + h) * 2 : a.part_ml + (slot * G + h) * 2;
        st_shared_out<!ACC>(ml, top);
        st_shared_out<!ACC>(ml + 1, all);
      }
    }
    if (!ACC && !whole && last_of(ticket, a.nonce, parts, &s_last))
      join_pieces<G, D, true>(a, inst, w0, parts, s_out, F::BUFFERS, s_m, s_inv);
    __syncthreads();
  }
}

// Adds the weights, and joins the pieces of instances that several workgroups went over.  Workgroup (0, instance) has the output,
// workgroup (1 + x, instance) the weights of 1024 rows.
constexpr int join_bytes(int g, int d) { return (kCacheDecodeWgs + 4) * g * 4 + 8 * g * d * 4; }
template <int G, int D>
__global__ __launch_bounds__(kThreads) void cache_join_kernel(DecodeArgs a, int wgs) {
  extern __shared__ __attribute__((aligned(16))) float s_join[];          // join_bytes
  __shared__ float s_m[G], s_inv[G];
  const int i = blockIdx.y, tid = threadIdx.x;
  const Seen s = seen_of(a.r.len[i], a.r.t_cap, a.window, a.n_first);
  const float scale = kLog2E / sqrtf((float)D);
  if (s.n == 0) return;
  const int j0 = ((int)blockIdx.x - 1) * 4 * kThreads;
  if (blockIdx.x > 0 && (j0 >= s.L || (j0 >= s.f && j0 + 4 * kThreads <= s.lo))) return;
  const unsigned long long at = a.before[i], groups = a.before[a.r.n_inst], per = share_of(groups, wgs);
  const int w0 = (int)(at / per), parts = groups == kAlone ? 1 : (int)((at + (unsigned)s.n - 1) / per) - w0 + 1;
  if (parts > 1) {
    join_pieces<G, D, false>(a, blockIdx.x == 0 ? i : -1, w0, parts, s_join, join_bytes(G, D), s_m, s_inv);
  } else if (tid < G) {
    s_m[tid] = reference(a.whole[((size_t)i * G + tid) * 2]);
    s_inv[tid] = over(1.f, a.whole[((size_t)i * G + tid) * 2 + 1]);
  }
  if (blockIdx.x == 0) return;
  __syncthreads();
  const int j = j0 + 4 * tid;
  if (j >= s.L || (j >= s.f && j + 4 <= s.lo)) return;     // (so j < t_cap, and j + 3 too: it is a multiple of 8)
  float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < G; ++h) {
    const float4v z = *reinterpret_cast<const float4v*>(a.logits + ((size_t)i * G + h) * a.r.t_cap + j);
#pragma unroll
    for (int r = 0; r < 4; ++r) add[r] += exp2_of(z[r], scale, s_m[h]) * s_inv[h];
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (s.row(j + r)) a.acc[(size_t)i * a.r.t_cap + j + r] += add[r];
}

template <typename T, int D, int G> hipError_t run(const DecodeArgs& a, hipStream_t st) {
  using F = Form<T, D, G>;
  if (a.acc != nullptr) cache_decode_kernel<T, D, G, true><<<F::WGS, kThreads, F::BUFFERS, st>>>(a);
  else cache_decode_kernel<T, D, G, false><<<F::WGS, kThreads, F::BUFFERS, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.acc == nullptr) return e;
  const unsigned columns = (unsigned)((a.r.t_cap + 4 * kThreads - 1) / (4 * kThreads));
  cache_join_kernel<G, D><<<dim3(1 + columns, a.r.n_inst), kThreads, join_bytes(G, D), st>>>(a, F::WGS);
  return hipGetLastError();
}
template <typename T, int D> hipError_t run_g(int g, const DecodeArgs& a, hipStream_t st) {
  return g == 1 ? run<T, D, 1>(a, st) : g == 2 ? run<T, D, 2>(a, st) : g == 4 ? run<T, D, 4>(a, st) : run<T, D, 8>(a, st);
}

}  // namespace

hipError_t launch_cache_decode(const Shape& s, const DecodeArgs& args, hipStream_t st) {
  DecodeArgs a = args;
  a.nonce = new_nonce(kTicketBits);
  if (s.kv_dtype == AP_BF16) return s.d == 128 ? run_g<bf16_t, 128>(s.g, a, st) : run_g<bf16_t, 64>(s.g, a, st);
  return s.d == 128 ? run_g<float, 128>(s.g, a, st) : run_g<float, 64>(s.g, a, st);
}

}  // namespace ap
