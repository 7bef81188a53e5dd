// Rows of caches with lengths of their own: new ones are appended, and caches beyond a budget lose those that gathered the least
// attention weight.
#include "cache_body.h"

namespace ap {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kPickThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 8;        // 16-byte pieces that a thread holds at a time

// K[i][L - n + r] = k_new[i][r], V the same: a copy of 16-byte pieces, a thread each, whose bound is the memory's rate.
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

// Order of floats as order of whole numbers; -0 counts as +0.
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned u = __float_as_uint(x == 0.f ? 0.f : x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Sum over the workgroup's threads before this one, and over all of them.
__device__ __forceinline__ int scan_before(int v, int* s_wave, int* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();                                         // s_wave may still be read from the scan before
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kPickThreads / 64; ++w) {
    if (w < wave) before += s_wave[w];
    total += s_wave[w];
  }
  *all = total;
  return before + x - v;
}

// One workgroup per instance: the rows that stay.  The m-th largest of the middle rows' weights is found digit by digit (11, 11 and 10
// bits of the ordered key, a histogram in LDS each); then the rows are gone through in order, and a prefix sum gives every row that stays
// its new place.  Weights move along: a row's new place is never behind its old one, and a round's weights are all read
// before any is written, so acc_out may be acc.
__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(CacheRows c, const float* acc, int budget, int n_first, int n_last,
                                                                  float* acc_out, int32_t* len_out, int32_t* __restrict__ kept) {
  __shared__ int s_hist[2048];
  __shared__ int s_wave[kPickThreads / 64];
  __shared__ unsigned s_prefix;
  __shared__ int s_need;
  const int i = blockIdx.x, tid = threadIdx.x;
  const int L = clamped(c.len[i], 0, c.t_cap);
  const float* w = acc + (size_t)i * c.t_cap;
  float* w_out = acc_out + (size_t)i * c.t_cap;
  kept += (size_t)i * budget;
  __syncthreads();                                         // everyone has the length before it may be overwritten
  if (L <= budget) {
    for (int j = tid; j < L; j += kPickThreads) {
      kept[j] = j;
      if (w_out != w) w_out[j] = w[j];
    }
    if (tid == 0) len_out[i] = L;
    return;
  }
  const int lo = n_first, hi = L - n_last;                 // the middle rows [lo, hi), more than `need` of them
  int need = budget - n_first - n_last;
  unsigned prefix = 0;                                     // the key of the last that stays; with need = 0 none does
  if (need > 0) {
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int pass = 0; pass < 3; ++pass) {
      for (int x = tid; x < 2048; x += kPickThreads) s_hist[x] = 0;
      __syncthreads();
      const int sh = shifts[pass], above = sh + bits[pass];
      for (int j = lo + tid; j < hi; j += kPickThreads) {
        const unsigned k = order_of(w[j]);
        if (pass == 0 || (k >> above) == (prefix >> above)) atomicAdd(&s_hist[(k >> sh) & ((1 << bits[pass]) - 1)], 1);
      }
      __syncthreads();
      // bins from the largest down, two a thread: the one in which the need is met
      const int b0 = 2047 - 2 * tid, h0 = s_hist[b0], h1 = s_hist[b0 - 1];
      int all;
      const int before = scan_before(h0 + h1, s_wave, &all);
      if (before < need && need <= before + h0 + h1) {
        const bool second = need > before + h0;
        s_prefix = prefix | ((unsigned)(b0 - (second ? 1 : 0)) << sh);
        s_need = need - before - (second ? h0 : 0);
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
    }
  }
  // `need` of the rows with the key `prefix` stay, the first ones, and all with a larger key
  const bool some = budget > n_first + n_last;
  int place = 0, ties = 0;
  for (int j0 = 0; j0 < L; j0 += kPickThreads) {
    const int j = j0 + tid;
    const bool in = j < L, middle = j >= lo && j < hi;
    const float x = in ? w[j] : 0.f;
    const unsigned k = order_of(x);
    const int tie = some && in && middle && k == prefix;
    int n_ties, n_stay;
    const int my_tie = ties + scan_before(tie, s_wave, &n_ties);
    const int stays = in && (!middle || (some && (k > prefix || (tie && my_tie < need))));
    const int at = place + scan_before(stays, s_wave, &n_stay);
    if (stays) {
      kept[at] = j;
      w_out[at] = x;
    }
    place += n_stay;
    ties += n_ties;
  }
  for (int j = budget + tid; j < L; j += kPickThreads) w_out[j] = 0.f;
  if (tid == 0) len_out[i] = budget;
}

// Row kept[j] of K and V becomes row j, in place.  A workgroup owns a column of 128 bytes of an instance's K or V, so nobody else reads or
// writes what it moves, and goes through the rows in order: a row's new place is never behind its old one, so that rows still to come
// are not overwritten; within a round, all rows have arrived in registers before one is written.
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(CacheRows c, u32x4* __restrict__ K, u32x4* __restrict__ V, int pieces,
                                                                  int budget, const int32_t* __restrict__ len_out,
                                                                  const int32_t* __restrict__ kept) {
  constexpr int W = 8, RPL = kMoveThreads / W;             // lanes a row, rows a load
  const int i = blockIdx.y, columns = pieces / W;
  u32x4* X = blockIdx.x < (unsigned)columns ? K : V;
  const int piece = (blockIdx.x % columns) * W + threadIdx.x % W, r = threadIdx.x / W;
  const int n = len_out[i];
  kept += (size_t)i * budget;
  for (int j0 = 0; j0 < n; j0 += RPL * kMoveLoads) {
    u32x4 x[kMoveLoads];
    bool moves[kMoveLoads];
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l) {
      const int j = j0 + l * RPL + r;
      const int src = j < n ? kept[j] : j;
      moves[l] = src != j;
      if (moves[l]) x[l] = X[row_at(c, i, src) * pieces + piece];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int l = 0; l < kMoveLoads; ++l) {
      size_t to;
      if (moves[l] && row_to_write(c, i, j0 + l * RPL + r, &to)) X[to * pieces + piece] = x[l];
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
  evict_pick_kernel<<<dim3(s.n_inst), kPickThreads, 0, st>>>(r, acc, budget, n_first, n_last, acc_out, len_out, kept);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pieces = pieces_of(s);
  evict_move_kernel<<<dim3(2 * pieces / 8, s.n_inst), kMoveThreads, 0, st>>>(r, static_cast<u32x4*>(K), static_cast<u32x4*>(V), pieces,
                                                                           budget, len_out, kept);
  return hipGetLastError();
}

}  // namespace ap
