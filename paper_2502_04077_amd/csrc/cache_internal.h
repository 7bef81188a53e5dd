// Caches whose instances have lengths of their own: what the calls on them (cache_api.hip) hand to the kernels.
#pragma once

#include "ap_internal.h"

namespace ap {

// Rows of the caches: instance i's row j lies at row i * t_cap + j of K and V, or, with a table, at row j % b of the page that the
// table names for block j / b.
struct CacheRows {
  const int32_t* table;    // [n_inst][nb_cap], or null
  const int32_t* len;      // [n_inst]
  int n_inst, t_cap, nb_cap, n_phys, lb;   // lb = log2(b)
};

struct DecodeArgs {
  CacheRows r;
  const void *q, *K, *V;
  int window, n_first;
  float *out, *acc;
  unsigned long long* before;   // workspace: [n_inst + 1] groups of 16 rows in the instances before
  float* whole;                 // workspace: [n_inst][g][2] maximum and sum of the instances that one workgroup goes over
  float *part_ml, *part_acc;    // workspace: [2 * kCacheDecodeWgs][g][2] and [..][g][d] of the others' pieces
  unsigned long long* tickets;  // workspace: [kCacheDecodeWgs][kTicketStride], without acc: pieces done of the instance that begins in a workgroup
  unsigned long long nonce;     // a number of this launch's own (new_nonce)
  float* logits;                // workspace: [n_inst][g][t_cap], with acc only
};

struct PrefillArgs {
  CacheRows r;
  const void *q, *K, *V;
  const int32_t* n_q;           // [n_inst], or null: q_cap each
  int q_cap, window, n_first;
  void* out;
  float* acc;
  float* stat;                  // workspace: [n_inst][stat_rows][2] maximum and 1 / sum of every row of q, with acc only
  float* sums;                  // workspace: [chunks][n_inst][tiles][128] columns' sums over a chunk of the queries, with acc only
  float *part_ml, *part_o;      // workspace: [splits][n_inst][q_cap * g][2] and [..][d], where the cache is in splits
  int splits;                   // set by the launcher, as the next ones
  int chunks, tiles, stat_rows; // set by the launcher: chunks of the queries; tiles of rows of q, and rows in whole tiles, an instance
};

constexpr int kCacheDecodeWgs = 1024;    // workgroups that share the rows of a decode call
constexpr int kPrefillRows = 128;        // rows of q per workgroup of a prefill; of the cache, for the columns' sums
// Workgroups that splits of the cache may come to, two a CU.  (g = 4, d = 128, 8 instances but where said; up to 256, 512, 1024 of them: 512 tokens
// behind 15 thousand rows 182, 158, 169 us, 128 behind 16 thousand 57, 55, 69, 1000 behind 3000 92, 92, 96, 300 of 1000 22.4, 25.5, 30.3; 16 behind
// 8000, 64 instances, 62, 61, 71.)
constexpr int kSplitWgs = 512;
// The join has a split a lane.  (4 tokens behind 32 thousand rows, one instance, by 32 and 64 splits 29.5 and 21.7 us, 83 and 153 in fp32.)
constexpr int kMostSplits = 64;
// Workgroups of the columns' sums that fill the chip.  (Up to 2048, 4096, 8192: chunks of 1365 and 2048 tokens with a window of 2048, whole calls,
// 289, 277, 285 us; a prompt of 8000 930, 925, 917.)
constexpr int kColumnWgs = 4096;
// Rows of q of an instance, in whole tiles.
inline int cache_stat_rows(const Shape& s, int q_cap) { return (q_cap * s.g + 63) / 64 * 64; }

struct CacheWs { size_t before, whole, part_ml, part_acc, tickets, logits, total; };     // decode, in bytes
CacheWs cache_decode_ws(const Shape& s, bool weights);
struct CacheQWs { size_t stat, sums, part_ml, part_o, total; };                                   // prefill, in bytes
CacheQWs cache_prefill_ws(const Shape& s, int q_cap, bool weights);

hipError_t launch_cache_append(const Shape& s, const CacheRows& r, const void* k_new, const void* v_new, const int32_t* n_new, int q_cap,
                               void* K, void* V, hipStream_t st);
hipError_t launch_cache_decode(const Shape& s, const DecodeArgs& a, hipStream_t st);
hipError_t launch_cache_prefill(const Shape& s, const PrefillArgs& a, hipStream_t st);
hipError_t launch_cache_evict(const Shape& s, const CacheRows& r, void* K, void* V, const float* acc, int budget, int n_first, int n_last,
                              float* acc_out, int32_t* len_out, int32_t* kept, hipStream_t st);

}  // namespace ap
