// Sequences that share pages and a beginning: what the calls on them (share_api.hip) hand to the kernels.
#pragma once

#include "cache_internal.h"

namespace ap {

// A pool and the table that names its pages.
struct Pages {
  int32_t* table;          // [n_inst][nb_cap]; entries outside the pool name no page
  int32_t* refs;           // [n_pages] how often the table names each page; 0: free
  int32_t* seg;            // [segments] free pages among each kSegment pages
  void *K, *V;
  int n_inst, t_cap, nb_cap, n_pages, lb, segments, row_pieces;      // lb = log2(b); 16-byte pieces of a row
};
constexpr int kSegment = 1024;
inline int page_segments(int n_pages) { return (int)(((long long)n_pages + kSegment - 1) / kSegment); }

// Workspace of the calls on pages, in bytes.  What a call needs is decided first (need, staged, kept, length), then free pages are picked
// (before, picked, taken), then all is carried out.
struct PagesWs {
  size_t head;             // 4 words: pages given out (0 where some lack), pages lacking; pages in use, pages to move
  size_t need;             // int32 [n_inst] pages needed
  size_t before;           // int32 [n_inst] pages needed by the instances before
  size_t length;           // int32 [n_inst] rows from now on (fork), -1: stays as it is
  size_t staged;           // int32 [n_inst][nb_cap] resize: the blocks that need a page; fork: the new table
  size_t picked;           // int32 [n_pages] free pages, the lowest first; compact: those in front of the pages in use
  size_t taken;            // int32 [segments] pages taken of each segment
  size_t from, rank;       // int32 [n_pages] compact: pages to move, and each one's place among them
  size_t total;
};
PagesWs pages_ws(const Shape& s, int n_pages);

struct ResizeArgs { Pages p; const int32_t *len, *n_new; int q_cap; int32_t* info; char* ws; PagesWs w; };
struct ForkArgs { Pages p; const int32_t *parent, *len; int32_t *len_out, *info; char* ws; PagesWs w; };
struct CompactArgs { Pages p; int32_t* info; char* ws; PagesWs w; };

hipError_t launch_pages_count(const Pages& p, hipStream_t st);
hipError_t launch_pages_resize(const ResizeArgs& a, hipStream_t st);
hipError_t launch_pages_fork(const ForkArgs& a, hipStream_t st);
hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t st);
// page_pieces: 16-byte pieces of a page of K, or V.  from, to: null: 0, 1, 2, ...
hipError_t launch_pages_copy(const void* K_src, const void* V_src, int n_src, const int32_t* from, void* K_dst, void* V_dst, int n_dst,
                             const int32_t* to, int n, int page_pieces, hipStream_t st);

// Groups of instances whose first rows are the same.  plan: what ap_cache_share makes of `group` and `shared`.
struct SharePlan {
  int4* inst;              // [n_inst] first member (the lowest); place of its group's first row in `member`; members, 1: alone; rows in common
  int4* groups;            // [n_inst] the same line of every group of several members, in the order of the first ones
  int32_t* pos;            // [n_inst] own place in `member`, -1: alone
  int32_t* member;         // [n_inst] the groups' members, groups by their first member, members ascending
  int32_t* count;          // [4] groups
};
size_t share_plan_bytes(const Shape& s);
SharePlan share_plan(const Shape& s, void* plan);

// Workgroups of the attention, two a CU.
constexpr int kShareWgs = 512;
constexpr int kNarrowRows = 32;     // rows of q of a tile up to which a wave has them alone

// Rows of q, `rows` an instance, are numbered twice: those of the instances, x < n_inst * rows, for what lies behind the beginnings; and n_inst * rows +
// those of the groups' members one after the other for the groups' beginnings.  The piece that workgroup w leaves of row x is number x + kPrefillRows * w; that
// wave w leaves of a tile of few rows, narrow0 + x + kNarrowRows * w.
struct SharedArgs {
  CacheRows r;
  const void *q, *K, *V;
  const int32_t* n_q;              // [n_inst], or null: q_cap each
  int q_cap, lg, rows, window, n_first, narrow0;      // lg = log2(g)
  void* out;
  SharePlan plan;
  int32_t *begun, *behind;         // workspace: [n_inst] whether there are pieces of the beginning that an instance is the first member of; of the rows behind
  int2* row;                       // workspace: [2 * n_inst * rows] of a row of q: the first of its pieces, and how many (a wave's: negative)
  int sized;                       // whether the sizes of the sources are in the workspace:
  int32_t* low;                    // [n_inst] with a window: by a group's first member, the lowest position of its queries
  unsigned long long* sizes;       // [whole blocks of sources][2] sizes of those in front in the block: of tiles with many rows of q, and with few
  unsigned long long* totals;      // [blocks][2]
  float *ml, *o;                   // workspace: [shared_pieces][2] maximum and sum, and [..][d]
};
// Pieces: those of workgroups, in front of narrow0, and of waves.
inline size_t shared_narrow0(const Shape& s, int q_cap) { return (size_t)2 * s.n_inst * q_cap * s.g + (size_t)kPrefillRows * kShareWgs; }
inline size_t shared_pieces(const Shape& s, int q_cap) {
  return shared_narrow0(s, q_cap) + (size_t)2 * s.n_inst * q_cap * s.g + (size_t)kNarrowRows * 4 * kShareWgs;
}
// Of so many sources at most, in whole blocks of 256.
inline size_t shared_sources(const Shape& s) { return ((size_t)s.n_inst + s.n_inst / 2 + 255) / 256 * 256; }
struct SharedWs { size_t begun, behind, row, low, sizes, totals, ml, o, total; };
SharedWs shared_ws(const Shape& s, int q_cap);

hipError_t launch_cache_share(const Shape& s, const int32_t* group, const int32_t* shared, const SharePlan& plan, hipStream_t st);
// decode: the output is fp32, and probabilities keep 24 bits; else it is of the kv dtype.
hipError_t launch_cache_shared(const Shape& s, const SharedArgs& a, bool decode, hipStream_t st);

}  // namespace ap
