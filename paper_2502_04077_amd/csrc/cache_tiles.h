// Tiles of a cache in LDS, and products with them, that the kernels with many rows of q share: 256 threads, a wave has 32 rows of q.
#pragma once

#include "cache_body.h"

namespace ap {
namespace {

constexpr int kThreads = 256, kWaves = 4;
typedef float float16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));


template <typename T, int D> struct Form {
  static constexpr int E = 16 / (int)sizeof(T);            // elements of a 16-byte piece
  static constexpr int PIECES = D / E;                     // pieces of a row
  static constexpr int TT = sizeof(T) == 2 ? 64 : 32;      // cache rows of a tile
  static constexpr int TB = TT / 32;                       // blocks of 32 of them
  static constexpr int KS = PIECES / 2;                    // pieces a lane contributes to a product over d
  static constexpr int DB = D / 32;                        // blocks of 32 output dims
  static constexpr int LOADS = TT * PIECES / kThreads;     // pieces a thread fetches of a tile of K, or V
  static constexpr int TILE = TT * PIECES;                 // pieces of a tile
  static constexpr int RPL = 64 / PIECES;                  // rows that a wave fetches with a load
  static constexpr int RW = TT / kWaves;                   // rows of a tile that a wave fetches
  static_assert(RPL * LOADS == RW, "a wave's rows");
  // Piece p of row r lies at place p ^ swizzle(r) of the row, so that the lanes of one LDS cycle use different banks: K is read a row
  // per lane, V (16 bits) in blocks of four rows by four pieces, half a wave at a time.
  __device__ static __forceinline__ int k_place(int r, int p) { return p ^ (r & (PIECES - 1)); }
  __device__ static __forceinline__ int v_place(int r, int p) {
    return sizeof(T) == 2 ? p ^ (PIECES == 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1)) : p;
  }
};

// SPAN: the rows [0, f) and [lo0, p1] of the cache are seen, f <= lo0.  ARGS: K, V and the caches' rows r.
// A wave fetches RW consecutive rows of a tile, which lie in one page, or in two of eight rows.  Rows that no query of the tile sees are not
// read: row `alt`, which is seen, stands in for them, and may be any row of the cache.  Wave-uniform.
struct Run {
  const char *k, *v;                                       // row 0 of the run, as if all of it lay together
  long long second;                                        // and what to add for its second eight rows, in bytes
  bool all;
  int j0, alt;
};
// The instance's part of the table, looked up through the scalar cache.
struct TablePages {
  const __attribute__((address_space(4))) int32_t* table;  // of this instance, or null
  size_t row0;                                             // contiguous: the instance's first row
  int lb, nb_cap, n_phys;
  __device__ __forceinline__ size_t at(int j) const {      // of row j, a multiple of 8
    if (table == nullptr) return row0 + j;
    const int block = j >> lb;
    const int page = clamped(table[block < nb_cap ? block : nb_cap - 1], 0, n_phys - 1);
    return ((size_t)page << lb) + (j & ((1 << lb) - 1));
  }
};
__device__ __forceinline__ TablePages pages_of(const CacheRows& r, int inst) {
  TablePages p;
  p.table = r.table == nullptr ? nullptr : (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(r.table + (size_t)inst * r.nb_cap);
  p.row0 = (size_t)inst * r.t_cap;
  p.lb = r.lb; p.nb_cap = r.nb_cap; p.n_phys = r.n_phys;
  return p;
}
template <typename F, typename ARGS, typename SPAN>
__device__ __forceinline__ Run run_of(const ARGS& a, const TablePages& pages, const SPAN& s, int t0, int wave) {
  constexpr size_t bytes = F::PIECES * 16;
  Run x;
  x.j0 = t0 + wave * F::RW;
  x.all = x.j0 + F::RW - 1 <= s.p1 && (x.j0 >= s.lo0 || x.j0 + F::RW <= s.f);
  int alt = x.j0;                                          // a row of the run that is seen, or one of another run
  if (x.j0 >= s.f) alt = x.j0 > s.lo0 ? x.j0 : s.lo0;
  if (alt > s.p1) alt = s.p1;
  x.alt = alt;
  const size_t at = pages.at(x.j0);
  x.k = static_cast<const char*>(a.K) + at * bytes;
  x.v = static_cast<const char*>(a.V) + at * bytes;
  x.second = F::RW == 16 && pages.lb == 3 && pages.table != nullptr ? ((long long)(pages.at(x.j0 + 8) - at) - 8) * (long long)bytes : 0;
  return x;
}
// Sends a tile of K (or V) to LDS: the lane chooses the piece, so that it lies where the swizzle says.
template <typename F, bool IS_V, typename ARGS, typename SPAN>
__device__ __forceinline__ void send_tile(const ARGS& a, int inst, const Run& run, const SPAN& s, int wave, unsigned lds) {
  constexpr unsigned bytes = F::PIECES * 16;
  const int lane = threadIdx.x & 63;
  const unsigned to = lds + wave * F::LOADS * 1024;
  auto row = [&](int l) { return l * F::RPL + lane / F::PIECES; };                   // of the run, which begins at a multiple of RW rows
  auto piece = [&](int l) {
    const int place = lane % F::PIECES;
    return IS_V ? F::v_place(row(l), place) : F::k_place(wave * F::RW + row(l), place);
  };
  if (run.all) {
#pragma unroll
    for (int l = 0; l < F::LOADS; ++l)
      to_lds<false>((IS_V ? run.v : run.k) + (l >= F::LOADS / 2 ? run.second : 0), row(l) * bytes + piece(l) * 16, to + l * 1024);
  } else {
#pragma unroll 1
    for (int l = 0; l < F::LOADS; ++l) {
      int j = run.j0 + row(l);
      if (j > s.p1 || (j >= s.f && j < s.lo0)) j = run.alt;
      to_lds_from(static_cast<const char*>(IS_V ? a.V : a.K) + row_at(a.r, inst, j) * bytes + piece(l) * 16, to + l * 1024);
    }
  }
}

// (32 rows of X in LDS) . (32 rows held as operands)^T, fp32: one block of scores.
template <typename T, int D>
__device__ __forceinline__ float16v product(const u32x4* X, int row0, const u32x4 (&b)[Form<T, D>::KS]) {
  using F = Form<T, D>;
  const int lane = threadIdx.x & 63, m = lane & 31, hb = lane >> 5;
  float16v c;
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
  for (int k = 0; k < F::KS; ++k) {
    const u32x4 x = X[(row0 + m) * F::PIECES + F::k_place(row0 + m, 2 * k + hb)];
    if constexpr (sizeof(T) == 2) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, b[k]), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(b[k][e]), c, 0, 0, 0);
    }
  }
  return c;
}

// Which of 16 registers' rows: register i of a block holds row 8 (i / 4) + 4 hb + i % 4.
__device__ __forceinline__ int reg_row(int i, int hb) { return 8 * (i >> 2) + 4 * hb + (i & 3); }

}  // namespace
}  // namespace ap
