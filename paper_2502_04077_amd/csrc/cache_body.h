// Device code that the kernels on caches with lengths of their own share.
#pragma once

#include "attention_body.h"
#include "cache_internal.h"

namespace ap {
namespace {

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Where row j of instance i lies, in rows of K and V.  Table entries outside the pool are clamped into it, as in the other calls.
__device__ __forceinline__ size_t row_at(const CacheRows& r, int i, int j) {
  if (r.table == nullptr) return (size_t)i * r.t_cap + j;
  const int page = clamped(r.table[(size_t)i * r.nb_cap + (j >> r.lb)], 0, r.n_phys - 1);
  return ((size_t)page << r.lb) + (j & ((1 << r.lb) - 1));
}
// The same for a row that is written: false where the table names no page of the pool.
__device__ __forceinline__ bool row_to_write(const CacheRows& r, int i, int j, size_t* at) {
  if (r.table == nullptr) { *at = (size_t)i * r.t_cap + j; return true; }
  const int page = r.table[(size_t)i * r.nb_cap + (j >> r.lb)];
  *at = ((size_t)page << r.lb) + (j & ((1 << r.lb) - 1));
  return page >= 0 && page < r.n_phys;
}

// The same for 8 consecutive rows from j on (a multiple of 8: they lie in one page), asked by a whole wave: the table is read through the
// scalar cache, so that the vector loads in flight are not waited for.
__device__ __forceinline__ size_t rows_at(const CacheRows& r, int i, int j) {
  if (r.table == nullptr) return (size_t)i * r.t_cap + j;
  typedef const __attribute__((address_space(4))) int32_t* cptr;
  const int block = j >> r.lb;
  const int page = clamped(((cptr)(uintptr_t)r.table)[(size_t)i * r.nb_cap + (block < r.nb_cap ? block : r.nb_cap - 1)], 0, r.n_phys - 1);
  return ((size_t)page << r.lb) + (j & ((1 << r.lb) - 1));
}

// A lane's value and that of the lane 32 (16) further on or back, in an order that both see alike; without a trip through LDS.
struct Two { float a, b; };
__device__ __forceinline__ Two across32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Two across16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float sum32(float x) { const Two t = across32(x); return t.a + t.b; }
__device__ __forceinline__ float sum16(float x) { const Two t = across16(x); return t.a + t.b; }
__device__ __forceinline__ float max32(float x) { const Two t = across32(x); return fmaxf(t.a, t.b); }
__device__ __forceinline__ float max16(float x) { const Two t = across16(x); return fmaxf(t.a, t.b); }

// Memory to LDS without registers, 16 bytes a lane: to lds + 16 * lane from base + off (base and lds the same for the whole wave), or from an
// address of the lane's own.  Written as asm because the compiler, which cannot tell the buffers apart, would wait for all of
// these loads before every read of LDS; whoever reads waits with landed<N>() until at most N later ones are under way.
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p);
}
template <bool ONCE> __device__ __forceinline__ void to_lds(const void* base, unsigned off, unsigned lds) {      // ONCE: nobody reads it again
  lds = __builtin_amdgcn_readfirstlane(lds);
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void to_lds_from(const void* p, unsigned lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
// The same past the XCD's L2: what workgroups of this launch wrote with st_shared_out.
__device__ __forceinline__ void shared_to_lds(const void* p, unsigned lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off sc1" ::"s"(lds), "v"(p) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// Reads of LDS are over: what they read may be overwritten.
__device__ __forceinline__ void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Exponents, in units of log2, are c * scale - m with one rounding, for m the largest product's whole number above.  From 2^24 on the
// product's own rounding, which m has, is some whole numbers itself (from 2^31 on more than an exponent of 32 bits): there, it is rounded as m
// was before m is subtracted, and the largest score has the exponent 0.  (-inf, of a head that has seen nothing, counts as far.)
__device__ __forceinline__ bool is_far(float m) { return !(fabsf(m) < 16777216.f); }
__device__ __forceinline__ float exp2_of(float c, float scale, float m) {           // exp2(c * scale - m) for any m but -inf
#pragma clang fp contract(off)
  const float x = c * scale;
  return exp2_fast(is_far(m) ? x - m : __builtin_fmaf(c, scale, -m));
}
__device__ __forceinline__ float brought_near(float c, float scale, float m) {      // the score whose exponent relative to 0 is c's relative to m
#pragma clang fp contract(off)
  const float x = c * scale;
  return (x - m) / scale;
}

// Bytes of a 16-byte piece are moved whatever their type.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

}  // namespace
}  // namespace ap
