// Attention of a chunk of new tokens per instance over its cache, which holds their rows already.  Query r of n lies at position
// p = L - n + r and sees the rows j <= p, with a window only those with j > p - window or j < n_first:
//
//   s_rhj = q_rh . K_j / sqrt(d),  P_rhj = exp(s_rhj - m_rh) / sum_j exp(s_rhj - m_rh),  out_rh = sum_j P_rhj V_j,
//   acc_j += sum_r sum_h P_rhj.
//
// The g heads of a group read the same K and V, so a workgroup's tile is 128 rows of q seen as [n * g][d], 32 a wave.  K and V go through
// LDS, 64 rows (fp32: 32) at a time, in two buffers that are filled from memory without registers.  Both products are made transposed,
// K q^T and V^T P^T: a lane then has scores, statistics and outputs of one query row, and the scores' registers are the second product's
// operand as they are, since the order of its contraction index is free.  V^T comes out of LDS by the transposing read.
//
// A prompt of 8190 tokens (8 instances, g = 4, d = 128) takes 556 us, 990 TFLOP/s of useful products, where a large library product
// reaches 1210.  What bounds it is the vector unit beside the matrix unit: a wave's tile has 32 exponentials and some 170 other instructions a
// lane for its 32 matrix instructions, some 1180 cycles and 1024, and a SIMD's two waves hardly cover each other - the cycles of both units
// add up to nearly all of the time -, and the clock, which falls to 1.8 GHz under it.  Tried and no faster: the next tile's scores beside
// this one's exponentials, three waves a SIMD with tiles of 32 rows, 256 rows a workgroup, a higher priority for the matrix phases.
// In fp32 (4000 tokens, 8 instances) 1125 us, 117 TFLOP/s, where a large library product reaches 154.
#include "cache_body.h"

namespace ap {
namespace {

constexpr int kThreads = 256, kWaves = 4;
// Tiles of a split.  (g = 4, d = 128: a chunk of 101 behind 416 rows, 8 instances, by splits of 1, 2, 4 tiles 15.6, 15.6, 16.9 us; 4 tokens
// behind 2000 rows 12.1, 11.8, 13.5; 300 of 1000 rows 25.5, 25.5, 23.0.)
constexpr int kLeastTiles = 2;
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

// What the queries of a tile see of an instance.
struct Span {
  int L, n, base;        // length, queries, position of query 0 (may be negative)
  int p0, p1;            // positions of the tile's first and last query
  int lo0, f;            // rows [0, f) and [lo0, p1] are seen by one of them at least, f <= lo0
  int tiles, ts, tb;     // tiles of TT rows: ts from 0 on, the others from tb
  __device__ __forceinline__ int tile(int u) const { return u < ts ? u : tb + (u - ts); }
};
template <int TT, int G>
__device__ __forceinline__ Span span_of(const CacheRows& r, const int32_t* n_q, int q_cap, int window, int n_first, int inst, int row0, int rows) {
  Span s;
  s.L = clamped(r.len[inst], 0, r.t_cap);
  s.n = n_q == nullptr ? q_cap : clamped(n_q[inst], 0, q_cap);
  s.base = s.L - s.n;
  const int last = row0 + rows < s.n * G ? row0 + rows : s.n * G;        // rows of q up to here
  s.p0 = s.base + row0 / G;
  s.p1 = s.base + (last - 1) / G;
  if (last <= row0) s.p1 = -1;
  s.lo0 = window > 0 && s.p0 >= window ? s.p0 - window + 1 : 0;
  s.f = n_first < s.lo0 ? n_first : s.lo0;
  if (s.p1 < 0) { s.tiles = s.ts = s.tb = 0; return s; }
  s.ts = (s.f + TT - 1) / TT;
  s.tb = s.lo0 / TT > s.ts ? s.lo0 / TT : s.ts;
  s.tiles = s.ts + (s.p1 / TT >= s.tb ? s.p1 / TT - s.tb + 1 : 0);
  return s;
}

// A wave fetches RW consecutive rows of a tile, which lie in one page, or in two of eight rows.  Rows that no query of the tile sees are not
// read: row `alt`, which is seen, stands in for them, and may be any row of the cache.  Wave-uniform.
struct Run {
  const char *k, *v;                                       // row 0 of the run, as if all of it lay together
  long long second;                                        // and what to add for its second eight rows, in bytes
  bool all;
  int j0, alt;
};
// The instance's part of the table, looked up through the scalar cache.
struct Pages {
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
__device__ __forceinline__ Pages pages_of(const CacheRows& r, int inst) {
  Pages p;
  p.table = r.table == nullptr ? nullptr : (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(r.table + (size_t)inst * r.nb_cap);
  p.row0 = (size_t)inst * r.t_cap;
  p.lb = r.lb; p.nb_cap = r.nb_cap; p.n_phys = r.n_phys;
  return p;
}
template <typename F> __device__ __forceinline__ Run run_of(const PrefillArgs& a, const Pages& pages, const Span& s, int t0, int wave) {
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
template <typename F, bool IS_V>
__device__ __forceinline__ void send_tile(const PrefillArgs& a, int inst, const Run& run, const Span& s, int wave, unsigned lds) {
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

// Workgroup b of tiles * n_inst: which instance and which tile.  Consecutive workgroups go to the 8 XCDs in turn, so instances are dealt
// eight at a time, one an XCD, whose L2 then serves one instance's K and V; the fewer than eight that are left share the XCDs.
struct Work { int inst, tile; };
__device__ __forceinline__ Work work_of(unsigned b, int tiles, int n_inst) {
  const unsigned whole = (unsigned)n_inst / 8 * 8, rest = (unsigned)n_inst - whole;
  if (b < whole * (unsigned)tiles) {
    const unsigned eight = b / (8u * tiles), x = b % (8u * tiles);
    return {(int)(eight * 8 + x % 8), (int)(x / 8)};
  }
  const unsigned x = b - whole * (unsigned)tiles;
  return {(int)(whole + x % rest), (int)(x / rest)};
}

template <typename T, int D, int G, bool STAT>
__global__ __launch_bounds__(kThreads) void cache_prefill_kernel(PrefillArgs a) {
  using F = Form<T, D>;
  extern __shared__ __attribute__((aligned(16))) u32x4 s_tiles[];         // [2][K, V][TILE]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hb = lane >> 5;
  const Work job = work_of(blockIdx.x, a.tiles, a.r.n_inst);
  const int inst = job.inst, row0 = (a.tiles - 1 - job.tile) * kPrefillRows;            // the longest ones first
  const Span s = span_of<F::TT, G>(a.r, a.n_q, a.q_cap, a.window, a.n_first, inst, row0, kPrefillRows);
  const int rows = s.n * G;                                // of q
  if (row0 >= rows) return;

  const int row = row0 + wave * 32 + n;                    // this lane's row of q; beyond the last it is computed and not stored
  const size_t q_row = (size_t)inst * a.q_cap * G + (row < rows ? row : rows - 1);
  u32x4 qf[F::KS];
#pragma unroll
  for (int k = 0; k < F::KS; ++k) qf[k] = static_cast<const u32x4*>(a.q)[q_row * F::PIECES + 2 * k + hb];
  const int p = s.base + (row < rows ? row : rows - 1) / G;               // its position
  const int lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;

  float16v o[F::DB];
#pragma unroll
  for (int b = 0; b < F::DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  float m = -INFINITY, sum = 0.f;                          // the sum over this lane's half of the cache rows
  const float scale = kLog2E / sqrtf((float)D);

  const unsigned buffers = lds_address(s_tiles);
  const Pages pages = pages_of(a.r, inst);
  // Tiles of the cache in splits: this workgroup's.
  const int each = (s.tiles + a.splits - 1) / a.splits > kLeastTiles ? (s.tiles + a.splits - 1) / a.splits : kLeastTiles;
  const int u_begin = a.splits == 1 ? 0 : (int)blockIdx.y * each;
  const int u_end = a.splits == 1 || s.tiles < u_begin + each ? s.tiles : u_begin + each;
  Run next;
  auto send = [&](int u) {                                 // tile u, whose rows are those of `next`
    const unsigned to = buffers + (u % 2) * 2 * F::TILE * 16;
    send_tile<F, false>(a, inst, next, s, wave, to);
    send_tile<F, true>(a, inst, next, s, wave, to + F::TILE * 16);
    next = run_of<F>(a, pages, s, s.tile(u + 1 < u_end ? u + 1 : u) * F::TT, wave);         // a tile ahead: the table's latency
  };
  if (u_begin < u_end) {
    next = run_of<F>(a, pages, s, s.tile(u_begin) * F::TT, wave);
    send(u_begin);
  }
  // (From here on the compiler counts no load of its own as under way, and waits for none in the loop.)
#pragma unroll
  for (int k = 0; k < F::KS; ++k) asm volatile("" : "+v"(qf[k]));
  for (int u = u_begin; u < u_end; ++u) {
    // This tile has landed; everybody is done with the buffer that is filled next.
    landed<0>();
    lds_read();
    __builtin_amdgcn_s_barrier();
    const int t0 = s.tile(u) * F::TT;
    const u32x4* Kt = s_tiles + (u % 2) * 2 * F::TILE;
    const u32x4* Vt = Kt + F::TILE;
    if (u + 1 < u_end) send(u + 1);
    float16v c[F::TB];
#pragma unroll
    for (int b = 0; b < F::TB; ++b) c[b] = product<T, D>(Kt, 32 * b, qf);
    // Every row of the tile is seen by every query of it, or the scores of those that are not become -inf.
    const bool all = t0 + F::TT - 1 <= s.p0 && (a.window <= 0 || t0 > s.p1 - a.window || t0 + F::TT <= a.n_first);
    if (!all) {
#pragma unroll
      for (int b = 0; b < F::TB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = t0 + 32 * b + reg_row(i, hb);
          c[b][i] = (j > p) | ((j < lo) & (j >= a.n_first)) ? -INFINITY : c[b][i];
        }
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
      // Probabilities are rounded to bf16 for the matrix unit; their sum is taken before.  That adds an error of the size of the output's own
      // rounding: relative to the definition, outputs of scores spread by 2 are off by 0.0024 (root mean square), 0.0017 if the rounding of the output
      // were all.  Two bf16 parts of each probability reach the latter, with half as many matrix instructions again and a third of the vector
      // unit's: a prompt 556 -> 742 us, a window with weights 272 -> 318, a chunk of 101 behind a prefix 15.6 -> 16.4.
#pragma unroll
      for (int k = 0; k < F::TT / 16; ++k) {
        bf16x8 pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[e] = (__bf16)c[k / 2][8 * (k % 2) + e];
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
            const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at);
            const bf16x4 y = __builtin_bit_cast(bf16x4, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) va[4 * half + e] = y[e];
          }
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb, o[b], 0, 0, 0);
        }
      }
    } else {
      const float* Vf = reinterpret_cast<const float*>(Vt);
#pragma unroll
      for (int b = 0; b < F::DB; ++b) {
        float16v x;                                        // of this tile alone, as the sums
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          x = __builtin_amdgcn_mfma_f32_32x32x2f32(Vf[reg_row(i, hb) * D + 32 * b + n], c[0][i], x, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] += x[i];
      }
    }
  }

  sum = sum32(sum);
  if (row >= rows) return;
  if (a.splits > 1) {                                      // (whatever its share: the join goes by the maximum)
    const size_t at = ((size_t)blockIdx.y * a.r.n_inst + inst) * a.q_cap * G + row;
    if (hb == 0) {
      a.part_ml[at * 2] = m;
      a.part_ml[at * 2 + 1] = sum;
    }
    if (u_begin < u_end) {
#pragma unroll
      for (int b = 0; b < F::DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          float4v y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = o[b][i + e];
          *reinterpret_cast<float4v*>(a.part_o + at * D + 32 * b + reg_row(i, hb)) = y;
        }
    }
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;           // a query that sees nothing has a zero output
  if (STAT && hb == 0) {
    float* st = a.stat + ((size_t)inst * a.stat_rows + row) * 2;
    st[0] = m == -INFINITY ? 0.f : m;
    st[1] = inv;
  }
  T* out = static_cast<T*>(a.out) + ((size_t)inst * a.q_cap * G + row) * D;
#pragma unroll
  for (int b = 0; b < F::DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * b + reg_row(i, hb);
      if constexpr (sizeof(T) == 2) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[b][i + e] * inv);
        *reinterpret_cast<bf16x4*>(out + d) = y;
      } else {
        float4v y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = o[b][i + e] * inv;
        *reinterpret_cast<float4v*>(out + d) = y;
      }
    }
}

// Joins the splits of the cache: a wave per row of q.
template <typename T, int D, int G>
__global__ __launch_bounds__(kThreads) void cache_prefill_join_kernel(PrefillArgs a) {
  constexpr int E = D / 64;                                // outputs of a lane
  const int inst = blockIdx.y, lane = threadIdx.x & 63, row = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int nq = a.n_q == nullptr ? a.q_cap : clamped(a.n_q[inst], 0, a.q_cap);
  if (row >= nq * G) return;
  const size_t at = (size_t)inst * a.q_cap * G + row, step = (size_t)a.r.n_inst * a.q_cap * G;
  // A lane has the statistics of a split (there are at most 64).
  const float m = lane < a.splits ? a.part_ml[(lane * step + at) * 2] : -INFINITY, l = lane < a.splits ? a.part_ml[(lane * step + at) * 2 + 1] : 0.f;
  const float top = wave_max(m), use = top == -INFINITY ? 0.f : top;
  const float f = exp2_fast(m - use), sum = wave_sum(f * l), inv = sum == 0.f ? 0.f : 1.f / sum;
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  constexpr int kAhead = 8;                                // loads under way
  for (int x0 = 0; x0 < a.splits; x0 += kAhead) {
    float v[kAhead][E];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int y = x0 + x < a.splits ? x0 + x : a.splits - 1;
#pragma unroll
      for (int e = 0; e < E; ++e) v[x][e] = a.part_o[(y * step + at) * D + lane * E + e];
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const float w = x0 + x < a.splits ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), x0 + x)) : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += w > 0.f ? w * v[x][e] : 0.f;                // (a split without tiles has left no sums)
    }
  }
  T* out = static_cast<T*>(a.out) + at * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (sizeof(T) == 2) out[e].bits = __builtin_bit_cast(uint16_t, (__bf16)(o[e] * inv));
    else out[e] = o[e] * inv;
  }
  if (a.acc != nullptr && lane == 0) {
    float* st = a.stat + ((size_t)inst * a.stat_rows + row) * 2;
    st[0] = use;
    st[1] = inv;
  }
}

// Tiles of kPrefillRows cache rows that an instance's queries see: rows [0, f) and [lo, L), f <= lo.
struct Columns {
  int L, nq, base, lo, f, tiles, ts, tb;
  __device__ __forceinline__ int tile(int u) const { return u < ts ? u : tb + (u - ts); }
};
__device__ __forceinline__ Columns columns_of(const PrefillArgs& a, int inst) {
  Columns c;
  c.L = clamped(a.r.len[inst], 0, a.r.t_cap);
  c.nq = a.n_q == nullptr ? a.q_cap : clamped(a.n_q[inst], 0, a.q_cap);
  c.base = c.L - c.nq;
  c.lo = a.window > 0 && c.base >= a.window ? c.base - a.window + 1 : 0;
  c.f = a.n_first < c.lo ? a.n_first : c.lo;
  c.ts = (c.f + kPrefillRows - 1) / kPrefillRows;
  c.tb = c.lo / kPrefillRows > c.ts ? c.lo / kPrefillRows : c.ts;
  c.tiles = c.L == 0 || c.nq == 0 ? 0 : c.ts + ((c.L - 1) / kPrefillRows >= c.tb ? (c.L - 1) / kPrefillRows - c.tb + 1 : 0);
  return c;
}

// Sums of the columns of P over a chunk of the query rows.  A workgroup has 128 cache rows, 32 a wave, held as operands; the queries go
// through LDS, 64 rows (fp32: 32) at a time.  A lane has scores of one query row, whose statistics are two registers, and of 16 cache
// rows, whose sums stay in registers to the end.
template <typename T, int D, int G>
__global__ __launch_bounds__(kThreads) void cache_weights_kernel(PrefillArgs a) {
  using F = Form<T, D>;
  constexpr int QT = F::TT, RING = 3, BUFFER = F::TILE + QT / 2;          // of a buffer, in pieces: the queries and their statistics
  __shared__ __attribute__((aligned(16))) u32x4 s_q[RING * BUFFER];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hb = lane >> 5;
  const int inst = blockIdx.y, chunk = blockIdx.z;
  const Columns col = columns_of(a, inst);
  if ((int)blockIdx.x >= col.tiles) return;
  const int t0 = col.tile(blockIdx.x) * kPrefillRows, L = col.L, base = col.base, rows = col.nq * G;
  // Rows of q in this chunk, whole tiles of them, that see one of the cache rows at least.
  const int all_tiles = (rows + QT - 1) / QT, each = (all_tiles + a.chunks - 1) / a.chunks;
  int begin = chunk * each * QT, end = begin + each * QT < rows ? begin + each * QT : rows;
  const int first_q = t0 - base > 0 ? t0 - base : 0;                          // the first query that lies at t0 or behind it
  if (begin < first_q * G) begin = first_q * G / QT * QT;
  if (a.window > 0 && t0 >= a.n_first) {                                      // and the last that still sees t0 + 127
    const long long last_q = (long long)t0 + kPrefillRows - 1 + a.window - 1 - base;
    if ((last_q + 1) * G < end) end = (int)((last_q + 1) * G);
  }
  const int j0 = t0 + 32 * wave;                           // this wave's cache rows
  const bool none = j0 >= L || (j0 >= col.f && j0 + 32 <= col.lo);          // that no query sees
  const float scale = kLog2E / sqrtf((float)D);
  float total[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) total[i] = 0.f;
  const u32x4* q = static_cast<const u32x4*>(a.q) + (size_t)inst * a.q_cap * G * F::PIECES;
  const float* stat = a.stat + (size_t)inst * a.stat_rows * 2;
  const unsigned lds = lds_address(s_q);
  const int tiles = begin < end ? (end - begin + QT - 1) / QT : 0;
  auto send = [&](int u) {
    const int r0 = begin + u * QT;
    const unsigned to = lds + (u % RING) * BUFFER * 16;
    // (behind the last row of q there is room for the statistics of a whole tile; what lies there is not used)
    if (wave == 0 && lane < QT / 2) to_lds_from(stat + (r0 + 2 * lane) * 2, to + F::TILE * 16);
#pragma unroll
    for (int l = 0; l < F::LOADS; ++l) {
      const int r = wave * F::RW + l * F::RPL + lane / F::PIECES, p = F::k_place(r, lane % F::PIECES);
      const int row = r0 + r < rows ? r0 + r : rows - 1;
      to_lds_from(q + (size_t)row * F::PIECES + p, to + (wave * F::LOADS + l) * 1024);
    }
  };
  if (tiles > 0) send(0);
  if (tiles > 1) send(1);
  u32x4 kf[F::KS];
  {
    const int j = j0 + n < L ? j0 + n : L - 1;
    const u32x4* k = static_cast<const u32x4*>(a.K) + row_at(a.r, inst, j) * F::PIECES + hb;
#pragma unroll
    for (int x = 0; x < F::KS; ++x) kf[x] = k[2 * x];
  }
#pragma unroll
  for (int x = 0; x < F::KS; ++x) asm volatile("" : "+v"(kf[x]));           // (they are there: the loop waits for none of them)
  for (int u = 0; u < tiles; ++u) {
    const int r0 = begin + u * QT;
    if (u + 1 < tiles) landed<F::LOADS>(); else landed<0>();                // this tile's; the next one's are under way
    lds_read();
    __builtin_amdgcn_s_barrier();                                           // ... of all waves; and everybody is done with the tile before
    if (u + 2 < tiles) send(u + 2);
    if (none) continue;
    const u32x4* Q = s_q + (u % RING) * BUFFER;
    const int r_last = r0 + QT < rows ? r0 + QT - 1 : rows - 1;
    const bool all = r0 + QT <= rows && j0 + 31 <= base + r0 / G &&
                     (a.window <= 0 || j0 > base + r_last / G - a.window || j0 + 32 <= a.n_first);
#pragma unroll
    for (int b = 0; b < F::TB; ++b) {
      float16v c;
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
      for (int k = 0; k < F::KS; ++k) {
        const u32x4 x = Q[(32 * b + n) * F::PIECES + F::k_place(32 * b + n, 2 * k + hb)];
        if constexpr (sizeof(T) == 2) {
          c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[k]), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[k][e]), __uint_as_float(x[e]), c, 0, 0, 0);
        }
      }
      struct Stat { float m, inv; };
      Stat st = reinterpret_cast<const Stat*>(Q + F::TILE)[32 * b + n];
      if (__any(is_far(st.m))) {
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = is_far(st.m) ? brought_near(c[i], scale, st.m) : c[i];
        st.m = is_far(st.m) ? 0.f : st.m;
      }
      if (all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) total[i] = __builtin_fmaf(exp2_fast(__builtin_fmaf(c[i], scale, -st.m)), st.inv, total[i]);
      } else {
        const int row = r0 + 32 * b + n, p = base + row / G, lo_q = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
        if (row >= rows) st.m = st.inv = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = j0 + reg_row(i, hb);
          const bool seen = (j <= p) & ((j >= lo_q) | (j < a.n_first)) & (st.inv > 0.f);
          const float w = exp2_fast(__builtin_fmaf(c[i], scale, -st.m)) * st.inv;
          total[i] += seen ? w : 0.f;
        }
      }
    }
  }
  // The lanes of a half have the same cache rows.
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    total[i] = lane_group_sum<16>(total[i]);
    total[i] = sum16(total[i]);
  }
  if (n == 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = j0 + reg_row(i, hb);
      if (j >= L) continue;
      if (a.chunks == 1) a.acc[(size_t)inst * a.r.t_cap + j] += total[i];
      else a.sums[(((size_t)chunk * a.r.n_inst + inst) * gridDim.x + blockIdx.x) * kPrefillRows + j - t0] = total[i];
    }
  }
}

// The chunks' sums, one after the other, so that the result does not depend on which was ready first.
__global__ __launch_bounds__(kPrefillRows) void cache_weights_add_kernel(PrefillArgs a) {
  const int inst = blockIdx.y;
  const Columns col = columns_of(a, inst);
  if ((int)blockIdx.x >= col.tiles) return;
  const int j = col.tile(blockIdx.x) * kPrefillRows + threadIdx.x;
  if (j >= col.L) return;
  float x = 0.f;
#pragma unroll 8
  for (int c = 0; c < a.chunks; ++c)
    x += a.sums[(((size_t)c * a.r.n_inst + inst) * gridDim.x + blockIdx.x) * kPrefillRows + threadIdx.x];
  a.acc[(size_t)inst * a.r.t_cap + j] += x;
}

// Most tiles of cache rows that an instance's queries can see.
static long long most_columns(const Shape& s, int q_cap, int window, int n_first) {
  const long long all = ((long long)s.t_cap + kPrefillRows - 1) / kPrefillRows;
  if (window <= 0) return all;
  const long long some = ((long long)n_first + kPrefillRows - 1) / kPrefillRows + ((long long)window + q_cap) / kPrefillRows + 2;
  return some < all ? some : all;
}
// Splits of the cache where the rows of q alone leave CUs without work: up to 512 workgroups, of at least kLeastTiles tiles.
static int cache_splits(const Shape& s, int q_cap, int window, int n_first) {
  const long long wgs = (((long long)q_cap * s.g + kPrefillRows - 1) / kPrefillRows) * s.n_inst;
  const long long rows = window > 0 && (long long)window + q_cap + n_first < s.t_cap ? (long long)window + q_cap + n_first : s.t_cap;
  const int tt = s.kv_dtype == AP_BF16 ? 64 : 32;
  long long splits = kSplitWgs / wgs, most = (rows + tt * kLeastTiles - 1) / (tt * kLeastTiles);
  if (splits > most) splits = most;
  if (splits > kMostSplits) splits = kMostSplits;
  return splits < 1 ? 1 : (int)splits;
}
// Workgroups of the columns' sums: chunks of the query rows, of at least 512 rows, where the tiles alone are few for the chip.  (Whole calls
// with weights, g = 4, d = 128.  Chunks of at least 256, 512, 1024 rows: 101 tokens behind 416 rows, 8 instances, 29.0, 31.9, 31.9 us, 1000
// behind 7000 255, 253, 252.  At most 8, 16, 32 chunks: a prompt of 4000 in one instance 92, 79, 83.)
static int column_chunks(const Shape& s, int q_cap, long long columns) {
  const long long q_rows = (long long)q_cap * s.g;
  long long chunks = (kColumnWgs + s.n_inst * columns - 1) / (s.n_inst * columns);
  if (chunks > (q_rows + 511) / 512) chunks = (q_rows + 511) / 512;
  if (chunks > 16) chunks = 16;
  return (int)chunks;
}

template <typename T, int D, int G> hipError_t run(const Shape& s, const PrefillArgs& a, hipStream_t st) {
  // (More buffers where a CU has one workgroup at most are no faster: with four, a chunk of 100 behind 400 rows, 8 instances, g = 4, d = 128,
  // 15.2 us and 15.3; 4 tokens behind 32 thousand rows, one instance 21.7 and 21.3, four 24.3 and 23.0.)
  const dim3 grid((unsigned)a.tiles * (unsigned)a.r.n_inst, a.splits);
  const size_t lds = (size_t)2 * 2 * Form<T, D>::TILE * 16;
  if (a.acc == nullptr) cache_prefill_kernel<T, D, G, false><<<grid, kThreads, lds, st>>>(a);
  else cache_prefill_kernel<T, D, G, true><<<grid, kThreads, lds, st>>>(a);
  if (a.splits > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    cache_prefill_join_kernel<T, D, G><<<dim3((a.q_cap * G + kWaves - 1) / kWaves, a.r.n_inst), kThreads, 0, st>>>(a);
  }
  if (a.acc == nullptr) return hipGetLastError();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 columns((unsigned)most_columns(s, a.q_cap, a.window, a.n_first), a.r.n_inst, a.chunks);
  cache_weights_kernel<T, D, G><<<columns, kThreads, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.chunks == 1) return e;
  cache_weights_add_kernel<<<dim3(columns.x, columns.y), kPrefillRows, 0, st>>>(a);
  return hipGetLastError();
}
template <typename T, int D> hipError_t run_g(const Shape& s, const PrefillArgs& a, hipStream_t st) {
  return s.g == 1 ? run<T, D, 1>(s, a, st) : s.g == 2 ? run<T, D, 2>(s, a, st) : s.g == 4 ? run<T, D, 4>(s, a, st) : run<T, D, 8>(s, a, st);
}

}  // namespace

hipError_t launch_cache_prefill(const Shape& s, const PrefillArgs& args, hipStream_t st) {
  PrefillArgs a = args;
  a.stat_rows = cache_stat_rows(s, a.q_cap);
  a.tiles = (int)(((long long)a.q_cap * s.g + kPrefillRows - 1) / kPrefillRows);
  a.splits = cache_splits(s, a.q_cap, a.window, a.n_first);
  a.chunks = a.acc == nullptr ? 1 : column_chunks(s, a.q_cap, most_columns(s, a.q_cap, a.window, a.n_first));
  if (s.kv_dtype == AP_BF16) return s.d == 128 ? run_g<bf16_t, 128>(s, a, st) : run_g<bf16_t, 64>(s, a, st);
  return s.d == 128 ? run_g<float, 128>(s, a, st) : run_g<float, 64>(s, a, st);
}

}  // namespace ap
