// Attention of groups of instances that begin with the same rows, over that beginning: it is read once for all of them.
//
// The members' queries are the rows of one product.  With S rows in common, for every row x of q of the group, at position p of its cache,
//
//   s_xj = q_x . K_j / sqrt(d),  m_x = max_j s_xj,  l_x = sum_j exp(s_xj - m_x),  o_x = sum_j exp(s_xj - m_x) V_j,   j < S that p sees;
//
// what lies behind the beginning is every instance's own (cache_decode.hip, cache_prefill.hip), and (m, l, o) of both are joined there.
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

// ---------------------------------------------------------------------------------------------------------------- the beginnings
// What a group's queries see of its beginning.
struct Begin {
  int lead, first, count, S;
  int p1, lo0, f;        // rows [0, f) and [lo0, p1], f <= lo0, each of which may be empty
  int tiles, ts, tb;     // tiles of TT rows: ts from 0 on, the others from tb
  __device__ __forceinline__ int tile(int u) const { return u < ts ? u : tb + (u - ts); }
};
// inst: any member's line of the plan.  Called by a thread.
template <int TT> __device__ __forceinline__ Begin begin_of(const BeginArgs& a, int4 inst) {
  Begin s;
  s.lead = inst.x; s.first = inst.y; s.count = inst.z;
  const bool several = inst.z > 1 && (unsigned)inst.x < (unsigned)a.r.n_inst && inst.y >= 0 && inst.z <= a.r.n_inst - inst.y;
  const int L = several ? clamped(a.r.len[s.lead], 0, a.r.t_cap) : 0;
  s.S = inst.w < L ? inst.w : L;
  s.lo0 = 0;
  s.p1 = s.S - 1;
  if (s.S > 0 && a.window > 0) {
    int p = 0x7fffffff;                                    // the lowest position of a query
    for (int x = 0; x < s.count; ++x) {
      const int i = a.b.plan.member[s.first + x];
      const int n = a.n_q == nullptr ? a.q_cap : clamped(a.n_q[i], 0, a.q_cap);
      const int base = clamped(a.r.len[i], 0, a.r.t_cap) - n;
      if (n > 0 && base < p) p = base;
    }
    s.lo0 = p >= a.window ? p - a.window + 1 : 0;
  }
  s.f = a.n_first < s.lo0 ? a.n_first : s.lo0;
  if (s.f > s.S) s.f = s.S;
  if (s.lo0 >= s.S) {                                      // the first rows alone
    s.lo0 = s.f;
    s.p1 = s.f - 1;
  }
  s.ts = (s.f + TT - 1) / TT;
  s.tb = s.lo0 / TT > s.ts ? s.lo0 / TT : s.ts;
  s.tiles = s.p1 < 0 ? 0 : s.ts + (s.p1 / TT >= s.tb ? s.p1 / TT - s.tb + 1 : 0);
  return s;
}
__device__ __forceinline__ unsigned long long units_of(const BeginArgs& a, const Begin& s) {
  return (unsigned long long)s.tiles * (unsigned)((s.count * a.b.rows + kPrefillRows - 1) / kPrefillRows);
}
constexpr int kLeastUnits = 2;      // of a workgroup

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

// A workgroup's share of the units, piece by piece: a tile of rows of q, 32 a wave, over consecutive tiles of the beginning.
template <typename T, int D, bool EXACT>
__global__ __launch_bounds__(kThreads) void cache_beginnings_kernel(BeginArgs a, int g) {
  using F = Form<T, D>;
  extern __shared__ __attribute__((aligned(16))) u32x4 s_tiles[];         // [2][K, V][TILE]
  __shared__ unsigned long long s_wave[kWaves], s_from;
  __shared__ int s_first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hb = lane >> 5;

  // Where this workgroup's share begins: every thread sums the units of consecutive groups.
  const int groups = clamped(*a.b.plan.count, 0, a.r.n_inst), chunk = (groups + kThreads - 1) / kThreads;
  const int i_begin = tid * chunk < groups ? tid * chunk : groups, i_end = i_begin + chunk < groups ? i_begin + chunk : groups;
  unsigned long long mine = 0;
  for (int i = i_begin; i < i_end; ++i) mine += units_of(a, begin_of<F::TT>(a, a.b.plan.groups[i]));
  unsigned long long upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long y = __shfl_up(upto, o, 64);
    if (lane >= o) upto += y;
  }
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  unsigned long long units = 0, ahead = upto - mine;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) ahead += s_wave[w];
    units += s_wave[w];
  }
  unsigned long long per = (units + gridDim.x - 1) / gridDim.x;
  if (per < kLeastUnits) per = kLeastUnits;
  unsigned long long done = (unsigned long long)blockIdx.x * per;         // units in front of the next one
  unsigned long long left = done < units ? (done + per < units ? per : units - done) : 0;
  if (left > 0 && ahead <= done && done < ahead + mine) {
    unsigned long long at = ahead;
    for (int i = i_begin; i < i_end; ++i) {
      const unsigned long long u = units_of(a, begin_of<F::TT>(a, a.b.plan.groups[i]));
      if (at <= done && done < at + u) {
        s_first = i;
        s_from = done - at;
      }
      at += u;
    }
  }
  // Where every instance's own rows begin.
  for (int i = blockIdx.x * kThreads + tid; i < a.r.n_inst; i += gridDim.x * kThreads) {
    const Begin s = begin_of<F::TT>(a, a.b.plan.inst[i]);
    a.b.start[i] = s.tiles > 0 ? s.S : 0;
  }
  if (left == 0) return;
  __syncthreads();
  unsigned long long from = s_from;

  const float scale = kLog2E / sqrtf((float)D);
  const unsigned buffers = lds_address(s_tiles);
  for (int gi = __builtin_amdgcn_readfirstlane(s_first); left > 0 && gi < groups; ++gi, from = 0) {
    const Begin s = begin_of<F::TT>(a, a.b.plan.groups[gi]);
    const unsigned long long all_units = units_of(a, s);
    while (left > 0 && from < all_units) {
      const int t = (int)(from / (unsigned)s.tiles), u_begin = (int)(from % (unsigned)s.tiles);
      const int u_end = (unsigned long long)(s.tiles - u_begin) < left ? s.tiles : u_begin + (int)left;
      const int parts = (int)((done - (unsigned)u_begin + (unsigned)s.tiles - 1) / per) - (int)blockIdx.x + 1;      // of this tile, from here on
      from += (unsigned)(u_end - u_begin);
      left -= (unsigned)(u_end - u_begin);
      done += (unsigned)(u_end - u_begin);

      // This lane's row of q, of all of the group's.  Rows that are none are computed as the group's first and not stored.
      const int x = t * kPrefillRows + wave * 32 + n;
      const int of = x / a.b.rows, rest = x % a.b.rows;
      const int inst = a.b.plan.member[s.first + (of < s.count ? of : 0)];
      const int n_q = a.n_q == nullptr ? a.q_cap : clamped(a.n_q[inst], 0, a.q_cap);
      const bool real = of < s.count && rest / g < n_q;
      const int p = clamped(a.r.len[inst], 0, a.r.t_cap) - n_q + rest / g;
      const int lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
      int p_min = real ? p : 0x7fffffff, p_max = real ? p : -1;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const int y = __shfl_xor(p_min, o, 64), z = __shfl_xor(p_max, o, 64);
        p_min = y < p_min ? y : p_min;
        p_max = z > p_max ? z : p_max;
      }
      p_min = __builtin_amdgcn_readfirstlane(p_min);
      p_max = __builtin_amdgcn_readfirstlane(p_max);
      const bool idle = p_max < 0;                         // a wave without rows (or whose rows see nothing)
      const size_t q_row = (size_t)inst * a.b.rows + (real ? rest : 0);
      u32x4 qf[F::KS];
#pragma unroll
      for (int k = 0; k < F::KS; ++k) qf[k] = static_cast<const u32x4*>(a.q)[q_row * F::PIECES + 2 * k + hb];

      float16v o[F::DB];
#pragma unroll
      for (int b = 0; b < F::DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
      float m = -INFINITY, sum = 0.f;                      // the sum over this lane's half of the cache rows

      const TablePages pages = pages_of(a.r, s.lead);
      __syncthreads();                                     // everybody is done with the piece before
      Run next = run_of<F>(a, pages, s, s.tile(u_begin) * F::TT, wave);
      auto send = [&](int u) {                             // tile u, whose rows are those of `next`
        const unsigned to = buffers + (u % 2) * 2 * F::TILE * 16;
        send_tile<F, false>(a, s.lead, next, s, wave, to);
        send_tile<F, true>(a, s.lead, next, s, wave, to + F::TILE * 16);
        next = run_of<F>(a, pages, s, s.tile(u + 1 < u_end ? u + 1 : u) * F::TT, wave);
      };
      send(u_begin);
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
        if (idle) continue;
        float16v c[F::TB];
        if constexpr (sizeof(T) == 2 || !EXACT) {
#pragma unroll
          for (int b = 0; b < F::TB; ++b) c[b] = product<T, D>(Kt, 32 * b, qf);
        } else {
          c[0] = product_in_parts<D>(Kt, qf);
        }
        // Every row of the tile is seen by every query of the wave, or the scores of those that are not become -inf.
        const bool all = t0 + F::TT <= s.S && t0 + F::TT - 1 <= p_min && (a.window <= 0 || t0 > p_max - a.window || t0 + F::TT <= a.n_first);
        if (!all) {
#pragma unroll
          for (int b = 0; b < F::TB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int j = t0 + 32 * b + reg_row(i, hb);
              c[b][i] = (j >= s.S) | (j > p) | ((j < lo) & (j >= a.n_first)) ? -INFINITY : c[b][i];
            }
        }
        float top = c[0][0];
#pragma unroll
        for (int b = 0; b < F::TB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, c[b][i]);
        top = max32(top);
        // The reference is a whole number in units of log2 (a change of it rounds nothing).  Exponents refer to 0 as long as nothing is seen, and
        // where it is far, as the scores are brought near then.
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
        float part[4] = {0.f, 0.f, 0.f, 0.f};              // (sums of a tile first: long caches lose fewer digits so)
#pragma unroll
        for (int b = 0; b < F::TB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            c[b][i] = exp2_fast(__builtin_fmaf(c[b][i], scale, -use));
            part[i & 3] += c[b][i];
          }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int k = 0; k < F::TT / 16; ++k) {
            // A probability is the sum of three numbers of bf16, 24 bits, where the output has 32 (EXACT); else it is rounded to one, as in a prefill.
            constexpr int PARTS = EXACT ? 3 : 1;
            bf16x8 pb[PARTS];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float y = c[k / 2][8 * (k % 2) + e];
#pragma unroll
              for (int w = 0; w < PARTS; ++w) {
                pb[w][e] = (__bf16)y;
                y -= (float)pb[w][e];
              }
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
              for (int w = PARTS - 1; w >= 0; --w) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[w], o[b], 0, 0, 0);
            }
          }
        } else {
          const float* Vf = reinterpret_cast<const float*>(Vt);
#pragma unroll
          for (int b = 0; b < F::DB; ++b) {
            float16v y;                                    // of this tile alone, as the sums
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              y = __builtin_amdgcn_mfma_f32_32x32x2f32(Vf[reg_row(i, hb) * D + 32 * b + n], c[0][i], y, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] += y[i];
          }
        }
      }
      sum = sum32(sum);
      if (real) {
        const size_t slot = (size_t)s.first * a.b.rows + x + (size_t)kPrefillRows * blockIdx.x;
        if (hb == 0 && u_begin == 0) a.b.row[(size_t)s.first * a.b.rows + x] = make_int2((int)slot, parts);
        if (hb == 0) {
          a.b.ml[slot * 2] = m;
          a.b.ml[slot * 2 + 1] = sum;
        }
#pragma unroll
        for (int b = 0; b < F::DB; ++b)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            float4v y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = o[b][i + e];
            *reinterpret_cast<float4v*>(a.b.o + slot * D + 32 * b + reg_row(i, hb)) = y;
          }
      }
    }
  }
}

template <typename T, int D> hipError_t run(const Shape& s, const BeginArgs& a, bool exact, hipStream_t st) {
  const size_t lds = (size_t)2 * 2 * Form<T, D>::TILE * 16;
  if (exact) cache_beginnings_kernel<T, D, true><<<kShareWgs, kThreads, lds, st>>>(a, s.g);
  else cache_beginnings_kernel<T, D, false><<<kShareWgs, kThreads, lds, st>>>(a, s.g);
  return hipGetLastError();
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

hipError_t launch_cache_beginnings(const Shape& s, const BeginArgs& a, bool exact, hipStream_t st) {
  if (s.kv_dtype == AP_BF16) return s.d == 128 ? run<bf16_t, 128>(s, a, exact, st) : run<bf16_t, 64>(s, a, exact, st);
  return s.d == 128 ? run<float, 128>(s, a, exact, st) : run<float, 64>(s, a, exact, st);
}

}  // namespace ap
