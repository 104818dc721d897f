// hs_logprobs.h — log probabilities of given tokens, entropies and top
// alternatives of rows of logits (gfx950).  Included by hs_misc.hip.
//
// With M = max x, Z = sum e^(x - M): the log probability of token t is
// x_t - M - log Z, the entropy log Z - (sum (x - M) e^(x - M)) / Z, a sum of
// two terms that are not negative.  Z is held as R = Z - 1, the sum without one
// instance of the maximum, and log Z as log1p(R), so that a nearly certain
// token's log probability keeps its digits.
#pragma once

#include "hs_device.h"

#include <cfloat>

namespace hs {
namespace {

using namespace dev;

// d = x - M is cut here as the factor of d e^d: e^-200 is 0 in fp32, and the
// product then 0 and not NaN
constexpr float LOGPROB_FAR = -200.f;

// Orders logits by value, the lowest index first among equals: larger keys
// first.  -0 counts as 0.
__device__ __forceinline__ uint64_t logit_key(float x, int i) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u >> 31 ? u & 0x7FFFFFFFu : ~u);
}

// A part of a row: its maximum, R of that maximum, sum d e^d with d = x - max, and
// whether it holds a NaN or +inf.
struct LogprobPart {
  float m, r, s1, bad;
};
// its share of the row's sums relative to the row's maximum M; `lead`: the part
// that gives M its one instance
__device__ __forceinline__ void add_part(const LogprobPart &p, float M, bool lead, float &r, float &s1) {
  if (p.m == -INFINITY) return;
  const float d = fmaxf(p.m - M, LOGPROB_FAR), w = __expf(d), z = 1.f + p.r;
  r += lead ? p.r : w * z;
  s1 += w * (p.s1 + d * z);
}

constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64;
// candidates that the selection's fast path holds
constexpr int LP_CAND = 1024;
// keys of a row's parts up to which all are candidates
constexpr int LP_FEW = 64;

// largest of the work group's values, in every thread
__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *s_tmp) {
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < LP_WAVES; ++w) v = max(v, s_tmp[w]);
  return v;
}

template <int PER>
__device__ __forceinline__ int wave_count(const uint32_t (&v)[PER], uint32_t c) {  // values from c on
  int n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) n += (int)__popcll(__ballot(v[i] >= c));
  return n;
}
// The k-th largest of PER * 64 values, PER to a lane, bit by bit: bits `from` down
// to `to` of it, those above given.
template <int PER>
__device__ __forceinline__ uint32_t wave_kth(const uint32_t (&v)[PER], int k, int from, int to, uint32_t t = 0) {
  for (int b = from; b >= to; --b)
    if (wave_count(v, t | 1u << b) >= k) t |= 1u << b;
  return t;
}

constexpr uint32_t ORD_LEAST = 0x007FFFFFu;  // -inf's order bits

// Hands the `top` largest of the work group's keys to put(rank, key), each once.
// for_each(floor, f) calls f(key) for those of the thread's own keys whose value
// reaches the floor (or for all of them); at least `top` keys reach floor_key.
// Keys are distinct.  The keys that reach the floor are gathered in LDS and
// ranked by counting; where they are more than fit, the largest is taken `top`
// times.  lds.n is 0 and that is seen by all threads.
struct SelectLds {
  __align__(16) uint64_t key[LP_CAND + 8];
  uint64_t tmp[LP_WAVES];
  int n;
};
template <class ForEach, class Put>
__device__ __forceinline__ void select_top(SelectLds &lds, int top, uint64_t floor_key, ForEach for_each, Put put) {
  for_each(key_value(floor_key), [&](uint64_t key) {
    if (key >= floor_key) {
      const int at = atomicAdd(&lds.n, 1);
      if (at < LP_CAND) lds.key[at] = key;
    }
  });
  __syncthreads();
  const int n = lds.n;
  if (n <= LP_CAND) {
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
      const uint64_t mine = lds.key[i];
      int rank = 0;
      for (int o = 0; o < n; o += 8) {
        u32x4 two[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) two[u] = *(const u32x4 *)&lds.key[o + 2 * u];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          rank += o + 2 * u < n && ((uint64_t)two[u][1] << 32 | two[u][0]) > mine;
          rank += o + 2 * u + 1 < n && ((uint64_t)two[u][3] << 32 | two[u][2]) > mine;
        }
      }
      if (rank < top) put(rank, mine);
    }
    return;
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < top; ++k) {
    uint64_t best = 0;
    for_each(key_value(floor_key), [&](uint64_t key) { best = key < last ? max(best, key) : best; });
    last = block_max(best, lds.tmp);
    if (threadIdx.x == 0) put(k, last);
  }
}

// a row's given token and its logit (0 outside the row), asked for early by the
// thread that puts the row
struct Given {
  int t;
  float x;
};
template <int DT>
__device__ __forceinline__ Given given_token(const LogprobArgs &a, int64_t row) {
  Given g{-1, 0.f};
  if (threadIdx.x == 0 && a.logprob) {
    g.t = a.tokens[a.act ? a.act[row] : row];
    if (g.t >= 0 && g.t < a.vocab) g.x = ld_elem<DT>(a.logits, row * a.ld + g.t);
  }
  return g;
}
// what a row's sums give
__device__ __forceinline__ void put_row(const LogprobArgs &a, int64_t row, const Given &g, bool none, float M, float r,
                                        float s1) {
  const float lz = log1pf(r);
  if (a.entropy) a.entropy[row] = none ? NAN : lz - s1 / (1.f + r);
  if (a.logprob) a.logprob[row] = g.t < 0 ? 0.f : none || g.t >= a.vocab ? NAN : g.x - M - lz;
}
__device__ __forceinline__ void put_top(const LogprobArgs &a, int64_t row, bool none, float M, float lz, int rank,
                                        uint64_t key) {
  if (a.top_ids) a.top_ids[row * a.top + rank] = none ? -1 : key_index(key);
  if (a.top_logprobs) a.top_logprobs[row * a.top + rank] = none ? NAN : key_value(key) - M - lz;
}

// a row without a distribution has no alternatives
__device__ __forceinline__ void put_no_top(const LogprobArgs &a, int64_t row) {
  for (int k = threadIdx.x; k < a.top; k += LP_THREADS) put_top(a, row, true, 0.f, 0.f, k, 0);
}

// parts that another work group of the same launch reads (past the caches of one
// XCD), or another launch
template <bool SAME, class T>
__device__ __forceinline__ T ld_part(const T *p) {
  if constexpr (SAME) return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else return *p;
}
template <class T>
__device__ __forceinline__ void st_part(bool same, T *p, T v) {
  if (same) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *p = v;
}
// the workspace: a counter for each row, the parts' sums, the parts' keys
__device__ __forceinline__ LogprobPart *row_parts(const LogprobArgs &a, int64_t row) {
  return (LogprobPart *)((char *)a.ws + LOGPROB_COUNTERS * 4) + row * a.parts;
}
__device__ __forceinline__ uint64_t *row_keys(const LogprobArgs &a, int64_t row) {
  return (uint64_t *)(row_parts(a, a.rows)) + row * a.parts * a.top;
}

// A work group joins a row's parts.  Every part gave its `top` largest keys in
// order (elements past the row's end among them: they have the lowest keys).
// The floor is the top-th largest of as many of the parts' first keys as a wave holds
// two to a lane, at least `top`: hardly more of all reach it (with the least of the
// parts' second keys 256 rows of 19 parts and twenty alternatives took 53.6 us, not
// 47.5).  Few keys are ranked without one, as fast as it is found.  Every wave joins
// the sums and finds the floor by itself; the keys are asked for beside them.
template <bool SAME>
__device__ __forceinline__ void join_parts(const LogprobArgs &a, int64_t row, const Given &given, SelectLds &lds) {
  constexpr int HOLD = 4;  // keys of a thread that stay in registers
  const int lane = threadIdx.x & 63;
  const LogprobPart *p = row_parts(a, row);
  const uint64_t *keys = row_keys(a, row);
  const int64_t n_keys = (int64_t)a.parts * a.top;
  uint64_t hold[HOLD];
#pragma unroll
  for (int u = 0; u < HOLD; ++u) {
    const int64_t i = u * LP_THREADS + threadIdx.x;
    hold[u] = i < n_keys ? ld_part<SAME>(&keys[i]) : 0;
  }
  // the first keys of the parts, part by part
  constexpr int PER = 2;
  const int n_first = min(a.parts, 64 * PER) * (a.top > 0 ? min(a.top, max(64 * PER / a.parts, 1)) : 0);
  uint64_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * 64 + lane, k = e / a.parts;
    key[i] = n_keys > LP_FEW && e < n_first ? ld_part<SAME>(&keys[(int64_t)(e - k * a.parts) * a.top + k]) : 0;
  }
  // parts lane, lane + 64, ..; the first of them kept
  auto part = [&](int c) { return LogprobPart{ld_part<SAME>(&p[c].m), ld_part<SAME>(&p[c].r), ld_part<SAME>(&p[c].s1), ld_part<SAME>(&p[c].bad)}; };
  const LogprobPart mine = lane < a.parts ? part(lane) : LogprobPart{-INFINITY, 0.f, 0.f, 0.f};
  float m = mine.m;
  bool bad = mine.bad != 0.f;
  for (int c = lane + 64; c < a.parts; c += 64) {
    m = fmaxf(m, ld_part<SAME>(&p[c].m));
    bad |= ld_part<SAME>(&p[c].bad) != 0.f;
  }
  const float M = wave_max(m);
  if (__ballot(bad) || M == -INFINITY) {
    if (threadIdx.x == 0) put_row(a, row, given, true, 0.f, 0.f, 0.f);
    put_no_top(a, row);
    return;
  }
  // the first part that holds the maximum leads
  int lead = mine.m == M ? lane : 0x7FFFFFFF;
  for (int c = lane + 64; c < a.parts && lead == 0x7FFFFFFF; c += 64)
    if (ld_part<SAME>(&p[c].m) == M) lead = c;
  for (int off = 32; off >= 1; off >>= 1) lead = min(lead, __shfl_xor(lead, off));
  float r = 0.f, s1 = 0.f;
  if (lane < a.parts) add_part(mine, M, lane == lead, r, s1);
  for (int c = lane + 64; c < a.parts; c += 64) add_part(part(c), M, c == lead, r, s1);
  r = wave_sum(r);
  s1 = wave_sum(s1);
  if (threadIdx.x == 0) {
    put_row(a, row, given, false, M, r, s1);
    lds.n = 0;
  }
  if (a.top <= 0) return;
  uint64_t low = 0;
  if (n_keys > LP_FEW) {
    uint32_t ord[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) ord[i] = (uint32_t)(key[i] >> 32);
    // as in k_logprobs: the upper half of the value's bits, all of them, the lowest places
    uint32_t kth = max(wave_kth(ord, a.top, 31, 16), ORD_LEAST), place = 0;
    if (wave_count(ord, kth) > a.top + 16) {
      kth = max(wave_kth(ord, a.top, 15, 0, kth & 0xFFFF0000u), ORD_LEAST);
      if (wave_count(ord, kth) > a.top + 16) {
        const int above = kth == ~0u ? 0 : wave_count(ord, kth + 1);
#pragma unroll
        for (int i = 0; i < PER; ++i) ord[i] = ord[i] == kth ? (uint32_t)key[i] : 0u;
        place = wave_kth(ord, a.top - above, 31, 0);
      }
    }
    low = (uint64_t)kth << 32 | place;
  }
  __syncthreads();
  const float lz = log1pf(r);
  select_top(
      lds, a.top, low,
      [&](float floor, auto f) {
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
          if (hold[u]) f(hold[u]);
        for (int64_t i = HOLD * LP_THREADS + threadIdx.x; i < n_keys; i += LP_THREADS) f(ld_part<SAME>(&keys[i]));
      },
      [&](int rank, uint64_t key) { put_top(a, row, false, M, lz, rank, key); });
}

// element i of a thread's raw words: as fp32
template <int DT, int NW>
__device__ __forceinline__ float raw_elem(const uint32_t (&w)[NW], int i) {
  if constexpr (DT == HS_F32) return __uint_as_float(w[i]);
  else return i & 1 ? hi_f32<DT>(w[i >> 1]) : lo_f32<DT>(w[i >> 1]);
}

// One work group takes one part of a row, NW words a thread, which stay in
// registers as they are: read once, all loads in flight together.  First the
// maximum, then the sums, then the alternatives: the top-th largest of the 256
// threads' own maxima is a value that at least `top` elements reach, and few more
// (one wave finds it, bit by bit with ballots, while the others sum).  A single
// alternative is the maximum's first place.  A NaN makes the sum NaN.  The exponentials
// are 2^(d log2 e) with the product rounded: off by |d| 2^-24 of themselves,
// as much as the rounding of d = x - M moves them.  A row of one
// part is finished here; of several, by the last of its work groups to arrive, or by
// k_logprobs_join.
//
// Measured: 256 rows of 152064 fp32 logits (156 MB), no alternatives 33 us, one 39,
// five 44, twenty 47; 1531 rows of 32003 bf16 logits (98 MB) 32, 38, 41, 44.  Neither the
// vector unit (issue 48 % of the cycles for fp32, 57 % for bf16) nor memory (3.8 TB/s) is
// full: each work group's load, maximum, barrier and sum come one after the other, five
// share a CU, and no register is left for the next part meanwhile; the alternatives add the
// floor's 16 ballots and the ranking.  16 rows of 152064: 7, 9.5, 12, 13 us, one row of 32000: 6, 8, 9.5, 11, the
// chain of one part and of the join.  A work group to a row that read it again for each
// pass took 1204 us for the 256 rows with twenty.
template <int DT, int NW>
__global__ __launch_bounds__(LP_THREADS, 5) void k_logprobs(LogprobArgs a) {
  constexpr int VEC = DT == HS_F32 ? 4 : 8, VPT = NW * VEC / 4, NV = NW / 4, PART = LP_THREADS * VPT;
  using S = typename Ty<DT>::S;
  __shared__ SelectLds s_sel;
  __shared__ float s_m[LP_WAVES], s_r[LP_WAVES], s_1[LP_WAVES];
  __shared__ int s_lead[LP_WAVES], s_last;
  __shared__ uint32_t s_ord[LP_THREADS];
  __shared__ uint32_t s_kth;
  __shared__ int s_first[LP_WAVES], s_tie;
  const int64_t row = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x % (uint32_t)a.parts), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // the last of several parts is read from further ahead, so that it is whole; what
  // the part before it has counts as lying past the row's end
  const int i0 = min(part * PART, max(0, a.vocab - PART)), n = min(a.vocab - i0, PART), skip0 = part * PART - i0;
  const S *x = (const S *)a.logits + row * a.ld + i0;
  // element e of vector u: VEC consecutive ones to a thread; rows start anywhere
  int tid = (int)threadIdx.x;
  auto index = [&](int u, int e) { return (u * LP_THREADS + tid) * VEC + e; };
  struct __attribute__((packed, aligned(sizeof(S)))) Loose {
    u32x4 w;
  };
  constexpr uint32_t NEG = DT == HS_F32 ? 0xFF800000u : DT == HS_F16 ? 0xFC00FC00u : 0xFF80FF80u;  // -inf
  uint32_t w[NW];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    if (n == PART || index(u, VEC - 1) < n) {
      *(u32x4 *)&w[4 * u] = ((const Loose *)(x + index(u, 0)))->w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[4 * u + k] = NEG;
        constexpr int PER = VEC / 4;
        uint32_t bits = NEG;
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (index(u, k * PER + e) < n) {
            const S v = x[index(u, k * PER + e)];
            if constexpr (DT == HS_F32) bits = __float_as_uint(v);
            else bits = (bits & ~(0xFFFFu << (16 * e))) | (uint32_t)v << (16 * e);
          }
        w[4 * u + k] = bits;
      }
    }
  }
  const Given given = given_token<DT>(a, row);
  if (skip0) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (index(i / VEC, i % VEC) < skip0) {
        if constexpr (DT == HS_F32) w[i] = NEG;
        else w[i >> 1] = i & 1 ? (w[i >> 1] & 0xFFFFu) | (NEG & 0xFFFF0000u) : (w[i >> 1] & 0xFFFF0000u) | (NEG & 0xFFFFu);
      }
  }
  // an element's index in the row, or past its end
  auto place = [&](int i) {
    const int k = index(i / VEC, i % VEC);
    return k < skip0 ? a.vocab + k : i0 + k;
  };
  // the words and places are opaque from one use to the next: 16-bit elements are
  // unpacked and places made again, not kept in registers
  auto keep = [&] {
    asm volatile("" : "+v"(tid));
    if constexpr (DT != HS_F32)
#pragma unroll
      for (int k = 0; k < NW; ++k) asm volatile("" : "+v"(w[k]));
  };
  float tm = -INFINITY;
#pragma unroll
  for (int i = 0; i < VPT; ++i) tm = fmaxf(tm, raw_elem<DT, NW>(w, i));
  keep();
  const float wm = wave_max(tm);
  if (lane == 0) s_m[wave] = wm;
  if (threadIdx.x == 0) s_sel.n = 0;
  const uint32_t bits = __float_as_uint(tm + 0.f), ord = bits >> 31 ? ~bits : bits | 0x80000000u;
  if (a.top > 1) s_ord[threadIdx.x] = ord;
  __syncthreads();
  float M = s_m[0];
#pragma unroll
  for (int w2 = 1; w2 < LP_WAVES; ++w2) M = fmaxf(M, s_m[w2]);
  // the place of the first of the thread's elements that is v (there is one)
  auto first_of = [&](float v) {
    int at = 0;
#pragma unroll
    for (int i = VPT - 1; i >= 0; --i) at = raw_elem<DT, NW>(w, i) == v ? i : at;
    keep();
    return place(at);
  };
  // The floor: one wave finds it while the others sum, another one in the next work group.
  // Among threads that share the top-th largest maximum the lowest places would come
  // first; where many share it, s_tie has the others wait for that.
  if (a.top > 1 && wave == (int)(blockIdx.x & (LP_WAVES - 1))) {
    uint32_t all[LP_WAVES];
#pragma unroll
    for (int i = 0; i < LP_WAVES; ++i) all[i] = s_ord[i * 64 + lane];
    // the upper half of the bits does, unless many threads share it
    // (no number orders below -inf, whose lower bits are set)
    uint32_t kth = max(wave_kth(all, a.top, 31, 16), ORD_LEAST);
    if (wave_count(all, kth) > a.top + 16) kth = max(wave_kth(all, a.top, 15, 0, kth & 0xFFFF0000u), ORD_LEAST);
    if (lane == 0) s_kth = kth, s_tie = wave_count(all, kth) > a.top + 16;
  }
  // every e^(x - M), the maximum's own 1 among them; without a number above -inf
  // the difference is to the lowest one, so that only a NaN, which the maximum passed
  // over, gives a NaN
  float r = 0.f, s1 = 0.f;
  const float ref = fmaxf(M, -FLT_MAX);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const float d = raw_elem<DT, NW>(w, i) - ref, e = __expf(d);
    r += e;
    s1 = __builtin_fmaf(fmaxf(d, LOGPROB_FAR), e, s1);
  }
  keep();
  r = wave_sum(r);
  s1 = wave_sum(s1);
  int first = 0x7FFFFFFF;
  if (a.top == 1 && wm == M) {
    if (tm == M) first = first_of(M);
    for (int off = 32; off >= 1; off >>= 1) first = min(first, __shfl_xor(first, off));
  }
  if (lane == 0) s_r[wave] = r, s_1[wave] = s1, s_first[wave] = first;
  __syncthreads();
  r = s1 = 0.f;
#pragma unroll
  for (int w2 = 0; w2 < LP_WAVES; ++w2) r += s_r[w2], s1 += s_1[w2];
  uint64_t floor_key = 0;
  if (a.top > 1) {
    const uint32_t kth = s_kth;
    floor_key = (uint64_t)kth << 32;
    if (s_tie) {
      uint32_t all[LP_WAVES];
#pragma unroll
      for (int i = 0; i < LP_WAVES; ++i) all[i] = s_ord[i * 64 + lane];
      const int above = kth == ~0u ? 0 : wave_count(all, kth + 1);
      __syncthreads();
      s_ord[threadIdx.x] = ord == kth ? (uint32_t)~first_of(tm) : 0u;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < LP_WAVES; ++i) all[i] = s_ord[i * 64 + lane];
      floor_key |= wave_kth(all, a.top - above, 31, 0);  // the largest complement is the lowest place
    }
  }
  if (M > -INFINITY && M < INFINITY && r < 1.f + 0x1p-4f) {
    // nearly certain: the difference would lose the rest's digits, so the rest is summed by
    // itself.  A thread with the maximum leaves its first instance out.
    const bool lead = tm == M;
    float rest = 0.f;
    bool out = lead;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const float v = raw_elem<DT, NW>(w, i);
      const bool skip = out && v == M;
      out &= !skip;
      rest += skip ? 0.f : __expf(v - M);
    }
    keep();
    rest = wave_sum(rest);
    const int leads = (int)__popcll(__ballot(lead));
    __syncthreads();
    if (lane == 0) s_r[wave] = rest, s_lead[wave] = leads;
    __syncthreads();
    r = 0.f;
    int n2 = 0;
#pragma unroll
    for (int w2 = 0; w2 < LP_WAVES; ++w2) r += s_r[w2], n2 += s_lead[w2];
    r += (float)(n2 - 1);
  } else {
    r -= 1.f;
  }
  const bool bad = !(r < INFINITY) || M == INFINITY;
  const bool whole = a.parts == 1, none = bad || M == -INFINITY;
  LogprobPart *mine = row_parts(a, row) + part;
  if (threadIdx.x == 0) {
    if (whole) {
      put_row(a, row, given, none, M, r, s1);
    } else {
      st_part(a.count, &mine->m, M);
      st_part(a.count, &mine->r, r);
      st_part(a.count, &mine->s1, s1);
      st_part(a.count, &mine->bad, bad ? 1.f : 0.f);
    }
  }
  if (whole && none) {
    put_no_top(a, row);
  } else if (a.top > 0 && !bad) {  // (the keys of a part with a NaN are not looked at)
    const float lz = log1pf(r);
    uint64_t *keys = row_keys(a, row) + (int64_t)part * a.top;
    if (a.top == 1) {
      if (threadIdx.x == 0) {
#pragma unroll
        for (int w2 = 0; w2 < LP_WAVES; ++w2) first = min(first, s_first[w2]);
        const uint64_t key = logit_key(M, first);
        if (whole) put_top(a, row, false, M, lz, 0, key);
        else st_part(a.count, keys, key);
      }
    } else select_top(
        s_sel, a.top, floor_key,
        [&](float floor, auto f) {
#pragma unroll
          for (int i = 0; i < VPT; ++i) {
            const float v = raw_elem<DT, NW>(w, i);
            if (v >= floor) f(logit_key(v, place(i)));
          }
          keep();
        },
        [&](int rank, uint64_t key) {
          if (whole) put_top(a, row, false, M, lz, rank, key);
          else st_part(a.count, &keys[rank], key);
        });
  }
  if (whole || !a.count) return;
  // Parts are stored and read past the caches of one XCD; every wave's stores are
  // done before the barrier, behind which one thread counts the work group in.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    // (as far apart as they may lie: counters in one cache line wait for each other, 9.4 us
    // against 7.3 for 16 rows of 19 parts without alternatives)
    uint32_t *c = (uint32_t *)a.ws + row * min(32, LOGPROB_COUNTERS / (int)a.rows);
    const bool last = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(a.parts - 1);
    if (last) st_part(true, c, 0u);  // for the next call
    s_last = last;
  }
  __syncthreads();
  if (s_last) join_parts<true>(a, row, given, s_sel);
}

// Rows past one launch's: 6.0 us for 1531 rows of two parts with one alternative, 5.4 for
// 256 rows of 19 parts with twenty, two dependent reads and the ranking.
template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_join(LogprobArgs a) {
  __shared__ SelectLds s_sel;
  join_parts<false>(a, blockIdx.x, given_token<DT>(a, blockIdx.x), s_sel);
}

template <int DT>
hipError_t logprobs_dt(LogprobArgs a, hipStream_t st) {
  constexpr int CE = Ty<DT>::CE / 4;  // elements of a word
  // rows that eight words a thread hold: fewer registers, and no thread without an
  // element (1531 rows of 2048 fp32 logits 7.4 us, with 32 words 11.2; one row 3.6 and 5.0)
  const bool small = a.vocab <= LP_THREADS * 8 * CE;
  constexpr int PART = LOGPROB_PART * CE;
  static_assert(LOGPROB_PART == LP_THREADS * 32, "a part is 32 words a thread");
  a.parts = small ? 1 : (int)(((int64_t)a.vocab + PART - 1) / PART);
  const int64_t groups = a.rows * a.parts;
  if (groups > INT32_MAX) return hipErrorInvalidValue;
  // One launch while the GPU holds all work groups at once, five to a CU: where more
  // wait, joining at the end of a work group keeps its place for longer than a second
  // launch takes (no alternatives, one launch against two: 64 rows of 152064 fp32
  // logits 12.4 and 13.1 us, 400 rows 54.8 and 46.3; one row of 32000 8.7 and 11.1).
  a.count = a.parts > 1 && groups <= LOGPROB_ONE_LAUNCH && a.rows <= LOGPROB_COUNTERS;
  if (small) HS_LAUNCH((k_logprobs<DT, 8>), dim3((uint32_t)groups), dim3(LP_THREADS), 0, st, a);
  else HS_LAUNCH((k_logprobs<DT, 32>), dim3((uint32_t)groups), dim3(LP_THREADS), 0, st, a);
  if (a.parts > 1 && !a.count) HS_LAUNCH((k_logprobs_join<DT>), dim3((uint32_t)a.rows), dim3(LP_THREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace

uint64_t logprob_workspace(int64_t rows, int vocab, int top) {
  const int64_t parts = logprob_parts(vocab);
  return parts > 1 ? LOGPROB_COUNTERS * 4 + (uint64_t)rows * parts * (sizeof(LogprobPart) + top * 8) : 0;
}

hipError_t launch_logprobs(int dtype, const LogprobArgs &a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  switch (dtype) {
    case HS_F32: return logprobs_dt<HS_F32>(a, st);
    case HS_F16: return logprobs_dt<HS_F16>(a, st);
    case HS_BF16: return logprobs_dt<HS_BF16>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace hs
