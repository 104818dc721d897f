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

namespace hs {
namespace {

using namespace dev;

// d = x - M is cut here: e^-200 is 0 in fp32, and d e^d then 0 and not NaN
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

// The k-th largest of the wave's 64 values (k in 1..64), bit by bit.
__device__ __forceinline__ uint32_t wave_kth(uint32_t v, int k) {
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | 1u << b;
    if ((int)__popcll(__ballot(v >= c)) >= k) t = c;
  }
  return t;
}

// Hands the `top` largest of the work group's keys to put(rank, key), each once.
// for_each(f) calls f(key) for the thread's own keys; floor_key is a key that at
// least `top` of all keys reach.  Keys are distinct.  The keys that reach the
// floor are gathered in LDS and ranked by counting; where they are more than fit,
// the largest is taken `top` times.
template <class ForEach, class Put>
__device__ __forceinline__ void select_top(int top, uint64_t floor_key, ForEach for_each, Put put) {
  __shared__ __align__(16) uint64_t s_key[LP_CAND + 2];
  __shared__ uint64_t s_tmp[LP_WAVES];
  __shared__ int s_n;
  __syncthreads();
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  for_each([&](uint64_t key) {
    if (key >= floor_key) {
      const int at = atomicAdd(&s_n, 1);
      if (at < LP_CAND) s_key[at] = key;
    }
  });
  __syncthreads();
  const int n = s_n;
  if (n <= LP_CAND) {
    if (threadIdx.x < 2) s_key[n + threadIdx.x] = 0;  // pads the pairs below
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
      const uint64_t mine = s_key[i];
      int rank = 0;
      for (int o = 0; o < n; o += 2) {
        const u32x4 two = *(const u32x4 *)&s_key[o];
        rank += ((uint64_t)two[1] << 32 | two[0]) > mine;
        rank += ((uint64_t)two[3] << 32 | two[2]) > mine;
      }
      if (rank < top) put(rank, mine);
    }
    return;
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < top; ++k) {
    uint64_t best = 0;
    for_each([&](uint64_t key) { best = key < last ? max(best, key) : best; });
    last = block_max(best, s_tmp);
    if (threadIdx.x == 0) put(k, last);
  }
}

// what a row's sums give
template <int DT>
__device__ __forceinline__ void put_row(const LogprobArgs &a, int64_t row, bool none, float M, float r, float s1) {
  const float lz = log1pf(r);
  if (a.entropy) a.entropy[row] = none ? NAN : lz - s1 / (1.f + r);
  if (a.logprob) {
    const int t = a.tokens[a.act ? a.act[row] : row];
    float v = NAN;
    if (t >= 0 && t < a.vocab) v = ld_elem<DT>(a.logits, row * a.ld + t) - M - lz;
    a.logprob[row] = t < 0 ? 0.f : none ? NAN : v;
  }
}
__device__ __forceinline__ void put_top(const LogprobArgs &a, int64_t row, bool none, float M, float lz, int rank,
                                        uint64_t key) {
  if (a.top_ids) a.top_ids[row * a.top + rank] = none ? -1 : key_index(key);
  if (a.top_logprobs) a.top_logprobs[row * a.top + rank] = none ? NAN : key_value(key) - M - lz;
}

// One work group takes one part of a row, VPT elements a thread, which stay in
// registers: read once, all loads in flight together.  First the maximum, then
// the sums, then the alternatives: a wave's top-th largest lane maximum is a
// value that at least `top` of its elements reach (bit by bit with ballots), so
// the largest of the waves' is a floor that few elements pass.  A row of one part
// is finished here.
template <int DT, int VPT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs(LogprobArgs a) {
  constexpr int VEC = DT == HS_F32 ? 4 : 8, NV = VPT / VEC;
  using S = typename Ty<DT>::S;
  __shared__ float s_m[LP_WAVES], s_r[LP_WAVES], s_1[LP_WAVES];
  __shared__ int s_bad[LP_WAVES], s_lead[LP_WAVES];
  __shared__ uint64_t s_t[LP_WAVES];
  const int64_t row = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x % (uint32_t)a.parts), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = part * (LP_THREADS * VPT), n = min(a.vocab - i0, LP_THREADS * VPT);
  const S *x = (const S *)a.logits + row * a.ld + i0;
  // element e of vector u: VEC consecutive ones to a thread; rows start anywhere
  auto index = [&](int u, int e) { return (u * LP_THREADS + (int)threadIdx.x) * VEC + e; };
  float v[VPT];
  if (n == LP_THREADS * VPT) {
    struct __attribute__((packed, aligned(sizeof(S)))) Loose {
      u32x4 w;
    };
    u32x4 w[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) w[u] = ((const Loose *)(x + index(u, 0)))->w;
#pragma unroll
    for (int u = 0; u < NV; ++u) unpack<DT>(w[u], v + u * VEC);
  } else {
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[u * VEC + e] = index(u, e) < n ? ld_elem<DT>(x, index(u, e)) : -INFINITY;
  }
  float tm = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    tm = fmaxf(tm, v[i]);
    bad |= !(v[i] < INFINITY);
  }
  // the floor of the alternatives
  if (a.top > 0) {
    const uint32_t u = __float_as_uint(tm + 0.f), ord = u >> 31 ? ~u : u | 0x80000000u;
    const uint32_t kth = wave_kth(ord, a.top);
    uint64_t floor_key = (uint64_t)kth << 32;
    // lanes that share it: the lowest indices among them come first
    const int above = (int)__popcll(__ballot(ord > kth)), share = (int)__popcll(__ballot(ord == kth));
    if (above + share > a.top) {
      int first = 0x7FFFFFFF;
      if (ord == kth)
#pragma unroll
        for (int i = VPT - 1; i >= 0; --i)
          if (v[i] == tm) first = index(i / VEC, i % VEC);
      // the largest complement is the lowest index
      floor_key |= wave_kth(ord == kth ? (uint32_t)~(i0 + first) : 0u, a.top - above);
    }
    if (lane == 0) s_t[wave] = floor_key;
  }
  const float wm = wave_max(tm);
  const bool wbad = __ballot(bad) != 0;
  if (lane == 0) s_m[wave] = wm, s_bad[wave] = wbad;
  __syncthreads();
  float M = s_m[0];
  uint64_t floor_key = a.top > 0 ? s_t[0] : 0;
  bool any_bad = s_bad[0];
#pragma unroll
  for (int w = 1; w < LP_WAVES; ++w) {
    M = fmaxf(M, s_m[w]);
    any_bad |= s_bad[w] != 0;
    if (a.top > 0) floor_key = max(floor_key, s_t[w]);
  }
  float r = 0.f, s1 = 0.f;
  int lead = 0;  // threads that leave out one instance of the maximum
  if (M > -INFINITY) {
    int skip = -1;
    if (tm == M) {
#pragma unroll
      for (int i = VPT - 1; i >= 0; --i) skip = v[i] == M ? i : skip;
      lead = 1;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const float d = fmaxf(v[i] - M, LOGPROB_FAR), e = __expf(d);
      r += e;
      s1 = __builtin_fmaf(d, e, s1);
    }
    // the instance itself added exactly e^0 = 1: the sum is made again without it
    if (skip >= 0) {
      r = 0.f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) r += i == skip ? 0.f : __expf(fmaxf(v[i] - M, LOGPROB_FAR));
    }
  }
  r = wave_sum(r);
  s1 = wave_sum(s1);
  const int wlead = (int)__popcll(__ballot(lead));
  if (lane == 0) s_r[wave] = r, s_1[wave] = s1, s_lead[wave] = wlead;
  __syncthreads();
  r = s1 = 0.f;
  lead = 0;
#pragma unroll
  for (int w = 0; w < LP_WAVES; ++w) r += s_r[w], s1 += s_1[w], lead += s_lead[w];
  r += (float)max(lead - 1, 0);
  const bool whole = a.parts == 1, none = any_bad || M == -INFINITY;
  if (threadIdx.x == 0) {
    if (whole) put_row<DT>(a, row, none, M, r, s1);
    else ((LogprobPart *)a.ws)[blockIdx.x] = LogprobPart{M, r, s1, any_bad ? 1.f : 0.f};
  }
  if (a.top <= 0) return;
  const float lz = log1pf(r);
  uint64_t *keys = (uint64_t *)((LogprobPart *)a.ws + a.rows * a.parts) + (int64_t)blockIdx.x * a.top;
  select_top(
      a.top, floor_key,
      [&](auto f) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) f(logit_key(v[i], i0 + index(i / VEC, i % VEC)));
      },
      [&](int rank, uint64_t key) {
        if (whole) put_top(a, row, none, M, lz, rank, key);
        else keys[rank] = key;
      });
}

// One work group joins a row's parts.  Every part gave its `top` largest keys in
// order (elements past the row's end among them: they have the lowest keys).
// The k-th keys of all parts, k = ceil(top / parts): at least `top` keys reach the
// least of them.
template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_join(LogprobArgs a) {
  __shared__ float s_m[LP_WAVES], s_r[LP_WAVES], s_1[LP_WAVES];
  __shared__ int s_bad[LP_WAVES];
  __shared__ uint64_t s_t[LP_WAVES], s_lead[LP_WAVES];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const LogprobPart *p = (const LogprobPart *)a.ws + row * a.parts;
  const uint64_t *keys = (const uint64_t *)((const LogprobPart *)a.ws + a.rows * a.parts) + row * a.parts * a.top;
  const int kth = a.top > 0 ? (a.top + a.parts - 1) / a.parts - 1 : 0;
  float m = -INFINITY;
  bool bad = false;
  uint64_t low = ~0ull;
  for (int c = threadIdx.x; c < a.parts; c += LP_THREADS) {
    m = fmaxf(m, p[c].m);
    bad |= p[c].bad != 0.f;
    if (a.top > 0) low = min(low, keys[(int64_t)c * a.top + kth]);
  }
  m = wave_max(m);
  for (int off = 32; off >= 1; off >>= 1) low = min(low, (uint64_t)__shfl_xor((unsigned long long)low, off));
  const bool wbad = __ballot(bad) != 0;
  if (lane == 0) s_m[wave] = m, s_bad[wave] = wbad, s_t[wave] = low;
  __syncthreads();
  float M = s_m[0];
  bool any_bad = s_bad[0];
  uint64_t floor_key = s_t[0];
#pragma unroll
  for (int w = 1; w < LP_WAVES; ++w) {
    M = fmaxf(M, s_m[w]);
    any_bad |= s_bad[w] != 0;
    floor_key = min(floor_key, s_t[w]);
  }
  // the first part that holds the maximum leads
  uint64_t first = ~0ull;
  for (int c = threadIdx.x; c < a.parts; c += LP_THREADS)
    if (p[c].m == M) first = min(first, (uint64_t)c);
  for (int off = 32; off >= 1; off >>= 1) first = min(first, (uint64_t)__shfl_xor((unsigned long long)first, off));
  if (lane == 0) s_lead[wave] = first;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < LP_WAVES; ++w) first = min(first, s_lead[w]);
  float r = 0.f, s1 = 0.f;
  for (int c = threadIdx.x; c < a.parts; c += LP_THREADS) add_part(p[c], M, (uint64_t)c == first, r, s1);
  r = wave_sum(r);
  s1 = wave_sum(s1);
  if (lane == 0) s_r[wave] = r, s_1[wave] = s1;
  __syncthreads();
  r = s1 = 0.f;
#pragma unroll
  for (int w = 0; w < LP_WAVES; ++w) r += s_r[w], s1 += s_1[w];
  const bool none = any_bad || M == -INFINITY;
  if (threadIdx.x == 0) put_row<DT>(a, row, none, M, r, s1);
  if (a.top <= 0) return;
  const float lz = log1pf(r);
  select_top(
      a.top, floor_key,
      [&](auto f) {
        for (int64_t i = threadIdx.x; i < (int64_t)a.parts * a.top; i += LP_THREADS) f(keys[i]);
      },
      [&](int rank, uint64_t key) { put_top(a, row, none, M, lz, rank, key); });
}

template <int DT>
hipError_t logprobs_dt(const LogprobArgs &a, hipStream_t st) {
  HS_LAUNCH((k_logprobs<DT, LOGPROB_PART / LP_THREADS>), dim3((uint32_t)(a.rows * a.parts)), dim3(LP_THREADS), 0, st, a);
  if (a.parts > 1) HS_LAUNCH((k_logprobs_join<DT>), dim3((uint32_t)a.rows), dim3(LP_THREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace

uint64_t logprob_workspace(int64_t rows, int vocab, int top) {
  const int64_t parts = logprob_parts(vocab);
  return parts > 1 ? (uint64_t)rows * parts * (sizeof(LogprobPart) + top * 8) : 0;
}

hipError_t launch_logprobs(int dtype, const LogprobArgs &a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.rows * a.parts > INT32_MAX) return hipErrorInvalidValue;
  switch (dtype) {
    case HS_F32: return logprobs_dt<HS_F32>(a, st);
    case HS_F16: return logprobs_dt<HS_F16>(a, st);
    case HS_BF16: return logprobs_dt<HS_BF16>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace hs
