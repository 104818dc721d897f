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

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *s_tmp) {
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < 16; ++w) v = max(v, s_tmp[w]);
  return v;
}
__device__ __forceinline__ float block_sum(float v, float *s_tmp) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < 16; ++w) v += s_tmp[w];
  return v;
}

// One work group takes a row: its largest element, its sums, then the
// alternatives one at a time, each the largest key below the one before.
template <int DT>
__global__ __launch_bounds__(1024) void k_logprobs(LogprobArgs a) {
  __shared__ uint64_t s_k[16];
  __shared__ float s_f[16];
  const int64_t row = blockIdx.x;
  using S = typename Ty<DT>::S;
  const S *x = (const S *)a.logits + row * a.ld;
  uint64_t top = 0;
  float bad = 0.f;
  for (int i = threadIdx.x; i < a.vocab; i += 1024) {
    const float v = ld_elem<DT>(x, i);
    if (!(v < INFINITY)) bad = 1.f;
    top = max(top, logit_key(v, i));
  }
  top = block_max(top, s_k);
  bad = block_sum(bad, s_f);
  const float M = key_value(top);
  const int at = key_index(top);
  const bool none = bad > 0.f || M == -INFINITY;  // no distribution
  float r = 0.f, s1 = 0.f;
  for (int i = threadIdx.x; i < a.vocab; i += 1024) {
    const float d = ld_elem<DT>(x, i) - M;
    const float e = i == at ? 0.f : expf(d);
    r += e;
    s1 += e > 0.f ? d * e : 0.f;
  }
  r = block_sum(r, s_f);
  s1 = block_sum(s1, s_f);
  const float lz = log1pf(r);
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[row] = none ? NAN : lz - s1 / (1.f + r);
    if (a.logprob) {
      const int t = a.tokens[row];
      a.logprob[row] = t < 0 ? 0.f : none || t >= a.vocab ? NAN : ld_elem<DT>(x, t) - M - lz;
    }
  }
  for (int k = 0; k < a.top; ++k) {
    if (k) {
      uint64_t best = 0;
      for (int i = threadIdx.x; i < a.vocab; i += 1024) {
        const uint64_t key = logit_key(ld_elem<DT>(x, i), i);
        if (key < top) best = max(best, key);
      }
      top = block_max(best, s_k);
    }
    if (threadIdx.x == 0) {
      if (a.top_ids) a.top_ids[row * a.top + k] = none ? -1 : key_index(top);
      if (a.top_logprobs) a.top_logprobs[row * a.top + k] = none ? NAN : key_value(top) - M - lz;
    }
  }
}

}  // namespace

hipError_t launch_logprobs(int dtype, const LogprobArgs &a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  const dim3 grid((uint32_t)a.rows), block(1024);
  switch (dtype) {
    case HS_F32: HS_LAUNCH(k_logprobs<HS_F32>, grid, block, 0, st, a); break;
    case HS_F16: HS_LAUNCH(k_logprobs<HS_F16>, grid, block, 0, st, a); break;
    case HS_BF16: HS_LAUNCH(k_logprobs<HS_BF16>, grid, block, 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hs
