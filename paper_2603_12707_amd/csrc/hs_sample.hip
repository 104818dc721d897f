// hs_sample.hip — a token drawn for each row of logits from a given uniform
// number, after temperature, top-k, top-p and min-p (gfx950).
//
// In falling order of the logits (the lowest index first among equals) every
// one of the three leaves a beginning of the row, and the draw is a walk down
// it.  A beginning is held as a value and a number: all logits above the value,
// and the first so many of those equal to it.  Weights are e^((x - max) / T) in 64
// bits: a draw falls on a token by the sum of up to all the weights before it, and
// in 32 bits one in some ten thousand would fall on its neighbour.
#include "hs_device.h"

#include <algorithm>
#include <cfloat>

namespace hs {
namespace {

using namespace dev;

// order of the values as whole numbers; -0 counts as 0
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k); }

constexpr int SM_THREADS = 1024, SM_WAVES = SM_THREADS / 64;

// A row's parameters, and whether they and u are numbers that make a draw.
struct SampleRow {
  double inv_t, u;
  float top_p, min_p;
  int top_k;
  bool greedy, bad;
};
__device__ __forceinline__ SampleRow sample_row(const SampleArgs &a, int64_t at) {
  SampleRow r;
  const float t = a.temperature ? a.temperature[at] : 1.f, u = a.u[at];
  r.top_p = a.top_p ? a.top_p[at] : 1.f;
  r.min_p = a.min_p ? a.min_p[at] : 0.f;
  const int k = a.top_k ? a.top_k[at] : 0;
  r.top_k = k <= 0 || k > a.vocab ? a.vocab : k;
  r.bad = !(t >= 0.f) || t == INFINITY || r.top_p != r.top_p || r.min_p != r.min_p || u != u;
  r.greedy = t == 0.f;
  r.inv_t = 1.0 / (double)t;
  r.u = u < 0.f ? 0.0 : u >= 1.f ? 1.0 - 0x1p-53 : (double)u;
  return r;
}

// ---------------------------------------------------------------------------
// a row by itself
// ---------------------------------------------------------------------------
template <class T, class Op>
__device__ __forceinline__ T block_reduce(T v, T *s, Op op) {
  for (int o = 32; o; o >>= 1) v = op(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < SM_WAVES; ++w) v = op(v, s[w]);
  return v;
}

// The whole draw by bisection over the 32 bits of a value, a pass over the row for
// each: every row is drawn from rightly, whatever it holds.
template <int DT>
__global__ __launch_bounds__(SM_THREADS) void k_sample_row(SampleArgs a) {
  __shared__ double s_d[SM_WAVES];
  __shared__ unsigned long long s_u[SM_WAVES];
  const int64_t row = blockIdx.x, slot = a.act ? a.act[row] : row;
  const char *x = (const char *)a.logits + row * a.ld * (DT == HS_F32 ? 4 : 2);
  const int V = a.vocab, tid = threadIdx.x;
  const SampleRow p = sample_row(a, slot);
  const auto add = [](double u, double v) { return u + v; };
  const auto addn = [](unsigned long long u, unsigned long long v) { return u + v; };
  const auto most = [](unsigned long long u, unsigned long long v) { return u > v ? u : v; };

  // the first of the largest, and whether the row has a distribution
  unsigned long long top = 0, odd = 0;
  for (int i = tid; i < V; i += SM_THREADS) {
    const float v = ld_elem<DT>(x, i);
    odd |= v != v || v == INFINITY;
    top = most(top, (unsigned long long)value_key(v) << 32 | (uint32_t)~i);
  }
  odd = block_reduce(odd, s_u, most);
  top = block_reduce(top, s_u, most);
  const uint32_t kmax = (uint32_t)(top >> 32);
  const float M = key_float(kmax);
  if (p.bad || odd || M == -INFINITY) {
    if (tid == 0) {
      a.tokens[slot] = -1;
      if (a.logprob) a.logprob[row] = NAN;
    }
    return;
  }
  if (p.greedy) {
    if (tid == 0) {
      a.tokens[slot] = (int)~(uint32_t)top;
      if (a.logprob) a.logprob[row] = 0.f;
    }
    return;
  }
  const auto weight = [&](float v) { return exp(((double)v - (double)M) * p.inv_t); };
  const auto count = [&](uint32_t from) {
    unsigned long long n = 0;
    for (int i = tid; i < V; i += SM_THREADS) n += value_key(ld_elem<DT>(x, i)) >= from;
    return (int64_t)block_reduce(n, s_u, addn);
  };
  const auto mass = [&](uint32_t from) {
    double z = 0.0;
    for (int i = tid; i < V; i += SM_THREADS) {
      const float v = ld_elem<DT>(x, i);
      if (value_key(v) >= from) z += weight(v);
    }
    return block_reduce(z, s_d, add);
  };
  // the beginning that is left: values above `edge`, and `ties` of those equal to it
  uint32_t edge = 0;
  int64_t ties = V;
  if (p.top_k < V) {
    for (int b = 31; b >= 0; --b)
      if (count(edge | 1u << b) >= p.top_k) edge |= 1u << b;
    ties = p.top_k - count(edge + 1);
  } else {
    edge = value_key(-FLT_MAX);  // -inf is never drawn
    ties = count(edge) - count(edge + 1);
  }
  if (edge < value_key(-FLT_MAX)) {
    edge = value_key(-FLT_MAX);
    ties = count(edge) - count(edge + 1);
  }
  double above = mass(edge + 1);
  if (p.top_p < 1.f) {
    const double want = (double)p.top_p * (above + (double)ties * weight(key_float(edge)));
    if (above >= want) {
      uint32_t t = 0;
      for (int b = 31; b >= 0; --b)
        if ((t | 1u << b) <= kmax && mass(t | 1u << b) >= want) t |= 1u << b;
      edge = t;
      above = mass(edge + 1);
      ties = count(edge) - count(edge + 1);
    }
    const double n = ceil((want - above) / weight(key_float(edge)));
    ties = n >= (double)ties ? ties : n > 1.0 ? (int64_t)n : 1;
  }
  if (p.min_p > 0.f) {
    // the least float that is not below it
    const double least = fmin((double)M + log((double)p.min_p) / p.inv_t, (double)M);
    float f = (float)fmax(least, -(double)FLT_MAX);
    if ((double)f < least) f = key_float(value_key(f) + 1);
    const uint32_t k = value_key(f);
    if (k > edge) {
      edge = k;
      above = mass(edge + 1);
      ties = count(edge) - count(edge + 1);
    }
  }
  const double z = above + (double)ties * weight(key_float(edge)), want = p.u * z;
  uint32_t v = edge;
  if (above > want) {
    v = 0;
    for (int b = 31; b >= 0; --b)
      if ((v | 1u << b) <= kmax && mass(v | 1u << b) > want) v |= 1u << b;
    above = mass(v + 1);
    ties = count(v) - count(v + 1);
  }
  const double w = weight(key_float(v));
  const double nth = floor((want - above) / w);
  int64_t left = nth >= (double)ties ? ties - 1 : nth > 0.0 ? (int64_t)nth : 0;
  // the left-th index that holds it
  for (int b = 0; b < V; b += SM_THREADS) {
    const int i = b + tid;
    const bool is = i < V && value_key(ld_elem<DT>(x, i)) == v;
    const uint64_t in = __ballot(is);
    __syncthreads();
    if ((tid & 63) == 0) s_u[tid >> 6] = (unsigned long long)__popcll(in);
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int o = 0; o < SM_WAVES; ++o) {
      if (o < tid >> 6) before += (int64_t)s_u[o];
      all += (int64_t)s_u[o];
    }
    if (left < all) {
      if (is && before + (int64_t)__popcll(in & ((1ull << (tid & 63)) - 1)) == left) {
        a.tokens[slot] = i;
        if (a.logprob) a.logprob[row] = (float)(((double)key_float(v) - (double)M) * p.inv_t - log(z));
      }
      return;
    }
    left -= all;
  }
}

}  // namespace

uint64_t sample_workspace(int64_t rows, int vocab) {
  (void)rows;
  (void)vocab;
  return 0;
}

hipError_t launch_sample(int dtype, const SampleArgs &a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  const dim3 grid((uint32_t)a.rows), block(SM_THREADS);
  switch (dtype) {
    case HS_F32: HS_LAUNCH((k_sample_row<HS_F32>), grid, block, 0, st, a); break;
    case HS_F16: HS_LAUNCH((k_sample_row<HS_F16>), grid, block, 0, st, a); break;
    case HS_BF16: HS_LAUNCH((k_sample_row<HS_BF16>), grid, block, 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hs
