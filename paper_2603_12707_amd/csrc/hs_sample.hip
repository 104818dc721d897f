// hs_sample.hip — a token drawn for each row of logits from a given uniform
// number, after temperature, top-k, top-p and min-p (gfx950).
//
// In falling order of the logits (the lowest index first among equals) every
// one of the three leaves a beginning of the row, and the draw is a walk down
// it.  Weights are e^((x - max) / T) in 64 bits: a draw falls on a token by the sum
// of up to all the weights before it, and in 32 bits one in some ten thousand would
// fall on its neighbour.
//
// No row is sorted.  A first launch cuts rows into parts that stay in registers
// and sums the weights of bins 1/16 wide in x / T, aligned to the same grid in every
// part.  A second one, a work group for a row, joins the bins, finds those in which
// the three borders and the draw lie, gathers their logits from the row, and sorts
// those few.
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

// 16 bytes of elements: rows start anywhere
template <int DT>
struct __attribute__((packed, aligned(sizeof(typename Ty<DT>::S)))) Loose {
  u32x4 w;
};
template <int DT>
__device__ __forceinline__ u32x4 ld_loose(const void *p) {
  return ((const Loose<DT> *)p)->w;
}

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
  r.u = u < 0.f ? 0.0 : u >= 1.f ? 1.0 - 0x1p-24 : (double)u;
  return r;
}
// the least float that min_p leaves, M at most
__device__ __forceinline__ float min_p_floor(const SampleRow &p, float M) {
  const double least = fmin((double)M + log((double)p.min_p) / p.inv_t, (double)M);
  float f = (float)fmax(least, -(double)FLT_MAX);
  if ((double)f < least) f = key_float(value_key(f) + 1);
  return f;
}

// Where a sum of weights and a border are equal by the definition (equal logits, a
// border at a whole number of them) roundings leave them this part of the row's
// weight apart at most, and they are taken as equal.
constexpr double SM_EQUAL = 0x1p-44;

// ---------------------------------------------------------------------------
// bins
// ---------------------------------------------------------------------------
// Bin b holds the logits with floor(x * 16 / T) = b; the product is rounded, but
// alike everywhere, and rounding keeps the order.  Counted from the bin of a
// part's (a row's) largest downward, the last of SM_BINS holds all that is lower.
constexpr int SM_BINS = 512;
constexpr double SM_FINE = 16.0;
// A weight relative to its bin's upper end, in (e^-1/16, 1], as a whole multiple of
// 2^-49: a part's 2^14 of them sum in 63 bits, in any order to the same.
constexpr double SM_ONE = 8.0;  // the number whose last place is 2^-49
__device__ __forceinline__ uint64_t bin_weight(double xs, double b) {
#pragma clang fp contract(off)  // xs is the rounded product that b comes from
  const double r = (xs - (b + 1.0)) * (1.0 / SM_FINE);  // -1/16 .. 0
  // e^r, the series' next term is 6e-15
  double e = __builtin_fma(r, 1.0 / 5040, 1.0 / 720);
  e = __builtin_fma(e, r, 1.0 / 120);
  e = __builtin_fma(e, r, 1.0 / 24);
  e = __builtin_fma(e, r, 1.0 / 6);
  e = __builtin_fma(e, r, 0.5);
  e = __builtin_fma(e, r, 1.0);
  e = __builtin_fma(e, r, 1.0);
  return __builtin_bit_cast(uint64_t, e + SM_ONE) - __builtin_bit_cast(uint64_t, SM_ONE);
}
// The same in the last bin, where all lies 32 below the part's largest: its whole
// sum is 1e-10 of that one's weight, and fp32 does for it.
__device__ __forceinline__ uint64_t tail_weight(double xs, double b) {
#pragma clang fp contract(off)
  const float e = __expf((float)fmax((xs - (b + 1.0)) * (1.0 / SM_FINE), -200.0));
  return __builtin_bit_cast(uint64_t, (double)e + SM_ONE) - __builtin_bit_cast(uint64_t, SM_ONE);
}

struct SamplePart {
  double top;     // the bin of its largest
  uint64_t best;  // that one's value key and ~index
  uint64_t odd;   // whether it holds a NaN or +inf
};
// a row's workspace: for each part its SamplePart, the bins' weights, their numbers
constexpr int64_t SM_PART_BYTES = sizeof(SamplePart) + SM_BINS * 12;
__host__ __device__ inline char *sample_ws(void *ws, int64_t row, int parts, int part) {
  return (char *)ws + (row * parts + part) * SM_PART_BYTES;
}

constexpr int SP_THREADS = 256, SP_WAVES = SP_THREADS / 64;
constexpr int SP_WORDS = 32;  // 4-byte words of a thread

// largest of the work group's values, in every thread
template <int WAVES>
__device__ __forceinline__ uint64_t block_most(uint64_t v, uint64_t *s_tmp) {
  for (int o = 32; o; o >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) v = max(v, s_tmp[w]);
  return v;
}

// A part of a row: its largest, and its bins.  One read of the logits, which stay
// in registers; the sums go through LDS, whole numbers that are added in any order.
template <int DT>
__global__ __launch_bounds__(SP_THREADS) void k_sample_parts(SampleArgs a) {
  constexpr int B = DT == HS_F32 ? 4 : 2, PER = 4 / B, PART = SP_THREADS * SP_WORDS * PER;
  __shared__ unsigned long long s_mass[SM_BINS];
  __shared__ uint32_t s_count[SM_BINS];
  __shared__ uint64_t s_tmp[SP_WAVES];
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts), tid = threadIdx.x;
  const SampleRow p = sample_row(a, a.act ? a.act[row] : row);
  const int first = part * PART, n = min(PART, a.vocab - first);
  const char *x = (const char *)a.logits + (row * a.ld + first) * B;
  // chunks of 16 bytes to a thread
  constexpr int CE = 16 / B, NC = SP_WORDS / 4;
  constexpr uint32_t NEG = DT == HS_F32 ? 0xFF800000u : DT == HS_F16 ? 0xFC00FC00u : 0xFF80FF80u;  // -inf
  u32x4 w[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int i = (c * SP_THREADS + tid) * CE;
    w[c] = u32x4{NEG, NEG, NEG, NEG};
    if (n == PART || i + CE <= n) {
      w[c] = ld_loose<DT>(x + i * B);
    } else {
#pragma unroll
      for (int e = 0; e < CE; ++e)
        if (i + e < n) {
          if constexpr (DT == HS_F32) {
            w[c][e] = ((const uint32_t *)x)[i + e];
          } else {
            const uint32_t h = ((const uint16_t *)x)[i + e];
            w[c][e / 2] = e & 1 ? (w[c][e / 2] & 0xFFFFu) | h << 16 : (w[c][e / 2] & 0xFFFF0000u) | h;
          }
        }
    }
  }
  const auto value = [&](int i) {  // element i of the thread's
    const uint32_t u = w[i / CE][i % CE / PER];
    if constexpr (DT == HS_F32) return __uint_as_float(u);
    else return i & 1 ? hi_f32<DT>(u) : lo_f32<DT>(u);
  };
  for (int i = tid; i < SM_BINS; i += SP_THREADS) {
    s_mass[i] = 0;
    s_count[i] = 0;
  }
  float m = -INFINITY;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < SP_WORDS * PER; ++i) {
    m = fmaxf(m, value(i));
    odd |= !(value(i) < INFINITY);
  }
  int at = INT32_MAX;
#pragma unroll
  for (int i = SP_WORDS * PER - 1; i >= 0; --i)
    if (value(i) == m) at = first + ((i / CE) * SP_THREADS + tid) * CE + i % CE;
  // (a part that ends early has -inf behind its end, which is not looked for)
  const uint64_t best = block_most<SP_WAVES>((uint64_t)value_key(m) << 32 | (uint32_t)~at, s_tmp);
  const bool any_odd = __syncthreads_or(odd);
  const float top = key_float((uint32_t)(best >> 32));
  const double s = p.inv_t * SM_FINE, b0 = floor((double)top * s);
  char *ws = sample_ws(a.ws, row, a.parts, part);
  if (tid == 0) *(SamplePart *)ws = SamplePart{b0, best, any_odd ? 1ull : 0ull};
  if (p.bad || p.greedy || any_odd || top == -INFINITY) return;
  const bool counts = p.top_k < a.vocab;
#pragma unroll
  for (int i = 0; i < SP_WORDS * PER; ++i) {
    const float v = value(i);
    const double xs = (double)v * s, b = floor(xs);
    const double d = b0 - b;
    if (d < SM_BINS - 1) {
      const int g = (int)d;
      atomicAdd(&s_mass[g], (unsigned long long)bin_weight(xs, b));
      if (counts) atomicAdd(&s_count[g], 1u);
    } else if (v > -INFINITY) {
      atomicAdd(&s_mass[SM_BINS - 1], (unsigned long long)tail_weight(xs, b0 - (SM_BINS - 1)));
      if (counts) atomicAdd(&s_count[SM_BINS - 1], 1u);
    }
  }
  __syncthreads();
  uint64_t *mass = (uint64_t *)(ws + sizeof(SamplePart));
  uint32_t *count = (uint32_t *)(mass + SM_BINS);
  for (int i = tid; i < SM_BINS; i += SP_THREADS) {
    mass[i] = s_mass[i];
    if (counts) count[i] = s_count[i];
  }
}

// ---------------------------------------------------------------------------
// draws
// ---------------------------------------------------------------------------
constexpr int SD_THREADS = 512, SD_WAVES = SD_THREADS / 64;
constexpr int SD_LIST = 4096;  // logits that are sorted
static_assert(SD_THREADS == SM_BINS, "a thread for each bin");

struct DrawLds {
  union {
    uint64_t list[SD_LIST];       // value key and ~index, sorted downward
    struct {                      // a row by itself
      unsigned long long mass[256];
      uint32_t count[256];
    } radix;
  };
  uint64_t sorted[1024];          // (ranked by counting)
  double upto[SM_BINS], before[SM_BINS], scale[SM_BINS];
  int count_before[SM_BINS];
  int start[SM_BINS];
  double list_before[SM_BINS];
  uint8_t need[SM_BINS];
  double tmp[SD_WAVES];
  uint64_t tmp_u[SD_WAVES];
  int tmp_n[SD_WAVES];
  int bk, bp0, bp1, bt0, bt1, n, pick, last;
  uint32_t digit;
  double above;
  uint64_t above_u, ties;
};

// sums over the threads before this one and up to it
__device__ __forceinline__ double block_scan(double v, double *s_tmp, double &total, double &before) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s_tmp[wave] = x;
  __syncthreads();
  double base = 0.0;
  total = 0.0;
#pragma unroll
  for (int w = 0; w < SD_WAVES; ++w) {
    if (w < wave) base += s_tmp[w];
    total += s_tmp[w];
  }
  const double prev = __shfl_up(x, 1);
  before = lane ? base + prev : base;
  return base + x;
}
__device__ __forceinline__ int block_scan(int v, int *s_tmp) {  // up to this thread
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();
  if (lane == 63) s_tmp[wave] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SD_WAVES; ++w)
    if (w < wave) v += s_tmp[w];
  return v;
}
__device__ __forceinline__ double block_largest(double v, double *s_tmp) {
  for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SD_WAVES; ++w) v = fmax(v, s_tmp[w]);
  return v;
}

// A row by itself, whatever it holds: each border and the draw by four passes over
// the row, a byte of the value each, over sums of the weights in whole multiples of
// a unit that no sum of the row overflows.  For rows whose border bins hold more than
// SD_LIST logits (flat ones, or many equal ones), or lie in the last bin.
template <int DT>
__device__ __attribute__((noinline)) void draw_alone(const SampleArgs &a, DrawLds &lds, const SampleRow &p, int64_t row,
                                                     int64_t slot, float M) {
  const char *x = (const char *)a.logits + row * a.ld * (DT == HS_F32 ? 4 : 2);
  const int V = a.vocab, tid = threadIdx.x;
  const int bits = 62 - (32 - __clz(V));  // V * 2^bits stays below 2^62
  const double unit = (double)(1ull << bits), least = (double)M;
  const auto weight = [&](float v) { return (uint64_t)rint(exp(((double)v - least) * p.inv_t) * unit); };
  // the value at which `cross` (of the number and the weight up to it) becomes true
  // first; all above it, and its ties
  uint32_t edge = 0;
  uint64_t above = 0, number = 0, ties = 0;
  const auto find = [&](auto cross, bool by_weight) {
    edge = 0;
    above = number = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) {
        lds.radix.mass[tid] = 0;
        lds.radix.count[tid] = 0;
      }
      __syncthreads();
      for (int i = tid; i < V; i += SD_THREADS) {
        const float v = ld_elem<DT>(x, i);
        const uint32_t k = value_key(v);
        if (shift == 24 || (k >> (shift + 8)) == (edge >> (shift + 8))) {
          atomicAdd(&lds.radix.count[k >> shift & 255], 1u);
          atomicAdd(&lds.radix.mass[k >> shift & 255], (unsigned long long)weight(v));
        }
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t m = above, n = number;
        int d = 255, last = -1;
        uint64_t lm = m, ln = n;
        for (; d >= 0; --d) {
          const uint64_t c = lds.radix.count[d];
          if (!c) continue;
          if (!by_weight || lds.radix.mass[d]) last = d, lm = m, ln = n;
          if (cross(n + c, m + lds.radix.mass[d])) break;
          n += c;
          m += lds.radix.mass[d];
        }
        if (d < 0) d = last, m = lm, n = ln;  // (rounding: the last that counts)
        lds.digit = (uint32_t)d;
        lds.above_u = m;
        lds.tmp_u[0] = n;
        lds.ties = lds.radix.count[d];
      }
      __syncthreads();
      edge |= lds.digit << shift;
      above = lds.above_u;
      number = lds.tmp_u[0];
      ties = lds.ties;
    }
  };
  if (p.top_k < V) {
    find([&](uint64_t n, uint64_t) { return n >= (uint64_t)p.top_k; }, false);
    ties = (uint64_t)p.top_k - number;
  } else {
    find([&](uint64_t n, uint64_t) { return n >= (uint64_t)V; }, false);
  }
  uint64_t total = above + ties * weight(key_float(edge));
  uint64_t kept = number + ties;  // of the row's beginning
  if (p.top_p < 1.f) {
    const double want = fmax((double)p.top_p * (double)total * (1 - SM_EQUAL), 0.5);
    const uint64_t most = kept;
    find([&](uint64_t, uint64_t m) { return (double)m >= want; }, true);
    const uint64_t w = weight(key_float(edge));
    const double n = ceil((want - (double)above) / (double)w);
    ties = min(n >= (double)ties ? ties : n > 1.0 ? (uint64_t)n : 1ull, most - number);
    total = above + ties * w;
    kept = number + ties;
  }
  if (p.min_p > 0.f) {
    const uint32_t k = value_key(min_p_floor(p, M));
    // how many reach it, and their weight
    __syncthreads();
    if (tid == 0) lds.radix.mass[0] = lds.radix.mass[1] = 0;
    __syncthreads();
    unsigned long long n = 0, m = 0;
    for (int i = tid; i < V; i += SD_THREADS) {
      const float v = ld_elem<DT>(x, i);
      if (value_key(v) >= k) {
        ++n;
        m += weight(v);
      }
    }
    atomicAdd(&lds.radix.mass[0], n);
    atomicAdd(&lds.radix.mass[1], m);
    __syncthreads();
    if (lds.radix.mass[0] < kept) {
      kept = lds.radix.mass[0];
      total = lds.radix.mass[1];
    }
  }
  const double want = (p.u + SM_EQUAL) * (double)total;
  find([&](uint64_t, uint64_t m) { return (double)m > want; }, true);
  const uint64_t w = weight(key_float(edge));
  const double nth = floor((want - (double)above) / (double)w);
  ties = min(ties, kept - number);
  int64_t left = nth >= (double)ties ? (int64_t)ties - 1 : nth > 0.0 ? (int64_t)nth : 0;
  // the left-th index that holds it
  for (int b = 0; b < V; b += SD_THREADS) {
    const int i = b + tid;
    const bool is = i < V && value_key(ld_elem<DT>(x, i)) == edge;
    const uint64_t in = __ballot(is);
    __syncthreads();
    if ((tid & 63) == 0) lds.tmp_n[tid >> 6] = (int)__popcll(in);
    __syncthreads();
    int before = 0, all = 0;
    for (int o = 0; o < SD_WAVES; ++o) {
      if (o < tid >> 6) before += lds.tmp_n[o];
      all += lds.tmp_n[o];
    }
    if (left < all) {
      if (is && before + (int)__popcll(in & ((1ull << (tid & 63)) - 1)) == left) {
        a.tokens[slot] = i;
        if (a.logprob) a.logprob[row] = (float)log((double)w / (double)total);
      }
      return;
    }
    left -= all;
  }
}

// A row's draw.  The sums of its bins say in which bins top-k and min-p end, and
// between which bounds the weight that top-k leaves, hence in which bins top-p ends,
// hence between which bounds the weight that is drawn from, and so the draw.  The
// logits of those bins (a few hundred, mostly) are gathered from the row and sorted;
// with the sums of the bins before theirs that gives each its place and the weight
// up to it, and with these the borders and the draw.  Bounds are wider by 1e-12 than
// sums are off.
template <int DT>
__global__ __launch_bounds__(SD_THREADS) void k_sample_draw(SampleArgs a) {
  constexpr int B = DT == HS_F32 ? 4 : 2, CE = 16 / B;
  __shared__ DrawLds lds;
  const int64_t row = blockIdx.x, slot = a.act ? a.act[row] : row;
  const int tid = threadIdx.x, V = a.vocab;
  const SampleRow p = sample_row(a, slot);
  // the parts' largest
  uint64_t best = 0, odd = 0;
  for (int i = tid; i < a.parts; i += SD_THREADS) {
    const SamplePart h = *(const SamplePart *)sample_ws(a.ws, row, a.parts, i);
    best = max(best, h.best);
    odd |= h.odd;
  }
  best = block_most<SD_WAVES>(best, lds.tmp_u);
  const bool any_odd = __syncthreads_or(odd != 0);
  const float M = key_float((uint32_t)(best >> 32));
  if (p.bad || any_odd || M == -INFINITY || p.greedy) {
    if (tid == 0) {
      const bool none = p.bad || any_odd || M == -INFINITY;
      a.tokens[slot] = none ? -1 : (int)~(uint32_t)best;
      if (a.logprob) a.logprob[row] = none ? NAN : 0.f;
    }
    return;
  }
  const double s = p.inv_t * SM_FINE, b0 = floor((double)M * s);
  const bool cut_k = p.top_k < V, cut_p = p.top_p < 1.f, cut_m = p.min_p > 0.f;

  // the row's bins, bin tid of each thread: from part i's bin tid - off
  const double scale = exp(-(double)tid / SM_FINE) * 0x1p-49;
  double w = 0.0;
  int count = 0;
  for (int i = 0; i < a.parts; ++i) {
    const char *ws = sample_ws(a.ws, row, a.parts, i);
    const SamplePart *h = (const SamplePart *)ws;
    if ((uint32_t)(h->best >> 32) == value_key(-INFINITY)) continue;
    const uint64_t *mass = (const uint64_t *)(ws + sizeof(SamplePart));
    const uint32_t *cnt = (const uint32_t *)(mass + SM_BINS);
    const int off = (int)fmin(b0 - h->top, (double)SM_BINS);
    if (tid < SM_BINS - 1 && tid >= off) {
      w += (double)mass[tid - off] * scale;
      if (cut_k) count += (int)cnt[tid - off];
    }
  }
  // what lies in the last one: bins of parts that reach past it
  double far = 0.0;
  int far_count = 0;
  for (int i = 0; i < a.parts; ++i) {
    const char *ws = sample_ws(a.ws, row, a.parts, i);
    const SamplePart *h = (const SamplePart *)ws;
    if ((uint32_t)(h->best >> 32) == value_key(-INFINITY)) continue;
    const uint64_t *mass = (const uint64_t *)(ws + sizeof(SamplePart));
    const uint32_t *cnt = (const uint32_t *)(mass + SM_BINS);
    const double off = b0 - h->top;
    if (tid + off >= SM_BINS - 1) {
      far += (double)mass[tid] * (exp(-(tid + off) / SM_FINE) * 0x1p-49);
      if (cut_k) far_count += (int)cnt[tid];
    }
  }
  double total, before;
  (void)block_scan(far, lds.tmp, total, before);
  if (tid == SM_BINS - 1) w = total;
  const double upto = block_scan(w, lds.tmp, total, before);
  lds.upto[tid] = upto;
  lds.before[tid] = before;
  lds.scale[tid] = scale;
  lds.need[tid] = 0;
  int count_upto = 0;
  if (cut_k) {
    // (-inf is not counted: a border past the last bin's numbers lies among them)
    const int fars = block_scan(far_count, lds.tmp_n);
    if (tid == SM_BINS - 1) count = fars;
    count_upto = block_scan(count, lds.tmp_n);
    lds.count_before[tid] = count_upto - count;
  }
  if (tid == 0) {
    lds.bk = lds.bp0 = lds.bp1 = lds.bt0 = lds.bt1 = SM_BINS;
    lds.n = 0;
    lds.pick = INT32_MAX;
    lds.last = -1;
  }
  __syncthreads();
  if (cut_k && count && count_upto >= p.top_k && count_upto - count < p.top_k) lds.bk = tid;
  __syncthreads();
  const int bk = lds.bk;  // SM_BINS: none
  const auto bound = [&](int b, bool after) {  // weight before, or after, bin b
    return b >= SM_BINS ? total : after ? lds.upto[b] : lds.before[b];
  };
  const double wider = 1e-12;
  if (cut_p) {
    const double lo = fmax((double)p.top_p * bound(bk, false) * (1 - wider), 0x1p-1070),
                 hi = fmax((double)p.top_p * bound(bk, true) * (1 + wider), 0x1p-1070);
    if (upto >= lo && before < lo) lds.bp0 = tid;
    if (upto >= hi && before < hi) lds.bp1 = tid;
  }
  const float floor_x = cut_m ? min_p_floor(p, M) : -INFINITY;
  const int bm = cut_m ? (int)fmin(b0 - floor((double)floor_x * s), (double)(SM_BINS - 1)) : SM_BINS;
  __syncthreads();
  const int bp0 = lds.bp0, bp1 = lds.bp1;
  const int e0 = min(bm, min(bk, bp0)), e1 = min(bm, min(bk, bp1));
  const double lo = p.u * bound(e0, false) * (1 - wider), hi = p.u * bound(e1, true) * (1 + wider);
  if (upto > lo && before <= lo) lds.bt0 = tid;
  if (upto > hi && before <= hi) lds.bt1 = tid;
  __syncthreads();
  const int bt0 = min(lds.bt0, e1), bt1 = min(lds.bt1, e1);
  const bool need = (tid == bk && (cut_p || bk <= e1)) || (cut_p && tid >= bp0 && tid <= bp1 && tid <= e1) ||
                    (tid == bm && bm <= e1) || (tid >= bt0 && tid <= bt1);
  if (need) lds.need[tid] = 1;
  // the last bin is not gathered, nor is what no bin holds
  const bool past = (need && tid == SM_BINS - 1) || bt1 >= SM_BINS || (cut_p && bp1 >= SM_BINS) ||
                    (cut_m && bm >= SM_BINS - 1 && bm <= e1);
  if (__syncthreads_or(past)) {
    draw_alone<DT>(a, lds, p, row, slot, M);
    return;
  }
  // the lowest bin that is asked for
  const int lowest = (int)block_most<SD_WAVES>(need ? (uint64_t)tid : 0, lds.tmp_u);
  // (a first sieve: a bin and more lower, for the roundings)
  const double edge = (b0 - lowest - 1.0) / s;
  const float sieve = (float)fmax(edge - fabs(edge) * 1e-6, -(double)FLT_MAX);
  const char *x = (const char *)a.logits + row * a.ld * B;
  const auto take = [&](float v, int i) {
    if (v >= sieve) {
      const double d = b0 - floor((double)v * s);
      if (d < SM_BINS - 1 && lds.need[(int)d]) {
        const int at = atomicAdd(&lds.n, 1);
        if (at < SD_LIST) lds.list[at] = (uint64_t)value_key(v) << 32 | (uint32_t)~i;
      }
    }
  };
  const int chunks = V / CE;
  for (int c = tid; c < chunks; c += 4 * SD_THREADS) {
    u32x4 q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = ld_loose<DT>(x + (int64_t)min(c + u * SD_THREADS, chunks - 1) * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (c + u * SD_THREADS < chunks) {
        float f[CE];
        unpack<DT>(q[u], f);
#pragma unroll
        for (int e = 0; e < CE; ++e) take(f[e], (c + u * SD_THREADS) * CE + e);
      }
  }
  for (int i = chunks * CE + tid; i < V; i += SD_THREADS) take(ld_elem<DT>(x, i), i);
  __syncthreads();
  const int n = lds.n;
  if (n > SD_LIST) {
    __syncthreads();
    draw_alone<DT>(a, lds, p, row, slot, M);
    return;
  }
  const uint64_t *sorted = lds.list;
  if (n <= 1024) {
    for (int i = tid; i < n; i += SD_THREADS) {
      const uint64_t mine = lds.list[i];
      int rank = 0;
      for (int o = 0; o < n; ++o) rank += lds.list[o] > mine;
      lds.sorted[rank] = mine;
    }
    sorted = lds.sorted;
  } else {
    int m = 2048;
    while (m < n) m *= 2;
    for (int i = n + tid; i < m; i += SD_THREADS) lds.list[i] = 0;
    for (int k = 2; k <= m; k *= 2)
      for (int j = k / 2; j; j /= 2) {
        __syncthreads();
        for (int i = tid; i < m / 2; i += SD_THREADS) {
          const int lo_i = i / j * 2 * j + i % j, hi_i = lo_i + j;
          const uint64_t u = lds.list[lo_i], v = lds.list[hi_i];
          if ((u < v) == ((lo_i & k) == 0)) {
            lds.list[lo_i] = v;
            lds.list[hi_i] = u;
          }
        }
      }
  }
  __syncthreads();
  // each thread's run of the list: weights, and the weight before it in the list
  constexpr int PER = SD_LIST / SD_THREADS;
  const int run = (n + SD_THREADS - 1) / SD_THREADS, i0 = min(n, tid * run), mine = min(n, i0 + run) - i0;
  double wt[PER], sum = 0.0;
  int bin[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    wt[i] = 0.0;
    bin[i] = 0;
    if (i < mine) {
      const double xs = (double)key_float((uint32_t)(sorted[i0 + i] >> 32)) * s, b = floor(xs);
      bin[i] = (int)(b0 - b);
      wt[i] = (double)bin_weight(xs, b) * lds.scale[bin[i]];
      sum += wt[i];
    }
  }
  double list_total, run_before;
  (void)block_scan(sum, lds.tmp, list_total, run_before);
  {
    double c = run_before;
    int prev = -1;
    if (mine && i0) prev = (int)(b0 - floor((double)key_float((uint32_t)(sorted[i0 - 1] >> 32)) * s));
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < mine) {
        if (bin[i] != prev) {
          lds.start[bin[i]] = i0 + i;
          lds.list_before[bin[i]] = c;
        }
        prev = bin[i];
        c += wt[i];
      }
  }
  __syncthreads();
  // weight before each and its place in the row
  double ahead[PER];
  bool in[PER];
  double c = run_before, kept = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    in[i] = i < mine;
    ahead[i] = 0.0;
    if (in[i]) {
      ahead[i] = lds.before[bin[i]] + (c - lds.list_before[bin[i]]);
      c += wt[i];
      if (cut_k) in[i] = lds.count_before[bin[i]] + (i0 + i - lds.start[bin[i]]) < p.top_k;
      if (in[i] && bin[i] == bk) kept = fmax(kept, ahead[i] + wt[i]);
    }
  }
  if (cut_p) {
    const double zk = bk < SM_BINS ? fmax(block_largest(kept, lds.tmp), lds.before[bk]) : total;
    const double want = fmax((double)p.top_p * zk * (1 - SM_EQUAL), 0x1p-1070);
#pragma unroll
    for (int i = 0; i < PER; ++i) in[i] = in[i] && ahead[i] < want;
  }
  kept = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (in[i]) {
      in[i] = key_float((uint32_t)(sorted[i0 + i] >> 32)) >= floor_x;
      if (in[i]) kept = fmax(kept, ahead[i] + wt[i]);
    }
  const double z = e1 < SM_BINS ? fmax(block_largest(kept, lds.tmp), bound(e0, false)) : total;
  const double want = (p.u + SM_EQUAL) * z;
  int pick = INT32_MAX, last = -1;
#pragma unroll
  for (int i = PER - 1; i >= 0; --i)
    if (in[i] && wt[i] > 0.0) {
      last = max(last, i0 + i);
      if (ahead[i] + wt[i] > want) pick = i0 + i;
    }
  if (pick < INT32_MAX) atomicMin(&lds.pick, pick);
  if (last >= 0) atomicMax(&lds.last, last);
  __syncthreads();
  const int at = lds.pick < INT32_MAX ? lds.pick : lds.last;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i < mine && i0 + i == at) {
      a.tokens[slot] = (int)~(uint32_t)sorted[at];
      if (a.logprob) a.logprob[row] = (float)log(wt[i] / z);
    }
}

inline int sample_parts(int vocab, int dtype) {
  const int part = SP_THREADS * SP_WORDS * (dtype == HS_F32 ? 1 : 2);
  return (int)(((int64_t)vocab + part - 1) / part);
}

template <int DT>
hipError_t sample_launch(SampleArgs a, hipStream_t st) {
  a.parts = sample_parts(a.vocab, DT);
  HS_LAUNCH((k_sample_parts<DT>), dim3((uint32_t)(a.rows * a.parts)), dim3(SP_THREADS), 0, st, a);
  HS_LAUNCH((k_sample_draw<DT>), dim3((uint32_t)a.rows), dim3(SD_THREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace

uint64_t sample_workspace(int64_t rows, int vocab) {
  return (uint64_t)rows * sample_parts(vocab, HS_F32) * SM_PART_BYTES;
}

hipError_t launch_sample(int dtype, const SampleArgs &a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  switch (dtype) {
    case HS_F32: return sample_launch<HS_F32>(a, st);
    case HS_F16: return sample_launch<HS_F16>(a, st);
    case HS_BF16: return sample_launch<HS_BF16>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace hs
