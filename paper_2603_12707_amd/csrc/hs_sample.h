// hs_sample.h — a token drawn for each row of logits from a given uniform
// number, after temperature, top-k, top-p and min-p (gfx950).  Included by
// hs_misc.hip.
//
// In falling order of the logits (the lowest index first among equals) every
// one of the three leaves a beginning of the row, and the draw is a walk down
// it.  Weights are e^((x - max) / T) in 64 bits: a draw falls on a token by the sum
// of up to all the weights before it, and in 32 bits one in some ten thousand would
// fall on its neighbour.
//
// No row is sorted.  The weights of bins 1/16 wide in x / T are summed, which says
// in which few of them the three borders and the draw lie; the logits of those are
// found in the row, cut into 64 parts a bin, and the same said of the parts; what is
// left is sorted.  A work group draws from a row, which it reads three or four times
// (L2 holds it).  The bins of long rows are summed by a launch before, in parts that
// stay in registers, on one grid.
#pragma once

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
  // (no weight reaches a min_p above 1: the first alone stays, whatever equals it)
  r.top_k = r.min_p > 1.f ? 1 : k <= 0 || k > a.vocab ? a.vocab : k;
  r.bad = !(t >= 0.f) || t == INFINITY || r.top_p != r.top_p || r.min_p != r.min_p || u != u;
  r.greedy = t == 0.f;
  r.inv_t = 1.0 / (double)t;
  r.u = u < 0.f ? 0.0 : u >= 1.f ? 1.0 - 0x1p-24 : (double)u;
  return r;
}
// the least float that min_p leaves, M at most (of a min_p above 1 top_k leaves the first)
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
constexpr int SM_BINS = 1024;
constexpr double SM_FINE = 16.0;
// A weight relative to its bin's upper end, in (e^-1/16, 1], as a whole multiple of
// 2^-48: a part's (or short row's) 2^15 of them at most sum in 64 bits, in any order to
// the same.
constexpr double SM_ONE = 16.0;  // the number whose last place is 2^-48
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
// The same in the last bin, where all lies 63 below the part's largest: its whole
// sum is 2^15 e^-63 of that one's weight at most, 2^-75, and fp32 does for it: its
// exponential is off by 2^-15 of itself (the argument, up to 200, is rounded to 2^-17 and its
// product with log2 e to 2^-16), 2^-90 of the part, where bounds are 1e-12 wide.  (Where a
// border lies among these the row is drawn from by itself.)
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

constexpr int SP_WORDS = 32;  // 4-byte words of a thread

// sum over the work group's threads up to this one
template <int WAVES>
__device__ __forceinline__ int block_scan(int v, int *s_tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();
  if (lane == 63) s_tmp[wave] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (w < wave) v += s_tmp[w];
  return v;
}
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

// Up to 32 words of logits for each of a work group's threads, in registers.
template <int DT, int THREADS>
struct Held {
  static constexpr int B = DT == HS_F32 ? 4 : 2, CE = 16 / B, PER = 4 / B, N = SP_WORDS * PER, ALL = THREADS * N;
  uint32_t w[SP_WORDS];
  int n;
  // n of them from x on; -inf past them
  __device__ __forceinline__ Held(const char *x, int n_) : n(n_) {
    constexpr uint32_t NEG = DT == HS_F32 ? 0xFF800000u : DT == HS_F16 ? 0xFC00FC00u : 0xFF80FF80u;
#pragma unroll
    for (int c = 0; c < SP_WORDS / 4; ++c) {
      const int i = (c * THREADS + (int)threadIdx.x) * CE;
      u32x4 t = {NEG, NEG, NEG, NEG};
      if (i + CE <= n) {
        t = ld_loose<DT>(x + i * B);
      } else {
#pragma unroll
        for (int e = 0; e < CE; ++e)
          if (i + e < n) {
            if constexpr (DT == HS_F32) {
              t[e] = ((const uint32_t *)x)[i + e];
            } else {
              const uint32_t h = ((const uint16_t *)x)[i + e];
              t[e / 2] = e & 1 ? (t[e / 2] & 0xFFFFu) | h << 16 : (t[e / 2] & 0xFFFF0000u) | h;
            }
          }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) w[4 * c + k] = t[k];
    }
  }
  // f(values of a chunk, the first one's index), in order
  template <class F>
  __device__ __forceinline__ void chunks(F f) {
#pragma unroll
    for (int c = 0; c < SP_WORDS / 4; ++c) {
      float v[CE];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // opaque from one use to the next: what is made of a word is made again, not
        // kept in registers
        asm volatile("" : "+v"(w[4 * c + k]));
      }
      unpack<DT>(u32x4{w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]}, v);
      f(v, (c * THREADS + (int)threadIdx.x) * CE);
    }
  }
};
// The same of a row in memory, of any length.
template <int DT, int THREADS>
struct Read {
  static constexpr int B = DT == HS_F32 ? 4 : 2, CE = 16 / B;
  const char *x;
  int n;
  template <class F>
  __device__ __forceinline__ void chunks(F f) const {
    const int whole = n / CE, tid = (int)threadIdx.x;
    constexpr int U = 4;  // loads in flight
    u32x4 q[U];
    for (int c = tid; c - tid < whole; c += U * THREADS) {
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = ld_loose<DT>(x + (int64_t)min(c + u * THREADS, whole - 1) * 16);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[CE];
        unpack<DT>(q[u], v);
        if (c + u * THREADS >= whole) {
#pragma unroll
          for (int e = 0; e < CE; ++e) v[e] = -INFINITY;
        }
        f(v, (c + u * THREADS) * CE);
      }
    }
    // what is left, less than a chunk
    float v[CE];
#pragma unroll
    for (int e = 0; e < CE; ++e) v[e] = -INFINITY;
    if (whole * CE + tid < n) v[0] = ld_elem<DT>(x, whole * CE + tid);
    f(v, whole * CE + tid);
  }
};

struct BinLds {
  unsigned long long mass[SM_BINS];
  uint32_t count[SM_BINS];
  uint64_t tmp[16];
  int tmp_n[16];
  int last;
};
// The largest of some logits (value key and ~index, counted from `first` on), and
// whether one is NaN or +inf.
template <class H, int THREADS>
__device__ __forceinline__ uint64_t row_best(H &h, int first, BinLds &lds, bool &odd) {
  float m = -INFINITY;
  int at = 0;
  odd = false;
  h.chunks([&](const float *v, int i) {
#pragma unroll
    for (int e = 0; e < H::CE; ++e) {
      odd |= !(v[e] < INFINITY);
      at = v[e] > m ? i + e : at;
      m = fmaxf(m, v[e]);
    }
  });
  odd = __syncthreads_or(odd);
  return block_most<THREADS / 64>((uint64_t)value_key(m) << 32 | (uint32_t)~(first + at), lds.tmp);
}
// Their bins from b0 down, in LDS.  The sums are of whole numbers, added in any
// order.  With top_k: among the largest of every chunk (16 bytes) there is a bin up
// to which top_k of them lie; what lies lower is left out.
template <class H, int THREADS>
__device__ __forceinline__ void row_bins(H &h, double s, double b0, int top_k, bool counts, BinLds &lds) {
  const int tid = threadIdx.x;
  for (int i = tid; i < SM_BINS; i += THREADS) {
    lds.mass[i] = 0;
    lds.count[i] = 0;
  }
  double most = INFINITY;
  __syncthreads();
  if (counts && top_k <= h.n / H::CE / 2) {
    h.chunks([&](const float *v, int) {
      float m = v[0];
#pragma unroll
      for (int e = 1; e < H::CE; ++e) m = fmaxf(m, v[e]);
      const double d = b0 - floor((double)m * s);
      if (d < SM_BINS - 1) atomicAdd(&lds.count[(int)d], 1u);
    });
    if (tid == 0) lds.last = SM_BINS;
    __syncthreads();
    constexpr int EACH = SM_BINS / THREADS;
    int own[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) sum += own[i] = (int)lds.count[tid * EACH + i];
    int n = block_scan<THREADS / 64>(sum, lds.tmp_n) - sum;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (n < top_k && n + own[i] >= top_k) lds.last = tid * EACH + i;
      n += own[i];
      lds.count[tid * EACH + i] = 0;
    }
    __syncthreads();
    most = lds.last;
  }
  h.chunks([&](const float *v, int) {
#pragma unroll
    for (int e = 0; e < H::CE; ++e) {
      const double xs = (double)v[e] * s, b = floor(xs), d = b0 - b;
      if (d <= most) {
        if (d < SM_BINS - 1) {
          const int g = (int)d;
          atomicAdd(&lds.mass[g], (unsigned long long)bin_weight(xs, b));
          if (counts) atomicAdd(&lds.count[g], 1u);
        } else if (v[e] > -INFINITY) {
          atomicAdd(&lds.mass[SM_BINS - 1], (unsigned long long)tail_weight(xs, b0 - (SM_BINS - 1)));
          if (counts) atomicAdd(&lds.count[SM_BINS - 1], 1u);
        }
      }
    }
  });
  __syncthreads();
}

// A part of a row: its largest, and its bins.  One read of the logits.  256 rows of
// 152064 take 54 us (2.9 TB/s): the additions in LDS and the 64-bit arithmetic bound it,
// not the read (22 us).  Leaving out what top_k cannot reach took it from 64 to 54;
// 256 threads and bins of half the range from 78 to 64.
constexpr int SP_THREADS = 512;
template <int DT>
__global__ __launch_bounds__(SP_THREADS) void k_sample_parts(SampleArgs a) {
  using H = Held<DT, SP_THREADS>;
  __shared__ BinLds lds;
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts), tid = threadIdx.x;
  const SampleRow p = sample_row(a, a.act ? a.act[row] : row);
  const int first = part * H::ALL;
  H h((const char *)a.logits + (row * a.ld + first) * H::B, min(H::ALL, a.vocab - first));
  bool odd;
  const uint64_t best = row_best<H, SP_THREADS>(h, first, lds, odd);
  const float top = key_float((uint32_t)(best >> 32));
  const double s = p.inv_t * SM_FINE, b0 = floor((double)top * s);
  char *ws = sample_ws(a.ws, row, a.parts, part);
  if (tid == 0) *(SamplePart *)ws = SamplePart{b0, best, odd ? 1ull : 0ull};
  if (p.bad || p.greedy || odd || top == -INFINITY) return;
  const bool counts = p.top_k < a.vocab;
  row_bins<H, SP_THREADS>(h, s, b0, p.top_k, counts, lds);
  uint64_t *mass = (uint64_t *)(ws + sizeof(SamplePart));
  uint32_t *count = (uint32_t *)(mass + SM_BINS);
  for (int i = tid; i < SM_BINS; i += SP_THREADS) {
    mass[i] = lds.mass[i];
    if (counts) count[i] = lds.count[i];
  }
}

// ---------------------------------------------------------------------------
// draws
// ---------------------------------------------------------------------------
constexpr int SD_THREADS = 1024, SD_WAVES = SD_THREADS / 64;
constexpr int SD_LIST = 2048;  // gathered logits that stay at hand
constexpr int SD_SUB = 64;     // parts that a bin is cut into
constexpr int SD_FEW = 1024;   // logits that are sorted
constexpr int SD_RUNS = 3;     // ranges of values that are looked for
static_assert(SD_THREADS == SM_BINS && SD_WAVES * SD_SUB == SD_THREADS && SD_FEW <= SD_THREADS, "a thread for each");

struct DrawLds {
  BinLds bins;                    // of the row, then the parts of its needed bins
  union {
    struct {
      uint64_t queue[SD_WAVES][128];  // a wave's logits (value key and ~index) that wait for 64 lanes
      int slot[SM_BINS];              // of a bin that is cut further, -1: not
    };
    struct {
      double few_before[SD_THREADS];
      int start[SD_THREADS];
    };
  };
  uint64_t list[SD_LIST];
  __align__(16) uint64_t few[SD_FEW + 8];
  uint64_t sorted[SD_FEW];
  double upto[SD_THREADS], before[SD_THREADS];
  int count_before[SD_THREADS];
  int slot_bin[SD_WAVES];
  uint8_t need[SD_THREADS];
  double tmp[SD_WAVES];
  float run_lo[SD_RUNS], run_hi[SD_RUNS];
  int bk, bp0, bp1, bt0, bt1, n, n_few, pick, last;
  uint32_t digit;
  double above;
  uint64_t number, ties;
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
__device__ __forceinline__ double block_largest(double v, double *s_tmp) {
  for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_tmp[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SD_WAVES; ++w) v = fmax(v, s_tmp[w]);
  return v;
}

// A sum of weights that are whole multiples of 2^-63, in any order the same: up to 2^30
// of them fit, their upper and lower 32 bits apart.
struct Mass {
  unsigned long long hi, lo;
  __device__ __forceinline__ void add(uint64_t w) {
    hi += w >> 32;
    lo += w & 0xFFFFFFFFu;
  }
  __device__ __forceinline__ void add(const Mass &m) {
    hi += m.hi;
    lo += m.lo;
  }
  __device__ __forceinline__ double value() const { return (double)hi * 0x1p32 + (double)lo; }
};

// A row by itself, whatever it holds: each border and the draw by four passes over
// the row, a byte of the value each, over sums of the weights in whole multiples of
// 2^-63 of the largest.  (Multiples of a unit that the row's sum takes in 64 bits, 2^-44 of
// 200000 logits, are a tenth faster and lose many small weights under a large one.)  For rows of which more
// than SD_FEW logits lie in the parts of bins that count (many equal ones, mostly), or whose
// borders lie in the last bin: some 200 us for 112677 bf16 logits of which thousands are
// equal.
template <int DT>
__device__ __attribute__((noinline)) void draw_alone(const SampleArgs &a, DrawLds &lds, const SampleRow &p, int64_t row,
                                                     int64_t slot, float M) {
  using H = Read<DT, SD_THREADS>;
  const int V = a.vocab, tid = threadIdx.x;
  const H h{(const char *)a.logits + row * a.ld * H::B, V};
  const char *x = h.x;
  const double least = (double)M;
  const auto weight = [&](float v) { return (uint64_t)rint(exp(((double)v - least) * p.inv_t) * 0x1p63); };
  const auto each = [&](auto f) {
    h.chunks([&](const float *v, int) {
      for (int e = 0; e < H::CE; ++e)
        if (v[e] > -INFINITY) f(v[e]);  // (-inf stands for what is past the row's end, and is never drawn)
    });
  };
  unsigned long long *const his = lds.bins.mass, *const los = lds.bins.mass + 256;
  // a number and a weight of every thread, summed
  const auto sum = [&](unsigned long long &n, Mass m) {
    unsigned long long *all = lds.bins.mass;
    __syncthreads();
    if (tid < 3) all[tid] = 0;
    __syncthreads();
    atomicAdd(&all[0], n);
    atomicAdd(&all[1], m.hi);
    atomicAdd(&all[2], m.lo);
    __syncthreads();
    n = all[0];
    return Mass{all[1], all[2]}.value();
  };
  // the value at which `cross` (of the number and the weight up to it) becomes true
  // first; all above it, and its ties
  uint32_t edge = 0;
  double above = 0.0;
  uint64_t number = 0, ties = 0;
  const auto find = [&](auto cross, bool by_weight) {
    edge = 0;
    number = 0;
    Mass over{0, 0};  // (thread 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) {
        his[tid] = los[tid] = 0;
        lds.bins.count[tid] = 0;
      }
      __syncthreads();
      // (a run of equal digits, of which there are many, is added at once)
      uint32_t digit = 0, n = 0;
      Mass m{0, 0};
      const auto put = [&] {
        if (!n) return;
        atomicAdd(&lds.bins.count[digit], n);
        atomicAdd(&his[digit], m.hi);
        atomicAdd(&los[digit], m.lo);
      };
      each([&](float v) {
        const uint32_t k = value_key(v);
        if (shift != 24 && (k >> (shift + 8)) != (edge >> (shift + 8))) return;
        if ((k >> shift & 255) != digit) {
          put();
          digit = k >> shift & 255;
          n = 0;
          m = Mass{0, 0};
        }
        ++n;
        m.add(weight(v));
      });
      put();
      __syncthreads();
      if (tid == 0) {
        Mass up = over, last_up = over;
        uint64_t n = number, last_n = n;
        int d = 255, last = -1;
        for (; d >= 0; --d) {
          const uint64_t c = lds.bins.count[d];
          if (!c) continue;
          const Mass of{his[d], los[d]};
          if (!by_weight || of.hi || of.lo) last = d, last_up = up, last_n = n;
          Mass to = up;
          to.add(of);
          if (cross(n + c, to.value())) break;
          n += c;
          up = to;
        }
        if (d < 0) d = last, up = last_up, n = last_n;  // (rounding: the last that counts)
        over = up;
        lds.digit = (uint32_t)d;
        lds.above = up.value();
        lds.number = n;
        lds.ties = lds.bins.count[d];
      }
      __syncthreads();
      edge |= lds.digit << shift;
      above = lds.above;
      number = lds.number;
      ties = lds.ties;
    }
  };
  unsigned long long kept = 0;  // of the row's beginning
  Mass row_mass{0, 0};
  each([&](float v) {
    ++kept;
    row_mass.add(weight(v));
  });
  double total = sum(kept, row_mass);
  if ((uint64_t)p.top_k < kept) {
    find([&](uint64_t n, double) { return n >= (uint64_t)p.top_k; }, false);
    kept = p.top_k;
    total = above + (double)(kept - number) * (double)weight(key_float(edge));
  }
  if (p.top_p < 1.f) {
    const double want = fmax((double)p.top_p * total * (1 - SM_EQUAL), 0.5);
    const uint64_t most = kept;
    find([&](uint64_t, double m) { return m >= want; }, true);
    const double w = (double)weight(key_float(edge));
    const double n = ceil((want - above) / w);
    ties = min(n >= (double)ties ? ties : n > 1.0 ? (uint64_t)n : 1ull, most - number);
    total = above + (double)ties * w;
    kept = number + ties;
  }
  if (p.min_p > 0.f) {
    // how many reach it, and their weight
    const float least_x = min_p_floor(p, M);
    unsigned long long n = 0;
    Mass m{0, 0};
    each([&](float v) {
      if (v >= least_x) {
        ++n;
        m.add(weight(v));
      }
    });
    const double reach = sum(n, m);
    if (n < kept) {
      kept = n;
      total = reach;
    }
  }
  const double want = (p.u + SM_EQUAL) * total;
  find([&](uint64_t, double m) { return m > want; }, true);
  const double w = (double)weight(key_float(edge));
  const double nth = floor((want - above) / w);
  ties = min(ties, kept - number);
  int64_t left = nth >= (double)ties ? (int64_t)ties - 1 : nth > 0.0 ? (int64_t)nth : 0;
  // the left-th index that holds it
  for (int b = 0; b < V; b += SD_THREADS) {
    const int i = b + tid;
    const bool is = i < V && value_key(ld_elem<DT>(x, i)) == edge;
    const uint64_t in = __ballot(is);
    __syncthreads();
    if ((tid & 63) == 0) lds.bins.tmp_n[tid >> 6] = (int)__popcll(in);
    __syncthreads();
    int before = 0, all = 0;
    for (int o = 0; o < SD_WAVES; ++o) {
      if (o < tid >> 6) before += lds.bins.tmp_n[o];
      all += lds.bins.tmp_n[o];
    }
    if (left < all) {
      if (is && before + (int)__popcll(in & ((1ull << (tid & 63)) - 1)) == left) {
        a.tokens[slot] = i;
        if (a.logprob) a.logprob[row] = (float)(((double)key_float(edge) - least) * p.inv_t - log(total * 0x1p-63));
      }
      return;
    }
    left -= all;
  }
}

// What a thread knows of its bin (or part of one): the weight and the number before
// it and up to it, in the row's falling order.
struct DrawBin {
  double before, upto, weight;
  int count_before, count;
};
struct DrawCuts {
  bool k, p, m;
  int bk, e0, e1;   // the bin in which top-k ends; bounds of the one in which all that stays ends (SD_THREADS: none)
  bool need, past;  // whether the thread's bin may hold a border or the draw; whether some bin could not be found
};
// Which bins top-k and min-p end in; between which bounds the weight lies that top-k
// leaves, hence the bins that top-p may end in; hence the bounds of the weight that
// is drawn from, and the bins that the draw may fall in.  Bounds are wider by 1e-12
// than sums are off.  bm: the bin that min-p's floor lies in.
__device__ __forceinline__ DrawCuts draw_cuts(DrawLds &lds, const SampleRow &p, const DrawBin &b, double total, int vocab,
                                              int bm) {
  constexpr int NONE = SD_THREADS;
  const int tid = threadIdx.x;
  DrawCuts c;
  c.k = p.top_k < vocab;
  c.p = p.top_p < 1.f;
  c.m = p.min_p > 0.f;
  __syncthreads();
  lds.before[tid] = b.before;
  lds.upto[tid] = b.upto;
  lds.count_before[tid] = b.count_before;
  if (tid == 0) lds.bk = lds.bp0 = lds.bp1 = lds.bt0 = lds.bt1 = NONE;
  __syncthreads();
  if (c.k && b.count && b.count_before < p.top_k && b.count_before + b.count >= p.top_k) lds.bk = tid;
  __syncthreads();
  c.bk = lds.bk;
  const auto bound = [&](int at, bool after) { return at >= NONE ? total : after ? lds.upto[at] : lds.before[at]; };
  const double wider = 1e-12;
  if (c.p) {
    const double lo = fmax((double)p.top_p * bound(c.bk, false) * (1 - wider), 0x1p-1070),
                 hi = fmax((double)p.top_p * bound(c.bk, true) * (1 + wider), 0x1p-1070);
    if (b.upto >= lo && b.before < lo) lds.bp0 = tid;
    if (b.upto >= hi && b.before < hi) lds.bp1 = tid;
    __syncthreads();
  }
  const int bp0 = lds.bp0, bp1 = lds.bp1;
  c.e0 = min(bm, min(c.bk, bp0));
  c.e1 = min(bm, min(c.bk, bp1));
  const double lo = p.u * bound(c.e0, false) * (1 - wider), hi = p.u * bound(c.e1, true) * (1 + wider);
  if (b.upto > lo && b.before <= lo) lds.bt0 = tid;
  if (b.upto > hi && b.before <= hi) lds.bt1 = tid;
  __syncthreads();
  const int bt0 = min(lds.bt0, c.e1), bt1 = min(lds.bt1, c.e1);
  // (a top-p that ends past what the others leave says nothing, nor then does top-k)
  c.need = (tid == c.bk && ((c.p && bp0 <= c.e1) || c.bk <= c.e1)) || (tid == bm && bm <= c.e1) ||
           (b.weight > 0.0 && ((c.p && tid >= bp0 && tid <= bp1 && tid <= c.e1) || (tid >= bt0 && tid <= bt1)));
  c.past = bt1 >= NONE || (c.p && c.e1 >= NONE);
  return c;
}

// A row's draw.  WHOLE: its bins are summed here; else its parts' are joined.  It is a
// chain of a dozen short phases with a barrier or two each: 31 us for one row of
// 32000, 56 for 16 of 152064, 65 for 256 of them, 260 for 1531 bf16 rows of 32003, six
// rows to a CU one after the other (88 KB of LDS and 128 registers of 1024 threads; with
// 64 registers it spills, and two at a time took 445).  The row in registers instead of read again took 545:
// the unrolled code does not fit the instruction cache.
template <int DT, bool WHOLE>
__global__ __launch_bounds__(SD_THREADS) void k_sample_draw(SampleArgs a) {
  using H = Read<DT, SD_THREADS>;
  __shared__ DrawLds lds;
  const int64_t row = blockIdx.x, slot = a.act ? a.act[row] : row;
  const int tid = threadIdx.x, V = a.vocab, lane = tid & 63, wave = tid >> 6;
  H h{(const char *)a.logits + row * a.ld * H::B, V};
  const SampleRow p = sample_row(a, slot);
  uint64_t best = 0;
  bool odd = false;
  if constexpr (WHOLE) {
    best = row_best<H, SD_THREADS>(h, 0, lds.bins, odd);
  } else {
    for (int i = tid; i < a.parts; i += SD_THREADS) {
      const SamplePart h = *(const SamplePart *)sample_ws(a.ws, row, a.parts, i);
      best = max(best, h.best);
      odd |= h.odd != 0;
    }
    odd = __syncthreads_or(odd);
    best = block_most<SD_WAVES>(best, lds.bins.tmp);
  }
  const float M = key_float((uint32_t)(best >> 32));
  if (p.bad || odd || M == -INFINITY || p.greedy) {
    if (tid == 0) {
      const bool none = p.bad || odd || M == -INFINITY;
      a.tokens[slot] = none ? -1 : (int)~(uint32_t)best;
      if (a.logprob) a.logprob[row] = none ? NAN : 0.f;
    }
    return;
  }
  const double s = p.inv_t * SM_FINE, b0 = floor((double)M * s);
  const bool cut_k = p.top_k < V;

  // the row's bins, one of each thread
  const auto bin_scale = [](int b) { return exp(-(double)b / SM_FINE) * 0x1p-48; };
  const double scale = bin_scale(tid);
  double w = 0.0, total, before;
  int count = 0;
  if constexpr (WHOLE) {
    row_bins<H, SD_THREADS>(h, s, b0, p.top_k, cut_k, lds.bins);
    w = (double)lds.bins.mass[tid] * scale;
    count = (int)lds.bins.count[tid];
  } else {
    // from part i's bin tid - off, and what reaches past the last; `list` holds the
    // parts' offsets
    double far = 0.0;
    int far_count = 0;
    for (int i0 = 0; i0 < a.parts; i0 += SD_LIST) {
      const int n = min(a.parts - i0, SD_LIST);
      __syncthreads();
      for (int i = tid; i < n; i += SD_THREADS) {
        const SamplePart *h = (const SamplePart *)sample_ws(a.ws, row, a.parts, i0 + i);
        const double off = (uint32_t)(h->best >> 32) == value_key(-INFINITY) ? -1.0 : b0 - h->top;
        lds.list[i] = __builtin_bit_cast(uint64_t, off);
      }
      __syncthreads();
      constexpr int U = 4;
      for (int j = 0; j < n; j += U) {
        uint64_t near_w[U], far_w[U];
        uint32_t near_n[U], far_n[U];
        double off[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          off[u] = j + u < n ? __builtin_bit_cast(double, lds.list[j + u]) : -1.0;
          const char *ws = sample_ws(a.ws, row, a.parts, i0 + min(j + u, n - 1)) + sizeof(SamplePart);
          const int to = (int)fmin(off[u], (double)SM_BINS);
          const bool near = to >= 0 && tid < SM_BINS - 1 && tid >= to, past = to >= 0 && tid + to >= SM_BINS - 1;
          near_w[u] = near ? ((const uint64_t *)ws)[tid - to] : 0;
          far_w[u] = past ? ((const uint64_t *)ws)[tid] : 0;
          near_n[u] = near && cut_k ? ((const uint32_t *)((const uint64_t *)ws + SM_BINS))[tid - to] : 0;
          far_n[u] = past && cut_k ? ((const uint32_t *)((const uint64_t *)ws + SM_BINS))[tid] : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          w += (double)near_w[u] * scale;
          if (far_w[u]) far += (double)far_w[u] * (exp(-(tid + off[u]) / SM_FINE) * 0x1p-48);
          count += (int)near_n[u];
          far_count += (int)far_n[u];
        }
      }
    }
    (void)block_scan(far, lds.tmp, total, before);
    if (tid == SM_BINS - 1) w = total;
    if (cut_k) {
      const int fars = block_scan<SD_WAVES>(far_count, lds.bins.tmp_n);
      if (tid == SM_BINS - 1) count = fars;
    }
  }
  DrawBin bin;
  bin.upto = block_scan(w, lds.tmp, total, bin.before);
  bin.weight = w;
  bin.count = count;
  // (-inf is not counted: top_k may end past the last number)
  bin.count_before = cut_k ? block_scan<SD_WAVES>(count, lds.bins.tmp_n) - count : 0;
  const float floor_x = p.min_p > 0.f ? min_p_floor(p, M) : -INFINITY;
  const int bm = p.min_p > 0.f ? (int)fmin(b0 - floor((double)floor_x * s), (double)(SM_BINS - 1)) : SD_THREADS;
  DrawCuts cut = draw_cuts(lds, p, bin, total, V, bm);
  // the needed bins in order; the last one is not cut further
  const uint64_t needed = __ballot(cut.need);
  if (lane == 0) lds.bins.tmp_n[wave] = (int)__popcll(needed);
  if (tid == 0) lds.n = lds.n_few = 0;
  const bool alone = __syncthreads_or(cut.past || (cut.need && tid == SM_BINS - 1));
  int mine = (int)__popcll(needed & ((1ull << lane) - 1)), slots = 0;
  for (int o = 0; o < SD_WAVES; ++o) {
    if (o < wave) mine += lds.bins.tmp_n[o];
    slots += lds.bins.tmp_n[o];
  }
  if (alone || slots > SD_WAVES) {
    __syncthreads();
    draw_alone<DT>(a, lds, p, row, slot, M);
    return;
  }
  lds.slot[tid] = cut.need ? mine : -1;
  if (cut.need) lds.slot_bin[mine] = tid;
  lds.bins.mass[tid] = 0;
  lds.bins.count[tid] = 0;
  __syncthreads();
  // ranges of values that cover them, wider than roundings: few logits outside the
  // bins are in them
  if (tid == 0) {
    for (int r = 0; r < SD_RUNS; ++r) {
      lds.run_lo[r] = INFINITY;
      lds.run_hi[r] = -INFINITY;
    }
    int r = -1;
    for (int i = 0; i < slots; ++i) {
      const int b = lds.slot_bin[i];
      if (r < 0 || (b != lds.slot_bin[i - 1] + 1 && r < SD_RUNS - 1)) {
        const double hi = (b0 - b + 1.0) / s;
        lds.run_hi[++r] = (float)fmin(hi + fabs(hi) * 0x1p-20 + 1e-37, (double)FLT_MAX);
      }
      const double lo = (b0 - b) / s;
      lds.run_lo[r] = (float)fmax(lo - fabs(lo) * 0x1p-20 - 1e-37, -(double)FLT_MAX);
    }
  }
  __syncthreads();
  float run_lo[SD_RUNS], run_hi[SD_RUNS];
#pragma unroll
  for (int r = 0; r < SD_RUNS; ++r) {
    run_lo[r] = lds.run_lo[r];
    run_hi[r] = lds.run_hi[r];
  }
  const float lowest = fminf(run_lo[0], fminf(run_lo[1], run_lo[2]));
  // Calls take(value, ~index), a wave's lanes together, for the row's logits in the
  // ranges.  They wait in a queue of the wave's until they fill its lanes.
  const auto each = [&](auto take) {
    int waiting = 0;
    const auto offer = [&](float v, int i) {
      bool in = v >= run_lo[0] && v <= run_hi[0];
#pragma unroll
      for (int r = 1; r < SD_RUNS; ++r) in |= v >= run_lo[r] && v <= run_hi[r];
      const uint64_t all = __ballot(in);
      if (!all) return;
      if (in)
        lds.queue[wave][waiting + (int)__popcll(all & ((1ull << lane) - 1))] = (uint64_t)value_key(v) << 32 | (uint32_t)~i;
      waiting += (int)__popcll(all);
      if (waiting >= 64) {
        waiting -= 64;
        const uint64_t k = lds.queue[wave][waiting + lane];
        take(key_float((uint32_t)(k >> 32)), (uint32_t)k);
      }
    };
    h.chunks([&](const float *v, int i) {
      float top = v[0];
#pragma unroll
      for (int e = 1; e < H::CE; ++e) top = fmaxf(top, v[e]);
      if (!__ballot(top >= lowest)) return;
#pragma unroll
      for (int e = 0; e < H::CE; ++e) offer(v[e], i + e);
    });
    if (lane < waiting) {
      const uint64_t k = lds.queue[wave][lane];
      take(key_float((uint32_t)(k >> 32)), (uint32_t)k);
    }
  };
  // the part of a bin that a logit lies in, -1: in none that is needed.  (xs - b of an xs
  // just below zero is rounded to 1: that lies in its bin's first part)
  const auto part = [&](float v, double &xs, double &b) {
    xs = (double)v * s;
    b = floor(xs);
    const double d = b0 - b;
    const int at = d < SM_BINS - 1 ? lds.slot[(int)d] : -1;
    return at < 0 ? -1 : at * SD_SUB + SD_SUB - 1 - min((int)((xs - b) * SD_SUB), SD_SUB - 1);
  };
  each([&](float v, uint32_t low) {
    double xs, b;
    const int at = part(v, xs, b);
    if (at < 0) return;
    atomicAdd(&lds.bins.mass[at], (unsigned long long)bin_weight(xs, b));
    atomicAdd(&lds.bins.count[at], 1u);
    const int to = atomicAdd(&lds.n, 1);
    if (to < SD_LIST) lds.list[to] = (uint64_t)value_key(v) << 32 | low;
  });
  __syncthreads();
  // the parts, each wave's of one bin
  w = count = 0;
  bin.before = bin.upto = total;
  bin.count_before = INT32_MAX / 2;
  if (wave < slots) {
    const int of = lds.slot_bin[wave];
    w = (double)lds.bins.mass[tid] * bin_scale(of);
    count = (int)lds.bins.count[tid];
    double up = w;
    int n = count;
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(up, o);
      const int z = __shfl_up(n, o);
      if (lane >= o) {
        up += y;
        n += z;
      }
    }
    const double prev = __shfl_up(up, 1);
    bin.before = lds.before[of] + (lane ? prev : 0.0);
    bin.upto = lds.before[of] + up;
    bin.count_before = lds.count_before[of] + n - count;
  }
  bin.count = count;
  bin.weight = w;
  double floor_s, floor_b;
  int bm2 = p.min_p > 0.f ? part(floor_x, floor_s, floor_b) : -1;
  if (bm2 < 0) bm2 = SD_THREADS;
  cut = draw_cuts(lds, p, bin, total, V, bm2);
  lds.need[tid] = cut.need;
  // (a part of a bin may hold more of a long row's than sum in 64 bits)
  if (__syncthreads_or(cut.past || count > 1 << 14)) {
    draw_alone<DT>(a, lds, p, row, slot, M);
    return;
  }
  // what is left
  const auto pick_up = [&](float v, uint32_t low) {
    double xs, b;
    const int at = part(v, xs, b);
    if (at >= 0 && lds.need[at]) {
      const int to = atomicAdd(&lds.n_few, 1);
      if (to < SD_FEW) lds.few[to] = (uint64_t)value_key(v) << 32 | low;
    }
  };
  if (lds.n <= SD_LIST) {
    for (int i = tid; i < lds.n; i += SD_THREADS) pick_up(key_float((uint32_t)(lds.list[i] >> 32)), (uint32_t)lds.list[i]);
  } else {
    each(pick_up);
  }
  __syncthreads();
  const int n = lds.n_few;
  if (n > SD_FEW) {
    __syncthreads();
    draw_alone<DT>(a, lds, p, row, slot, M);
    return;
  }
  if (tid < n) {
    const uint64_t key = lds.few[tid];
    int rank = 0;
    for (int o = 0; o < n; o += 8) {
      u32x4 two[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) two[u] = *(const u32x4 *)&lds.few[o + 2 * u];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        rank += o + 2 * u < n && ((uint64_t)two[u][1] << 32 | two[u][0]) > key;
        rank += o + 2 * u + 1 < n && ((uint64_t)two[u][3] << 32 | two[u][2]) > key;
      }
    }
    lds.sorted[rank] = key;
  }
  if (tid == 0) {
    lds.pick = INT32_MAX;
    lds.last = -1;
  }
  __syncthreads();
  // each one's weight, and the weight before it and its place in the row
  double wt = 0.0, xs, b, all;
  int at = -1, at_prev = -1;
  float v = 0.f;
  if (tid < n) {
    v = key_float((uint32_t)(lds.sorted[tid] >> 32));
    if (tid) at_prev = part(key_float((uint32_t)(lds.sorted[tid - 1] >> 32)), xs, b);
    at = part(v, xs, b);
    wt = (double)bin_weight(xs, b) * bin_scale((int)(b0 - b));
  }
  (void)block_scan(wt, lds.tmp, all, before);  // (its barriers end the use of `slot`)
  if (tid < n && at != at_prev) {
    lds.start[at] = tid;
    lds.few_before[at] = before;
  }
  __syncthreads();
  bool in = tid < n;
  double ahead = 0.0;
  if (in) {
    ahead = lds.before[at] + (before - lds.few_before[at]);
    if (cut.k) in = lds.count_before[at] + (tid - lds.start[at]) < p.top_k;
  }
  if (cut.p) {
    const double kept = block_largest(in && at == cut.bk ? ahead + wt : 0.0, lds.tmp);
    const double zk = cut.bk < SD_THREADS ? fmax(kept, lds.before[cut.bk]) : total;
    in = in && ahead < fmax((double)p.top_p * zk * (1 - SM_EQUAL), 0x1p-1070);
  }
  in = in && v >= floor_x;
  const double kept = block_largest(in ? ahead + wt : 0.0, lds.tmp);
  const double z = cut.e1 < SD_THREADS ? fmax(kept, lds.before[cut.e0]) : total;
  const double want = (p.u + SM_EQUAL) * z;
  if (in && wt > 0.0) {
    atomicMax(&lds.last, tid);
    if (ahead + wt > want) atomicMin(&lds.pick, tid);
  }
  __syncthreads();
  if (tid == (lds.pick < INT32_MAX ? lds.pick : lds.last)) {
    a.tokens[slot] = (int)~(uint32_t)lds.sorted[tid];
    if (a.logprob) a.logprob[row] = (float)log(wt / z);
  }
}

// A row of T logits or fewer, a thread for each: sorted by counting, then as the
// definition has it.  Up to 256; for 613 rows of 1020 counting among all took 121 us,
// bins 100.
template <int DT, int T>
__global__ __launch_bounds__(T) void k_sample_few(SampleArgs a) {
  constexpr int WAVES = T / 64;
  __shared__ __align__(16) uint64_t s_key[T + 8], s_sorted[T];
  __shared__ double s_d[WAVES];
  __shared__ int s_pick, s_last;
  const int64_t row = blockIdx.x, slot = a.act ? a.act[row] : row;
  const int tid = threadIdx.x, V = a.vocab, lane = tid & 63, wave = tid >> 6;
  const SampleRow p = sample_row(a, slot);
  const float x = tid < V ? ld_elem<DT>((const char *)a.logits + row * a.ld * (DT == HS_F32 ? 4 : 2), tid) : -INFINITY;
  const bool odd = __syncthreads_or(!(x < INFINITY));
  const uint64_t key = (uint64_t)value_key(x) << 32 | (uint32_t)~tid;
  s_key[tid] = key;
  if (tid == 0) {
    s_pick = INT32_MAX;
    s_last = -1;
  }
  __syncthreads();
  int rank = 0;
  const int n = (V + 7) / 8 * 8;  // (what lies past the row ranks below it)
  for (int o = 0; o < n; o += 8) {
    u32x4 two[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) two[u] = *(const u32x4 *)&s_key[o + 2 * u];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      rank += o + 2 * u < V && ((uint64_t)two[u][1] << 32 | two[u][0]) > key;
      rank += o + 2 * u + 1 < V && ((uint64_t)two[u][3] << 32 | two[u][2]) > key;
    }
  }
  if (tid < V) s_sorted[rank] = key;
  __syncthreads();
  const float M = key_float((uint32_t)(s_sorted[0] >> 32));
  if (p.bad || odd || M == -INFINITY || p.greedy) {
    if (tid == 0) {
      const bool none = p.bad || odd || M == -INFINITY;
      a.tokens[slot] = none ? -1 : (int)~(uint32_t)s_sorted[0];
      if (a.logprob) a.logprob[row] = none ? NAN : 0.f;
    }
    return;
  }
  const float v = tid < V ? key_float((uint32_t)(s_sorted[tid] >> 32)) : -INFINITY;
  bool in = tid < V && tid < p.top_k;
  const double w = in ? exp(((double)v - (double)M) * p.inv_t) : 0.0;
  double upto = w;
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 63) s_d[wave] = upto;
  __syncthreads();
  double z = 0.0;
#pragma unroll
  for (int o = 0; o < WAVES; ++o) {
    if (o < wave) upto += s_d[o];
    z += s_d[o];
  }
  if (p.top_p < 1.f) in = in && (tid == 0 || upto - w < (double)p.top_p * z * (1 - SM_EQUAL));
  if (p.min_p > 0.f) in = in && v >= min_p_floor(p, M);
  // the weight up to the last that stays
  double top = in ? upto : 0.0;
  for (int o = 32; o; o >>= 1) top = fmax(top, __shfl_xor(top, o));
  __syncthreads();
  if (lane == 0) s_d[wave] = top;
  __syncthreads();
  z = 0.0;
#pragma unroll
  for (int o = 0; o < WAVES; ++o) z = fmax(z, s_d[o]);
  if (in && w > 0.0) {
    atomicMax(&s_last, tid);
    if (upto > (p.u + SM_EQUAL) * z) atomicMin(&s_pick, tid);
  }
  __syncthreads();
  if (tid == (s_pick < INT32_MAX ? s_pick : s_last)) {
    a.tokens[slot] = (int)~(uint32_t)s_sorted[tid];
    if (a.logprob) a.logprob[row] = (float)log(w / z);
  }
}

// Rows up to this long are drawn from in one launch: for a few of them a second one and
// its read of what the first wrote cost more than a work group's summing of 32768 logits
// (one row of 32000 is 31 us against 19 + 10 and a launch).  For many it is the other way
// round: 1531 bf16 rows of 32003 take 264 us, and took 175 with their bins in a launch of
// their own and draws by 512 threads in 62 KB of LDS, two to a CU.  The rule does not
// look at how many rows there are.
constexpr int SAMPLE_WHOLE = 32768;
// parts of a row; 0: it has none
inline int sample_parts(int vocab, int dtype) {
  const int per = SP_WORDS * SP_THREADS * (dtype == HS_F32 ? 1 : 2);
  return vocab <= SAMPLE_WHOLE ? 0 : (int)(((int64_t)vocab + per - 1) / per);
}

template <int DT>
hipError_t sample_launch(SampleArgs a, hipStream_t st) {
  a.parts = sample_parts(a.vocab, DT);
  if (a.vocab <= 64) {
    HS_LAUNCH((k_sample_few<DT, 64>), dim3((uint32_t)a.rows), dim3(64), 0, st, a);
  } else if (a.vocab <= 256) {
    HS_LAUNCH((k_sample_few<DT, 256>), dim3((uint32_t)a.rows), dim3(256), 0, st, a);
  } else if (!a.parts) {
    HS_LAUNCH((k_sample_draw<DT, true>), dim3((uint32_t)a.rows), dim3(SD_THREADS), 0, st, a);
  } else {
    HS_LAUNCH((k_sample_parts<DT>), dim3((uint32_t)(a.rows * a.parts)), dim3(SP_THREADS), 0, st, a);
    HS_LAUNCH((k_sample_draw<DT, false>), dim3((uint32_t)a.rows), dim3(SD_THREADS), 0, st, a);
  }
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
