// hs_paged.h — a paged KV cache in the model's own type (gfx950): new rows
// normalised, turned and stored, and attention over it where rows of a group
// share their first positions.  Included by hs_attn.hip.
#pragma once

#include "hs_device.h"

#include <algorithm>
#include <cfloat>

namespace hs {
namespace {

using namespace dev;

// element offset of layer a.layer's K (sel 0) or V (1) of head j in a block
__device__ __forceinline__ int64_t paged_slab(const PagedRef &c, int64_t block, int sel, int j, int hd) {
  return block * c.block_elems + ((((int64_t)c.layer * 2 + sel) * c.n_kv + j) << c.bt_log2) * hd;
}
// The block of (sequence, position), or -1: outside the table, without a
// block, or a number that is no block of the cache.
__device__ __forceinline__ int64_t paged_block(const PagedRef &c, int seq, int pos) {
  const int k = pos >> c.bt_log2;
  if ((uint32_t)seq >= (uint32_t)c.n_seqs || pos < 0 || k >= c.table_ld) return -1;
  const int64_t b = c.table[(int64_t)seq * c.table_ld + k];
  return (uint64_t)b < (uint64_t)c.n_blocks ? b : -1;
}

// ---------------------------------------------------------------------------
// rows stored
// ---------------------------------------------------------------------------
constexpr int APPEND_THREADS = 256;
constexpr int APPEND_ROWS = 4;  // most rows of a work group

// cos and sin of the angle at * freq.  The product and the whole turns taken off
// it are in 64 bits (an angle of 2^30 keeps 2^-23 of a radian); what is left, half a
// turn at most, goes through fp32.
__device__ __forceinline__ void turn(int at, double freq, float &c, float &s) {
  const double t = (double)at * freq * 0.15915494309189535;  // turns
  const float r = 2.f * (float)(t - rint(t));                // half turns
  sincospif(r, &s, &c);
}

// New rows of a layer.  x of query and key heads becomes x / sqrt(mean x^2 + eps) * gain
// (with a gain), then pair i of its first 2 pairs channels, (i, i + pairs) or
// (2 i, 2 i + 1), is turned by angles_at[axis[i]][row] * freq[i]: all in fp32, rounded
// once.  Keys and values go to the row's place in the cache, queries to q_out.
//
// The work is a copy.  A work group takes some rows (or a part of one row's
// heads), computes the rows' cosines and sines once for all heads (64 bits, into
// LDS) and gives each head to HD / 8 lanes, 8 channels a lane; a half-apart pair's
// other channel comes from the lane that holds it.  The next head is asked for before
// one is worked on.  14370 rows of 28 + 8 heads of 128, with norms and three axes: 102 us,
// 2.6 TB/s both ways (121 without that); 32 rows of 96 heads: 4 us.
template <int DT, int HD>
__global__ __launch_bounds__(APPEND_THREADS) void k_paged_append(PagedRows a, int rows_wg, int heads_wg) {
  constexpr int B = DT == HS_F32 ? 4 : 2, L = HD / 8, GROUPS = APPEND_THREADS / L;
  constexpr int W = DT == HS_F32 ? 8 : 4;  // words of a lane's 8 channels
  __shared__ float2 cs[APPEND_ROWS][HD / 2];
  const int parts = (a.n_heads + 2 * a.c.n_kv + heads_wg - 1) / heads_wg;
  const int row0 = blockIdx.x / parts * rows_wg, h0 = blockIdx.x % parts * heads_wg;
  const int rows = min(rows_wg, a.n - row0), heads = min(heads_wg, a.n_heads + 2 * a.c.n_kv - h0);
  const int items = rows * heads;
  const int lane = threadIdx.x % L, e0 = lane * 8;
  for (int i = threadIdx.x; i < rows * a.pairs; i += APPEND_THREADS) {
    const int r = i / a.pairs, p = i - r * a.pairs;
    const int axis = a.axes ? min(max(a.axes[p], 0), a.n_axes - 1) : 0;
    float c, s;
    turn(a.angles_at[(int64_t)axis * a.n + row0 + r], a.freq[p], c, s);
    cs[r][p] = float2{c, s};
  }
  // a half-apart pair's other channels, 8 of them in one lane as pairs is a multiple of 8
  const bool early = e0 < a.pairs, paired = e0 < 2 * a.pairs;
  const int other = !a.adjacent && paired ? (early ? lane + a.pairs / 8 : lane - a.pairs / 8) : lane;
  const auto load8 = [](const char *p, uint32_t(&w)[W]) {
#pragma unroll
    for (int u = 0; u < W; u += 4) {
      const u32x4 t = ld16(p + u * 4);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[u + x] = t[x];
    }
  };
  const auto widen = [](const uint32_t(&v)[W], float *o) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (DT == HS_F32) o[e] = __uint_as_float(v[e]);
      else o[e] = e & 1 ? hi_f32<DT>(v[e / 2]) : lo_f32<DT>(v[e / 2]);
    }
  };
  // the lane's and its other's gains
  uint32_t gains[2][2][W];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const char *gain = (const char *)(k ? a.k_gain : a.q_gain);
    if (gain) {
      load8(gain + e0 * B, gains[k][0]);
      load8(gain + other * 8 * B, gains[k][1]);
    }
  }
  // item `it` is head h0 + it % heads of row row0 + it / heads
  const auto fetch = [&](int it, uint32_t(&w)[W]) {
    const int r = it / heads, h = h0 + it - r * heads;
    const int64_t row = row0 + r;
    const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.c.n_kv;
    const int j = is_q ? h : is_k ? h - a.n_heads : h - a.n_heads - a.c.n_kv;
    load8((const char *)(is_q ? a.q : is_k ? a.k : a.v) +
              (is_q ? row * a.ld_q + j * a.ld_q_head : row * a.ld + j * a.ld_head) * B + e0 * B,
          w);
  };
  uint32_t next[W];
  if ((int)threadIdx.x / L < items) fetch(threadIdx.x / L, next);
  __syncthreads();
  for (int it = threadIdx.x / L; it < items; it += GROUPS) {
    const int r = it / heads, h = h0 + it - r * heads;
    const int64_t row = row0 + r;
    const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.c.n_kv;
    const int j = is_q ? h : is_k ? h - a.n_heads : h - a.n_heads - a.c.n_kv;
    uint32_t w[W];
#pragma unroll
    for (int u = 0; u < W; ++u) w[u] = next[u];
    // (q_out may be q: an item's place is written after its own load, and no other's)
    if (it + GROUPS < items) fetch(it + GROUPS, next);
    char *dst;
    if (is_q) {
      dst = (char *)a.q_out + (row * a.ld_q_out + j * a.ld_q_out_head) * B;
    } else {
      const int pos = a.pos[row];
      const int64_t b = paged_block(a.c, a.seqs ? a.seqs[row] : (int)row, pos);
      dst = b < 0 ? nullptr
                  : (char *)a.c.blocks + (paged_slab(a.c, b, is_k ? 0 : 1, j, HD) +
                                          (int64_t)(pos & ((1 << a.c.bt_log2) - 1)) * HD) * B;
    }
    if (is_q || is_k) {
      float f[8], g[8], gain[8];
      widen(w, f);
      const bool norm = (is_q ? a.q_gain : a.k_gain) != nullptr;
      float rs = 1.f;
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(f[e], f[e], ss);
        ss = group_sum<L>(ss);
        rs = 1.f / sqrtf(ss * (1.f / HD) + a.eps);
        widen(gains[is_q ? 0 : 1][0], gain);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= rs * gain[e];
      }
      if (a.adjacent) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          if (e0 + e < 2 * a.pairs) {
            const float2 t = cs[r][(e0 + e) / 2];
            const float x = f[e], y = f[e + 1];
            f[e] = x * t.x - y * t.y;
            f[e + 1] = x * t.y + y * t.x;
          }
      } else if (a.pairs) {
        const int from = (int)(threadIdx.x & 63) - lane + other;
        uint32_t v[W];
#pragma unroll
        for (int u = 0; u < W; ++u) v[u] = (uint32_t)__shfl((int)w[u], from);
        widen(v, g);
        if (norm) widen(gains[is_q ? 0 : 1][1], gain);
        if (paired) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (norm) g[e] *= rs * gain[e];
            const float2 t = cs[r][(early ? e0 : e0 - a.pairs) + e];
            f[e] = early ? f[e] * t.x - g[e] * t.y : g[e] * t.y + f[e] * t.x;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < W; ++u) {
        if constexpr (DT == HS_F32) w[u] = __float_as_uint(f[u]);
        else w[u] = pack2<DT>(f[2 * u], f[2 * u + 1]);
      }
    }
    if (dst) {
#pragma unroll
      for (int u = 0; u < W; u += 4) *(u32x4 *)(dst + e0 * B + u * 4) = u32x4{w[u], w[u + 1], w[u + 2], w[u + 3]};
    }
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
constexpr int PG_WAVES = 4;
constexpr int PG_STRIPE = PG_WAVES * 32;  // positions that a work group takes at a time
// 16-bit parts in which a weight enters the second product: 22 bits of it in f16, 24 in
// bf16.  (With two parts of bf16, 16 bits, outputs were rounded to another number than
// an fp32 form's often enough to differ by 2.8e-4 in norm for large groups, 8e-5 now.
// The third part costs those 14 % and others 2 to 3 %.)
template <int DT>
constexpr int PG_PARTS = DT == HS_BF16 ? 3 : 2;
// Weights are 2^(score - m).  o / l does not depend on m, which moves only where a
// wave's tile has a score that passes it by more than PG_UP, and then to PG_TO below that
// column's largest.  The weights of fp32 and bf16 may fall as low as they like.  Those of
// f16 end at 2^-24, so m moves down too, where a column's largest is less than PG_LOW
// above it: o and l are fp32 and hold what came before.  So a weight is off by 2^-34 of the
// largest up to its tile, and by 2^-26 of the largest in its tile, at most.  (With m at
// the largest of all, thousands of equal positions 2^-25 below one vanished; following
// them costs 3 % of large groups and 4 % of drafts.)  m stays within PG_DOWN of where it
// was highest, so that o is finite; scores that far down weigh nothing.
template <int DT>
constexpr float PG_UP = DT == HS_F16 ? 15.f : 8.f;
template <int DT>
constexpr float PG_TO = DT == HS_F16 ? 9.f : 0.f;
constexpr float PG_LOW = 1.f, PG_DOWN = 48.f;
// f16: where m moves to for a tile whose largest score is top, `over` of it
__device__ __forceinline__ float moved(float m, float top, float over, float highest) {
  if (!(over > PG_UP<HS_F16> || over < PG_LOW) || top == -INFINITY) return m;
  const float mn = fmaxf(top - PG_TO<HS_F16>, highest - PG_DOWN);
  return top - mn > PG_UP<HS_F16> ? top : mn;  // (scores so large that the difference is rounded)
}
// two weights in parts
template <int DT>
__device__ __forceinline__ void weight_parts(float p0, float p1, uint32_t (&w)[PG_PARTS<DT>]) {
#pragma unroll
  for (int i = 0; i < PG_PARTS<DT>; ++i) {
    w[i] = pack2<DT>(p0, p1);
    p0 -= lo_f32<DT>(w[i]);
    p1 -= hi_f32<DT>(w[i]);
  }
}

__device__ __forceinline__ int paged_most(const PagedRef &c) {
  return (int)min((int64_t)c.table_ld << c.bt_log2, (int64_t)INT32_MAX);
}
__device__ __forceinline__ int paged_shared(const PagedAttn &a, int g) {
  return max(0, min(min(a.shared[g], a.max_shared), paged_most(a.c)));
}
__device__ __forceinline__ int paged_seq(const PagedAttn &a, int row) { return a.seqs ? a.seqs[row] : row; }
__device__ __forceinline__ int paged_length(const PagedAttn &a, int row, int seq) {
  if ((uint32_t)seq >= (uint32_t)a.c.n_seqs) return 0;
  return max(0, min(min(a.lens[row], a.max_len), paged_most(a.c)));
}
// What a row attends over: positions [lo, hi) of its own (or of its group's
// first sequence, where it is shorter than what the group shares), and whether
// the shared ones before them come from the group.
struct PagedRow {
  int seq, lo, hi;
  bool grouped;
};
__device__ __forceinline__ PagedRow paged_row(const PagedAttn &a, int row) {
  PagedRow r;
  r.seq = paged_seq(a, row);
  r.lo = 0;
  r.hi = paged_length(a, row, r.seq);
  r.grouped = false;
  // its group: starts[g] <= row < starts[g + 1]
  const int lane = threadIdx.x & 63;
  for (int b = 0; b < a.n_groups; b += 64) {
    const int i = min(b + lane, a.n_groups - 1), start = a.starts[i], end = a.starts[i + 1], shared = paged_shared(a, i);
    const uint64_t in = __ballot(b + lane < a.n_groups && start <= row && row < end);
    if (!in) continue;
    const int at = (int)__builtin_ctzll(in), sh = __shfl(shared, at), first = __shfl(start, at);
    if (sh > 0 && r.hi >= sh) {
      r.lo = sh;
      r.grouped = true;
    } else if (sh > 0) {
      r.seq = paged_seq(a, min(max(first, 0), a.n - 1));
    }
    break;
  }
  return r;
}

// a row's partials: [row][head][slot], slots 0 .. n_own - 1 of its own
// positions, then n_pre of the shared ones
__device__ __forceinline__ int64_t paged_slot(const PagedAttn &a, int64_t row, int head, int slot) {
  return (row * a.n_heads + head) * (a.n_own + a.n_pre) + slot;
}

// The unit-th tile of columns (the heads of a group's rows that share a KV head, row by
// row, `per` at most to a tile), counted group by group: the group's first row and
// number (-1: there is no such tile), the tile's first column and its columns, and
// the positions that the group, and that any group, shares.
struct PagedUnit {
  int first, group, col0, cols, shared, longest;
};
__device__ __forceinline__ PagedUnit paged_unit(const PagedAttn &a, int unit, int per, int G) {
  const int lane = threadIdx.x & 63;
  PagedUnit u{0, -1, 0, 0, 0, 0};
  int left = unit, longest = 0;
  for (int b = 0; b < a.n_groups; b += 64) {
    const int i = b + lane;
    int s = 0, e = 0, shared = 0;
    if (i < a.n_groups) {
      s = min(max(a.starts[i], 0), a.n);
      e = min(max(a.starts[i + 1], s), a.n);
      shared = paged_shared(a, i);
    }
    longest = max(longest, shared);
    int sum = ((e - s) * G + per - 1) / per;
    const int mine = sum;
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o);
      if (lane >= o) sum += v;
    }
    const uint64_t in = __ballot(left < sum);
    if (in && u.group < 0) {
      const int at = (int)__builtin_ctzll(in);
      left -= __builtin_amdgcn_readfirstlane(__shfl(sum, at) - __shfl(mine, at));
      u.first = __builtin_amdgcn_readfirstlane(__shfl(s, at));
      u.group = b + at;
      u.col0 = left * per;
      u.cols = min((__builtin_amdgcn_readfirstlane(__shfl(e, at)) - u.first) * G - u.col0, per);
      u.shared = __builtin_amdgcn_readfirstlane(__shfl(shared, at));
    }
    left -= __builtin_amdgcn_readfirstlane(__shfl(sum, 63));
  }
  for (int o = 32; o; o >>= 1) longest = max(longest, __shfl_xor(longest, o));
  u.longest = __builtin_amdgcn_readfirstlane(longest);
  return u;
}

// Attention of up to 16 CT query columns (a column is a head of a row) over a
// range of positions of one KV head: a row's own positions (PRE false: the
// columns are the heads of one row, CT 1), or the positions that a group of rows
// shares.  One work group takes a split of the range, each wave stripes of 32
// positions on its own, straight from memory into registers.
//
// Scores are S^T = K Q^T, 16 positions x 16 columns: lane (g, c) then holds those
// of positions 4 g .. 4 g + 3 for column c, which is how the second product, O^T +=
// V^T P^T, takes them.  Its k slots of lane group g are positions 4 g .. 4 g + 3 of
// both tiles of a stripe; its rows are channels: a lane loads VE = HD / 16
// consecutive channels of those positions, and row m of tile dt is channel VE m +
// dt.  P enters in parts of the type (PG_PARTS).  fp32 runs on the fp32 products.
//
// Loads go through buffer descriptors made for a tile of 16 positions, which
// end where the positions do: what lies past them reads as zeros.
//
// 256 rows of 1 to 2048 positions and 4 KV heads take 114 us, 4.7 TB/s: memory, with two
// work groups to a CU (registers) and rows of uneven length.  Short rows are a chain of
// loads (group, length, block number, first tiles): 23 us for 32 rows of 32 heads and
// some 200 positions.
template <int HD>
struct AttnLds {
  __align__(16) float o[PG_WAVES][16][HD + 4];
  float m[PG_WAVES][16], l[PG_WAVES][16];
};
template <int DT, int HD, int CT, bool PRE>
__device__ __forceinline__ void attn_columns(const PagedAttn &a, uint32_t block, AttnLds<HD> &lds) {
  constexpr int B = DT == HS_F32 ? 4 : 2;
  constexpr int KCH = HD * B / 64;  // 16-byte chunks of a K row's quarter
  constexpr int VE = HD / 16, VW = VE * B / 4;  // channels of a lane, and their words
  auto &s_o = lds.o;
  auto &s_m = lds.m, &s_l = lds.l;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.n_heads / a.c.n_kv;
  const int ns = PRE ? a.n_pre : a.n_own;
  const int j = block % a.c.n_kv, split = block / a.c.n_kv % ns, unit = block / a.c.n_kv / ns;
  int first = unit, col0 = 0, cols = G, seq, lo = 0, hi, total;
  if constexpr (PRE) {
    const PagedUnit t = paged_unit(a, unit, 16 * CT, G);
    if (t.group < 0) return;
    first = t.first;
    col0 = t.col0;
    cols = t.cols;
    seq = paged_seq(a, first);
    hi = t.shared;
    total = t.longest;
  } else {
    const PagedRow r = paged_row(a, unit);
    seq = __builtin_amdgcn_readfirstlane(r.seq);
    lo = __builtin_amdgcn_readfirstlane(r.lo);
    hi = __builtin_amdgcn_readfirstlane(r.hi);
    total = hi - (lo & ~15);
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  // this split's stripes, of whole ones from the tile of the first position on; groups
  // are cut at equal lengths, so that all splits of long and short ones are alike
  const int base = lo & ~15;
  const int per = max(0, (int)((((int64_t)total + ns - 1) / ns + PG_STRIPE - 1) / PG_STRIPE * PG_STRIPE));
  const int s0 = (int)min((int64_t)hi, base + (int64_t)split * per), s1 = (int)min((int64_t)hi, (int64_t)s0 + per);

  u32x4 q[CT][KCH];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int cc = ct * 16 + c;
    const int r = (col0 + cc) / G, h = j * G + col0 + cc - r * G;
    const char *src = (const char *)a.q + (((int64_t)first + r) * a.ld_q + (int64_t)h * HD) * B + g * 16;
#pragma unroll
    for (int k = 0; k < KCH; ++k) q[ct][k] = cc < cols ? ld16(src + k * 64) : u32x4{0u, 0u, 0u, 0u};
  }

  struct Buf {
    u32x4 k[2][KCH];
    uint32_t v[2][4][VW];
    bool any[2];
  };
  const bool known = (uint32_t)seq < (uint32_t)a.c.n_seqs;
  const int64_t *trow = a.c.table + (known ? (int64_t)seq * a.c.table_ld : 0);
  const int in_block = (1 << a.c.bt_log2) - 1;
  auto load = [&](Buf &b, int pos) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int p0 = pos + 16 * u, at = p0 >> a.c.bt_log2;
      const bool ask = known && p0 < s1 && at < a.c.table_ld;
      const int64_t num = ask ? trow[at] : -1;
      b.any[u] = (uint64_t)num < (uint64_t)a.c.n_blocks;
      const int64_t blk = b.any[u] ? num : 0;
      const uint32_t bytes = b.any[u] ? (uint32_t)min(16, s1 - p0) * (HD * B) : 0u;
      const int64_t inner = (int64_t)(p0 & in_block) * HD;
      const rsrc_t kr = make_rsrc((const char *)a.c.blocks + (paged_slab(a.c, blk, 0, j, HD) + inner) * B, bytes);
      const rsrc_t vr = make_rsrc((const char *)a.c.blocks + (paged_slab(a.c, blk, 1, j, HD) + inner) * B, bytes);
      const int skip = PRE ? 0 : lo - p0;  // rows before the first position
      const uint32_t ko = !PRE && c < skip ? BUF_OOB : (uint32_t)(c * HD * B + g * 16);
#pragma unroll
      for (int k = 0; k < KCH; ++k) b.k[u][k] = PRE ? bld16(kr, ko + k * 64) : bld16_stream(kr, ko + k * 64);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t vo = !PRE && 4 * g + i < skip ? BUF_OOB : (uint32_t)((4 * g + i) * HD * B + c * VE * B);
        if constexpr (VW == 2) {
          const u32x2 t = bld8(vr, vo);
          b.v[u][i][0] = t[0];
          b.v[u][i][1] = t[1];
        } else {
#pragma unroll
          for (int x = 0; x < VW; x += 4) {
            const u32x4 t = PRE ? bld16(vr, vo + x * 4) : bld16_stream(vr, vo + x * 4);
#pragma unroll
            for (int y = 0; y < 4; ++y) b.v[u][i][x + y] = t[y];
          }
        }
      }
    }
  };

  const float c2 = a.scale * 1.4426950408889634f;
  float m[CT], l[CT], highest[CT];  // (the highest m: f16)
  f32x4 o[CT][VE];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = highest[ct] = -INFINITY;
    l[ct] = 0.f;
#pragma unroll
    for (int dt = 0; dt < VE; ++dt) o[ct][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](const Buf &b, int pos) {
    f32x4 s[CT][2];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[ct][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KCH; ++k) s[ct][u] = mma<DT>(b.k[u][k], q[ct][k], s[ct][u]);
        s[ct][u] *= c2;
      }
    if (!b.any[0] || !b.any[1] || pos < lo || pos + 32 > s1) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = pos + 16 * u + 4 * g + i;
          if (!b.any[u] || p < lo || p >= s1) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][u][i] = -INFINITY;
          }
        }
    }
    uint32_t ps[CT][PG_PARTS<DT>][4];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[ct][u][i]);
      // m is the same for the four lanes of a column
      bool move = __ballot(top - m[ct] > PG_UP<DT>);
      if constexpr (DT == HS_F16) {
        uint64_t low = __ballot(top - m[ct] < PG_LOW);
        low &= low >> 32;
        move |= (low & low >> 16 & 0xFFFF) != 0;
      }
      if (move) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        float mn = fmaxf(m[ct], top);
        if constexpr (DT == HS_F16) {
          mn = moved(m[ct], top, top - m[ct], highest[ct]);
          highest[ct] = fmaxf(highest[ct], mn);
        }
        const float corr = m[ct] == mn ? 1.f : __builtin_amdgcn_exp2f(m[ct] - mn);
        l[ct] *= corr;
#pragma unroll
        for (int dt = 0; dt < VE; ++dt) o[ct][dt] *= corr;
        m[ct] = mn;
      }
      const float ref = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[ct][u][i] = __builtin_amdgcn_exp2f(s[ct][u][i] - ref);
          l[ct] += s[ct][u][i];
        }
      if constexpr (DT != HS_F32) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          uint32_t w[PG_PARTS<DT>];
          weight_parts<DT>(s[ct][x >> 1][2 * (x & 1)], s[ct][x >> 1][2 * (x & 1) + 1], w);
#pragma unroll
          for (int i = 0; i < PG_PARTS<DT>; ++i) ps[ct][i][x] = w[i];
        }
      }
    }
    if constexpr (DT == HS_F32) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int dt = 0; dt < VE; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
              o[ct][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.v[u][i][dt]), s[ct][u][i], o[ct][dt],
                                                               0, 0, 0);
    } else {
#pragma unroll
      for (int dt = 0; dt < VE; ++dt) {
        u32x4 av;
        const uint32_t sel = dt & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          av[2 * u] = __builtin_amdgcn_perm(b.v[u][1][dt / 2], b.v[u][0][dt / 2], sel);
          av[2 * u + 1] = __builtin_amdgcn_perm(b.v[u][3][dt / 2], b.v[u][2][dt / 2], sel);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < PG_PARTS<DT>; ++i)
            o[ct][dt] = mma<DT>(av, u32x4{ps[ct][i][0], ps[ct][i][1], ps[ct][i][2], ps[ct][i][3]}, o[ct][dt]);
      }
    }
  };
  Buf b0, b1;
  int pos = s0 + wave * 32;
  load(b0, pos);
  for (; pos < s1; pos += 2 * PG_STRIPE) {
    load(b1, pos + PG_STRIPE);
    step(b0, pos);
    if (pos + PG_STRIPE >= s1) break;
    load(b0, pos + 2 * PG_STRIPE);
    step(b1, pos + PG_STRIPE);
  }

  // the waves' results, 16 columns at a time
  const bool whole = a.n_own + a.n_pre == 1;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    if (ct * 16 >= cols) break;
    if (ct) __syncthreads();
    l[ct] += __shfl_xor(l[ct], 16);
    l[ct] += __shfl_xor(l[ct], 32);
    if (g == 0) {
      s_m[wave][c] = m[ct];
      s_l[wave][c] = l[ct];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int dt = 0; dt < VE; dt += 4)
        *(f32x4 *)&s_o[wave][c][VE * (4 * g + i) + dt] =
            f32x4{o[ct][dt][i], o[ct][dt + 1][i], o[ct][dt + 2][i], o[ct][dt + 3][i]};
    __syncthreads();
    for (int x = tid; x < 16 * HD / 4; x += 64 * PG_WAVES) {
      const int cc = x / (HD / 4), e = x % (HD / 4) * 4;
      if (ct * 16 + cc >= cols) continue;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < PG_WAVES; ++w) M = fmaxf(M, s_m[w][cc]);
      float den = 0.f;
      f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < PG_WAVES; ++w) {
        // (a wave that saw no score keeps -inf and zeros; one that saw NaN alone has NaN sums)
        const float k = s_m[w][cc] == M ? 1.f : __builtin_amdgcn_exp2f(s_m[w][cc] - M);
        den += k * s_l[w][cc];
        num += k * *(const f32x4 *)&s_o[w][cc][e];
      }
      const int r = (col0 + ct * 16 + cc) / G, h = j * G + col0 + ct * 16 + cc - r * G;
      const int64_t row = first + r;
      if (whole) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = den == 0.f ? 0.f : num[i] / den;
        const int64_t at = row * a.ld_out + (int64_t)h * HD + e;
        st_elem2<DT>(a.out, at, f[0], f[1]);
        st_elem2<DT>(a.out, at + 2, f[2], f[3]);
      } else {
        const int64_t at = paged_slot(a, row, h, PRE ? a.n_own + split : split);
        *(f32x4 *)(a.part_o + at * HD + e) = num;
        if (e == 0) {
          a.part_ml[at * 2] = M;
          a.part_ml[at * 2 + 1] = den;
        }
      }
    }
  }
}

// Attention of a tile of query columns over the positions that their group shares,
// in 16-bit types.  The waves, of 32 columns each, share the K and V of 64 positions,
// which are copied straight into LDS a tile ahead.  Scores are S^T = K Q^T, 32
// positions x 32 columns: lane (h, c) holds those of positions 8 i + 4 h + 0 .. 3 for
// column c, and these are its k slots of the second product, O^T += V^T P^T, with
// the rows of V taken in the same order.  Output row m of tile dt is channel VE m +
// dt: a lane reads VE = HD / 32 consecutive channels of eight positions.  P enters
// in parts, as in attn_columns.  16-byte chunk j of K's row p lies at chunk j ^ p, so
// that the 32 rows that a product reads spread over the banks.
//
// 256 rows of 28 heads over 32768 positions in bf16: 271 us, 440 TFLOP/s by the
// definition's operations, 890 with the parts of P.  A wave's tile is 2048 cycles of
// products and more than that of vector instructions, and two waves to a SIMD overlap
// them in part: the matrix cores are busy 48 % of the time, the vector units 53 %.
// With P in two parts (1536 cycles of products) it was 219: eight waves copy half as much a
// column as four (242 to 231 us), columns that rows lie across fill the tiles (219).  Tiles of
// 32 positions, three under way: 267; K, V and weights through registers alone, a wave to
// itself: 304.
// Few columns (HALVES 2: 64 at most) are two waves' each; the other two take the same
// columns over the other half of each tile, and the halves are joined in LDS.
template <int HD>
struct SharedLds {
  __align__(16) unsigned char kv[2][2][64 * HD * 2];
  int rows[2][4];
};
template <int DT, int HD, int WAVES, int HALVES>
__device__ __forceinline__ void shared_columns(const PagedAttn &a, uint32_t block, SharedLds<HD> &lds) {
  constexpr int NU = 2 / HALVES;  // runs of 32 positions that a wave takes of a tile
  constexpr int KK = HD / 16, VE = HD / 32, ROW = HD * 2, CHUNKS = ROW / 16;
  constexpr int TILE = 64, GROUP = 16 * ROW;  // bytes of 16 positions
  constexpr int PARTS = GROUP / 1024;         // copies of 1 KB of them
  constexpr int ROWS = 1024 / ROW;            // rows of a copy
  auto &s_kv = lds.kv;
  auto &s_rows = lds.rows;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.n_heads / a.c.n_kv;
  const int j = block % a.c.n_kv, split = block / a.c.n_kv % a.n_pre, unit = block / a.c.n_kv / a.n_pre;
  const PagedUnit t = paged_unit(a, unit, 32 * WAVES / HALVES, G);
  if (t.group < 0) return;
  const int seq = __builtin_amdgcn_readfirstlane(paged_seq(a, t.first));
  const int hi = t.shared, cols = t.cols;
  // (groups are cut at equal lengths, so that all splits of long and short ones are alike)
  const int per = ((t.longest + a.n_pre - 1) / a.n_pre + TILE - 1) / TILE * TILE;
  const int s0 = min((int64_t)hi, (int64_t)split * per), s1 = min((int64_t)hi, (int64_t)s0 + per);
  const int mine = HALVES == 2 ? wave & 1 : wave, u0 = HALVES == 2 ? wave >> 1 : 0;  // columns, first run
  const int col = mine * 32 + c;
  const bool some = mine * 32 < cols;  // whether the wave has columns
  const int row = t.first + (t.col0 + col) / G, head = j * G + (t.col0 + col) % G;
  u32x4 q[KK];
#pragma unroll
  for (int k = 0; k < KK; ++k)
    q[k] = col < cols ? ld16((const char *)a.q + ((int64_t)row * a.ld_q + (int64_t)head * HD) * 2 + k * 32 + h * 16)
                      : u32x4{0u, 0u, 0u, 0u};

  // wave w copies 16 of the tile's positions, K and V of them or, with eight waves, one
  const bool known = (uint32_t)seq < (uint32_t)a.c.n_seqs;
  const int64_t *trow = a.c.table + (known ? (int64_t)seq * a.c.table_ld : 0);
  const int in_block = (1 << a.c.bt_log2) - 1, part16 = wave & 3;
  // lane i holds the block of the wave's positions of the i-th tile from pos on (-1: none)
  const auto blocks64 = [&](int pos) {
    const int64_t p0 = (int64_t)pos + lane * TILE + 16 * part16, at = p0 >> a.c.bt_log2;
    int64_t num = -1;
    if (known && p0 < s1 && at < a.c.table_ld) num = trow[at];
    return (uint64_t)num < (uint64_t)a.c.n_blocks ? (int)num : -1;
  };
  uint32_t k_off[PARTS];
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    const int r = i * ROWS + lane / CHUNKS, ch = lane % CHUNKS;  // row of the 16, chunk of LDS
    k_off[i] = (uint32_t)(r * ROW + (CHUNKS == 16 ? ch ^ r : ch ^ (r >> 1 & 7)) * 16);
  }
  const auto copy = [&](int buf, int pos, int num) {
    const int p0 = pos + 16 * part16, n = num >= 0 ? min(16, s1 - p0) : 0;
    const int64_t blk = max(num, 0), inner = (int64_t)(p0 & in_block) * HD;
    const uint32_t bytes = (uint32_t)n * ROW;
#pragma unroll
    for (int sel = 0; sel < 2; ++sel) {
      if (WAVES == 8 && wave / 4 != sel) continue;
      const uint64_t at = (uint64_t)((const char *)a.c.blocks + (paged_slab(a.c, blk, sel, j, HD) + inner) * 2);
      const u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, (uint32_t)BUF_WORD3};
      const uint32_t to = lds_addr(&s_kv[buf][sel][part16 * GROUP]);
#pragma unroll
      for (int i = 0; i < PARTS; ++i)
        if (sel) dma_1k(r, (uint32_t)lane * 16, i * 1024, to + i * 1024);
        else dma_1k(r, k_off[i], 0, to + i * 1024);
    }
    if (lane == 0 && wave < 4) s_rows[buf][wave] = n;
  };

  // the scale's sign goes into the queries, so that the largest product has the largest
  // score; of scale 0 the queries are zeros
  float c2 = a.scale * 1.4426950408889634f;
  if (!(c2 > 0.f)) {
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) q[k][w] = c2 == 0.f ? 0u : q[k][w] ^ 0x80008000u;
    c2 = c2 == 0.f ? 1.f : -c2;
  }
  float m = -INFINITY, l = 0.f, highest = -INFINITY;
  f32x16 o[VE];
#pragma unroll
  for (int dt = 0; dt < VE; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  // `part`: some of the tile's positions have no rows
  const auto step = [&](int buf, auto part) {
    const unsigned char *kt = s_kv[buf][0] + u0 * 32 * ROW, *vt = s_kv[buf][1] + u0 * 32 * ROW;
    // chunk 2 k + h of row c, at its place; made anew for every tile, not kept in registers
    int first = (h ^ (CHUNKS == 16 ? c & 15 : c >> 1 & 7)) * 16 + c * ROW;
    asm volatile("" : "+v"(first));
    f32x16 s[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int u = 0; u < NU; ++u) s[u] = mma32<DT>(*(const u32x4 *)(kt + u * 32 * ROW + (first ^ (k * 32))), q[k], s[u]);
    if constexpr (part) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4 & 1) + 4 * h + i % 4 >= s_rows[buf][2 * (u0 + u) + i / 8]) s[u][i] = -INFINITY;
    }
    // scores less m
    const float ref = m == -INFINITY ? 0.f : m;
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[u][i] = __builtin_fmaf(s[u][i], c2, -ref);
        top = fmaxf(top, s[u][i]);
      }
    bool move = __ballot(top > PG_UP<DT> || m == -INFINITY);
    if constexpr (DT == HS_F16) {
      const uint64_t low = __ballot(top < PG_LOW);
      move |= (uint32_t)(low & low >> 32) != 0;
    }
    if (move) {
      top = fmaxf(top, __shfl_xor(top, 32));
      float mn = fmaxf(m, ref + top);
      if constexpr (DT == HS_F16) {
        mn = moved(m, ref + top, m == -INFINITY ? INFINITY : top, highest);
        highest = fmaxf(highest, mn);
      }
      const float up = mn == -INFINITY ? 0.f : mn - ref;
      const float corr = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < VE; ++dt) o[dt] *= corr;
      m = mn;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[u][i] -= up;
          // (of scores so large that their sum with m is rounded; NaN stays)
          if constexpr (DT == HS_F16) s[u][i] = s[u][i] > PG_UP<DT> ? PG_UP<DT> : s[u][i];
        }
    }
    u32x4 ps[PG_PARTS<DT>];
    const auto parts = [&](int x) {  // of 16 positions
      float sum = 0.f;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float p0 = __builtin_amdgcn_exp2f(s[x / 2][8 * (x & 1) + 2 * y]);
        const float p1 = __builtin_amdgcn_exp2f(s[x / 2][8 * (x & 1) + 2 * y + 1]);
        sum += p0 + p1;
        uint32_t w[PG_PARTS<DT>];
        weight_parts<DT>(p0, p1, w);
#pragma unroll
        for (int i = 0; i < PG_PARTS<DT>; ++i) ps[i][y] = w[i];
      }
      l += sum;
    };
    parts(0);
#pragma unroll
    for (int x = 0; x < 2 * NU; ++x) {
      u32x4 px[PG_PARTS<DT>];
#pragma unroll
      for (int i = 0; i < PG_PARTS<DT>; ++i) px[i] = ps[i];
      const unsigned char *vp = vt + (16 * x + 4 * h) * ROW + c * (VE * 2);
      uint32_t v[8][VE / 2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned char *at = vp + (i < 4 ? i : i + 4) * ROW;
        if constexpr (VE == 4) {
          const u32x2 two = *(const u32x2 *)at;
          v[i][0] = two[0];
          v[i][1] = two[1];
        } else {
          v[i][0] = *(const uint32_t *)at;
        }
      }
      if (x < 2 * NU - 1) parts(x + 1);
      u32x4 av[VE];
#pragma unroll
      for (int dt = 0; dt < VE; ++dt) {
        const uint32_t sel = dt & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
        for (int y = 0; y < 4; ++y) av[dt][y] = __builtin_amdgcn_perm(v[2 * y + 1][dt / 2], v[2 * y][dt / 2], sel);
      }
#pragma unroll
      for (int k = 0; k < PG_PARTS<DT>; ++k)
#pragma unroll
        for (int dt = 0; dt < VE; ++dt) o[dt] = mma32<DT>(av[dt], px[k], o[dt]);
      // the vector unit works on the next weights while the matrix cores multiply: a
      // product, then what fits behind it
#pragma unroll
      for (int i = 0; i < PG_PARTS<DT> * VE; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 6, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int nums = blocks64(s0), tile = 0;
  copy(0, s0, __builtin_amdgcn_readlane(nums, 0));
  int buf = 0;
  for (int pos = s0; pos < s1; pos += TILE) {
    dma_sync<0>();
    if (pos + TILE < s1) {
      if ((++tile & 63) == 0) nums = blocks64(pos + TILE);
      copy(buf ^ 1, pos + TILE, __builtin_amdgcn_readlane(nums, tile & 63));
    }
    if (some) {
      const int rows = s_rows[buf][0] + s_rows[buf][1] + s_rows[buf][2] + s_rows[buf][3];
      if (__builtin_amdgcn_readfirstlane(rows) == TILE) step(buf, std::false_type{});
      else step(buf, std::true_type{});
    }
    buf ^= 1;
  }
  dma_sync<0>();  // (an empty split has copies under way)
  l += __shfl_xor(l, 32);
  if constexpr (HALVES == 2) {
    f32x4 *half = (f32x4 *)&s_kv[0][0][0] + mine * 64 + lane;  // a wave's 16 bytes a lane, 128 lanes apart
    f32x2 *half_ml = (f32x2 *)((f32x4 *)&s_kv[0][0][0] + 4 * VE * 128) + mine * 64 + lane;
    static_assert((4 * VE * 16 + 8) * 128 <= sizeof(s_kv), "the halves fit");
    if (u0) {
#pragma unroll
      for (int dt = 0; dt < VE; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) half[(dt * 4 + i / 4) * 128] = f32x4{o[dt][i], o[dt][i + 1], o[dt][i + 2], o[dt][i + 3]};
      *half_ml = f32x2{m, l};
    }
    __syncthreads();
    if (u0) return;
    const f32x2 other = *half_ml;
    const float top = fmaxf(m, other[0]);
    const float k0 = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), k1 = other[0] == top ? 1.f : __builtin_amdgcn_exp2f(other[0] - top);
    m = top;
    l = k0 * l + k1 * other[1];
#pragma unroll
    for (int dt = 0; dt < VE; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 y = half[(dt * 4 + i / 4) * 128];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[dt][i + e] = k0 * o[dt][i + e] + k1 * y[e];
      }
  }
  if (col >= cols) return;
  const int64_t at = paged_slot(a, row, head, a.n_own + split);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float *to = a.part_o + at * HD + VE * (8 * (i / 4) + 4 * h + i % 4);
    if constexpr (VE == 4) *(f32x4 *)to = f32x4{o[0][i], o[1][i], o[2][i], o[3][i]};
    else *(f32x2 *)to = f32x2{o[0][i], o[1][i]};
  }
  if (h == 0) *(f32x2 *)(a.part_ml + at * 2) = f32x2{m, l};
}

// Rows' own positions.
template <int DT, int HD>
__global__ __launch_bounds__(64 * PG_WAVES) void k_paged_own(PagedAttn a) {
  __shared__ AttnLds<HD> lds;
  attn_columns<DT, HD, 1, false>(a, blockIdx.x, lds);
}
// The first `pre` work groups take the shared positions, the others the rows' own: one
// launch, in which the ones' arithmetic and the others' reads overlap.
template <int DT, int HD, int HALVES>
__global__ __launch_bounds__(64 * PG_WAVES, DT == HS_F32 ? 1 : 2) void k_paged_both(PagedAttn a, uint32_t pre) {
  __shared__ union {
    AttnLds<HD> own;
    SharedLds<HD> shared;
  } lds;
  if (blockIdx.x >= pre) attn_columns<DT, HD, 1, false>(a, blockIdx.x - pre, lds.own);
  else if constexpr (DT == HS_F32) attn_columns<DT, HD, 2, true>(a, blockIdx.x, lds.own);
  else shared_columns<DT, HD, PG_WAVES, HALVES>(a, blockIdx.x, lds.shared);
}
// Shared positions of large groups: eight waves, all of a CU's registers.
template <int DT, int HD>
__global__ __launch_bounds__(512, 2) void k_paged_shared(PagedAttn a) {
  __shared__ SharedLds<HD> lds;
  shared_columns<DT, HD, 8, 1>(a, blockIdx.x, lds);
}

// A row's partials joined, in the order of their slots; a thread takes four channels,
// eight slots at a time: 6 us for 67 rows of 28 heads in 13 slots (a work group to a row
// and a slot at a time: 21), 10 for 256 rows in 10.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_paged_join(PagedAttn a) {
  const int heads_wg = 256 / (HD / 4), parts = (a.n_heads + heads_wg - 1) / heads_wg;
  const int row = blockIdx.x / parts;
  const int h = blockIdx.x % parts * heads_wg + threadIdx.x / (HD / 4), e = threadIdx.x % (HD / 4) * 4;
  const int slots = paged_row(a, row).grouped ? a.n_own + a.n_pre : a.n_own;
  if (h >= a.n_heads) return;
  const int64_t at = paged_slot(a, row, h, 0);
  const f32x2 *ml = (const f32x2 *)(a.part_ml + at * 2);
  const f32x4 *po = (const f32x4 *)(a.part_o + at * HD + e);
  float M = -INFINITY, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 8;
  for (int s0 = 0; s0 < slots; s0 += U) {
    f32x2 w[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = min(s0 + u, slots - 1);
      w[u] = ml[s];
      o[u] = po[s * (HD / 4)];
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, w[u][0]);
    const float k0 = M == top ? 1.f : __builtin_amdgcn_exp2f(M - top);
    M = top;
    den *= k0;
    num *= k0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u < slots) {
        const float k = w[u][0] == M ? 1.f : __builtin_amdgcn_exp2f(w[u][0] - M);
        den += k * w[u][1];
        num += k * o[u];
      }
  }
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = den == 0.f ? 0.f : num[i] / den;
  const int64_t to = (int64_t)row * a.ld_out + (int64_t)h * HD + e;
  st_elem2<DT>(a.out, to, f[0], f[1]);
  st_elem2<DT>(a.out, to + 2, f[2], f[3]);
}

template <int DT, int HD>
hipError_t attn_launch(const PagedAttn &a, hipStream_t st) {
  const dim3 block(64 * PG_WAVES);
  const uint32_t own = (uint32_t)((int64_t)a.n * a.n_own * a.c.n_kv), pre = (uint32_t)(a.pre_units * a.n_pre * a.c.n_kv);
  if (!a.n_pre) {
    HS_LAUNCH((k_paged_own<DT, HD>), dim3(own), block, 0, st, a);
  } else if constexpr (DT == HS_F32) {
    HS_LAUNCH((k_paged_both<DT, HD, 1>), dim3(pre + own), block, 0, st, a, pre);
  } else if (a.tile == 256) {
    HS_LAUNCH((k_paged_shared<DT, HD>), dim3(pre), dim3(512), 0, st, a);
    HS_LAUNCH((k_paged_own<DT, HD>), dim3(own), block, 0, st, a);
  } else if (a.tile == 128) {
    HS_LAUNCH((k_paged_both<DT, HD, 1>), dim3(pre + own), block, 0, st, a, pre);
  } else {
    HS_LAUNCH((k_paged_both<DT, HD, 2>), dim3(pre + own), block, 0, st, a, pre);
  }
  if (a.n_own + a.n_pre > 1) {
    const int heads_wg = 256 / (HD / 4);
    const int64_t groups = (int64_t)a.n * ((a.n_heads + heads_wg - 1) / heads_wg);
    HS_LAUNCH((k_paged_join<DT, HD>), dim3((uint32_t)groups), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

template <int DT, int HD>
hipError_t append_launch(const PagedRows &a, hipStream_t st) {
  const int heads = a.n_heads + 2 * a.c.n_kv, at_once = APPEND_THREADS / (HD / 8);
  // heads to a work group: as many as it holds at once, more where 2048 work groups have
  // more; they are some of a row's, or those of up to APPEND_ROWS rows
  const int64_t want = std::max<int64_t>(at_once, (int64_t)a.n * heads / 2048);
  const int rows_wg = (int)std::min<int64_t>(std::max<int64_t>(want / heads, 1), APPEND_ROWS);
  const int heads_wg = want >= heads ? heads : (int)std::min<int64_t>((want + at_once - 1) / at_once * at_once, heads);
  const int parts = (heads + heads_wg - 1) / heads_wg;
  const int64_t groups = ((int64_t)a.n + rows_wg - 1) / rows_wg * parts;
  HS_LAUNCH((k_paged_append<DT, HD>), dim3((uint32_t)groups), dim3(APPEND_THREADS), 0, st, a, rows_wg, heads_wg);
  return hipGetLastError();
}

}  // namespace

// columns of a tile, splits of the shared and of the own positions
void paged_plan(int dtype, int64_t n, int n_heads, int n_kv, int max_len, int n_groups, int max_shared, PagedAttn *a) {
  const int G = n_heads / n_kv;
  a->n_groups = n_groups;
  a->n_pre = a->n_own = 1;
  // work groups: two to a CU.  (Four times as many splits of the own positions took 33 us
  // against 29 for 67 rows of 1..1664, 29 against 23 for 32 rows of 32..384)
  auto splits = [&](int64_t groups, int64_t positions, int64_t least) {
    const int64_t target = 512;
    int64_t s = std::max<int64_t>(1, target / std::max<int64_t>(groups, 1));
    s = std::min(s, (positions + least - 1) / least);
    return (int)std::min<int64_t>(std::max<int64_t>(s, 1), PAGED_MAX_SPLITS);
  };
  if (n_groups && max_shared > 0) {
    // eight waves where most groups fill them: each K and V tile is then copied once for
    // twice the columns
    const int64_t mean = (n * G + n_groups - 1) / n_groups;
    a->tile = dtype == HS_F32 ? 32 : mean > 192 ? 256 : mean > 64 ? 128 : 64;
    a->pre_units = std::min<int64_t>(n, n * G / a->tile + n_groups);
    // groups of one tile each, or one group of many: about so many tiles hold columns
    const int64_t units = std::max<int64_t>(n_groups, (n * G + a->tile - 1) / a->tile);
    // (several groups are of several lengths: twice the splits, of which some are empty)
    a->n_pre = splits((units * n_kv * (a->tile == 256 ? 2 : 1) + (n_groups > 1)) / (n_groups > 1 ? 2 : 1), max_shared, 256);
    // tiles of a group that read the same positions go to the same XCD (work group
    // index modulo 8), whose L2 then holds them, where that leaves nine tenths of the
    // work groups
    if (units > n_groups) {
      int s = a->n_pre;
      while (s > 1 && s * n_kv % 8) --s;
      if (s * n_kv % 8 == 0 && s * 10 >= a->n_pre * 9) a->n_pre = s;
    }
    a->n_own = splits(n * n_kv, std::max(1, max_len - max_shared), 256);
    // one round of work groups rather than a second with a few, while splits are short
    while (a->tile < 256 && a->n_pre > 1 && (units * a->n_pre + n * a->n_own) * n_kv > 512 &&
           max_shared / (a->n_pre - 1) <= 512)
      --a->n_pre;
  } else {
    a->tile = 16;
    a->pre_units = 0;
    a->n_pre = 0;
    a->n_own = splits(n * n_kv, max_len, 256);
  }
}

hipError_t launch_paged_attention(int dtype, int head_dim, const PagedAttn &a, hipStream_t st) {
  if (head_dim == 64) {
    if (dtype == HS_F32) return attn_launch<HS_F32, 64>(a, st);
    if (dtype == HS_F16) return attn_launch<HS_F16, 64>(a, st);
    if (dtype == HS_BF16) return attn_launch<HS_BF16, 64>(a, st);
  } else if (head_dim == 128) {
    if (dtype == HS_F32) return attn_launch<HS_F32, 128>(a, st);
    if (dtype == HS_F16) return attn_launch<HS_F16, 128>(a, st);
    if (dtype == HS_BF16) return attn_launch<HS_BF16, 128>(a, st);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_append(int dtype, int head_dim, const PagedRows &a, hipStream_t st) {
  if (head_dim == 64) {
    if (dtype == HS_F32) return append_launch<HS_F32, 64>(a, st);
    if (dtype == HS_F16) return append_launch<HS_F16, 64>(a, st);
    if (dtype == HS_BF16) return append_launch<HS_BF16, 64>(a, st);
  } else if (head_dim == 128) {
    if (dtype == HS_F32) return append_launch<HS_F32, 128>(a, st);
    if (dtype == HS_F16) return append_launch<HS_F16, 128>(a, st);
    if (dtype == HS_BF16) return append_launch<HS_BF16, 128>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace hs
