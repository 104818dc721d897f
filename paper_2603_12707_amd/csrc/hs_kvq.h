// hs_kvq.h — the KV cache held in 4 bits (gfx950): storing rows, fetching them
// back, and decode attention over it.  Included by hs_misc.hip.
//
// A row's elements are E2M1 numbers (sign, 2 exponent bits, 1 mantissa bit:
// 0, 1/2, 1, 3/2, 2, 3, 4, 6) in groups of 32 that share one power of two, a
// byte holding its exponent + 127.  With a = max |x| of a group the power is
// the least 2^e with a < 7 * 2^e: a is then 3.5 * 2^e at least (but where e is the
// least that there is) and rounds to 4 or 6, and as 7 lies half way between 6 and
// the next step, saturating at 6 moves an element by less than 2^e, which is half
// of the widest step.  Rounding is to nearest, ties to even.  A value takes at most
// 2 significant bits, so it is exact in f16 and in bf16, and gfx950 converts
// both ways in one full-rate instruction for two elements.
#pragma once

#include "hs_device.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace hs {
namespace {

using namespace dev;

// bounds of the exponent byte: every value is a number of the row type (f16:
// 1/2 * 2^-23 is its least subnormal, 6 * 2^13 is finite), and not subnormal in
// fp32 and bf16
template <int DT>
struct KvqByte {
  static constexpr int lo = DT == HS_F16 ? 104 : 2, hi = DT == HS_F16 ? 140 : 252;
};
constexpr uint32_t KVQ_NAN = 255;  // the byte of a group that held a NaN or an infinity: 32 NaNs

// The 4-bit elements of eight values and their group's exponent byte; the group
// is the aligned quad of lanes.
template <int DT>
__device__ __forceinline__ uint32_t kvq_encode(const float *x, uint32_t &byte) {
  uint32_t top = 0;  // bits of |x| order as |x| does, infinities and NaN last
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_QUAD_1032, 0xF, 0xF, false));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_QUAD_2301, 0xF, 0xF, false));
  // 7 is 1.75 * 2^2: a quarter added to the mantissa carries from 1.75 on
  const int b = min(max((int)((top + 0x00200000u) >> 23) - 2, KvqByte<DT>::lo), KvqByte<DT>::hi);
  const bool bad = top >= 0x7F800000u;
  byte = bad ? KVQ_NAN : (uint32_t)b;
  const float s = __uint_as_float((uint32_t)b << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return bad ? 0u : w;
}

// elements 2 B, 2 B + 1 of a word of eight, times the scale, as two of the type
template <int DT, int B>
__device__ __forceinline__ uint32_t kvq_pair(uint32_t w, float s) {
  if constexpr (DT == HS_F16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, B));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, B));
}
__device__ __forceinline__ void kvq_decode(uint32_t w, float s, float *f) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
  f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1], f[4] = c[0], f[5] = c[1], f[6] = d[0], f[7] = d[1];
}
__device__ __forceinline__ float kvq_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight elements at p (16-byte aligned), as fp32 and back
template <int DT>
__device__ __forceinline__ void ld8(const void *p, float *f) {
  if constexpr (DT == HS_F32) {
    unpack<DT>(ld16(p), f);
    unpack<DT>(ld16((const float *)p + 4), f + 4);
  } else {
    unpack<DT>(ld16(p), f);
  }
}
template <int DT>
__device__ __forceinline__ void st8(void *p, const float *f) {
  if constexpr (DT == HS_F32) {
    *(u32x4 *)p = pack<DT>(f);
    *((u32x4 *)p + 1) = pack<DT>(f + 4);
  } else {
    *(u32x4 *)p = pack<DT>(f);
  }
}

// element c of row's output
__device__ __forceinline__ int64_t kvq_out_at(const KvqAttn &a, int64_t row, int c, int hd) {
  return a.out_packed ? packed_x_index((int)row, c, (a.n_heads * hd / 8 + 15) / 16) : row * a.ld_out + c;
}

// row's positions
__device__ __forceinline__ int kvq_length(const KvqAttn &a, int64_t row, int seq) {
  if ((uint32_t)seq >= (uint32_t)a.c.n_seqs) return 0;
  int len = a.lens[a.len_by_seq ? (int64_t)seq : row];
  // in 64 bits, so that no length wraps
  len = (int)min((int64_t)len + a.len_add, (int64_t)a.max_len);
  if (a.cap) len = min(len, a.cap[seq]);
  return (int)min((int64_t)len, (int64_t)a.c.table_ld << a.c.bt_log2);
}

// The block of (sequence, position), or -1: outside the table, without a
// block, or a number that is no block of the cache.
__device__ __forceinline__ int64_t kvq_block(const KvqRef &c, int seq, int pos) {
  const int k = pos >> c.bt_log2;
  if ((uint32_t)seq >= (uint32_t)c.n_seqs || pos < 0 || k >= c.table_ld) return -1;
  const int64_t id = c.table[(int64_t)seq * c.table_ld + k];
  return (uint64_t)id < (uint64_t)c.n_blocks ? id : -1;
}
// bytes of a span (16 positions of one layer, K or V, and head)
__host__ __device__ constexpr int kvq_span_bytes(int hd) { return hd / 2 * 17; }
// the span that holds position pos of block id
__device__ __forceinline__ uint8_t *kvq_span(const KvqRef &c, int hd, int64_t id, int sel, int head, int pos) {
  const int in = pos & ((1 << c.bt_log2) - 1);
  return c.blocks + id * c.block_bytes +
         ((((int64_t)(c.layer * 2 + sel) * c.n_kv + head) << (c.bt_log2 - 4)) + (in >> 4)) * kvq_span_bytes(hd);
}

// row's sequence and position
__device__ __forceinline__ void kvq_place(const KvqRows &a, int row, int &seq, int &pos) {
  seq = a.seqs ? a.seqs[row] : a.seq >= 0 ? a.seq : row;
  pos = !a.pos ? a.pos0 + row : !a.pos_by_seq ? a.pos[row] : (uint32_t)seq < (uint32_t)a.c.n_seqs ? a.pos[seq] : -1;
}

// One thread takes eight elements; a work group takes one head of K or V of
// 2048 / HD consecutive rows, so that a prefill pass's rows fill whole spans of 16
// positions in one place (with all heads of a row in one work group, whose spans
// other work groups share, the pass below took 11.4 us).
// Bound by the bytes: 14370 bf16 rows of 4 heads of 128 (29 MB in, 7.8 MB out) are
// stored in 10.1 us, 3.7 TB/s both ways together, and fetched in 9.5; a copy of
// gigabytes moves 4.8.  A step's 32 rows of 32 heads take 2.6 and 2.4 us, a launch's
// least.
template <int DT, int HD>
struct KvqLine {
  static constexpr int CPR = HD / 8, ROWS = 256 / CPR, SB = DT == HS_F32 ? 4 : 2;
  int row, c, hi, head, sel;
  __device__ __forceinline__ explicit KvqLine(const KvqRows &a) {
    row = (int)blockIdx.x * ROWS + (int)threadIdx.x / CPR;
    c = (int)threadIdx.x % CPR;
    hi = (int)blockIdx.y;
    sel = a.sel;
    if (sel < 0) sel = hi >= a.heads, hi -= sel * a.heads;
    head = a.head0 + hi;
  }
  __device__ __forceinline__ int64_t at(const KvqRows &a, int r) const {
    return ((int64_t)r * a.ld + (int64_t)hi * a.ld_head + c * 8) * SB;
  }
};

template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_append(KvqRows a) {
  const KvqLine<DT, HD> t(a);
  if (t.row >= a.n) return;
  int seq, pos;
  kvq_place(a, t.row, seq, pos);
  const int64_t at = t.at(a, a.row_by_seq ? seq : t.row);
  float f[8];
  ld8<DT>((const char *)(t.sel ? a.v : a.k) + at, f);
  uint32_t byte;
  const uint32_t w = kvq_encode<DT>(f, byte);
  int64_t id = kvq_block(a.c, seq, pos);
  if (id >= 0 && a.cap && pos >= a.cap[seq]) id = -1;
  if (id >= 0) {
    uint8_t *span = kvq_span(a.c, HD, id, t.sel, t.head, pos);
    ((uint32_t *)span)[(pos & 15) * t.CPR + t.c] = w;
    if ((t.c & 3) == 0) span[HD * 8 + (t.c >> 2) * 16 + (pos & 15)] = (uint8_t)byte;
  }
  char *val = (char *)(t.sel ? a.v_out : a.k_out);
  if (val) {
    kvq_decode(w, kvq_scale(byte), f);
    st8<DT>(val + at, f);
  }
}

// The reverse: rows of K and V in the row type; a place without a block gives zeros.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_read(KvqRows a) {
  const KvqLine<DT, HD> t(a);
  if (t.row >= a.n) return;
  int seq, pos;
  kvq_place(a, t.row, seq, pos);
  const int64_t id = kvq_block(a.c, seq, pos);
  uint32_t w = 0, byte = KvqByte<DT>::lo;
  if (id >= 0) {
    const uint8_t *span = kvq_span(a.c, HD, id, t.sel, t.head, pos);
    w = ((const uint32_t *)span)[(pos & 15) * t.CPR + t.c];
    byte = span[HD * 8 + (t.c >> 2) * 16 + (pos & 15)];
  }
  float f[8];
  kvq_decode(w, kvq_scale(byte), f);
  st8<DT>((char *)(t.sel ? a.v_out : a.k_out) + t.at(a, t.row), f);
}

// Decode attention over the 4-bit cache.  One work group = (split of the row's
// positions, row, KV head j); each of its NW waves takes tiles of 64 positions
// and keeps an online softmax for the G query heads of the head in the 16
// columns of the matrix products.
//
// Scores: S^T = K Q^T with 16 positions as rows.  Lane (li, lg) = (lane % 16,
// lane / 16).  K is converted (HD / 4 elements of a position a lane, one group's
// scale) and Q enters the MFMA 16x16x32 as it is in the 16-bit types, as three bf16
// parts in fp32: every product is exact, every sum fp32.  (The scaled MFMA
// 16x16x128 would take K as it lies in memory, but its own sums are good to 2^-16 of
// the largest product only, measured, and its Q would be e4m3 parts under one power of
// two a head: a loud channel took the others' digits.)  Row r of the tile's product t is position
// 16 (r / 4) + 4 t + r % 4, so that a lane ends up with the scores of the 16
// consecutive positions 16 lg .. for head li, which is the B operand of
// O^T += V^T P^T (MFMA 16x16x32): positions 8 m .. 8 m + 7 of each lane group are
// the k range of MFMA m.  For V^T a lane reads its HD / 16 channels of those 16
// positions, converts pairs of channels (exact in the 16-bit type) and pairs the
// positions with v_perm.  P enters as the sum of parts in that type: two of f16 (22
// bits), three of bf16 (24 bits); every sum is fp32, that of P taken before it is cut.
//
// Each wave copies its tiles straight into LDS, K and V alike as they lie in
// memory, a tile and a half ahead, through buffer ranges that end at the last span
// with a position (past it LDS gets zeros and nothing is fetched).  The waits count
// the wave's own copies, so that the waves never meet before the end.  Blocks of 64
// positions and more (WIDE) hold a tile whole; smaller ones are copied span by span.
//
// Measured: 256 rows of 1024 .. 8192 positions (bf16, 28/4 heads of 128; 645 MB)
// 115 us, 5.6 TB/s; from a graph 121, of which the copies alone take 105 and the
// arithmetic alone 89: they overlap for the most part.  (109 with the scaled MFMA and P in
// two parts, for scores off by up to 2^-16 of their largest product and P's bits from the
// 17th on; K and V through registers took 139.)  32 rows of 608 .. 960 (f16, 32/32
// heads; 110 MB) 25 us, from a graph 27: the copies alone 19, the arithmetic alone 21, the
// vector unit a third busy and the matrix cores a ninth: 1024 work groups of uneven length
// in 768 places, each a chain of few tiles.  Two rows of 120000 .. 131072 (bf16; 137 MB)
// 35 us, 37 from a graph, the copies alone 31 and the arithmetic 32, 20 at the read rate:
// the ramp, the last tiles and the join of 32 splits are in each.  One row of 700 8 us: the
// length, the block number and the first tile's copy one after the other, 2 us a tile, the
// merge.
template <int DT>
constexpr int KVQ_MMA = DT == HS_F16 ? HS_F16 : HS_BF16;
template <int DT>
constexpr int KVQ_P_PARTS = DT == HS_F16 ? 2 : 3;
template <int DT>
constexpr int KVQ_Q_PARTS = DT == HS_F32 ? 3 : 1;
constexpr int KVQ_TILE = 64, KVQ_PLANES = 3;
// Rows are started longest first where some CU takes more than one work group and the
// longest rows take a while: up to this many rows, from more positions on.  28/4 heads, in
// their own order and longest first: 250 rows of 1024 .. 8192 140 and 121 us, 66 rows 64.6
// and 57.1, 160 rows of 400 .. 2000 34.9 and 30.2, of 200 .. 1000 22.7 and 21.8.
constexpr int KVQ_CUS = 256, KVQ_RANK_MOST = 256, KVQ_RANK_FROM = 1024;
typedef const __attribute__((address_space(4))) int64_t ConstI64;

// as dma_1k_stream, four bytes a lane
__device__ __forceinline__ void dma_dwords_stream(u32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen nt lds" ::"s"(lds), "v"(voff),
               "s"(rsrc), "s"(soff)
               : "memory");
}
// at most N of this wave's copies still in flight
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// this wave's LDS reads done
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// In units of the base-2 exponent: a column's probabilities are 2^(s - m) for a
// reference m that is put KVQ_BIAS below the largest score when a score passes it
// by more than KVQ_BIAS + KVQ_SLACK, and o and l are rescaled then.  f16 parts
// reach from 2^16 down to 2^-24 only: the bias puts the largest probability at
// 2^11 at least, so that what is dropped is below 2^-36 of it.  The other types
// have fp32's range.
template <int DT>
constexpr float KVQ_BIAS = DT == HS_F16 ? 11.f : 0.f;
template <int DT>
constexpr float KVQ_SLACK = DT == HS_F16 ? 4.f : 11.5f;
// From this reference on, scores are rounded before it is subtracted (as in
// prefill attention: below it one fma leaves s - m off by at most half an ulp of
// m, 2^-5, the same factor in o and l).
constexpr float KVQ_ROUND_FROM = 0x1p20f;

// word x of a matrix operand of parts: R(f0) | R(f1) << 16, and what is left
template <int MT>
__device__ __forceinline__ uint32_t take_part(float &f0, float &f1) {
  const uint32_t w = pack2<MT>(f0, f1);
  f0 -= lo_f32<MT>(w);
  f1 -= hi_f32<MT>(w);
  return w;
}

// The same of fp32 numbers of any size, cut to their upper 16 bits and not rounded: three
// parts hold all 24 bits either way, and the largest numbers do not round to infinity.
__device__ __forceinline__ uint32_t cut_part(float &f0, float &f1) {
  const uint32_t a = __float_as_uint(f0), b = __float_as_uint(f1);
  f0 -= __uint_as_float(a & 0xFFFF0000u);
  f1 -= __uint_as_float(b & 0xFFFF0000u);
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// past the caches of one XCD
__device__ __forceinline__ void st_agent(float *p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float ld_agent(const float *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The z-th longest row (the lower number first among equals) of at most 256, which
// every wave finds by itself: the largest length that more than z rows reach, bit by
// bit, then the row among those of that length.
__device__ __forceinline__ int kvq_ranked_row(const KvqAttn &a, int z) {
  constexpr int PER = KVQ_RANK_MOST / 64;
  const int lane = threadIdx.x & 63;
  int len[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int r = k * 64 + lane;
    len[k] = r < a.n ? max(kvq_length(a, r, a.seqs ? a.seqs[r] : r), 0) : -1;
  }
  auto reach = [&](int v) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) n += (int)__popcll(__ballot(len[k] >= v));
    return n;
  };
  int t = 0;
  for (int b = 31 - __builtin_clz(a.max_len); b >= 0; --b)
    if (reach(t | 1 << b) > z) t |= 1 << b;
  int left = z - reach(t + 1), row = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const uint64_t same = __ballot(len[k] == t);
    const int n = (int)__popcll(same);
    if (left >= 0 && left < n)
      row = k * 64 + (int)__builtin_ctzll(__ballot(((same >> lane) & 1) &&
                                                   (int)__popcll(same & ((1ull << lane) - 1)) == left));
    left -= n;
  }
  return __builtin_amdgcn_readfirstlane(row);
}

template <int DT, int HD, int NW, bool WIDE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(DT == HS_F32 || NW == 8 ? 2 : 3))) void k_kvq_attn(KvqAttn a) {
  constexpr int MT = KVQ_MMA<DT>, PP = KVQ_P_PARTS<DT>, QP = KVQ_Q_PARTS<DT>;
  constexpr int VB = HD / 32;             // bytes of a lane's V elements of one position
  constexpr int ND = HD / 16;             // 16-channel tiles of the output
  constexpr int SPAN = kvq_span_bytes(HD);
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  constexpr int PLANE = 4 * SPAN;
  __shared__ __align__(1024) unsigned char s_mem[NW * KVQ_PLANES * PLANE];
  const int G = a.n_heads / a.c.n_kv;
  // every row's first split comes before any row's second: the empty ones are last
  const int64_t bid = blockIdx.x, per = (int64_t)a.n * a.c.n_kv;
  const int split = (int)(bid / per), j = (int)(bid % a.c.n_kv);
  const int z = (int)(bid % per / a.c.n_kv);
  const int row = a.order ? a.order[z] : a.rank ? kvq_ranked_row(a, z) : z;
  const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seq = a.seqs ? a.seqs[row] : row;
  const int t0 = split * a.S;
  // the first tiles' block numbers are asked for beside the length
  // (through the scalar cache: the copies below clobber memory for all that the compiler knows)
  constexpr int NB = WIDE ? 1 : 4;  // of a tile: its block, or its spans' blocks
  struct Ids {
    int64_t id[NB];
  };
  const bool known = (uint32_t)seq < (uint32_t)a.c.n_seqs;
  const ConstI64 *tab = (const ConstI64 *)(uintptr_t)(a.c.table + (known ? (int64_t)seq * a.c.table_ld : 0));
  const int room = (int)min((int64_t)a.c.table_ld << a.c.bt_log2, (int64_t)INT32_MAX);
  auto lookup = [&](int t, int before) {  // places from `before` on have none
    Ids w;
#pragma unroll
    for (int s = 0; s < NB; ++s) {
      const int p = t0 + t * KVQ_TILE + s * 16;
      w.id[s] = p < before ? tab[p >> a.c.bt_log2] : -1;
    }
    return w;
  };
  auto settle = [&](Ids w, int t, int end) {
#pragma unroll
    for (int s = 0; s < NB; ++s)
      if (t0 + t * KVQ_TILE + s * 16 >= end || (uint64_t)w.id[s] >= (uint64_t)a.c.n_blocks) w.id[s] = -1;
    return w;
  };
  const Ids first = lookup(wave, room), second = lookup(wave + NW, room);
  const int len = kvq_length(a, row, seq);
  const int64_t rh = (int64_t)row * a.n_heads + j * G;  // first (row, head) of the group
  // the row's splits that have a position; a single one writes the output itself,
  // unless every split's partial is wanted (a.nat)
  const int live = a.nat ? a.n_split : max(1, (len + a.S - 1) / a.S);
  if (split >= live) return;
  if (t0 >= len) {
    for (int i = threadIdx.x; i < G * HD; i += 64 * NW) {
      const int h = i / HD, e = i - h * HD;
      if (live == 1) {
        st_elem<DT>(a.out, kvq_out_at(a, row, (j * G + h) * HD + e, HD), 0.f);
      } else {
        a.part_o[((rh + h) * a.n_split + split) * HD + e] = 0.f;
        if (e == 0) {
          a.part_ml[((rh + h) * a.n_split + split) * 2] = -INFINITY;
          a.part_ml[((rh + h) * a.n_split + split) * 2 + 1] = 0.f;
        }
      }
    }
    return;
  }
  // the split's positions: t0 .. end - 1.  The last one takes what is left: a replayed step may
  // serve a request of a larger capacity than any that S was made for.
  const int end = split == a.n_split - 1 ? len : min(t0 + a.S, len);
  const int n_tiles = (end - t0 + KVQ_TILE - 1) / KVQ_TILE;
  const int64_t kin = ((int64_t)(a.c.layer * 2) * a.c.n_kv + j) << (a.c.bt_log2 - 4);  // spans before the head's
  const int64_t vin = kin + ((int64_t)a.c.n_kv << (a.c.bt_log2 - 4));
  const int in_mask = (1 << a.c.bt_log2) - 1;

  // the wave's ring of planes, a plane being a tile's four K or V spans
  constexpr int COPIES = WIDE ? PLANE / 1024 + 1 : 8;  // of a plane
  unsigned char *ring = s_mem + wave * (KVQ_PLANES * PLANE);
  const uint32_t ring0 = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  const int kspan = li >> 2, vgrp = HD == 128 ? li >> 2 : li >> 3;
  // K (v = 0) or V of tile t into plane `slot` of the ring
  auto copy = [&](int t, const Ids &w, int v, int slot) {
    const int p0 = t0 + t * KVQ_TILE;
    const uint32_t lds = ring0 + slot * PLANE;
    if constexpr (WIDE) {
      const uint64_t at = (uint64_t)(uintptr_t)a.c.blocks + (uint64_t)max(w.id[0], (int64_t)0) * a.c.block_bytes +
                          (uint64_t)((v ? vin : kin) + ((p0 & in_mask) >> 4)) * SPAN;
      const uint32_t bytes = w.id[0] < 0 ? 0u : (uint32_t)((min(end - p0, KVQ_TILE) + 15) / 16 * SPAN);
      const u32x4 r{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, (uint32_t)BUF_WORD3};
#pragma unroll
      for (int x = 0; x < PLANE / 1024; ++x) dma_1k_stream(r, lane * 16, x * 1024, lds + x * 1024);
      if (lane < PLANE % 1024 / 4) dma_dwords_stream(r, lane * 4, PLANE / 1024 * 1024, lds + PLANE / 1024 * 1024);
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint64_t at = (uint64_t)(uintptr_t)a.c.blocks + (uint64_t)max(w.id[s], (int64_t)0) * a.c.block_bytes +
                            (uint64_t)((v ? vin : kin) + (((p0 + s * 16) & in_mask) >> 4)) * SPAN;
        const u32x4 r{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, w.id[s] < 0 ? 0u : (uint32_t)SPAN, (uint32_t)BUF_WORD3};
        if (lane < HD / 2) dma_1k_stream(r, lane * 16, 0, lds + s * SPAN);
        if (lane < HD / 8) dma_dwords_stream(r, lane * 4, HD * 8, lds + s * SPAN + HD * 8);
      }
    }
  };

  // the reference (base-2 units) and this lane's share of the sum; the reference
  // starts at the lowest finite number, so that s - m is a number for s = -inf
  float m = -FLT_MAX, l = 0.f;
  bool big = true;  // some column's |m| >= KVQ_ROUND_FROM (wave-uniform)
  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  // The first planes' copies go out before the query is read; plane x + 3 (K and
  // V of the wave's tiles in turn) follows as soon as plane x is read.  After the
  // wait for a plane at most two that were asked for later are in flight.
  static_assert(KVQ_PLANES == 3, "the order of the copies below");
  Ids nxt = settle(second, wave + NW, end);
  auto held_of = [&](const Ids &w) {  // bit s: span s has a block
    if constexpr (WIDE) return w.id[0] >= 0 ? 15u : 0u;
    else return (w.id[0] >= 0 ? 1u : 0u) | (w.id[1] >= 0 ? 2u : 0u) | (w.id[2] >= 0 ? 4u : 0u) | (w.id[3] >= 0 ? 8u : 0u);
  };
  uint32_t held_cur;
  {
    const Ids cur = settle(first, wave, end);
    held_cur = held_of(cur);
    if (wave < n_tiles) {
      copy(wave, cur, 0, 0);
      copy(wave, cur, 1, 1);
    }
  }
  if (wave + NW < n_tiles) copy(wave + NW, nxt, 0, 2);
  int slot = 0;  // of the tile's K
  auto next_slot = [](int x) { return x == KVQ_PLANES - 1 ? 0 : x + 1; };
  // Q^T operand: head li of the group (zeros past it)
  // (a negative scale's sign goes to Q, so that the scores' order is that of the products)
  const float sign = a.scale < 0.f ? -1.f : 1.f;
  u32x4 qh[QP][HD / 32];  // in the 16-bit type, or its parts
#pragma unroll
  for (int c = 0; c < HD / 32; ++c) {
    const char *at = (const char *)a.q + ((int64_t)row * a.ld_q + (j * G + li) * HD + lg * (HD / 4) + c * 8) * SB;
    if constexpr (DT == HS_F16) {
      typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
      u32x4 w{0u, 0u, 0u, 0u};
      if (li < G) w = ld16(at);
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // (an infinity becomes a NaN, as in the other types)
        const uint32_t word = w[x];
        const f16x2 v = __builtin_bit_cast(f16x2, word);
        const f16x2 zero{(_Float16)0.f, (_Float16)0.f}, sg{(_Float16)sign, (_Float16)sign};
        qh[0][c][x] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(v, zero, v * sg));
      }
    } else {
      float f[8] = {};
      if (li < G) ld8<DT>(at, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __builtin_fmaf(f[e], 0.f, f[e] * sign);
#pragma unroll
      for (int p = 0; p < QP; ++p)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          qh[p][c][x] = DT == HS_F32 ? cut_part(f[2 * x], f[2 * x + 1]) : pack2<MT>(f[2 * x], f[2 * x + 1]);
    }
  }
  const float c2 = fabsf(a.scale) * 1.44269504088896341f;

  for (int t = wave; t < n_tiles; t += NW) {
    const int p0 = t0 + t * KVQ_TILE;
    const bool one = t + NW < n_tiles, two = t + 2 * NW < n_tiles;  // tiles that follow
    const int vslot = next_slot(slot);
    const unsigned char *kp = ring + slot * PLANE, *vp = ring + vslot * PLANE;
    const Ids far = settle(lookup(t + 2 * NW, end), t + 2 * NW, end);
    if (one) wait_copies<2 * COPIES>();  // V, and the next tile's K
    else wait_copies<COPIES>();
    f32x4 sc[4];
    constexpr int FGRP = HD == 128 ? 0 : 1;  // lane groups to a group of 32, as a shift
    const u32x4 ks = *(const u32x4 *)(kp + kspan * SPAN + HD * 8 + (lg >> FGRP) * 16);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint32_t *at = (const uint32_t *)(kp + kspan * SPAN + (4 * x + (li & 3)) * (HD / 2) + lg * (HD / 8));
      const float s = __uint_as_float((ks[x] >> (8 * (li & 3))) << 23);  // (exponent bits alone)
      sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        const uint32_t w = at[c];
        const u32x4 kv{kvq_pair<MT, 0>(w, s), kvq_pair<MT, 1>(w, s), kvq_pair<MT, 2>(w, s), kvq_pair<MT, 3>(w, s)};
#pragma unroll
        for (int p = QP - 1; p >= 0; --p) sc[x] = mma<MT>(kv, qh[p][c], sc[x]);
      }
    }
    if (one) {
      wait_lds();
      copy(t + NW, nxt, 1, slot);
      wait_copies<2 * COPIES>();  // the next tile's K and V
    } else {
      wait_copies<0>();
    }
    uint32_t vc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned char *at = vp + lg * SPAN + i * (HD / 2) + li * VB;
      if constexpr (HD == 128) vc[i] = *(const uint32_t *)at;
      else vc[i] = *(const uint16_t *)at;
    }
    u32x4 vs = *(const u32x4 *)(vp + lg * SPAN + HD * 8 + vgrp * 16);
    // which of the lane's 16 positions count: all of them in a whole tile
    const bool held = (held_cur >> lg) & 1;
    const int left = end - p0 - 16 * lg;
    const bool whole = p0 + KVQ_TILE <= end && held_cur == 15u;
    if (!whole) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!held || 4 * x + i >= left) {
            sc[x][i] = -INFINITY;
            vc[4 * x + i] = 0u;                       // what lies there may be NaN
            vs[x] &= ~(255u << (8 * i));
          }
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, sc[x][i]);
    tmax *= c2;
    if (__ballot(tmax > m + (KVQ_BIAS<DT> + KVQ_SLACK<DT>))) {
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
      const float mn = fmaxf(m, tmax - KVQ_BIAS<DT>);
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= corr;
      m = mn;
      big = __ballot(fabsf(mn) >= KVQ_ROUND_FROM) != 0;
    }
    const float mul = big ? 1.f : c2, sub = big ? 0.f : m;
    if (big) {
#pragma clang fp contract(off)
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[x][i] = sc[x][i] * c2 - m;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[x][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x][i], mul, -sub));
    if (!whole) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[x][i] = !held || 4 * x + i >= left ? 0.f : sc[x][i];
    }
    // the conversion reads bits 23 .. 30 of its scale, the exponent, alone
    float vf[16];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      vf[4 * x] = __uint_as_float(vs[x] << 23);
      vf[4 * x + 1] = __uint_as_float(vs[x] << 15);
      vf[4 * x + 2] = __uint_as_float(vs[x] << 7);
      vf[4 * x + 3] = __uint_as_float(vs[x] >> 1);
    }
    u32x4 pb[2][PP];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float f0 = sc[2 * h + (x >> 1)][2 * (x & 1)], f1 = sc[2 * h + (x >> 1)][2 * (x & 1) + 1];
        l += f0 + f1;
#pragma unroll
        for (int p = 0; p < PP; ++p) pb[h][p][x] = take_part<MT>(f0, f1);
      }
    auto pv = [&](auto bc) {
      constexpr int B = decltype(bc)::value;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 lo, hi;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t w0 = kvq_pair<MT, B>(vc[8 * h + 2 * x], vf[8 * h + 2 * x]);
          const uint32_t w1 = kvq_pair<MT, B>(vc[8 * h + 2 * x + 1], vf[8 * h + 2 * x + 1]);
          lo[x] = __builtin_amdgcn_perm(w1, w0, 0x05040100u);
          hi[x] = __builtin_amdgcn_perm(w1, w0, 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < PP; ++p) {
          o[2 * B] = mma<MT>(lo, pb[h][p], o[2 * B]);
          o[2 * B + 1] = mma<MT>(hi, pb[h][p], o[2 * B + 1]);
        }
      }
    };
    pv(std::integral_constant<int, 0>{});
    pv(std::integral_constant<int, 1>{});
    if constexpr (HD == 128) {
      pv(std::integral_constant<int, 2>{});
      pv(std::integral_constant<int, 3>{});
    }
    if (two) {
      wait_lds();
      copy(t + 2 * NW, far, 0, vslot);
    }
    held_cur = held_of(nxt);
    nxt = far;
    slot = next_slot(vslot);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // merge the waves: lane (li, lg) holds channels d = (4 lg + i) (HD / 16) + dt of head li
  __shared__ float s_m[NW][16], s_l[NW][16];
  float(*s_o)[16][HD + 1] = (float(*)[16][HD + 1]) s_mem;  // over the rings
  static_assert(16 * (HD + 1) * 4 <= KVQ_PLANES * PLANE, "the merge fits the rings");
  if (lg == 0) {
    s_m[wave][li] = m;
    s_l[wave][li] = l;
  }
  __syncthreads();
  if (li < G)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_o[wave][li][(4 * lg + i) * ND + dt] = o[dt][i];
  __syncthreads();
  for (int i = threadIdx.x; i < G * HD; i += 64 * NW) {
    const int h = i / HD, e = i - h * HD;
    float M = s_m[0][h];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][h]);
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float wt = __builtin_amdgcn_exp2f(s_m[w][h] - M);
      num += wt * s_o[w][h][e];
      den += wt * s_l[w][h];
    }
    const float mp = den == 0.f ? -INFINITY : a.nat ? M * 0.693147180559945309f : M;  // -inf: no position held
    const int64_t at = (rh + h) * a.n_split + split;
    if (live == 1) {
      st_elem<DT>(a.out, kvq_out_at(a, row, (j * G + h) * HD + e, HD), den == 0.f ? 0.f : num / den);
    } else if (a.count) {
      st_agent(&a.part_o[at * HD + e], num);
      if (e == 0) {
        st_agent(&a.part_ml[at * 2], mp);
        st_agent(&a.part_ml[at * 2 + 1], den);
      }
    } else {
      a.part_o[at * HD + e] = num;
      if (e == 0) {
        a.part_ml[at * 2] = mp;
        a.part_ml[at * 2 + 1] = den;
      }
    }
  }
  if (!a.count || live == 1) return;
  // The row's last work group to arrive joins the splits.  Partials are stored and
  // read at agent scope, past the caches of one XCD; each wave's are done before
  // the barrier, behind which one thread counts the work group in.
  int &s_last = *(int *)&s_m[0][0];
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    // (counters as far apart as they may lie, so that few share a cache line)
    uint32_t *c = a.count + (row * a.c.n_kv + j) * min(32, KVQ_COUNTERS / (a.n * a.c.n_kv));
    const bool last = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(live - 1);
    if (last) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next call
    s_last = last;
  }
  __syncthreads();
  if (!s_last) return;
  float *jm = (float *)s_mem, *jl = jm + 16 * KVQ_JOIN_SPLITS;
  static_assert(sizeof(s_mem) >= 2 * 16 * KVQ_JOIN_SPLITS * 4, "maxima and sums of the splits");
  for (int i = threadIdx.x; i < G * live; i += 64 * NW) {
    const int h = i / live, s = i - h * live;
    jm[h * KVQ_JOIN_SPLITS + s] = ld_agent(&a.part_ml[((rh + h) * a.n_split + s) * 2]);
    jl[h * KVQ_JOIN_SPLITS + s] = ld_agent(&a.part_ml[((rh + h) * a.n_split + s) * 2 + 1]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * HD; i += 64 * NW) {
    const int h = i / HD, e = i - h * HD;
    const float *hm = jm + h * KVQ_JOIN_SPLITS, *hl = jl + h * KVQ_JOIN_SPLITS;
    float M = -FLT_MAX;
    for (int s = 0; s < live; ++s) M = fmaxf(M, hm[s]);
    float num = 0.f, den = 0.f;
    constexpr int AHEAD = 8;
    for (int s0 = 0; s0 < live; s0 += AHEAD) {
      float v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) v[u] = ld_agent(&a.part_o[((rh + h) * a.n_split + min(s0 + u, live - 1)) * HD + e]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const float w = s0 + u < live ? __builtin_amdgcn_exp2f(hm[min(s0 + u, live - 1)] - M) : 0.f;
        num += w * v[u];
        den += w * hl[min(s0 + u, live - 1)];
      }
    }
    st_elem<DT>(a.out, kvq_out_at(a, row, (j * G + h) * HD + e, HD), den == 0.f ? 0.f : num / den);
  }
}

// o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the splits of a (row,
// head); zeros where none holds a position.  HD / 4 threads take a split's
// partial, 1024 / HD splits at a time, several of them in flight.  64 splits of 28
// heads: 4.6 us, two dependent reads (beside 20 us of attention over 131072 positions).
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_combine(KvqAttn a) {
  constexpr int TPS = HD / 4, PARTS = 256 / TPS, AHEAD = 4;
  __shared__ float s_w[KVQ_MAX_SPLITS];
  __shared__ float s_m[4], s_d[4];
  __shared__ __align__(16) float s_n[PARTS][HD];
  const int h = blockIdx.x % a.n_heads;
  const int64_t row = blockIdx.x / a.n_heads, base = (row * a.n_heads + h) * a.n_split;
  const int ns = (kvq_length(a, row, a.seqs ? a.seqs[row] : (int)row) + a.S - 1) / a.S;
  if (ns <= 1) return;  // written already
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = threadIdx.x % TPS, part = threadIdx.x / TPS;
  static_assert(KVQ_MAX_SPLITS <= 256, "one split's maximum and sum per thread");
  float m = -FLT_MAX, l = 0.f;
  if ((int)threadIdx.x < ns) {
    m = fmaxf(a.part_ml[(base + threadIdx.x) * 2], -FLT_MAX);
    l = a.part_ml[(base + threadIdx.x) * 2 + 1];
  }
  const float wm = wave_max(m);
  if (lane == 0) s_m[wave] = wm;
  __syncthreads();
  const float M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  const float w = __builtin_amdgcn_exp2f(m - M), wd = wave_sum(w * l);
  s_w[threadIdx.x] = w;
  if (lane == 0) s_d[wave] = wd;
  __syncthreads();
  const float den = (s_d[0] + s_d[1]) + (s_d[2] + s_d[3]);
  const f32x4 *po = (const f32x4 *)(a.part_o + base * HD) + c;
  f32x4 num{0.f, 0.f, 0.f, 0.f};
  int s = part;
  for (; s + (AHEAD - 1) * PARTS < ns; s += AHEAD * PARTS) {
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = po[(int64_t)(s + u * PARTS) * TPS];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) num += s_w[s + u * PARTS] * v[u];
  }
  for (; s < ns; s += PARTS) num += s_w[s] * po[(int64_t)s * TPS];
  *(f32x4 *)&s_n[part][c * 4] = num;
  __syncthreads();
  const int e = threadIdx.x;
  if (e >= HD) return;
  float v = 0.f;
#pragma unroll
  for (int p = 0; p < PARTS; ++p) v += s_n[p][e];
  st_elem<DT>(a.out, kvq_out_at(a, row, h * HD + e, HD), den == 0.f ? 0.f : v / den);
}

template <int DT, int HD>
hipError_t kvq_rows(const KvqRows &a, bool read, hipStream_t st) {
  const int rows = KvqLine<DT, HD>::ROWS, lines = (a.sel < 0 ? 2 : 1) * a.heads;
  if (lines > 65535) return hipErrorInvalidValue;
  const dim3 grid((a.n + (int64_t)rows - 1) / rows, lines);
  if (read) HS_LAUNCH((k_kvq_read<DT, HD>), grid, dim3(256), 0, st, a);
  else HS_LAUNCH((k_kvq_append<DT, HD>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int DT>
hipError_t kvq_rows_dt(int hd, const KvqRows &a, bool read, hipStream_t st) {
  if (hd == 64) return kvq_rows<DT, 64>(a, read, st);
  if (hd == 128) return kvq_rows<DT, 128>(a, read, st);
  return hipErrorInvalidValue;
}
hipError_t kvq_rows_any(int dtype, int hd, const KvqRows &a, bool read, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  switch (dtype) {
    case HS_F32: return kvq_rows_dt<HS_F32>(hd, a, read, st);
    case HS_F16: return kvq_rows_dt<HS_F16>(hd, a, read, st);
    case HS_BF16: return kvq_rows_dt<HS_BF16>(hd, a, read, st);
  }
  return hipErrorInvalidValue;
}

// Waves of a work group: eight while there are no more pairs than CUs, four where
// several work groups share a CU (their LDS holds three).  bf16 rows of 3000 .. 4000 in 256
// pairs take 29.8 us with eight and 33.0 with four, in 288 pairs 48.2 and 42.9 (f16: 27.2
// and 30.7, 41.8 and 38.4).
int kvq_waves(int64_t pairs) { return pairs <= 256 ? 8 : 4; }

template <int DT, int HD, int NW>
void kvq_attn_start(const KvqAttn &a, uint32_t grid, hipStream_t st) {
  if ((1 << a.c.bt_log2) >= KVQ_TILE) HS_LAUNCH((k_kvq_attn<DT, HD, NW, true>), dim3(grid), dim3(64 * NW), 0, st, a);
  else HS_LAUNCH((k_kvq_attn<DT, HD, NW, false>), dim3(grid), dim3(64 * NW), 0, st, a);
}
template <int DT, int HD>
hipError_t kvq_attn_hd(KvqAttn a, hipStream_t st) {
  const int64_t grid = (int64_t)a.n * a.c.n_kv * a.n_split;
  if (grid > INT32_MAX || a.n_split > KVQ_MAX_SPLITS) return hipErrorInvalidValue;
  a.rank = !a.order && a.n_split == 1 && a.n > 1 && a.n <= KVQ_RANK_MOST && a.max_len > KVQ_RANK_FROM &&
           grid > KVQ_CUS;
  if (kvq_waves((int64_t)a.n * a.c.n_kv) == 8) kvq_attn_start<DT, HD, 8>(a, (uint32_t)grid, st);
  else kvq_attn_start<DT, HD, 4>(a, (uint32_t)grid, st);
  return hipGetLastError();
}
template <int DT, int HD>
hipError_t kvq_combine_hd(const KvqAttn &a, hipStream_t st) {
  const int64_t rows = (int64_t)a.n * a.n_heads;
  if (rows > INT32_MAX || a.n_split > KVQ_MAX_SPLITS || a.nat) return hipErrorInvalidValue;
  HS_LAUNCH((k_kvq_combine<DT, HD>), dim3((uint32_t)rows), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int DT>
hipError_t kvq_attn_dt(int hd, bool combine, const KvqAttn &a, hipStream_t st) {
  if (hd == 64) return combine ? kvq_combine_hd<DT, 64>(a, st) : kvq_attn_hd<DT, 64>(a, st);
  if (hd == 128) return combine ? kvq_combine_hd<DT, 128>(a, st) : kvq_attn_hd<DT, 128>(a, st);
  return hipErrorInvalidValue;
}
hipError_t kvq_attn_any(int dtype, int hd, bool combine, const KvqAttn &a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  switch (dtype) {
    case HS_F32: return kvq_attn_dt<HS_F32>(hd, combine, a, st);
    case HS_F16: return kvq_attn_dt<HS_F16>(hd, combine, a, st);
    case HS_BF16: return kvq_attn_dt<HS_BF16>(hd, combine, a, st);
  }
  return hipErrorInvalidValue;
}

__global__ __launch_bounds__(256) void k_kvq_stage(PackedRows pk, int hd, KvqStage s) {
  const int r = (int)blockIdx.x * 256 + threadIdx.x, rows = pk.cu[pk.n];
  if (r < pk.n) {
    s.start[pk.req[r]] = (int64_t)pk.cu[r] * hd;
    s.bt[pk.req[r]] = rows;
  }
  if (r >= rows) return;
  const int i = packed_request(&pk, r);
  s.seqs[r] = pk.req[i];
  s.pos[r] = r - pk.cu[i];
}

}  // namespace


// Splits where there are at most half as many (row, KV head) pairs as CUs: as many
// as the CUs hold at once (a work group of eight waves takes one), but none without
// a tile for each of its waves, and none up to 1024 positions, where joining takes
// the time of the two tiles a wave that it would save (one row of 768, 32/32 heads:
// 9.2 us whole, 10.1 in two).
void kvq_split_policy(int64_t n, int n_kv, int max_len, int *S, int *n_split) {
  const int64_t pairs = std::max<int64_t>(1, n * n_kv);
  constexpr int LEAST = 8 * KVQ_TILE;
  const int64_t most = max_len <= 2 * LEAST ? 1 : ((int64_t)max_len + LEAST - 1) / LEAST;
  const int64_t ns = std::max<int64_t>(1, std::min(std::min(256 / pairs, most), (int64_t)KVQ_MAX_SPLITS));
  const int64_t s = ((max_len + ns - 1) / ns + 255) / 256 * 256;
  *S = (int)std::min<int64_t>(s, 1 << 30);
  *n_split = (int)((max_len + s - 1) / s);
}

hipError_t launch_kvq_append(int dtype, int head_dim, const KvqRows &a, hipStream_t st) {
  return kvq_rows_any(dtype, head_dim, a, false, st);
}
hipError_t launch_kvq_read(int dtype, int head_dim, const KvqRows &a, hipStream_t st) {
  return kvq_rows_any(dtype, head_dim, a, true, st);
}
hipError_t launch_kvq_attention(int dtype, int head_dim, const KvqAttn &a, hipStream_t st) {
  return kvq_attn_any(dtype, head_dim, false, a, st);
}
hipError_t launch_kvq_combine(int dtype, int head_dim, const KvqAttn &a, hipStream_t st) {
  return a.n_split > 1 ? kvq_attn_any(dtype, head_dim, true, a, st) : hipSuccess;
}
hipError_t launch_kvq_stage(const PackedRows &pk, int head_dim, const KvqStage &s, hipStream_t st) {
  const int rows = std::max(pk.cu[pk.n], pk.n);
  if (rows <= 0) return hipSuccess;
  HS_LAUNCH(k_kvq_stage, dim3((rows + 255) / 256), dim3(256), 0, st, pk, head_dim, s);
  return hipGetLastError();
}

}  // namespace hs
