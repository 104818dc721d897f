// hs_kvq.h — the KV cache held in 4 bits (gfx950): storing rows, fetching them
// back, and decode attention over it.  Included by hs_misc.hip.
//
// A row's elements are E2M1 numbers (sign, 2 exponent bits, 1 mantissa bit:
// 0, 1/2, 1, 3/2, 2, 3, 4, 6) in groups of 32 that share one power of two, a
// byte holding its exponent + 127.  With a = max |x| of a group the power is
// the least 2^e with a < 7 * 2^e: the group's largest element then rounds to
// 4 or 6 (or to 3 below 3.5), and as 7 lies half way between 6 and the next
// step, saturating at 6 moves an element by less than 2^e, which is half of
// the widest step.  Rounding is to nearest, ties to even.  A value takes at most
// 2 significant bits, so it is exact in f16 and in bf16, and gfx950 converts
// both ways in one full-rate instruction for two elements.
#pragma once

#include "hs_device.h"

#include <algorithm>
#include <cfloat>

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

// One thread takes eight elements of a row of K or V.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_append(KvqRows a) {
  constexpr int CPR = HD / 8;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(t % CPR);
  const int64_t line = t / CPR;
  const int hi = (int)(line % a.heads), head = a.head0 + hi;
  const int64_t rs = line / a.heads;
  const int sel = a.sel < 0 ? (int)(rs & 1) : a.sel;
  const int row = (int)(a.sel < 0 ? rs >> 1 : rs);
  if (row >= a.n) return;
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  int seq, pos;
  kvq_place(a, row, seq, pos);
  const int64_t at = ((int64_t)(a.row_by_seq ? seq : row) * a.ld + (int64_t)hi * a.ld_head + c * 8) * SB;
  float f[8];
  ld8<DT>((const char *)(sel ? a.v : a.k) + at, f);
  uint32_t byte;
  const uint32_t w = kvq_encode<DT>(f, byte);
  int64_t id = kvq_block(a.c, seq, pos);
  if (id >= 0 && a.cap && pos >= a.cap[seq]) id = -1;
  if (id >= 0) {
    uint8_t *span = kvq_span(a.c, HD, id, sel, head, pos);
    ((uint32_t *)span)[(pos & 15) * CPR + c] = w;
    if ((c & 3) == 0) span[HD * 8 + (c >> 2) * 16 + (pos & 15)] = (uint8_t)byte;
  }
  char *val = (char *)(sel ? a.v_out : a.k_out);
  if (val) {
    kvq_decode(w, kvq_scale(byte), f);
    st8<DT>(val + at, f);
  }
}

// The reverse: rows of K and V in the row type; a place without a block gives zeros.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_read(KvqRows a) {
  constexpr int CPR = HD / 8;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(t % CPR);
  const int64_t line = t / CPR;
  const int hi = (int)(line % a.heads), head = a.head0 + hi;
  const int64_t rs = line / a.heads;
  const int sel = a.sel < 0 ? (int)(rs & 1) : a.sel;
  const int row = (int)(a.sel < 0 ? rs >> 1 : rs);
  if (row >= a.n) return;
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  int seq, pos;
  kvq_place(a, row, seq, pos);
  const int64_t id = kvq_block(a.c, seq, pos);
  uint32_t w = 0, byte = KvqByte<DT>::lo;
  if (id >= 0) {
    const uint8_t *span = kvq_span(a.c, HD, id, sel, head, pos);
    w = ((const uint32_t *)span)[(pos & 15) * CPR + c];
    byte = span[HD * 8 + (c >> 2) * 16 + (pos & 15)];
  }
  float f[8];
  kvq_decode(w, kvq_scale(byte), f);
  st8<DT>((char *)(sel ? a.v_out : a.k_out) + ((int64_t)row * a.ld + (int64_t)hi * a.ld_head + c * 8) * SB, f);
}

// Decode attention over the 4-bit cache.  One work group = (split of the row's
// positions, row, KV head j); each of its NW waves takes tiles of 64 positions
// and keeps an online softmax for the G query heads of the head in the 16
// columns of the matrix products.
//
// Scores: S^T = K Q^T, MFMA 16x16x32 with 16 positions as rows.  Lane (li, lg) =
// (lane % 16, lane / 16) converts HD / 4 consecutive elements of its position,
// one load and one group's scale, straight into A operands; the order of the
// elements inside the contraction is the same for Q.  Row r of the tile's
// product t is position 16 (r / 4) + 4 t + r % 4, so that a lane ends up with
// the scores of the 16 consecutive positions 16 lg .. for head li, which is the
// B operand of O^T += V^T P^T: positions 8 m .. 8 m + 7 of each lane group are
// the k range of MFMA m.  For V^T a lane reads its HD / 16 channels of those 16
// positions, converts pairs of channels and pairs the positions with v_perm; no
// value goes through LDS.  The 4-bit values are exact in the 16-bit type, P
// enters as the sum of parts in that type (two: 16 bits and more; fp32: three,
// 24 bits, and Q alike), every sum is fp32.
//
// Blocks of 64 positions and more (WIDE) hold a tile whole: it is read through a
// buffer range that ends at its last span, past which nothing is fetched.
// Smaller blocks are found span by span, per lane.
template <int DT>
constexpr int KVQ_MMA = DT == HS_F16 ? HS_F16 : HS_BF16;
template <int DT>
constexpr int KVQ_P_PARTS = DT == HS_F32 ? 3 : 2;
template <int DT>
constexpr int KVQ_Q_PARTS = DT == HS_F32 ? 3 : 1;
constexpr int KVQ_TILE = 64;
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

template <int DT, int HD, int NW, bool WIDE>
__global__ __launch_bounds__(64 * NW) void k_kvq_attn(KvqAttn a) {
  constexpr int MT = KVQ_MMA<DT>, PP = KVQ_P_PARTS<DT>, QP = KVQ_Q_PARTS<DT>;
  constexpr int NC = HD / 32;             // words of a lane's K elements: k steps of the scores
  constexpr int VB = HD / 32;             // bytes of a lane's V elements of one position
  constexpr int ND = HD / 16;             // 16-channel tiles of the output
  constexpr int SPAN = kvq_span_bytes(HD);
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  const int G = a.n_heads / a.c.n_kv;
  // every row's first split comes before any row's second: the empty ones are last
  const int64_t bid = blockIdx.x, per = (int64_t)a.n * a.c.n_kv;
  const int split = (int)(bid / per), j = (int)(bid % a.c.n_kv);
  const int z = (int)(bid % per / a.c.n_kv);
  const int row = a.order ? a.order[z] : z;
  const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seq = a.seqs ? a.seqs[row] : row;
  const int len = kvq_length(a, row, seq);
  const int t0 = split * a.S;
  const int64_t rh = (int64_t)row * a.n_heads + j * G;  // first (row, head) of the group
  if (t0 >= len) {
    for (int i = threadIdx.x; i < G * HD; i += 64 * NW) {
      const int h = i / HD, e = i - h * HD;
      if (a.n_split == 1) {
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
  const int end = min(t0 + a.S, len);  // the split's positions: t0 .. end - 1
  const int n_tiles = (end - t0 + KVQ_TILE - 1) / KVQ_TILE;
  const int64_t *tab = a.c.table + (int64_t)seq * a.c.table_ld;
  const int64_t kin = ((int64_t)(a.c.layer * 2) * a.c.n_kv + j) << (a.c.bt_log2 - 4);  // spans before the head's
  const int64_t vin = kin + ((int64_t)a.c.n_kv << (a.c.bt_log2 - 4));
  const int in_mask = (1 << a.c.bt_log2) - 1;

  // Q^T operand: head li of the group (zeros past it)
  u32x4 qb[QP][NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float f[8] = {};
    if (li < G) ld8<DT>((const char *)a.q + ((int64_t)row * a.ld_q + (j * G + li) * HD + lg * (HD / 4) + c * 8) * SB, f);
    // (a negative scale's sign goes to Q, so that the scores' order is that of the products)
    if (a.scale < 0.f)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = -f[e];
#pragma unroll
    for (int p = 0; p < QP; ++p)
#pragma unroll
      for (int x = 0; x < 4; ++x) qb[p][c][x] = take_part<MT>(f[2 * x], f[2 * x + 1]);
  }
  const float c2 = fabsf(a.scale) * 1.44269504088896341f;

  // a tile's data in flight: K words and scale bytes, V words and scale bytes
  uint32_t kc[4][NC], vc[16];
  u32x4 ks, vs;
  struct At {           // where a tile is
    int64_t kid, vid;   // WIDE: the tile's block, twice; else the blocks of the lane's K and V spans
  };
  const int kspan = li >> 2, kgrp = HD == 128 ? lg : lg >> 1, vgrp = HD == 128 ? li >> 2 : li >> 3;
  auto find = [&](int t) {
    At w{-1, -1};
    if (t >= n_tiles) return w;
    const int p0 = t0 + t * KVQ_TILE;
    if constexpr (WIDE) {
      w.kid = tab[p0 >> a.c.bt_log2];
    } else {
      // past the last span: that span again
      const int last = (end - 1) & ~15;
      w.kid = tab[min(p0 + kspan * 16, last) >> a.c.bt_log2];
      w.vid = tab[min(p0 + lg * 16, last) >> a.c.bt_log2];
      if ((uint64_t)w.vid >= (uint64_t)a.c.n_blocks) w.vid = -1;
    }
    if ((uint64_t)w.kid >= (uint64_t)a.c.n_blocks) w.kid = -1;
    if constexpr (WIDE) w.vid = w.kid;
    return w;
  };
  auto range = [&](int t, int64_t id, int64_t in) {  // WIDE: the tile's spans
    const int p0 = t0 + t * KVQ_TILE, spans = (min(end - p0, KVQ_TILE) + 15) / 16;
    return make_rsrc(a.c.blocks + max(id, (int64_t)0) * a.c.block_bytes + (in + ((p0 & in_mask) >> 4)) * SPAN,
                     id < 0 || t >= n_tiles ? 0u : (uint32_t)(spans * SPAN));
  };
  auto load_k = [&](int t, const At &w) {
    if constexpr (WIDE) {
      const rsrc_t r = range(t, w.kid, kin);
      const uint32_t o = kspan * SPAN + (li & 3) * (HD / 2) + lg * (HD / 8);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (HD == 128) *(u32x4 *)kc[x] = bld16_stream(r, o + x * 4 * (HD / 2));
        else *(u32x2 *)kc[x] = bld8(r, o + x * 4 * (HD / 2));
      }
      ks = bld16_stream(r, kspan * SPAN + HD * 8 + kgrp * 16);
    } else if (t < n_tiles) {
      const int p = min(t0 + t * KVQ_TILE + kspan * 16, (end - 1) & ~15);
      const uint8_t *s = a.c.blocks + max(w.kid, (int64_t)0) * a.c.block_bytes + (kin + ((p & in_mask) >> 4)) * SPAN;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint8_t *at = s + (4 * x + (li & 3)) * (HD / 2) + lg * (HD / 8);
        if constexpr (HD == 128) *(u32x4 *)kc[x] = *(const u32x4 *)at;
        else *(u32x2 *)kc[x] = *(const u32x2 *)at;
      }
      ks = *(const u32x4 *)(s + HD * 8 + kgrp * 16);
    }
  };
  auto load_v = [&](int t, const At &w) {
    if constexpr (WIDE) {
      const rsrc_t r = range(t, w.vid, vin);
      const uint32_t o = lg * SPAN + li * VB;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (HD == 128) vc[i] = bld4(r, o + i * (HD / 2));
        else vc[i] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, o + i * (HD / 2), 0, 0);
      }
      vs = bld16_stream(r, lg * SPAN + HD * 8 + vgrp * 16);
    } else if (t < n_tiles) {
      const int p = min(t0 + t * KVQ_TILE + lg * 16, (end - 1) & ~15);
      const uint8_t *s = a.c.blocks + max(w.vid, (int64_t)0) * a.c.block_bytes + (vin + ((p & in_mask) >> 4)) * SPAN;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (HD == 128) vc[i] = *(const uint32_t *)(s + i * (HD / 2) + li * VB);
        else vc[i] = *(const uint16_t *)(s + i * (HD / 2) + li * VB);
      }
      vs = *(const u32x4 *)(s + HD * 8 + vgrp * 16);
    }
  };

  // the reference (base-2 units) and this lane's share of the sum; the reference
  // starts at the lowest finite number, so that s - m is a number for s = -inf
  float m = -FLT_MAX, l = 0.f;
  bool big = true;  // some column's |m| >= KVQ_ROUND_FROM (wave-uniform)
  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  At cur = find(wave), nxt = find(wave + NW);
  load_k(wave, cur);
  load_v(wave, cur);
  for (int t = wave; t < n_tiles; t += NW) {
    const int p0 = t0 + t * KVQ_TILE;
    f32x4 sc[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float s = kvq_scale((ks[x] >> (8 * (li & 3))) & 255u);
      sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4 kv{kvq_pair<MT, 0>(kc[x][c], s), kvq_pair<MT, 1>(kc[x][c], s), kvq_pair<MT, 2>(kc[x][c], s),
                       kvq_pair<MT, 3>(kc[x][c], s)};
#pragma unroll
        for (int p = 0; p < QP; ++p) sc[x] = mma<MT>(kv, qb[p][c], sc[x]);
      }
    }
    load_k(t + NW, nxt);
    // which of the lane's 16 positions count: all of them in a whole tile
    const bool held = cur.vid >= 0;
    const int left = end - p0 - 16 * lg;
    const bool whole = p0 + KVQ_TILE <= end && __ballot(!held) == 0;
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
    float vf[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) vf[i] = kvq_scale((vs[i >> 2] >> (8 * (i & 3))) & 255u);
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
    load_v(t + NW, nxt);
    cur = nxt;
    nxt = find(t + 2 * NW);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // merge the waves: lane (li, lg) holds channels d = (4 lg + i) (HD / 16) + dt of head li
  __shared__ float s_m[NW][16], s_l[NW][16];
  __shared__ float s_o[NW][16][HD + 1];
  if (lg == 0) {
    s_m[wave][li] = m;
    s_l[wave][li] = l;
  }
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
    if (a.n_split == 1) {
      // no position held: zeros
      st_elem<DT>(a.out, kvq_out_at(a, row, (j * G + h) * HD + e, HD), den == 0.f ? 0.f : num / den);
    } else {
      a.part_o[((rh + h) * a.n_split + split) * HD + e] = num;
      if (e == 0) {
        a.part_ml[((rh + h) * a.n_split + split) * 2] = den == 0.f ? -INFINITY : a.nat ? M * 0.693147180559945309f : M;
        a.part_ml[((rh + h) * a.n_split + split) * 2 + 1] = den;
      }
    }
  }
}

// o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the splits of a (row,
// head), in split order; zeros where none holds a position
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_combine(KvqAttn a) {
  constexpr int PARTS = 256 / HD;
  __shared__ float s_w[KVQ_MAX_SPLITS], s_l[KVQ_MAX_SPLITS], s_n[PARTS][HD];
  const int h = blockIdx.x % a.n_heads, ns = a.n_split;
  const int64_t row = blockIdx.x / a.n_heads, base = (row * a.n_heads + h) * ns;
  const int e = threadIdx.x % HD, part = threadIdx.x / HD;
  for (int s = threadIdx.x; s < ns; s += 256) {
    s_w[s] = a.part_ml[(base + s) * 2];
    s_l[s] = a.part_ml[(base + s) * 2 + 1];
  }
  __syncthreads();
  float M = -FLT_MAX;
  for (int s = 0; s < ns; ++s) M = fmaxf(M, s_w[s]);
  float num = 0.f, den = 0.f;
  for (int s = 0; s < ns; ++s) den += __builtin_amdgcn_exp2f(s_w[s] - M) * s_l[s];
  for (int s = part; s < ns; s += PARTS) num += __builtin_amdgcn_exp2f(s_w[s] - M) * a.part_o[(base + s) * HD + e];
  s_n[part][e] = num;
  __syncthreads();
  if (part) return;
#pragma unroll
  for (int p = 1; p < PARTS; ++p) num += s_n[p][e];
  st_elem<DT>(a.out, kvq_out_at(a, row, h * HD + e, HD), den == 0.f ? 0.f : num / den);
}

template <int DT, int HD>
hipError_t kvq_rows(const KvqRows &a, bool read, hipStream_t st) {
  const int64_t threads = (int64_t)a.n * (a.sel < 0 ? 2 : 1) * a.heads * (HD / 8), grid = (threads + 255) / 256;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (read) HS_LAUNCH((k_kvq_read<DT, HD>), dim3((uint32_t)grid), dim3(256), 0, st, a);
  else HS_LAUNCH((k_kvq_append<DT, HD>), dim3((uint32_t)grid), dim3(256), 0, st, a);
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

template <int DT, int HD>
hipError_t kvq_attn_hd(const KvqAttn &a, hipStream_t st) {
  const int64_t grid = (int64_t)a.n * a.c.n_kv * a.n_split, rows = (int64_t)a.n * a.n_heads;
  if (grid > INT32_MAX || rows > INT32_MAX || a.n_split > KVQ_MAX_SPLITS) return hipErrorInvalidValue;
  if ((1 << a.c.bt_log2) >= KVQ_TILE) HS_LAUNCH((k_kvq_attn<DT, HD, 4, true>), dim3((uint32_t)grid), dim3(256), 0, st, a);
  else HS_LAUNCH((k_kvq_attn<DT, HD, 4, false>), dim3((uint32_t)grid), dim3(256), 0, st, a);
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

void kvq_split_policy(int64_t n, int n_kv, int max_len, int *S, int *n_split) {
  constexpr int ROUND = 4 * KVQ_TILE;  // one tile for each wave
  const int64_t pairs = std::max<int64_t>(1, n * n_kv), want = (2048 + pairs - 1) / pairs;
  const int64_t most = ((int64_t)max_len + ROUND - 1) / ROUND;
  const int64_t ns = std::max<int64_t>(1, std::min(std::min(want, most), (int64_t)KVQ_MAX_SPLITS));
  const int64_t s = ((max_len + ns - 1) / ns + ROUND - 1) / ROUND * ROUND;
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
