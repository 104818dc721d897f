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

// weight of a part with maximum m_part in a softmax with maximum m_all
__device__ __forceinline__ float kvq_weight(float m_part, float m_all) {
  return m_part == -INFINITY ? 0.f : expf(m_part - m_all);
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

// One thread takes eight elements of a row of K or V.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_append(KvqRows a) {
  constexpr int CPR = HD / 8;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(t % CPR);
  const int64_t line = t / CPR;
  const int head = (int)(line % a.c.n_kv);
  const int64_t rs = line / a.c.n_kv;
  const int sel = (int)(rs & 1);
  const int row = (int)(rs >> 1);
  if (row >= a.n) return;
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  const int64_t at = ((int64_t)row * a.ld + (int64_t)head * a.ld_head + c * 8) * SB;
  float f[8];
  ld8<DT>((const char *)(sel ? a.v : a.k) + at, f);
  uint32_t byte;
  const uint32_t w = kvq_encode<DT>(f, byte);
  const int seq = a.seqs ? a.seqs[row] : row;
  const int pos = !a.pos_by_seq ? a.pos[row] : (uint32_t)seq < (uint32_t)a.c.n_seqs ? a.pos[seq] : -1;
  const int64_t id = a.cap && pos >= 0 && pos >= a.cap[seq] ? -1 : kvq_block(a.c, seq, pos);
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
  const int head = (int)(line % a.c.n_kv);
  const int64_t rs = line / a.c.n_kv;
  const int sel = (int)(rs & 1);
  const int row = (int)(rs >> 1);
  if (row >= a.n) return;
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  const int seq = a.seqs ? a.seqs[row] : row, pos = a.pos[row];
  const int64_t id = kvq_block(a.c, seq, pos);
  uint32_t w = 0, byte = KvqByte<DT>::lo;
  if (id >= 0) {
    const uint8_t *span = kvq_span(a.c, HD, id, sel, head, pos);
    w = ((const uint32_t *)span)[(pos & 15) * CPR + c];
    byte = span[HD * 8 + (c >> 2) * 16 + (pos & 15)];
  }
  float f[8];
  kvq_decode(w, kvq_scale(byte), f);
  st8<DT>((char *)(sel ? a.v_out : a.k_out) + ((int64_t)row * a.ld + (int64_t)head * a.ld_head + c * 8) * SB, f);
}

// Decode attention: one work group takes one query head of one row; each of its
// 4 waves walks positions, HD / 8 lanes to a position, with an online softmax per
// group of lanes that is merged at the end.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_kvq_attn(KvqAttn a) {
  constexpr int CPR = HD / 8, TPW = 64 / CPR;
  const int h = blockIdx.x % a.n_heads;
  const int64_t row = blockIdx.x / a.n_heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane % CPR, tg = lane / CPR, head = h / (a.n_heads / a.c.n_kv);
  const int seq = a.seqs ? a.seqs[row] : (int)row;
  const int len = kvq_length(a, row, seq);
  constexpr int SB = DT == HS_F32 ? 4 : 2;
  float q[8], o[8] = {};
  ld8<DT>((const char *)a.q + (row * a.ld_q + h * HD + c * 8) * SB, q);
  float m = -INFINITY, l = 0.f;
  for (int p0 = 0; p0 < len; p0 += 4 * TPW) {
    const int pos = p0 + wave * TPW + tg;
    const int64_t id = pos < len ? kvq_block(a.c, seq, pos) : -1;
    float k[8] = {}, v[8] = {};
    if (id >= 0) {
      const uint8_t *ks = kvq_span(a.c, HD, id, 0, head, pos), *vs = kvq_span(a.c, HD, id, 1, head, pos);
      const int at = (pos & 15) * CPR + c, mark = HD * 8 + (c >> 2) * 16 + (pos & 15);
      kvq_decode(((const uint32_t *)ks)[at], kvq_scale(ks[mark]), k);
      kvq_decode(((const uint32_t *)vs)[at], kvq_scale(vs[mark]), v);
    }
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) d += q[e] * k[e];
    d = group_sum<CPR>(d);
    if (id < 0) continue;
    const float s = d * a.scale, mn = fmaxf(m, s), corr = kvq_weight(m, mn), p = expf(s - mn);
    l = l * corr + p;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * corr + p * v[e];
    m = mn;
  }
  __shared__ float s_m[4 * TPW], s_l[4 * TPW], s_o[4 * TPW][HD];
  const int slot = wave * TPW + tg;
  if (c == 0) s_m[slot] = m, s_l[slot] = l;
#pragma unroll
  for (int e = 0; e < 8; ++e) s_o[slot][c * 8 + e] = o[e];
  __syncthreads();
  for (int e = threadIdx.x; e < HD; e += 256) {
    float M = -INFINITY, num = 0.f, den = 0.f;
    for (int s = 0; s < 4 * TPW; ++s) M = fmaxf(M, s_m[s]);
    for (int s = 0; s < 4 * TPW; ++s) {
      const float w = kvq_weight(s_m[s], M);
      num += w * s_o[s][e];
      den += w * s_l[s];
    }
    st_elem<DT>(a.out, row * a.ld_out + h * HD + e, M == -INFINITY ? 0.f : num / den);
  }
}

template <int DT, int HD>
hipError_t kvq_rows(const KvqRows &a, bool read, hipStream_t st) {
  const int64_t threads = (int64_t)a.n * 2 * a.c.n_kv * (HD / 8), grid = (threads + 255) / 256;
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

template <int DT>
hipError_t kvq_attn_dt(int hd, const KvqAttn &a, hipStream_t st) {
  const int64_t grid = (int64_t)a.n * a.n_heads;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (hd == 64) HS_LAUNCH((k_kvq_attn<DT, 64>), dim3((uint32_t)grid), dim3(256), 0, st, a);
  else if (hd == 128) HS_LAUNCH((k_kvq_attn<DT, 128>), dim3((uint32_t)grid), dim3(256), 0, st, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kvq_append(int dtype, int head_dim, const KvqRows &a, hipStream_t st) {
  return kvq_rows_any(dtype, head_dim, a, false, st);
}
hipError_t launch_kvq_read(int dtype, int head_dim, const KvqRows &a, hipStream_t st) {
  return kvq_rows_any(dtype, head_dim, a, true, st);
}
hipError_t launch_kvq_attention(int dtype, int head_dim, const KvqAttn &a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  switch (dtype) {
    case HS_F32: return kvq_attn_dt<HS_F32>(head_dim, a, st);
    case HS_F16: return kvq_attn_dt<HS_F16>(head_dim, a, st);
    case HS_BF16: return kvq_attn_dt<HS_BF16>(head_dim, a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace hs
