"""Plain 64-bit forms of the 4-bit cache's operators and of token log probabilities, on the CPU."""
from __future__ import annotations

import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SIZES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
E_RANGE = {"f32": (-125, 125), "bf16": (-125, 125), "f16": (-23, 13)}


def quantize(x, dtype):
    """(codes int64 [..., hd], e + 127 int64 [..., hd / 32] (255: NaN), values float64) of rows x."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~torch.isfinite(g).all(-1)
    a = torch.where(torch.isfinite(g), g, 0.0).abs().amax(-1)
    lo, hi = E_RANGE[dtype]
    e = torch.full(a.shape, hi, dtype=torch.int64)
    for k in range(hi - 1, lo - 1, -1):  # the least e with a < 7 * 2^e
        e = torch.where(a < 7.0 * 2.0 ** k, k, e)
    y = torch.where(torch.isfinite(g), g, 0.0) / (2.0 ** e.double()).unsqueeze(-1)
    d = (y.abs().unsqueeze(-1) - SIZES).abs()
    near = d.amin(-1, keepdim=True)
    tie = (d == near).sum(-1) > 1  # two sizes as near: the even code
    first = d.argmin(-1)
    code = torch.where(tie & (first % 2 == 1), first + 1, first)
    code = code + 8 * torch.signbit(g).long()
    code = torch.where(bad.unsqueeze(-1), 0, code)
    val = SIZES[code % 8] * torch.where(code >= 8, -1.0, 1.0) * (2.0 ** e.double()).unsqueeze(-1)
    val = torch.where(bad.unsqueeze(-1), math.nan, val)
    return code.reshape(x.shape), torch.where(bad, 255, e + 127), val.reshape(x.shape)


class Layout:
    """A cache's blocks (uint8 CPU tensor) seen by place."""

    def __init__(self, blocks, table, n_layers, n_kv, hd, bt):
        self.shape = (-1, n_layers, 2, n_kv, bt // 16, hd // 2 * 17)
        self.b = blocks.cpu().reshape(-1)[: blocks.numel() // self.block_bytes(n_layers, n_kv, hd, bt)
                                          * self.block_bytes(n_layers, n_kv, hd, bt)].reshape(self.shape)
        self.table, self.hd, self.bt = table.cpu(), hd, bt

    @staticmethod
    def block_bytes(n_layers, n_kv, hd, bt):
        return 2 * n_layers * n_kv * bt * hd * 17 // 32

    def block(self, seq, pos):
        k = pos // self.bt
        if not 0 <= seq < self.table.shape[0] or pos < 0 or k >= self.table.shape[1]:
            return -1
        i = int(self.table[seq, k])
        return i if 0 <= i < self.b.shape[0] else -1

    def put(self, layer, sel, seq, pos, codes, bytes_):
        """One row [n_kv, hd] of codes and its bytes [n_kv, hd / 32]."""
        i = self.block(seq, pos)
        if i < 0:
            return
        span = self.b[i, layer, sel, :, pos % self.bt // 16]
        r = pos % 16
        span[:, r * (self.hd // 2) : (r + 1) * (self.hd // 2)] = (codes[:, 0::2] + 16 * codes[:, 1::2]).to(torch.uint8)
        span[:, self.hd * 8 + r :: 16] = bytes_.to(torch.uint8)

    def rows(self, layer, sel, seq, length):
        """(values float64 [n_kv, length, hd], held bool [length])."""
        n_kv = self.b.shape[3]
        out, held = torch.zeros(n_kv, length, self.hd, dtype=torch.float64), torch.zeros(length, dtype=torch.bool)
        for p0 in range(0, length, self.bt):
            i, n = self.block(seq, p0), min(self.bt, length - p0)
            if i < 0:
                continue
            raw = self.b[i, layer, sel]  # [n_kv, spans, bytes]
            w = raw[..., : self.hd * 8].reshape(n_kv, self.bt, self.hd // 2).long()
            code = torch.stack((w % 16, w // 16), -1).reshape(n_kv, self.bt, self.hd)
            e = raw[..., self.hd * 8 :].reshape(n_kv, -1, self.hd // 32, 16).transpose(-1, -2).reshape(n_kv, self.bt, -1)
            s = torch.where(e == 255, math.nan, 2.0 ** (e.double() - 127)).repeat_interleave(32, -1)
            v = SIZES[code % 8] * torch.where(code >= 8, -1.0, 1.0) * s
            out[:, p0 : p0 + n], held[p0 : p0 + n] = v[:, :n], True
        return out, held


def attention(layout, layer, q, lengths, seqs=None, scale=None, max_len=None):
    """(out float64 [n, heads, hd], weight float64: sum p |v|, reach: max of scale * sum |q k|)."""
    n, heads, hd = q.shape
    n_kv = layout.b.shape[3]
    scale = hd ** -0.5 if scale is None else scale
    out, mass, reach = torch.zeros(n, heads, hd, dtype=torch.float64), torch.zeros(n, heads, hd, dtype=torch.float64), 0.0
    for r in range(n):
        seq = r if seqs is None else int(seqs[r])
        length = int(lengths[r])
        length = min(length, layout.table.shape[1] * layout.bt, max_len or 2 ** 31)
        if length <= 0 or not 0 <= seq < layout.table.shape[0]:
            continue
        k, held = layout.rows(layer, 0, seq, length)
        v, _ = layout.rows(layer, 1, seq, length)
        if not held.any():
            continue
        k, v = k[:, held], v[:, held]
        g = q[r].double().cpu().reshape(n_kv, heads // n_kv, hd)
        s = torch.einsum("jgd,jpd->jgp", g, k) * scale
        reach = max(reach, float(torch.einsum("jgd,jpd->jgp", g.abs(), k.abs()).nan_to_num().max()) * abs(scale))
        p = torch.softmax(s, -1)
        out[r] = torch.einsum("jgp,jpd->jgd", p, v).reshape(heads, hd)
        mass[r] = torch.einsum("jgp,jpd->jgd", p, v.abs()).reshape(heads, hd)
    return out, mass, reach


def attention_tolerance(out, mass, reach, dtype, hd):
    """How far a sum in fp32 may be off.  A score sums hd exact products in fp32: off by at most hd 2^-24 of the sum
    of their sizes, and again 2^-22 of its own size where it is scaled and the maximum subtracted; exp adds 2^-22.
    That is the relative error of a weight, which enters numerator and denominator.  The probabilities enter the
    second product with 16 bits at least in the 16-bit types (2^-17), 24 in fp32, and both sums are fp32 sums over at
    most 2^9 partial sums per lane (2^-15 at the worst of signs, of the weighted sizes).  A weight below 2^-126 is no
    normal fp32 number and may come out as 0: 2^-126 of each value, whose sizes sum to less than 2^26 here (at most
    2^17 positions, values below 2^9), against a sum of weights of 1 at least: 2^-100."""
    weight = reach * (hd * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -22
    inner = 2 * weight + (2.0 ** -17 if dtype != "f32" else 2.0 ** -23) + 2.0 ** -15 * (0.125 if dtype == "f32" else 1)
    tiny = {"f16": 2.0 ** -25, "bf16": 2.0 ** -100, "f32": 2.0 ** -100}[dtype]  # f16: half its least subnormal
    return HALF_STEP[dtype] * out.abs() + inner * mass + tiny


def logprobs(x, tokens, top):
    """(logprob, entropy, ids, top logprobs) in float64 of rows x (CPU)."""
    rows, V = x.shape
    x = x.double()
    lp, ent = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    ids, tops = torch.zeros(rows, top, dtype=torch.int64), torch.zeros(rows, top, dtype=torch.float64)
    for r in range(rows):
        t = int(tokens[r])
        if torch.isnan(x[r]).any() or bool((x[r] == math.inf).any()) or bool((x[r] == -math.inf).all()):
            ent[r], ids[r], tops[r] = math.nan, -1, math.nan
            lp[r] = 0.0 if t < 0 else math.nan
            continue
        d = x[r] - x[r].max()
        e = d.exp()
        at = int(d.argmax())
        rest = e.clone()
        rest[at] = 0.0
        lz = math.log1p(float(rest.sum()))
        ent[r] = lz - float(torch.where(e > 0, d * e, 0.0).sum()) / (1.0 + float(rest.sum()))
        lp[r] = 0.0 if t < 0 else math.nan if t >= V else float(d[t]) - lz
        order = torch.sort(x[r], descending=True, stable=True)
        ids[r], tops[r] = order.indices[:top], order.values[:top] - x[r].max() - lz
    return lp, ent, ids, tops


def logprob_tolerance(lp):
    """log Z: every e^d is off by a few 2^-24 of d (e^d matters for d down to about -16) and of itself, and the sum
    adds at most 2^6 times 2^-24: 2^-18 of Z at the most, 2^-17 with the logarithm's own; the differences x - M - log Z
    are rounded twice, 2^-23 of their size."""
    return 2.0 ** -17 + 2.0 ** -22 * lp.abs().nan_to_num(posinf=0.0, neginf=0.0)
