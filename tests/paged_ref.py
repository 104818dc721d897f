"""Plain 64-bit forms of the paged cache's operators and of the token draw, on the CPU, and how far fp32 work may be off."""
from __future__ import annotations

import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def blocks(n, layers, kv, block, hd, dtype, seed=0, fill=None):
    """A cache's blocks on the GPU: unit normal, or one value throughout."""
    if fill is not None:
        return torch.full((n, layers, 2, kv, block, hd), fill, dtype=DT[dtype], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, layers, 2, kv, block, hd, device="cuda", generator=g).to(DT[dtype])


def turned(x, gain, eps, freq, axes, at, adjacent):
    """(x normalised and turned, a bound of its fp32 error): x [n][heads][hd], at [axes][n], all on the CPU."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    # sum of squares (a tree of 11 additions), root, quotient, two products: 16 roundings of 2^-24 at most
    err = x.abs() * 2.0 ** -20
    p = 0 if freq is None else len(freq)
    if not p:
        return x, err if gain is not None else 0 * err
    axis = torch.zeros(p, dtype=torch.int64) if axes is None else axes.long()
    angle = (at.double()[axis] * freq[:, None]).T[:, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    one = x[..., 0 : 2 * p : 2] if adjacent else x[..., :p]
    two = x[..., 1 : 2 * p : 2] if adjacent else x[..., p : 2 * p]
    a, b = one * cos - two * sin, one * sin + two * cos
    rest = x[..., 2 * p :]
    join = lambda u, v: torch.cat(  # noqa: E731
        ((torch.stack((u, v), -1).flatten(-2),) if adjacent else (u, v)) + (rest,), -1)
    # cos and sin: the angle is off by 2^-52 of itself (the product and the turns) and by 2^-23, a turn's half rounded to
    # fp32, and the functions by 2^-22; products and their sum by 2^-23.  The channels past the pairs pass
    off = (one.abs() + two.abs()) * (2.0 ** -20 + angle.abs() * 2.0 ** -51)
    e = join(off, off)
    e[..., 2 * p :] = 0
    return join(a, b), e + (err if gain is not None else 0)


def half_step(want, dtype):
    """A rounding's error: half a step relative to the value, and half the least subnormal."""
    info = torch.finfo(DT[dtype])
    return want.abs() * info.eps / 2 + info.smallest_normal * info.eps / 2


def attention(q, cache, table, layer, lengths, seqs, starts=None, shared=None, scale=None, max_len=None):
    """(out, bound of its error before the last rounding) of decode attention: all on the CPU, in 64 bits."""
    n, heads, hd = q.shape
    kv, block = cache.shape[3], cache.shape[4]
    dtype = next(k for k, v in DT.items() if v is q.dtype)
    scale = hd ** -0.5 if scale is None else scale
    out = torch.zeros(n, heads, hd, dtype=torch.float64)
    tol = torch.zeros(n, heads, hd, dtype=torch.float64)
    most = table.shape[1] * block
    for r in range(n):
        s, length = int(seqs[r]), int(lengths[r])
        if not 0 <= s < len(table):
            continue
        length = max(0, min(length, most, max_len or most))
        common, lead = 0, s
        for g in range(0 if starts is None else len(shared)):
            if int(starts[g]) <= r < int(starts[g + 1]):
                common, lead = int(shared[g]), int(seqs[int(starts[g])])
        places = []
        for p in range(length):
            t = lead if p < common else s
            b = int(table[t, p // block]) if 0 <= t < len(table) else -1
            if 0 <= b < len(cache):
                places.append((b, p % block))
        if not places:
            continue
        b, i = (torch.tensor(v) for v in zip(*places))
        k = cache[b, layer, 0, :, i].double().transpose(0, 1)  # [kv, positions, hd]
        v = cache[b, layer, 1, :, i].double().transpose(0, 1)
        qr = q[r].double().reshape(kv, -1, hd)
        score = torch.matmul(qr, k.transpose(1, 2)) * scale
        p = torch.softmax(score, -1)
        out[r] = torch.matmul(p, v).reshape(heads, hd)
        # a score is off by its products' sum in fp32, its scaling and the difference to the maximum
        size = torch.matmul(qr.abs(), k.abs().transpose(1, 2)).amax(-1, keepdim=True) * abs(scale)
        score_off = size * (hd + 8) * 2.0 ** -24 * 2
        # the weights' last bits (two parts of the type), exponentials, and sums of the positions in fp32
        weight_off = {"f32": 2.0 ** -22, "f16": 2.0 ** -21, "bf16": 2.0 ** -16}[dtype] + (len(places) / 32 + 64) * 2.0 ** -23
        tol[r] = (torch.matmul(p, v.abs()) * (2 * score_off + weight_off)).reshape(heads, hd)
    return out, tol


def draw(x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, log probabilities) drawn from the definition, row by row in 64 bits."""
    rows, vocab = x.shape
    tokens, lps = [], []
    at = lambda t, r, d: d if t is None else float(t[r])  # noqa: E731
    for r in range(rows):
        t, k, p, least, uu = (at(temperature, r, 1.0), at(top_k, r, 0), at(top_p, r, 1.0), at(min_p, r, 0.0),
                              float(u[r]))
        row = x[r].double()
        if not t >= 0 or math.isinf(t) or p != p or least != least or uu != uu or bool(torch.isnan(row).any()) or \
                float(row.max()) in (math.inf, -math.inf):
            tokens.append(-1)
            lps.append(math.nan)
            continue
        v, order = torch.sort(row, dim=-1, descending=True, stable=True)
        if t == 0:
            tokens.append(int(order[0]))
            lps.append(0.0)
            continue
        logw = (v - v[0]) / t
        logw = logw[: int(k) if 0 < k < vocab else vocab]
        w = torch.exp(logw)
        if p < 1:
            upto = torch.cumsum(w, 0)
            keep = max(1, int((upto - w < p * upto[-1]).sum()))
            w, logw = w[:keep], logw[:keep]
        if least > 0:
            keep = max(1, int((w >= least).sum()))
            w, logw = w[:keep], logw[:keep]
        upto = torch.cumsum(w, 0)
        uu = min(max(uu, 0.0), 1.0 - 2.0 ** -24)
        i = min(int((upto <= uu * upto[-1]).sum()), int((w > 0).sum()) - 1)
        tokens.append(int(order[i]))
        lps.append(float(logw[i] - torch.log(upto[-1])))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(lps, dtype=torch.float64)
