"""A paged cache's operators and token sampling, as a program that answers many questions on one prompt calls them.

Three kinds of case:

  append   new rows of queries, keys and values of one layer: queries and keys normalised for each head (where the model
           does that) and turned by their positions, keys and values stored at their places in a paged cache.
  attend   attention of one query row at a time over the first positions of its sequence in such a cache, the query
           heads of a group sharing one KV head; rows whose sequences begin with the same positions (answers drawn from
           one prompt, questions about one image, tokens drafted for one sequence) are given as a group, and the
           shared positions are read through the first row's blocks.  A row of length zero gives zeros.
  sample   a token drawn for each row of logits from a given uniform number, after temperature, top-k, top-p and min-p.

The cache.  A block of block_tokens positions is, for every layer, K then V, KV head, position, channel; a table holds
the block numbers of every sequence, negative where there is none.

The rotation.  Pair i of a head's first 2 pairs channels, (i, i + pairs) or (2 i, 2 i + 1), is turned by
position[axis[i]] * frequency[i]; channels past them stay.  The norm before it is x / sqrt(mean x^2 + eps) * gain.

The draw.  With x a row's logits in falling order (the lowest index first among equals) and w = exp((x - max x) / T):
the first k stay; of these the shortest beginning whose weights sum to top_p of theirs; of these the ones with
w >= min_p; the first always stays.  The token is the first whose weights, summed up to it, exceed u times their sum.
T = 0 takes the first.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def _append(name, dtype, seqs, rows, heads, kv, hd, block, layers=1, norm=False, axes=1, pairs=None, adjacent=False,
            theta=1e4, far=0):
    c = dict(kind="append", dtype=dtype, seqs=seqs, rows=rows, heads=heads, kv=kv, hd=hd, block=block, layers=layers,
             norm=norm, axes=axes, pairs=pairs or hd // 2, adjacent=adjacent, theta=theta, far=far)
    return dict(c, name=name) if name else c


def _attend(name, dtype, n, groups, heads, kv, hd, block, shared, more, layers=1, drafts=1, alone=0, empty=0):
    c = dict(kind="attend", dtype=dtype, n=n, groups=groups, heads=heads, kv=kv, hd=hd, block=block,
             shared_lo=shared[0], shared_hi=shared[1], lo=more[0], hi=more[1], layers=layers, drafts=drafts,
             alone=alone, empty=empty)
    return dict(c, name=name) if name else c


def _sample(name, dtype, rows, vocab, spread=2.5, banned=0.0, greedy=False, top_k=True, top_p=True, min_p=True):
    c = dict(kind="sample", dtype=dtype, rows=rows, vocab=vocab, spread=spread, banned=banned, greedy=greedy,
             top_k=top_k, top_p=top_p, min_p=min_p)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step's new rows, one for each of 32 requests (latency)
        _append("append_f16_step", "f16", 32, 32, 32, 32, 128, 256, layers=2),
        # one question's rows in fp32 after a long document, with norms and half of each head turned
        _append("append_f32_norm", "f32", 1, 623, 4, 4, 64, 16, norm=True, pairs=16, adjacent=True, far=1000000),
        # a packed prefill pass of 16 requests with their image positions
        _append("append_bf16_pass", "bf16", 16, 14370, 28, 4, 128, 256, layers=2, norm=True, axes=3, theta=1e6),
        # the smallest: three fp32 answers to one question about an image
        _attend("attend_f32_b3", "f32", 3, 1, 4, 4, 64, 16, (576, 576), (1, 32), layers=2),
        # 32 questions about one image, a KV head for every query head
        _attend("attend_f16_b32", "f16", 32, 1, 32, 32, 128, 64, (576, 576), (32, 384), layers=2),
        # 16 requests with five drafted tokens each to be checked
        _attend("attend_bf16_drafts", "bf16", 80, 16, 28, 4, 128, 256, (1024, 8192), (1, 5), drafts=5),
        # an odd batch: five prompts with several answers each, some rows alone, some without a position yet
        _attend("attend_bf16_b67", "bf16", 67, 5, 28, 4, 128, 32, (512, 4096), (1, 1664), layers=3, alone=9, empty=2),
        # the largest: 256 answers to one long document
        _attend("attend_bf16_b256", "bf16", 256, 1, 28, 4, 128, 256, (32768, 32768), (1, 2048)),
        # one answer's step
        _sample("sample_f32_b1", "f32", 1, 32000),
        # a batch's step over the largest vocabulary, the temperature and top-p alone
        _sample("sample_f32_b16", "f32", 16, 152064, top_k=False, min_p=False),
        # many rows of half-precision logits, an odd vocabulary with banned words, greedy rows among them
        _sample("sample_bf16_b1531", "bf16", 1531, 32003, banned=0.25, greedy=True),
        # the largest batch over the largest vocabulary
        _sample("sample_f32_b256", "f32", 256, 152064, greedy=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attend", "attend", "sample"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind == "sample":
        vocab = _log(rng, 2, 200000)
        rows = min(_log(rng, 1, 4096), max(1, 256 * 152064 // vocab))
        some = lambda: rng.random() < 0.6  # noqa: E731
        return _sample(None, dtype, rows, vocab, rng.choice((0.7, 2.5, 5.0)), rng.choice((0.0, 0.25)), some(), some(),
                       some(), some())
    hd, group, kv = rng.choice((64, 128)), rng.choice((1, 2, 4, 7, 8)), rng.choice((1, 2, 4, 8, 32))
    if kind == "append":
        rows = _log(rng, 1, 14370)
        while rows * kv * (group + 2) * hd > 14370 * 36 * 128:
            rows //= 2
        rows, axes = max(1, rows), rng.choice((1, 3))
        return _append(None, dtype, _log(rng, 1, min(rows, 64)), rows, group * kv, kv, hd, rng.choice((16, 64, 256)),
                       layers=rng.choice((1, 2)), norm=rng.random() < 0.5, axes=axes,
                       pairs=rng.choice((hd // 2, hd // 2, hd // 4)), adjacent=rng.random() < 0.3,
                       theta=rng.choice((1e4, 1e6)), far=rng.choice((0, 100000)))
    block = rng.choice((16, 32, 64, 256, 1024))
    drafts = rng.choice((1, 1, 4))
    n = _log(rng, 1, 256)
    if drafts > 1:
        n = max(drafts, n // drafts * drafts)
        groups, alone = n // drafts, 0
    else:
        alone = rng.choice((0, 0, n // 4))
        groups = rng.choice((0, 1, _log(rng, 1, max(1, n // 2)))) if n - alone else 0
        if not groups:
            alone = n
    shared = _log(rng, block, 65536) if groups else 0
    more = rng.randint(drafts, 16) if drafts > 1 else _log(rng, 1, 8192)
    fp32 = 4 if dtype == "f32" else 1  # fp32 products run at a fraction of the others' rate

    def too_much():
        flops = n * (shared + more) * group * kv * hd * fp32
        bytes_ = (groups * shared + n * more) * kv * hd * (2 if fp32 > 1 else 1)
        return flops > 256 * 34000 * 28 * 128 or bytes_ > 256 * 4096 * 4 * 128

    while too_much():
        if shared > 64 and groups * shared + 1 > more:
            shared //= 2
        elif more > 16:
            more //= 2
        elif drafts > 1 and n > drafts:
            n = max(drafts, n // 2 // drafts * drafts)
            groups = n // drafts
        elif n > 1 and drafts == 1:
            n, groups, alone = n // 2, min(groups, max(1, n // 4)) if groups else 0, 0
            alone = 0 if groups else n
        else:
            break
    lo = max(1, int(shared * rng.uniform(0.3, 1.0))) if shared else 0
    return _attend(None, dtype, n, groups, group * kv, kv, hd, block, (lo, shared), (drafts if drafts > 1 else 1, more),
                   layers=rng.choice((1, 2)), drafts=drafts, alone=alone, empty=1 if n > 4 and drafts == 1 else 0)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(shape, gen, loud):
    """Rows of heads: unit normal with some channels several times larger, as projections give them."""
    x = torch.randn(*shape, device="cuda", generator=gen)
    return x * (1.0 + loud * (torch.rand(shape[-1], device="cuda", generator=gen) > 0.9))


def _between(lo, hi, n, gen):
    return torch.randint(lo, hi + 1, (n,), device="cuda", generator=gen, dtype=torch.int32)


def _prepare_sample(s, c, gen):
    rows, vocab = c["rows"], c["vocab"]
    x = torch.randn(rows, vocab, device="cuda", generator=gen) * c["spread"]
    # in half of the rows the model is fairly sure of a few tokens
    sure = torch.randint(0, vocab, (rows, 4), device="cuda", generator=gen)
    x.scatter_add_(1, sure, (torch.rand(rows, 1, device="cuda", generator=gen) < 0.5) * 10.0 *
                   torch.rand(rows, 4, device="cuda", generator=gen))
    if c["banned"]:
        x.masked_fill_(torch.rand(x.shape, device="cuda", generator=gen) < c["banned"], -math.inf)
        x[:, 0] = 0.0
    s["logits"] = x.to(DTYPES[c["dtype"]])
    pick = lambda *v: torch.tensor(v, device="cuda")[  # noqa: E731
        torch.randint(0, len(v), (rows,), device="cuda", generator=gen)].contiguous()
    s["u"] = torch.rand(rows, device="cuda", generator=gen)
    s["temperature"] = 0.5 + 0.8 * torch.rand(rows, device="cuda", generator=gen)
    if c["greedy"]:
        s["temperature"] *= torch.rand(rows, device="cuda", generator=gen) > 0.1
    s["top_k"] = pick(0, 20, 50, 1000).to(torch.int32) if c["top_k"] else None
    s["top_p"] = pick(1.0, 0.9, 0.95) if c["top_p"] else None
    s["min_p"] = pick(0.0, 0.02, 0.1) if c["min_p"] else None
    if own:
        import paper_2603_12707_amd as hs
        s["workspace"] = hs.sample_tokens_workspace(rows, vocab)
    return s


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "sample":
        return _prepare_sample(s, c, gen)
    dt, block, kv, hd = DTYPES[c["dtype"]], c["block"], c["kv"], c["hd"]
    c["layer"] = c["layers"] - 1
    if c["kind"] == "append":
        n, rows = c["seqs"], c["rows"]
        # the rows of the sequences back to back, each from a position of its own on (a decode step: one row each)
        share = torch.full((n,), rows // n, device="cuda", dtype=torch.int64)
        share[: rows % n] += 1
        first = torch.randint(0, 600, (n,), device="cuda", generator=gen, dtype=torch.int64)
        seqs = torch.repeat_interleave(torch.arange(n, device="cuda"), share, output_size=rows)
        at = torch.arange(rows, device="cuda") - (share.cumsum(0) - share)[seqs] + first[seqs]
        s["seqs"], s["positions"] = seqs.to(torch.int32), at.to(torch.int32)
        turn = at + (torch.randint(0, c["far"], (1,), device="cuda", generator=gen) if c["far"] else 0)
        # an image's rows: time, height and width; text goes on from there
        side = 24
        s["angles_at"] = (turn[None] if c["axes"] == 1 else
                          torch.stack((turn // (side * side), turn // side % side + turn // 512, turn % side))
                          ).to(torch.int32).contiguous()
        width = -(-(-(-rows // n) + 601) // block)
        s["table"] = torch.randperm(n * width, device="cuda", generator=gen).reshape(n, width)
        s["blocks"] = torch.zeros(n * width, c["layers"], 2, kv, block, hd, dtype=dt, device="cuda")
        s["q"] = _rows((rows, c["heads"], hd), gen, 4.0).to(dt)
        s["k"] = _rows((rows, kv, hd), gen, 4.0).to(dt)
        s["v"] = _rows((rows, kv, hd), gen, 4.0).to(dt)
        pair = torch.arange(c["pairs"], device="cuda", dtype=torch.float64)
        s["frequencies"] = c["theta"] ** (-pair / c["pairs"])
        # of the pairs a quarter turns with the time, the rest with height and width
        s["axes"] = (None if c["axes"] == 1 else
                     torch.where(pair < c["pairs"] // 4, 0, torch.where(pair < c["pairs"] * 5 // 8, 1, 2)).to(torch.int32))
        gain = lambda: (1.0 + 0.3 * torch.randn(hd, device="cuda", generator=gen)).to(dt)  # noqa: E731
        s["q_gain"], s["k_gain"] = (gain(), gain()) if c["norm"] else (None, None)
        if own:
            import paper_2603_12707_amd as hs
            s["cache"] = hs.PagedCache(s["blocks"], s["table"])
            s["rope"] = hs.Rope(s["frequencies"], axes=s["axes"], adjacent=c["adjacent"])
        return s
    n, groups = c["n"], c["groups"]
    in_groups = n - c["alone"]
    starts = (torch.arange(groups + 1, device="cuda") * in_groups // max(1, groups)).to(torch.int32)
    shared = (_between(c["shared_lo"], c["shared_hi"], max(1, groups), gen)[:groups] // block * block
              if c["drafts"] == 1 else _between(c["shared_lo"], c["shared_hi"], groups, gen)).to(torch.int32)
    row = torch.arange(n, device="cuda")
    group = (torch.searchsorted(starts.long(), row, right=True) - 1).clamp(min=0, max=max(0, groups - 1))
    before = torch.where(row < in_groups, shared[group] if groups else 0 * row, 0 * row).to(torch.int64)
    if c["drafts"] > 1:
        # a group's rows are the next tokens of one sequence
        seqs, sequences = group, groups
        lengths = before + 1 + row - starts.long()[group]
    else:
        seqs, sequences = row, n
        lengths = before + _between(c["lo"], c["hi"], n, gen)
        lengths[: c["empty"]] = 0
    longest = c["shared_hi"] + c["hi"]
    width = max(1, -(-longest // block))
    column = torch.arange(width, device="cuda")[None]
    # every sequence has blocks of its own, but for the whole ones that its group shares: those are the first row's
    table = (torch.arange(sequences, device="cuda") * width)[:, None] + column
    if groups and c["drafts"] == 1:
        lead = starts.long()[group]
        table = torch.where(column < (before // block)[:, None], (lead * width)[:, None] + column, table)
    last = torch.zeros(sequences, dtype=torch.int64, device="cuda").scatter_reduce_(0, seqs, lengths, "amax")
    held = column < (-(-torch.maximum(last, torch.zeros_like(last) if c["drafts"] > 1 else before) // block))[:, None]
    names = torch.zeros(sequences * width, dtype=torch.int64, device="cuda")
    names[table[held]] = 1
    n_blocks = max(1, int(names.sum()))
    places = torch.randperm(n_blocks, device="cuda", generator=gen)
    table = torch.where(held, places[(names.cumsum(0) - 1).clamp(min=0)[table]], torch.full_like(table, -1))
    s["table"] = table.contiguous()
    s["blocks"] = torch.zeros(n_blocks, c["layers"], 2, kv, block, hd, dtype=dt, device="cuda")
    for sel in range(2):  # the layer that is read is filled
        s["blocks"][:, c["layer"], sel] = _rows((n_blocks, kv, block, hd), gen, 4.0).to(dt)
    s["q"] = (torch.randn(n, c["heads"], hd, device="cuda", generator=gen) * 1.2).to(dt)
    s["lengths"], s["seqs"] = lengths.to(torch.int32), seqs.to(torch.int32)
    s["starts"], s["shared"] = (starts, shared) if groups else (None, None)
    s["max_len"], s["max_shared"] = longest, c["shared_hi"]
    # what a group holds at most, and how far a row reaches past what it shares
    s["most"] = -(-in_groups // groups) if groups else 0
    s["tail"] = c["hi"]
    if own:
        import paper_2603_12707_amd as hs
        s["cache"] = hs.PagedCache(s["blocks"], s["table"])
        s["workspace"] = s["cache"].attention_workspace(n, c["heads"], s["max_len"], n_groups=groups,
                                                        max_shared=s["max_shared"])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _turned(x, gain, s):
    """float32 rows [n, heads, hd], normalised and turned."""
    c = s["case"]
    x = x.float()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    at = s["angles_at"].double()
    angle = (at[0][:, None] if s["axes"] is None else at[s["axes"].long()].T) * s["frequencies"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    p = c["pairs"]
    a, b = (x[..., 0 : 2 * p : 2], x[..., 1 : 2 * p : 2]) if c["adjacent"] else (x[..., :p], x[..., p : 2 * p])
    one, two = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((one, two), -1).flatten(-2) if c["adjacent"] else torch.cat((one, two), -1)
    return torch.cat((turned, x[..., 2 * p :]), -1)


def _plain_append(s):
    c = s["case"]
    dt, at = s["q"].dtype, s["positions"].long()
    block = s["table"][s["seqs"].long(), at // c["block"]]
    head = torch.arange(c["kv"], device=at.device)[None]
    place = (block[:, None], head, (at % c["block"])[:, None])
    s["blocks"][:, c["layer"], 0][place] = _turned(s["k"], s["k_gain"], s).to(dt)
    s["blocks"][:, c["layer"], 1][place] = s["v"]
    return {"q": _turned(s["q"], s["q_gain"], s).to(dt), "blocks": s["blocks"]}


def _positions(s, sequences, at, sel):
    """float32 [m, kv, positions, hd] of the cache's rows at positions `at` [m, positions] of the sequences."""
    c = s["case"]
    block = s["table"][sequences[:, None], (at // c["block"]).clamp(max=s["table"].shape[1] - 1)].clamp(min=0)
    head = torch.arange(c["kv"], device=at.device)[None, :, None]
    return s["blocks"][:, c["layer"], sel][block[:, None], head, (at % c["block"])[:, None]].float()


def _plain_attend(s):
    c = s["case"]
    n, kv, hd, dev = c["n"], c["kv"], c["hd"], s["q"].device
    per = c["heads"] // kv
    q = s["q"].float().reshape(n, kv, per, hd) * (1.0 / math.sqrt(hd))
    lengths, seqs, row = s["lengths"].long(), s["seqs"].long(), torch.arange(n, device=dev)
    grouped = s["starts"] is not None
    before = torch.zeros_like(lengths)
    if grouped:
        starts = s["starts"].long()
        group = torch.searchsorted(starts, row, right=True) - 1
        inside = group < c["groups"]
        group = group.clamp(max=c["groups"] - 1)
        place = torch.where(inside, row - starts[group], s["most"])
        before = torch.where(inside, s["shared"].long()[group], 0)
        at = torch.arange(s["max_shared"], device=dev)
        first = seqs[starts[:-1]]
        packed = torch.zeros(c["groups"], kv, s["most"] + 1, per, hd, device=dev)
        packed[group, :, place] = q
        keys = _positions(s, first, at[None].expand(len(first), -1), 0).transpose(-1, -2).contiguous()
        score = torch.matmul(packed.reshape(c["groups"], kv, -1, hd), keys).reshape(*packed.shape[:-1], -1)
        score = score[group, :, place]  # [n, kv, per, positions]
        seen = at[None] < torch.minimum(before, lengths)[:, None]
        early = score.masked_fill_(~seen[:, None, None], -math.inf)
    reach = before[:, None] + torch.arange(s["tail"], device=dev)
    late = torch.matmul(q, _positions(s, seqs, reach, 0).transpose(-1, -2).contiguous())
    late.masked_fill_((reach >= lengths[:, None])[:, None, None], -math.inf)
    top = late.amax(-1, keepdim=True)
    if grouped:
        top = torch.maximum(top, early.amax(-1, keepdim=True))
    top = top.clamp(min=-3e38)
    late = torch.exp(late - top)
    total = late.sum(-1, keepdim=True)
    out = torch.matmul(late, _positions(s, seqs, reach, 1))
    if grouped:
        early = torch.exp(early - top)
        total = total + early.sum(-1, keepdim=True)
        weights = torch.zeros(c["groups"], kv, s["most"] + 1, per, s["max_shared"], device=dev)
        weights[group, :, place] = early * inside[:, None, None, None]
        values = _positions(s, first, at[None].expand(len(first), -1), 1)
        part = torch.matmul(weights.reshape(c["groups"], kv, -1, s["max_shared"]), values)
        part = part.reshape(c["groups"], kv, s["most"] + 1, per, hd)[group, :, place]
        out = out + part * inside[:, None, None, None]
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.reshape(n, c["heads"], hd).to(s["q"].dtype)


def _plain_sample(s):
    x, ids = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True)
    rows, vocab = x.shape
    t = s["temperature"].double()[:, None]
    k = torch.full_like(t, vocab) if s["top_k"] is None else s["top_k"].double()[:, None]
    k = torch.where(t == 0, 1.0, torch.where(k <= 0, float(vocab), k))
    x = x.double()
    w = torch.exp((x - x[:, :1]) / torch.where(t == 0, 1.0, t))
    kept = torch.arange(vocab, device=x.device)[None] < k
    if s["top_p"] is not None:
        upto = torch.cumsum(torch.where(kept, w, 0.0), -1)
        total = upto[:, -1:]
        p = s["top_p"].double()[:, None]
        kept &= (upto - w < p * total) | (p >= 1)
        del upto
    if s["min_p"] is not None:
        kept &= w >= s["min_p"].double()[:, None]
    kept[:, 0] = True
    w = torch.where(kept, w, 0.0)
    upto = torch.cumsum(w, -1)
    total = upto[:, -1:]
    at = (upto <= s["u"].double()[:, None] * total).sum(-1, keepdim=True)
    at = torch.minimum(at, (w > 0).sum(-1, keepdim=True) - 1)
    return {"token": ids.gather(-1, at)[:, 0].to(torch.int32),
            "logprob": torch.log(w.gather(-1, at) / total)[:, 0].float()}


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[kind](s)
    if kind == "append":
        q = s["cache"].append(s["case"]["layer"], s["k"], s["v"], s["positions"], seqs=s["seqs"], q=s["q"],
                              rope=s["rope"], angles_at=s["angles_at"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        return {"q": q, "blocks": s["blocks"]}
    if kind == "attend":
        return s["cache"].attention(s["case"]["layer"], s["q"], s["lengths"], seqs=s["seqs"], group_starts=s["starts"],
                                    shared=s["shared"], max_len=s["max_len"], max_shared=s["max_shared"],
                                    workspace=s["workspace"])
    import paper_2603_12707_amd as hs
    token, logprob = hs.sample_tokens(s["logits"], s["u"], s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                      min_p=s["min_p"], workspace=s["workspace"])
    return {"token": token, "logprob": logprob}


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "append":
        read = c["rows"] * (c["heads"] + 2 * c["kv"]) * c["hd"]
        return {"bytes": 2 * read * b + 4 * c["rows"] * (2 + c["axes"]), "flops": 8 * read}
    if c["kind"] == "attend":
        heads, some = c["heads"] * c["hd"], c["n"] - c["empty"]
        shared, more = (c["shared_lo"] + c["shared_hi"]) / 2, (c["lo"] + c["hi"]) / 2
        if c["drafts"] > 1:
            held, more = c["groups"] * (shared + c["drafts"]), (1 + c["drafts"]) / 2
        else:
            held = c["groups"] * shared + some * more
        return {"bytes": held * 2 * c["kv"] * c["hd"] * b + 2 * c["n"] * heads * b,
                "flops": 4 * heads * (some * more + (c["n"] - c["alone"]) * shared)}
    # each weight is an exponential and a sum in 64 bits
    return {"bytes": c["rows"] * (c["vocab"] * b + 28), "flops": 10 * c["rows"] * c["vocab"]}


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _exact_append(s):
    c = s["case"]
    pairs, hd = c["pairs"], c["hd"]
    at = s["angles_at"].double()
    axis = torch.zeros(pairs, dtype=torch.int64, device="cuda") if s["axes"] is None else s["axes"].long()
    angle = torch.empty(c["rows"], pairs, dtype=torch.float64, device="cuda")
    for i in range(pairs):
        angle[:, i] = at[axis[i]] * s["frequencies"][i]
    # a pair is a complex number that is multiplied by e^(i angle)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rows(x, gain):
        x = x.double()
        if gain is not None:
            x = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / hd + EPS) * gain.double()
        x = x.clone()
        if c["adjacent"]:
            z = torch.complex(x[..., : 2 * pairs : 2].contiguous(), x[..., 1 : 2 * pairs : 2].contiguous()) * turn
            x[..., : 2 * pairs : 2], x[..., 1 : 2 * pairs : 2] = z.real, z.imag
        else:
            z = torch.complex(x[..., :pairs].contiguous(), x[..., pairs : 2 * pairs].contiguous()) * turn
            x[..., :pairs], x[..., pairs : 2 * pairs] = z.real, z.imag
        return x

    blocks = s["blocks"].double()
    where = s["positions"].long()
    number = s["table"].gather(1, (where // c["block"]).reshape(1, -1).expand(c["seqs"], -1))
    number = number[s["seqs"].long(), torch.arange(c["rows"], device="cuda")]
    k, v = rows(s["k"], s["k_gain"]), s["v"].double()
    for j in range(c["kv"]):
        blocks[number, c["layer"], 0, j, where % c["block"]] = k[:, j]
        blocks[number, c["layer"], 1, j, where % c["block"]] = v[:, j]
    return {"q": rows(s["q"], s["q_gain"]), "blocks": blocks}


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(c["n"], c["heads"], c["hd"], dtype=torch.float64, device="cuda")
    starts = [] if s["starts"] is None else s["starts"].tolist()
    shared = [] if s["shared"] is None else s["shared"].tolist()
    seqs, lengths = s["seqs"].tolist(), s["lengths"].tolist()
    lead = {r: (starts[g], shared[g]) for g in range(len(shared)) for r in range(starts[g], starts[g + 1])}
    for r in range(c["n"]):
        if not lengths[r]:
            continue
        first, common = lead.get(r, (r, 0))
        rows = []
        for sequence, lo, hi in ((seqs[first], 0, min(common, lengths[r])), (seqs[r], common, lengths[r])):
            if hi > lo:
                numbers = s["table"][sequence, : -(-hi // c["block"])]
                part = s["blocks"][numbers, c["layer"]].permute(1, 2, 0, 3, 4).reshape(2, c["kv"], -1, c["hd"])
                rows.append(part[:, :, lo:hi].double())
        k, v = torch.cat(rows, 2)
        q = s["q"][r].double().reshape(c["kv"], -1, c["hd"])
        p = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(c["hd"]), -1)
        out[r] = torch.bmm(p, v).reshape(c["heads"], c["hd"])
    return out


def _exact_sample(s):
    x = s["logits"].double()
    rows, vocab = x.shape
    token, logprob = [], []
    par = {k: (None if s[k] is None else s[k].tolist()) for k in ("temperature", "top_k", "top_p", "min_p", "u")}
    for r in range(rows):
        t = par["temperature"][r]
        k = par["top_k"][r] if par["top_k"] else 0
        k = 1 if t == 0 else vocab if k <= 0 else min(k, vocab)
        v, order = torch.sort(x[r], dim=-1, descending=True, stable=True)
        logw = (v - v[0]) / (t or 1.0)
        logw = logw[:k]
        if par["top_p"] and par["top_p"][r] < 1:
            share = torch.softmax(logw, 0).cumsum(0)
            logw = logw[: 1 + int((share < par["top_p"][r]).sum())]
        if par["min_p"] and par["min_p"][r] > 0:
            logw = logw[: max(1, int((logw >= math.log(par["min_p"][r])).sum()))]
        share = torch.softmax(logw, 0).cumsum(0)
        at = min(int((share <= par["u"][r]).sum()), int((logw > -math.inf).sum()) - 1)
        token.append(order[at])
        logprob.append(torch.log_softmax(logw, 0)[at])
    return {"token": torch.stack(token).to(torch.int32), "logprob": torch.stack(logprob)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](s)
