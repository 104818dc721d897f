"""The 4-bit cache on the GPU against plain 64-bit forms: what is stored byte by byte, what is fetched, and decode
attention over it, at the sizes, layouts and places where they can go wrong."""
from __future__ import annotations

import math

import pytest
import torch

import kvq_ref as R

pytestmark = pytest.mark.gpu


def make(hs, n_seqs, table_ld, n_layers, n_kv, hd, bt, seed=0, fill=0xFF, spare=2, held=None):
    """A cache whose every byte is `fill` (255: NaN groups), with shuffled block numbers."""
    g = torch.Generator().manual_seed(seed)
    total = n_seqs * table_ld + spare
    bb = hs.kvq_block_bytes(n_layers, n_kv, hd, bt)
    blocks = torch.full((total * bb + 5,), fill, dtype=torch.uint8, device="cuda")
    table = torch.randperm(total, generator=g)[: n_seqs * table_ld].reshape(n_seqs, table_ld)
    table = table.cuda()
    return hs.QuantCache(blocks, table, n_layers, n_kv, hd, bt), blocks, table


def rows(n, n_kv, hd, dtype, seed, device="cuda"):
    """Rows of many magnitudes, exact ties, zero groups and negative zeros among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, n_kv, hd, generator=g)
    x *= 2.0 ** torch.randint(-6, 7, (n, n_kv, hd // 32), generator=g).float().repeat_interleave(32, -1)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, -0.25, -0.75, -2.5, 0.0, -0.0, 6.9375, 3.4375])
    x[0, 0, :16] = ties
    x[0, 0, 16:32] = 0.5
    if n > 1:
        x[1, 0, :32] = 0.0
        x[1, 0, 3] = -0.0
    return x.to(R.DT[dtype]).to(device)


def expect_blocks(blocks, table, cfg, layer, dtype, k, v, seqs, pos):
    lay = R.Layout(blocks, table, *cfg)
    vals = []
    for sel, x in ((0, k), (1, v)):
        code, byte, val = R.quantize(x.cpu(), dtype)
        for i in range(x.shape[0]):
            lay.put(layer, sel, int(seqs[i]), int(pos[i]), code[i], byte[i])
        vals.append(val)
    return lay, vals


def same(got, want64):
    """Equal values, NaN in the same places."""
    got = got.double().cpu()
    return torch.equal(torch.isnan(got), torch.isnan(want64)) and torch.equal(got.nan_to_num(), want64.nan_to_num())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd,n_kv,bt", [(64, 1, 16), (128, 4, 32), (64, 3, 256), (128, 1, 1024)])
def test_append_stores_exactly_the_rounded_rows(dtype, hd, n_kv, bt):
    """Every byte of the cache: those of the rows stored, and every other as it was."""
    import paper_2603_12707_amd as hs
    n_seqs, n_layers = 3, 2
    cache, blocks, table = make(hs, n_seqs, 2, n_layers, n_kv, hd, bt, fill=0x5A)
    n = 37
    g = torch.Generator().manual_seed(5)
    place = torch.randperm(n_seqs * 2 * bt, generator=g)[:n] if n_seqs * 2 * bt >= n else None
    seqs, pos = (place // (2 * bt)).int(), (place % (2 * bt)).int()
    k, v = rows(n, n_kv, hd, dtype, 1), rows(n, n_kv, hd, dtype, 2)
    lay, (kv, vv) = expect_blocks(blocks, table, (n_layers, n_kv, hd, bt), 1, dtype, k, v, seqs, pos)
    want = blocks.cpu().clone()
    want[: lay.b.numel()] = lay.b.reshape(-1)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    cache.append(1, k, v, pos.cuda(), seqs=seqs.cuda(), k_values=ko, v_values=vo)
    assert torch.equal(blocks.cpu(), want)
    assert same(ko, kv) and same(vo, vv)
    rk, rv = cache.read(1, pos.cuda(), R.DT[dtype], seqs=seqs.cuda())
    assert same(rk, kv) and same(rv, vv)
    # |x - value| <= 2^e: half the widest step
    x = k.double().cpu()
    e = torch.frexp(x.reshape(n, n_kv, -1, 32).abs().amax(-1).clamp(min=2.0 ** -20)).exponent - 2
    assert ((x - kv).abs().reshape(n, n_kv, -1, 32) <= (2.0 ** e.double()).unsqueeze(-1)).all()


def test_every_half_precision_number_is_rounded_right():
    """All finite bf16 and f16 numbers below 7 times the group's power, the power set by one element of the group."""
    import paper_2603_12707_amd as hs
    for dtype in ("bf16", "f16"):
        allx = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(R.DT[dtype])
        allx = allx[torch.isfinite(allx)]
        allx = allx[: allx.numel() // 124 * 124].reshape(-1, 1, 124)
        for lead in (6.0, 1.0, 6.0 * 2.0 ** -10):
            x = allx.clone()
            x = torch.where(x.float().abs() <= lead, x, torch.zeros_like(x))
            x = torch.cat([x.reshape(-1, 1, 4, 31), torch.full((x.shape[0], 1, 4, 1), lead, dtype=x.dtype)], -1)
            x = x.reshape(-1, 1, 128).contiguous()
            n = x.shape[0]
            cache, blocks, table = make(hs, 1, -(-n // 256), 1, 1, 128, 256)
            pos = torch.arange(n, dtype=torch.int32, device="cuda")
            ko, vo = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
            cache.append(0, x.cuda(), x.cuda(), pos, seqs=torch.zeros_like(pos), k_values=ko, v_values=vo)
            assert same(ko, R.quantize(x, dtype)[2])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_extremes_and_non_finite_groups(dtype):
    """The largest and smallest numbers of the type, and groups with a NaN or an infinity (32 NaNs, the others kept)."""
    import paper_2603_12707_amd as hs
    cache, blocks, table = make(hs, 1, 1, 1, 1, 128, 16)
    big, tiny = torch.finfo(R.DT[dtype]).max, torch.finfo(R.DT[dtype]).smallest_normal
    x = torch.zeros(8, 1, 128, dtype=torch.float64)
    x[0, 0, :4] = torch.tensor([big, -big, big / 2, big / 16])
    x[0, 0, 32:36] = torch.tensor([tiny, -tiny, tiny * 4, tiny / 8 if dtype == "f16" else tiny])
    x[1, 0, 0] = math.nan
    x[1, 0, 40] = math.inf
    x[1, 0, 70] = -math.inf
    x[1, 0, 100] = 1.0
    x[2, 0, :] = tiny
    x[3, 0, ::32] = torch.tensor([2.0 ** -14, 6e4, 1.0, 2.0 ** 15]).to(torch.float64)
    x = x.to(R.DT[dtype]).cuda()
    pos = torch.arange(8, dtype=torch.int32, device="cuda")
    cache.append(0, x, x, pos, seqs=torch.zeros_like(pos))
    k, v = cache.read(0, pos, R.DT[dtype], seqs=torch.zeros_like(pos))
    want = R.quantize(x.cpu(), dtype)[2]
    assert same(k, want) and same(v, want)


def test_rows_that_have_no_place_are_not_stored():
    """Negative and far positions, sequences outside the table, blocks that are negative or past the buffer."""
    import paper_2603_12707_amd as hs
    cache, blocks, table = make(hs, 2, 3, 1, 2, 64, 16, fill=0x11)
    table[0, 1], table[1, 0], table[1, 2] = -1, 10 ** 9, table.numel() + 2
    before = blocks.clone()
    seqs = torch.tensor([0, 0, 0, -1, 2, 1, 1, 0, 2 ** 31 - 1, -2 ** 31, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([-1, 48, 16, 0, 0, 3, 40, 2 ** 31 - 1, 5, 5, -2 ** 31], dtype=torch.int32, device="cuda")
    k = rows(11, 2, 64, "f16", 3)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    cache.append(0, k, k, pos, seqs=seqs, k_values=ko, v_values=vo)
    assert torch.equal(blocks, before)
    assert same(ko, R.quantize(k.cpu(), "f16")[2])  # values come for every row
    rk, rv = cache.read(0, pos, torch.float16, seqs=seqs)
    assert not rk.any() and not rv.any()


@pytest.mark.parametrize("layout", ["rows", "heads", "wide", "alias"])
def test_append_and_read_take_strides(layout):
    import paper_2603_12707_amd as hs
    n, n_kv, hd = 9, 2, 64
    cache, blocks, table = make(hs, 1, 1, 1, n_kv, hd, 16)
    k, v = rows(n, n_kv, hd, "bf16", 4), rows(n, n_kv, hd, "bf16", 5)
    if layout == "heads":
        kk, vv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    elif layout == "wide":
        pad = torch.full((n, 5, hd + 8), 7.0, dtype=k.dtype, device="cuda")
        kk, vv = pad.clone()[:, 1:3, :hd], pad.clone()[:, 1:3, :hd]
        kk.copy_(k), vv.copy_(v)
    else:
        kk, vv = k.clone(), v.clone()
    pos = torch.arange(n, dtype=torch.int32, device="cuda").flip(0).contiguous()
    zero = torch.zeros_like(pos)
    cache.append(0, kk, vv, pos, seqs=zero, **(dict(k_values=kk, v_values=vv) if layout == "alias" else {}))
    if layout == "alias":
        assert same(kk, R.quantize(k.cpu(), "bf16")[2]) and same(vv, R.quantize(v.cpu(), "bf16")[2])
    ko = torch.empty_strided(kk.shape, kk.stride(), dtype=kk.dtype, device="cuda")
    vo = torch.empty_strided(kk.shape, kk.stride(), dtype=kk.dtype, device="cuda")
    cache.read(0, pos, torch.bfloat16, seqs=zero, k=ko, v=vo)
    assert same(ko, R.quantize(k.cpu(), "bf16")[2]) and same(vo, R.quantize(v.cpu(), "bf16")[2])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def fill_and_check(hs, dtype, lengths, heads, n_kv, hd, bt, *, n_layers=1, layer=0, table_ld=None, seqs=None, seed=0,
                   max_len=None, scale=None, spread=1.0, punch=None, workspace=None):
    lens = torch.tensor(lengths, dtype=torch.int32)
    n_seqs = len(lengths) if seqs is None else max(seqs) + 1
    longest = max(1, max(lengths))
    table_ld = table_ld or -(-longest // bt)
    cache, blocks, table = make(hs, n_seqs, table_ld, n_layers, n_kv, hd, bt, seed=seed)
    seq_len = [0] * n_seqs
    for r, ln in enumerate(lengths):
        s = r if seqs is None else seqs[r]
        seq_len[s] = max(seq_len[s], min(ln, table_ld * bt))
    at = [(s, p) for s in range(n_seqs) for p in range(max(0, seq_len[s]))]
    g = torch.Generator().manual_seed(seed + 1)
    if at:
        sq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*at))
        k = (torch.randn(len(at), n_kv, hd, generator=g) * spread).to(R.DT[dtype]).cuda()
        v = torch.randn(len(at), n_kv, hd, generator=g).to(R.DT[dtype]).cuda()
        cache.append(layer, k, v, pos, seqs=sq)
    if punch:
        punch(blocks, table)
    q = (torch.randn(len(lengths), heads, hd, generator=g) * 1.5).to(R.DT[dtype]).cuda()
    sq = None if seqs is None else torch.tensor(seqs, dtype=torch.int32, device="cuda")
    got = cache.attention(layer, q, lens.cuda(), seqs=sq, max_len=max_len, scale=scale, workspace=workspace)
    lay = R.Layout(blocks, table, n_layers, n_kv, hd, bt)
    want, mass, reach = R.attention(lay, layer, q.cpu(), lens, seqs, scale, max_len)
    tol = R.attention_tolerance(want, mass, reach, dtype, hd)
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), float((err - tol).max())
    return cache, q, lens.cuda(), got


EDGE = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,n_kv,hd,bt", [(4, 4, 64, 16), (28, 4, 128, 32), (2, 2, 128, 64), (16, 1, 64, 256),
                                              (6, 2, 128, 1024), (32, 2, 128, 128), (14, 2, 64, 32)])
def test_attention_at_every_edge_length(dtype, heads, n_kv, hd, bt):
    import paper_2603_12707_amd as hs
    fill_and_check(hs, dtype, EDGE, heads, n_kv, hd, bt, n_layers=2, layer=1, seed=heads)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", [[5000], [4097, 1, 0, 2500], [1024] * 3 + [1023, 1025]],
                         ids=["one", "ragged", "even"])
def test_attention_over_long_rows(dtype, lengths):
    import paper_2603_12707_amd as hs
    fill_and_check(hs, dtype, lengths, 8, 2, 128, 64, seed=3)
    fill_and_check(hs, dtype, lengths, 2, 2, 64, 512, seed=4)


@pytest.mark.parametrize("heads,n_kv,hd", [(4, 4, 64), (28, 4, 128)])
def test_fp32_rows_keep_fp32_precision(heads, n_kv, hd):
    """As a whole: the roundings of fp32 sums (2^-24 of each of a few terms, of either sign) are below 2^-20 of the
    result in the 2-norm; a product of fewer bits than fp32 anywhere on the way is not."""
    import paper_2603_12707_amd as hs
    cache, q, lens, got = fill_and_check(hs, "f32", [620, 90, 1500], heads, n_kv, hd, 32, seed=17)
    want = R.attention(R.Layout(cache.blocks, cache.table, 1, n_kv, hd, 32), 0, q.cpu(), lens.cpu())[0]
    assert float((got.double().cpu() - want).norm() / want.norm()) < 2.0 ** -20


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_a_loud_query_channel_costs_the_others_nothing(dtype, hd):
    """One query channel 2^14 above the others, over a group of K 2^14 below the others: both ends of the product count
    alike, and every element keeps all its bits.  Each head against a tolerance of its own."""
    import paper_2603_12707_amd as hs
    cache, blocks, table = make(hs, 1, 2, 1, 1, hd, 64)
    g = torch.Generator().manual_seed(hd)
    k, v = torch.randn(100, 1, hd, generator=g) * 0.5, torch.randn(100, 1, hd, generator=g)
    k[..., :32] *= 2.0 ** -14
    q = torch.randn(2, 2, hd, generator=g)
    q[:, 0, 5] = torch.tensor([1.25, -1.75]) * 2.0 ** 14
    k, v, q = (x.to(R.DT[dtype]).cuda() for x in (k, v, q))
    pos = torch.arange(100, dtype=torch.int32, device="cuda")
    cache.append(0, k, v, pos, seqs=torch.zeros_like(pos))
    lens = torch.tensor([100, 61], dtype=torch.int32)
    got = cache.attention(0, q, lens.cuda(), seqs=torch.zeros(2, dtype=torch.int32, device="cuda"), scale=1.0)
    lay = R.Layout(blocks, table, 1, 1, hd, 64)
    for h in range(2):
        want, mass, reach = R.attention(lay, 0, q[:, h : h + 1].cpu(), lens, [0, 0], 1.0)
        err = (got[:, h : h + 1].double().cpu() - want).abs()
        assert (err <= R.attention_tolerance(want, mass, reach, dtype, hd)).all(), (h, float(err.max()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_probabilities_keep_their_bits(dtype):
    """Two values that all but cancel: a position with most of the weight whose value is 0, and two with 1 and -1 whose
    scores differ by 2^-13.  A score is at most two exact products whose sum is exact; scaling it by log2(e) and taking
    the reference away leaves it off by less than 2^-23, the exponential by 2^-23 of itself, and the sums of three terms
    and the division by a few 2^-24 more: the weights by less than 2^-21 of themselves, and the output by 2^-20 of the sum
    of their sizes.  (With the probabilities in 16 bits it would be off by up to 2^-18.)"""
    import paper_2603_12707_amd as hs
    hd, n, heads = 64, 8, 16
    cache, blocks, table = make(hs, 1, 1, 1, 1, hd, 16)
    k, v = torch.zeros(3, 1, hd), torch.zeros(3, 1, hd)
    k[1:, 0, 0], k[1, 0, 32], k[2, 0, 32] = -1.0, 1.0, -1.0
    v[1], v[2] = 1.0, -1.0
    q = torch.zeros(n, heads, hd)
    q[..., 0] = (0.05 + 0.65 * torch.arange(n * heads).reshape(n, heads) / (n * heads)).to(R.DT[dtype]).float()
    q[..., 32] = 2.0 ** -14
    k, v, q = (x.to(R.DT[dtype]).cuda() for x in (k, v, q))
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    cache.append(0, k, v, pos, seqs=torch.zeros_like(pos))
    lens, seqs = torch.full((n,), 3, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)
    got = cache.attention(0, q, lens.cuda(), seqs=seqs.cuda(), scale=1.0).double().cpu()
    want, mass, _ = R.attention(R.Layout(blocks, table, 1, 1, hd, 16), 0, q.cpu(), lens, seqs, 1.0)
    tol = R.HALF_STEP[dtype] * want.abs() + 2.0 ** -20 * mass
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() - tol).max())


@pytest.mark.parametrize("heads", [2, 8])
def test_fp32_queries_reach_to_the_largest_number(heads):
    """A query element of the largest finite number over keys small enough for finite scores: not an infinity on the way."""
    import paper_2603_12707_amd as hs
    hd, big = 128, torch.finfo(torch.float32).max
    cache, blocks, table = make(hs, 1, 3, 1, 2, hd, 16)
    g = torch.Generator().manual_seed(heads)
    k, v = torch.randn(40, 2, hd, generator=g), torch.randn(40, 2, hd, generator=g)
    k[..., 32:64] *= 2.0 ** -124
    q = torch.randn(2, heads, hd, generator=g)
    q[0, :, 40], q[1, 0, 33], q[1, 1, 63] = big, -big, big * (1 - 2.0 ** -9)
    k, v, q = k.cuda(), v.cuda(), q.cuda()
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    cache.append(0, k, v, pos, seqs=torch.zeros_like(pos))
    lens = torch.tensor([40, 33], dtype=torch.int32)
    got = cache.attention(0, q, lens.cuda(), seqs=torch.zeros(2, dtype=torch.int32, device="cuda"))
    want, mass, reach = R.attention(R.Layout(blocks, table, 1, 2, hd, 16), 0, q.cpu(), lens, [0, 0])
    assert torch.isfinite(got).all()
    assert ((got.double().cpu() - want).abs() <= R.attention_tolerance(want, mass, reach, "f32", hd)).all()


def test_attention_over_very_long_rows():
    import paper_2603_12707_amd as hs
    fill_and_check(hs, "bf16", [70001, 3], 7, 1, 128, 1024, seed=6)
    fill_and_check(hs, "f16", [40000], 1, 1, 64, 16, seed=7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_masks_what_has_no_block(dtype):
    """Blocks missing at the start, inside and at the end, and numbers that are no block of the cache; a row all of
    whose blocks are missing gives zeros."""
    import paper_2603_12707_amd as hs

    def punch(blocks, table):
        table[0, 0], table[0, 5], table[1, 19] = -1, 10 ** 12, -7
        table[2, :] = -1
        table[3, :18] = -1

    for bt in (16, 64):
        fill_and_check(hs, dtype, [20 * bt, 20 * bt - 5, 300, 20 * bt], 8, 2, 128, bt, table_ld=20, punch=punch, seed=8)


def test_attention_rows_share_sequences_and_lengths_are_bounded():
    """Rows of one sequence at several lengths; lengths past max_len, past the table, and negative; sequences outside
    the table give zeros."""
    import paper_2603_12707_amd as hs
    fill_and_check(hs, "f16", [100, 37, 1, 100, 0, 64], 4, 4, 64, 32, seqs=[0, 0, 0, 1, 1, 0], seed=9)
    fill_and_check(hs, "bf16", [100, 37, 99], 4, 2, 64, 16, max_len=50, seed=10)
    cache, q, lens, got = fill_and_check(hs, "bf16", [64, 64, 64, 64], 4, 2, 64, 16, seed=11)
    sq = torch.tensor([0, -1, 4, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out = cache.attention(0, q, torch.full_like(lens, 2 ** 31 - 1), seqs=sq)
    assert torch.equal(out[0], got[0]) and not out[1:].any()
    out = cache.attention(0, q, torch.tensor([-1, -2 ** 31, 0, 64], dtype=torch.int32, device="cuda"))
    assert not out[:3].any() and torch.equal(out[3], got[3])


@pytest.mark.parametrize("n", [200, 256])
def test_many_rows_are_started_longest_first(n):
    """More work groups than the GPU holds: every row once, whatever the lengths (equal ones, none, the bound's own)."""
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(n)
    lengths = torch.randint(0, 90, (n,), generator=g).tolist()
    lengths[n // 2], lengths[3], lengths[n - 1] = 2100, 2048, 2100
    lengths[10:80] = [33] * 70
    fill_and_check(hs, "bf16", lengths, 8, 4, 64, 256, seed=18, max_len=2100)
    fill_and_check(hs, "f16", [7] * n, 4, 4, 64, 64, seed=19, max_len=4096, seqs=[i % 5 for i in range(n)])


@pytest.mark.parametrize("scale,spread", [(1.0, 30.0), (1e-6, 1.0), (-0.125, 1.0), (40.0, 8.0), (0.0, 1.0)],
                         ids=["peaked", "flat", "negative", "huge", "zero"])
def test_attention_of_other_scales(scale, spread):
    import paper_2603_12707_amd as hs
    for dtype in ("f16", "bf16", "f32"):
        fill_and_check(hs, dtype, [513, 70], 8, 2, 64, 64, scale=scale, spread=spread, seed=12)


def test_many_rows_and_many_heads():
    """More rows than a grid's second dimension takes, each as in a smaller call; and a cache of hundreds of heads."""
    import paper_2603_12707_amd as hs
    cache, q, lens, want = fill_and_check(hs, "bf16", [(37 * i) % 90 for i in range(300)], 4, 1, 64, 32, seed=22,
                                          seqs=[i % 7 for i in range(300)])
    n = 70000
    at = torch.arange(n, device="cuda") % 300
    got = cache.attention(0, q[at], lens[at], seqs=(at % 7).int())
    assert torch.equal(got, want[at])
    fill_and_check(hs, "f16", [70, 0, 33], 600, 300, 64, 16, seed=23)


def test_attention_takes_strides_and_leaves_other_memory_alone():
    import paper_2603_12707_amd as hs
    cache, q, lens, want = fill_and_check(hs, "bf16", [200, 31, 0, 77], 4, 2, 64, 32, seed=13)
    wide = torch.full((6, 9, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    qs, out = wide.clone()[1:5, 2:6], wide.clone()
    qs.copy_(q)
    cache.attention(0, qs, lens, out=out[1:5, 3:7])
    assert torch.equal(out[1:5, 3:7], want)
    out[1:5, 3:7] = 3.0
    assert torch.equal(out, wide)
    # one row, one head: no stride is looked at
    one = cache.attention(0, q[:1, :2].contiguous(), lens[:1])
    assert one.shape == (1, 2, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_that_nothing_uses_are_not_looked_at(dtype):
    """One row has no row stride, one head no head stride, whatever the tensors say of them."""
    import paper_2603_12707_amd as hs
    hd = 64
    odd = lambda x, st: torch.as_strided(x, x.shape, st)  # noqa: E731
    cache, blocks, table = make(hs, 2, 2, 1, 1, hd, 16)
    k, v = rows(20, 1, hd, dtype, 50), rows(20, 1, hd, dtype, 51)
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    zero = torch.zeros_like(pos)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    cache.append(0, odd(k, (hd, 5, 1)), odd(v, (hd, 7, 1)), pos, seqs=zero, k_values=odd(ko, (hd, 1, 1)), v_values=vo)
    want = [R.quantize(x.cpu(), dtype)[2] for x in (k, v)]
    for got, w in zip((ko, vo), want):
        assert torch.equal(got.double().cpu(), w)
    rk, rv = cache.read(0, pos, k.dtype, seqs=zero, k=odd(torch.empty_like(k), (hd, 3, 1)), v=torch.empty_like(v))
    assert torch.equal(rk.double().cpu(), want[0]) and torch.equal(rv.double().cpu(), want[1])
    q = rows(1, 4, hd, dtype, 52)
    one = cache.attention(0, q, pos[19:])
    out = torch.empty_like(q)
    cache.attention(0, odd(q, (1, hd, 1)), pos[19:], out=odd(out, (37, hd, 1)))
    assert torch.equal(out, one)
    wide, blocks, table = make(hs, 1, 1, 1, 3, hd, 16)
    k, v = rows(1, 3, hd, dtype, 53), rows(1, 3, hd, dtype, 54)
    wide.append(0, odd(k, (3, hd, 1)), odd(v, (1, hd, 1)), pos[:1], seqs=zero[:1])
    rk, rv = wide.read(0, pos[:1], k.dtype, seqs=zero[:1], k=odd(torch.empty_like(k), (11, hd, 1)))
    for got, x in ((rk, k), (rv, v)):
        assert torch.equal(got.double().cpu(), R.quantize(x.cpu(), dtype)[2])


def test_attention_passes_a_nan_group_on_to_its_own_heads():
    """A NaN stored in a row that is attended reaches the outputs of its KV head's rows and of no other; one behind
    the last position reaches none."""
    import paper_2603_12707_amd as hs
    for sel in (0, 1):
        cache, blocks, table = make(hs, 2, 4, 1, 2, 64, 16, fill=0)
        k = rows(64, 2, 64, "f16", 20)
        bad = k.clone()
        bad[40, 1, 3] = math.nan
        pos = torch.arange(64, dtype=torch.int32, device="cuda")
        for s in range(2):
            pair = (bad, k) if sel == 0 else (k, bad)
            cache.append(0, *(pair if s else (k, k)), pos, seqs=torch.full_like(pos, s))
        q = rows(2, 8, 64, "f16", 21)
        out = cache.attention(0, q, torch.tensor([64, 64], dtype=torch.int32, device="cuda"))
        assert torch.isfinite(out[0]).all() and torch.isfinite(out[1, :4]).all()
        nan = torch.isnan(out[1, 4:])
        assert nan.all() if sel == 0 else (nan[:, :32].all() and not nan[:, 32:].any())
        out = cache.attention(0, q, torch.tensor([64, 40], dtype=torch.int32, device="cuda"))
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("length,n_kv", [(3000, 2), (40000, 1)], ids=["joined", "combined"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_a_nan_in_one_of_several_splits_reaches_the_output(length, n_kv, dtype):
    """A NaN key group in one split alone, through the join of the last work group and through the combine kernel:
    the outputs of its head are NaN, the other heads' and rows' are not."""
    import paper_2603_12707_amd as hs
    hd = 64
    cache, blocks, table = make(hs, 2, -(-length // 64), 1, n_kv, hd, 64, fill=0)
    for at in (length // 3, length - 5, 7):
        blocks.zero_()  # rows of zeros but for a few, the one at `at` with a NaN
        pos = torch.arange(at - 5, min(at + 11, length), dtype=torch.int32, device="cuda")
        k, v = rows(len(pos), n_kv, hd, dtype, 60), rows(len(pos), n_kv, hd, dtype, 61)
        k[5, n_kv - 1, 3] = math.nan
        cache.append(0, k, v, pos, seqs=torch.zeros_like(pos))
        q = rows(2, 4 * n_kv, hd, dtype, 62)
        out = cache.attention(0, q, torch.tensor([length, length], dtype=torch.int32, device="cuda"))
        assert torch.isnan(out[0, -4:]).all()
        assert torch.isfinite(out[0, :-4]).all() and torch.isfinite(out[1]).all()
        short = cache.attention(0, q, torch.tensor([at, length], dtype=torch.int32, device="cuda"))
        assert torch.isfinite(short).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,n_kv,hd", [(4, 4, 64), (14, 2, 128)])
def test_queries_that_are_not_finite_reach_their_own_head_alone(dtype, heads, n_kv, hd):
    """An infinity or a NaN in a query head makes its output NaN (also where every score would be -inf), no other's.
    The others are within their tolerance and not always what they were bit for bit: a wave moves the references of
    its heads together, and a NaN score moves none, so that o and l are rounded at other places."""
    import paper_2603_12707_amd as hs
    cache, blocks, table = make(hs, 1, 8, 1, n_kv, hd, 16)
    k = rows(100, n_kv, hd, dtype, 30).abs() + 1.0
    v = rows(100, n_kv, hd, dtype, 31)
    pos = torch.arange(100, dtype=torch.int32, device="cuda")
    zero = torch.zeros_like(pos)
    cache.append(0, k, v, pos, seqs=zero)
    q = rows(4, heads, hd, dtype, 32)
    lens = torch.full((4,), 100, dtype=torch.int32)
    want, mass, reach = R.attention(R.Layout(blocks, table, 1, n_kv, hd, 16), 0, q.cpu(), lens, [0] * 4, None, None)
    tol = R.attention_tolerance(want, mass, reach, dtype, hd)
    q[0, 1, hd - 1], q[1, 0, 0], q[2, heads - 1, 33] = -math.inf, math.inf, math.nan
    got = cache.attention(0, q, lens.cuda(), seqs=zero[:4]).double().cpu()
    bad = torch.zeros(4, heads, dtype=torch.bool)
    bad[0, 1] = bad[1, 0] = bad[2, heads - 1] = True
    assert torch.isnan(got[bad]).all()
    assert ((got - want).abs() <= tol)[~bad].all()


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB whose rows live in its last blocks."""
    import paper_2603_12707_amd as hs
    n_kv, hd, bt = 4, 128, 1024
    bb = hs.kvq_block_bytes(2, n_kv, hd, bt)
    n_blocks = (5 << 30) // bb
    blocks = torch.full((n_blocks * bb,), 0xFF, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_blocks - 1, 0], [n_blocks - 2, n_blocks - 3]], device="cuda")
    cache = hs.QuantCache(blocks, table, 2, n_kv, hd, bt)
    small = blocks[: 4 * bb].clone()
    near = hs.QuantCache(small, torch.tensor([[3, 0], [2, 1]], device="cuda"), 2, n_kv, hd, bt)
    n = 1500
    seqs = torch.tensor([0] * n + [1] * n, dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n, dtype=torch.int32, device="cuda")] * 2)
    k, v = rows(2 * n, n_kv, hd, "bf16", 30), rows(2 * n, n_kv, hd, "bf16", 31)
    q = rows(2, 28, hd, "bf16", 32)
    lens = torch.tensor([n, n - 1], dtype=torch.int32, device="cuda")
    outs = []
    for c in (cache, near):
        c.append(1, k, v, pos, seqs=seqs)
        outs.append((c.attention(1, q, lens), *c.read(1, pos, torch.bfloat16, seqs=seqs)))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert torch.equal(blocks[(n_blocks - 1) * bb :], small[3 * bb :])


def test_calls_are_deterministic_and_run_on_the_current_stream():
    import paper_2603_12707_amd as hs
    cache, q, lens, want = fill_and_check(hs, "bf16", [3000, 17, 901], 28, 4, 128, 64, seed=14)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = cache.attention(0, q, lens)
        b = cache.attention(0, q, lens)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, want) and torch.equal(b, want)
    ws = cache.attention_workspace(3, 28, 3000, torch.bfloat16)
    ws[2048:].fill_(0xFF)  # only the first 2048 bytes are kept between calls
    c = cache.attention(0, q, lens, max_len=3000, workspace=ws)
    d = cache.attention(0, q, lens, max_len=3000, workspace=ws)
    assert torch.equal(c, d) and not ws[:2048].any()
    # the same workspace serves another shape, and the first one again
    fill_and_check(hs, "f16", [1200, 5, 700, 900], 4, 4, 64, 16, seed=16, workspace=ws)
    assert torch.equal(cache.attention(0, q, lens, max_len=3000, workspace=ws), c)


def test_append_and_attention_in_a_replayed_graph():
    """A step (append the new row, attend over one more position) captured once and replayed, the program's own work
    between the replays; every replay against the eager calls on a second cache."""
    import paper_2603_12707_amd as hs
    pair = []
    for _ in range(2):
        cache, blocks, table = make(hs, 3, 12, 1, 4, 128, 64, seed=15)
        k, v = rows(600, 4, 128, "bf16", 40), rows(600, 4, 128, "bf16", 41)
        pos = torch.arange(200, dtype=torch.int32, device="cuda").repeat(3)
        cache.append(0, k, v, pos, seqs=torch.arange(3, device="cuda", dtype=torch.int32).repeat_interleave(200))
        pair.append((cache, blocks))
    g = torch.Generator(device="cuda").manual_seed(3)
    lens = torch.tensor([200, 150, 1], dtype=torch.int32, device="cuda")
    new, q = (torch.randn(3, 4, 128, device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn(3, 28, 128, device="cuda", generator=g).bfloat16()
    out, ws = torch.empty_like(q), pair[0][0].attention_workspace(3, 28, 700)
    mine = lens.clone()

    def step():
        pair[0][0].append(0, new, new, mine)
        mine.add_(1)
        pair[0][0].attention(0, q, mine, max_len=700, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(5):
        new.copy_(torch.randn(new.shape, device="cuda", generator=g))
        q.copy_(torch.randn(q.shape, device="cuda", generator=g))
        pair[1][0].append(0, new, new, lens)
        lens.add_(1)
        want = pair[1][0].attention(0, q, lens, max_len=700)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        assert torch.equal(mine, lens)
    assert torch.equal(pair[0][1], pair[1][1])
