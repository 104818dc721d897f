"""The paged cache's operators on the GPU against plain 64-bit forms: rows normalised, turned and stored, and attention
with shared beginnings."""
from __future__ import annotations

import math

import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator().manual_seed(seed)


def close(got, want, off, dtype):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    bound = R.half_step(want, dtype) + off * (1 + torch.finfo(R.DT[dtype]).eps)
    worst = ((got - want).abs() / bound)[fine].max() if fine.any() else 0.0
    assert worst <= 1.0, float(worst)


# ---------------------------------------------------------------------------
# rows
# ---------------------------------------------------------------------------
def rows_case(hs, dtype, hd, kv, heads, n, block=32, layers=2, pairs=None, axes=0, adjacent=False, norm=False, far=0,
              seed=0, strided=False, in_place=False):
    g = gen(seed)
    dt = R.DT[dtype]
    width = -(-(n + 5) // block) + 1
    table = torch.randperm(2 * width, generator=g).reshape(2, width)
    blocks = R.blocks(2 * width, layers, kv, block, hd, dtype, fill=-7.0)
    cache = hs.PagedCache(blocks, table.cuda())
    wide = (heads + 2 * kv) * hd + (16 if strided else 0)
    qkv = torch.randn(n, wide, generator=g).to(dt).cuda()
    q, k, v = (qkv[:, o : o + h * hd].unflatten(-1, (h, hd)) for o, h in
               ((0, heads), (heads * hd, kv), ((heads + kv) * hd, kv)))
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    seqs = torch.randint(0, 2, (n,), generator=g, dtype=torch.int32)
    positions = torch.arange(n, dtype=torch.int32) + 3
    if n > 4:
        positions[1] = -1            # not stored
        seqs[2] = 2                  # outside the table
        positions[3] = width * block  # past it
    at = (torch.randint(-3, 4096, (max(axes, 1), n), generator=g) + far).to(torch.int32)
    pairs = hd // 2 if pairs is None else pairs
    freq = hs.rope_frequencies(1e4, pairs) if pairs else None
    ax = torch.randint(0, axes, (pairs,), generator=g, dtype=torch.int32) if axes > 1 else None
    rope = hs.Rope(freq, axes=None if ax is None else ax.cuda(), adjacent=adjacent, n_axes=max(axes, 1)) if pairs else None
    gains = [(1 + 0.3 * torch.randn(hd, generator=g)).to(dt) for _ in range(2)] if norm else [None, None]
    q0, k0, v0 = q.cpu(), k.cpu(), v.cpu()
    out = cache.append(layers - 1, k, v, positions.cuda(), seqs=seqs.cuda(), q=q if heads else None, rope=rope,
                       angles_at=at.cuda() if pairs else None, eps=1e-5, q_out=q if in_place else None,
                       q_gain=gains[0].cuda() if norm and heads else None, k_gain=gains[1].cuda() if norm else None)
    f = None if freq is None else freq.cpu()
    if heads:
        close(out, *R.turned(q0, gains[0], 1e-5, f, ax, at, adjacent), dtype)
        assert not in_place or out is q
    want, off = R.turned(k0, gains[1], 1e-5, f, ax, at, adjacent)
    expect = torch.full(blocks.shape, -7.0, dtype=torch.float64)
    bound = torch.zeros_like(expect)
    for i in range(n):
        p, s = int(positions[i]), int(seqs[i])
        if 0 <= p < width * block and s < 2:
            b = int(table[s, p // block])
            expect[b, -1, 0, :, p % block], bound[b, -1, 0, :, p % block] = want[i], off[i]
            expect[b, -1, 1, :, p % block] = v0[i].double()
    close(blocks, expect, bound, dtype)
    same = expect.clone()
    same[:, -1, 0] = 0
    got = blocks.double().cpu()
    got[:, -1, 0] = 0
    assert torch.equal(got, same)  # values and all that is not stored, bit for bit


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd,kv,heads,n", [(64, 1, 1, 1), (128, 2, 8, 1), (128, 4, 28, 37), (64, 3, 3, 130),
                                           (128, 32, 32, 5), (64, 2, 0, 9)])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_are_turned_and_stored(dtype, hd, kv, heads, n, norm):
    import paper_2603_12707_amd as hs
    rows_case(hs, dtype, hd, kv, heads, n, norm=norm, seed=n + hd)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd,pairs,axes,adjacent", [(128, 0, 0, False), (128, 16, 1, False), (128, 24, 3, False),
                                                    (128, 64, 3, True), (64, 8, 2, True), (64, 24, 8, False),
                                                    (64, 32, 3, False)])
def test_every_way_to_turn(dtype, hd, pairs, axes, adjacent):
    import paper_2603_12707_amd as hs
    rows_case(hs, dtype, hd, 2, 6, 33, pairs=pairs, axes=axes, adjacent=adjacent, norm=axes != 1, seed=pairs + axes)


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 4200, -(1 << 31) + 8])
@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions(far, adjacent):
    import paper_2603_12707_amd as hs
    rows_case(hs, "f32", 64, 2, 2, 40, far=far, adjacent=adjacent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_a_wider_projection_in_place(dtype):
    import paper_2603_12707_amd as hs
    rows_case(hs, dtype, 128, 4, 28, 70, norm=True, strided=True)
    rows_case(hs, dtype, 128, 4, 28, 70, norm=True, strided=True, in_place=True)
    rows_case(hs, dtype, 64, 2, 14, 3000, block=256, pairs=16, strided=True, in_place=True)


def test_many_rows_in_large_blocks():
    import paper_2603_12707_amd as hs
    rows_case(hs, "bf16", 128, 4, 28, 5003, block=1024, axes=3, norm=True)


def test_many_heads_of_some_rows():
    """A row's heads over several work groups, several passes each."""
    import paper_2603_12707_amd as hs
    rows_case(hs, "f32", 64, 32, 256, 300, block=64, axes=2, norm=True)
    rows_case(hs, "bf16", 128, 32, 512, 61, block=64, axes=1, norm=True, in_place=True)


def test_angles_default_to_positions():
    import paper_2603_12707_amd as hs
    n, hd = 9, 64
    blocks = R.blocks(2, 1, 2, 16, hd, "f32", fill=0.0)
    cache = hs.PagedCache(blocks, torch.tensor([[0, 1]], device="cuda"))
    k = torch.randn(n, 2, hd, generator=gen(1)).cuda()
    pos = torch.arange(7, 7 + n, dtype=torch.int32, device="cuda")
    seqs = torch.zeros(n, dtype=torch.int32, device="cuda")
    rope = hs.Rope(hs.rope_frequencies(1e6, 32))
    cache.append(0, k, k, pos, seqs=seqs, rope=rope)
    one = blocks.clone()
    cache.append(0, k, k, pos, seqs=seqs, rope=rope, angles_at=pos[None].contiguous())
    assert torch.equal(one, blocks) and bool((one != 0).any())


def test_rows_that_hold_nan_or_zeros():
    """A NaN stays in its own head; a head of zeros is normalised to zeros."""
    import paper_2603_12707_amd as hs
    blocks = R.blocks(1, 1, 2, 16, 64, "f32", fill=0.0)
    cache = hs.PagedCache(blocks, torch.zeros(1, 1, dtype=torch.int64, device="cuda"))
    k = torch.ones(2, 2, 64, device="cuda")
    k[0, 0, 5] = math.nan
    k[1, 1] = 0.0
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    pos = torch.arange(2, dtype=torch.int32, device="cuda")
    cache.append(0, k, k, pos, seqs=zero, rope=hs.Rope(hs.rope_frequencies(1e4, 32)),
                 k_gain=torch.ones(64, device="cuda"))
    got = blocks[0, 0, 0]
    assert bool(torch.isnan(got[0, 0]).all()) and bool(torch.isfinite(got[1]).all())
    assert bool((got[1, 1] == 0).all())
    assert torch.equal(torch.isnan(blocks[0, 0, 1, :, :2]), torch.isnan(k.transpose(0, 1)))


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def grouped(n, groups, shared, more, block, seed, alone=0, sequences=None):
    """(lengths, table, starts, shared, blocks): n rows in `groups` groups and `alone` by themselves, each with blocks
    of its own behind the whole ones that its group shares."""
    g = gen(seed)
    inside = n - alone
    starts = (torch.arange(groups + 1) * inside // max(groups, 1)).int()
    sh = torch.tensor([shared[i % len(shared)] for i in range(groups)], dtype=torch.int32)
    before = torch.zeros(n, dtype=torch.int64)
    for i in range(groups):
        before[starts[i] : starts[i + 1]] = int(sh[i])
    lengths = before + torch.tensor([more[i % len(more)] for i in range(n)])
    width = max(1, -(-int(lengths.max()) // block))
    total = n * width
    table = torch.randperm(total, generator=g).reshape(n, width)
    for i in range(groups):
        a, b = int(starts[i]), int(starts[i + 1])
        if a < b:
            table[a:b, : int(sh[i]) // block] = table[a, : int(sh[i]) // block].clone()
    return lengths.int(), table, starts, sh, total


def attend_case(hs, dtype, hd, kv, group, lengths, table, total, block, starts=None, shared=None, seqs=None, layers=2,
                seed=0, scale=None, max_len=None, max_shared=None, blocks=None, loud=1.0, q=None):
    g = gen(seed)
    n, heads = len(lengths), kv * group
    blocks = R.blocks(total, layers, kv, block, hd, dtype, seed) if blocks is None else blocks
    cache = hs.PagedCache(blocks, table.cuda())
    if q is None:
        q = (torch.randn(n, heads, hd, generator=g) * loud).to(R.DT[dtype])
    kw = {}
    if starts is not None:
        kw = dict(group_starts=starts.cuda(), shared=shared.cuda(), max_shared=max_shared)
    got = cache.attention(layers - 1, q.cuda(), lengths.cuda(), seqs=None if seqs is None else seqs.cuda(), scale=scale,
                          max_len=max_len, **kw)
    own = torch.arange(n) if seqs is None else seqs
    want, off = R.attention(q, blocks.cpu(), table, layers - 1, lengths, own, starts, shared, scale, max_len)
    close(got, want, off, dtype)
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kv,group", [(1, 1), (2, 4), (1, 16), (4, 7), (3, 3)])
def test_rows_of_every_length(dtype, hd, kv, group):
    import paper_2603_12707_amd as hs
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257, 511, 700, -4]
    lengths, table, _, _, total = grouped(len(lens), 0, [], lens, 16, hd)
    attend_case(hs, dtype, hd, kv, group, lengths, table, total, 16, seed=group)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kv,group,n,groups,alone", [(1, 1, 3, 1, 0), (4, 1, 70, 1, 0), (2, 7, 40, 3, 5),
                                                     (1, 16, 9, 2, 0), (2, 2, 150, 2, 1), (1, 3, 64, 64, 0)])
def test_shared_beginnings(dtype, hd, kv, group, n, groups, alone):
    import paper_2603_12707_amd as hs
    block = 32
    lengths, table, starts, shared, total = grouped(n, groups, [576, 96, 320], [1, 40, 5, 200, 33], block, n, alone)
    attend_case(hs, dtype, hd, kv, group, lengths, table, total, block, starts, shared, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,groups,kv,group", [(74, 1, 1, 7), (40, 1, 2, 16), (90, 2, 1, 5), (140, 70, 1, 2),
                                               (200, 130, 1, 1)])
def test_large_groups(dtype, hd, n, groups, kv, group):
    """Tiles of 256 columns that rows lie across, and of 128; more groups than a wave has lanes."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(n, groups, [320, 1088, 64], [1, 40, 5, 0], 64, n)
    attend_case(hs, dtype, hd, kv, group, lengths, table, total, 64, starts, shared, layers=1, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shared", [[1], [15], [16], [17], [100], [0], [128], [129, 0, 7]])
def test_shared_beginnings_that_end_anywhere(dtype, shared):
    """Also within a block: the first row's positions count, whatever the others' blocks hold."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, sh, total = grouped(24, 3, shared, [0, 1, 16, 3, 130], 16, 3)
    attend_case(hs, dtype, 64, 2, 4, lengths, table, total, 16, starts, sh, seed=len(shared))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_shorter_than_what_their_group_shares(dtype):
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(12, 2, [300, 200], [5, 60], 32, 4)
    lengths[1], lengths[4], lengths[7], lengths[10] = 0, 299, 3, 200
    lengths[0] = 40  # the first row too
    attend_case(hs, dtype, 128, 2, 4, lengths, table, total, 32, starts, shared)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_drafted_tokens_of_sequences(dtype):
    """Rows that are the next tokens of one sequence, which share all that was there before."""
    import paper_2603_12707_amd as hs
    block, per = 64, 5
    before = torch.tensor([700, 64, 1, 129])
    table = torch.randperm(4 * 12, generator=gen(1)).reshape(4, 12)
    seqs = torch.arange(4).repeat_interleave(per).int()
    lengths = (before[seqs.long()] + 1 + torch.arange(4 * per) % per).int()
    starts = (torch.arange(5) * per).int()
    attend_case(hs, dtype, 128, 2, 7, lengths, table, 48, block, starts, before.int(), seqs)
    # a prompt's rows: nothing shared, each sees those before it
    seqs = torch.zeros(130, dtype=torch.int32)
    attend_case(hs, dtype, 64, 2, 2, torch.arange(1, 131).int(), table, 48, block, seqs=seqs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_places_without_a_block(dtype):
    """Missing blocks, numbers past the cache and sequences outside the table are masked, in front, in the shared
    beginning and in tails."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(10, 2, [160], [90, 10], 16, 5)
    table = table.clone()
    table[:5, 2] = -1          # in the first group's beginning
    table[3, 11] = total       # in a tail
    table[4, 10:] = -5         # a whole tail
    table[5:, :10] = 1 << 40   # all that the second group shares
    table[9] = -1              # and a row's own
    seqs = torch.arange(10).int()
    seqs[1] = 10               # outside
    attend_case(hs, dtype, 64, 2, 3, lengths, table, total, 16, starts, shared, seqs)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_lies_past_the_lengths_is_not_looked_at(dtype):
    """NaN and infinities behind every row, behind the shared positions, and in a row's own blocks in their place."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(9, 2, [100, 77], [30, 3, 61], 32, 6)
    blocks = R.blocks(total, 2, 2, 32, 64, dtype, 3)
    clean = torch.zeros(total, 32, dtype=torch.bool)
    for r in range(9):
        lead, sh = (0, 100) if r < int(starts[1]) else (int(starts[1]), 77)
        for p in range(int(lengths[r])):
            clean[table[lead if p < sh else r, p // 32], p % 32] = True
    bad = (~clean).nonzero().cuda()
    blocks[bad[:, 0], :, 0, :, bad[:, 1]] = math.nan
    blocks[bad[:, 0], :, 1, :, bad[:, 1]] = math.inf
    attend_case(hs, dtype, 64, 2, 4, lengths, table, total, 32, starts, shared, blocks=blocks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("loud", [30.0, 1000.0])
def test_loud_scores(dtype, loud):
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(60, 1, [200], [1, 70], 16, 7)
    attend_case(hs, dtype, 128, 1, 4, lengths, table, total, 16, starts, shared, loud=loud)
    lengths, table, starts, shared, total = grouped(20, 2, [200], [1, 70], 16, 7)
    attend_case(hs, dtype, 64, 2, 4, lengths, table, total, 16, starts, shared, loud=loud)


def test_a_nan_query_is_its_own():
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(6, 1, [64], [20], 16, 8)
    q = torch.randn(6, 4, 64, generator=gen(2)).to(torch.bfloat16)
    q[2, 1, 3] = math.nan
    attend_case(hs, "bf16", 64, 2, 2, lengths, table, total, 16, starts, shared, q=q)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_scale_and_bounds(dtype):
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(8, 2, [96], [50, 120], 16, 9)
    attend_case(hs, dtype, 64, 2, 2, lengths, table, total, 16, starts, shared, scale=-0.3)
    attend_case(hs, dtype, 64, 2, 2, lengths, table, total, 16, starts, shared, scale=0.0)
    l2, t2, s2, h2, n2 = grouped(50, 1, [96], [50, 120], 16, 9)
    for scale in (-0.3, 0.0):
        attend_case(hs, dtype, 64, 1, 6, l2, t2, n2, 16, s2, h2, scale=scale)
    # lengths past max_len are cut
    attend_case(hs, dtype, 64, 2, 2, lengths, table, total, 16, starts, shared, max_len=140, max_shared=96)


@pytest.mark.parametrize("max_shared", [0, 10, 32, 95])
def test_more_shared_than_max_shared(max_shared):
    """What lies past max_shared is read through each row's own blocks, which share it too."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(8, 2, [96], [50, 120], 16, 9)
    attend_case(hs, "bf16", 64, 2, 2, lengths, table, total, 16, starts, shared, max_shared=max_shared)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,shared,more", [(1, 0, 30000), (2, 9000, 3000), (33, 5000, 400)])
def test_long_rows_in_several_splits(dtype, n, shared, more):
    import paper_2603_12707_amd as hs
    lengths, table, starts, sh, total = grouped(n, 1 if shared else 0, [shared], [more, more // 3], 256, n)
    if shared:
        attend_case(hs, dtype, 64, 1, 4, lengths, table, total, 256, starts, sh, layers=1)
    else:
        attend_case(hs, dtype, 64, 1, 4, lengths, table, total, 256, layers=1)


def test_strided_queries_and_outputs_and_one_workspace():
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(10, 2, [300], [40, 9], 32, 11)
    blocks = R.blocks(total, 1, 2, 32, 64, "bf16", 1)
    cache = hs.PagedCache(blocks, table.cuda())
    wide = torch.randn(10, 704, generator=gen(3)).to(torch.bfloat16).cuda()
    q = wide[:, 8 : 8 + 512].unflatten(-1, (8, 64))
    out = torch.full((10, 600), 5.0, dtype=torch.bfloat16, device="cuda")
    kw = dict(group_starts=starts.cuda(), shared=shared.cuda(), max_len=512, max_shared=300)
    ws = cache.attention_workspace(10, 8, 512, n_groups=2, max_shared=300)
    ws.random_(0, 256)  # nothing in it is needed
    got = cache.attention(0, q, lengths.cuda(), out=out[:, :512].unflatten(-1, (8, 64)), workspace=ws, **kw)
    plain = cache.attention(0, q.contiguous(), lengths.cuda(), **kw)
    assert torch.equal(got, plain) and bool((out[:, 512:] == 5).all())
    again = cache.attention(0, q, lengths.cuda(), workspace=ws, **kw)
    assert torch.equal(again, plain)


def test_groups_change_between_replays():
    import paper_2603_12707_amd as hs
    n, block = 24, 32
    lengths, table, starts, shared, total = grouped(n, 3, [320, 64, 200], [30, 100], block, 12)
    blocks = R.blocks(total, 1, 2, block, 128, "bf16", 2)
    cache = hs.PagedCache(blocks, table.cuda())
    q = torch.randn(n, 8, 128, generator=gen(4)).to(torch.bfloat16).cuda()
    held = dict(lengths=lengths.cuda(), group_starts=starts.cuda(), shared=shared.cuda())
    ws = cache.attention_workspace(n, 8, 512, n_groups=3, max_shared=400)
    out = torch.empty_like(q)
    call = lambda o: cache.attention(0, q, held["lengths"], group_starts=held["group_starts"],  # noqa: E731
                                     shared=held["shared"], max_len=512, max_shared=400, out=o, workspace=ws)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for turn in range(4):
        if turn:  # other groups, lengths and tables, in the same tensors
            l2, t2, s2, h2, _ = grouped(n, 3, [32 * turn, 100], [7 * turn, 60], block, 20 + turn)
            t3 = torch.full(table.shape, -1)
            t3[:, : min(t2.shape[1], table.shape[1])] = t2[:, : table.shape[1]]
            held["lengths"].copy_(l2)
            held["group_starts"].copy_(torch.tensor([0, turn, turn + 9, n]) if turn > 1 else s2)
            held["shared"].copy_(h2)
            cache.table.copy_(t3 % total)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(torch.empty_like(q)))
        want, off = R.attention(q.cpu(), blocks.cpu(), cache.table.cpu(), 0, held["lengths"].cpu(), torch.arange(n),
                                held["group_starts"].cpu(), held["shared"].cpu(), max_len=512)
        close(out, want, off, "bf16")


def test_on_another_stream():
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(12, 2, [300], [40, 9], 32, 13)
    cache = hs.PagedCache(R.blocks(total, 1, 2, 32, 64, "f16", 5), table.cuda())
    q = torch.randn(12, 4, 64, generator=gen(5)).half().cuda()
    kw = dict(group_starts=starts.cuda(), shared=shared.cuda())
    lens = lengths.cuda()
    want = cache.attention(0, q, lens, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cache.attention(0, q, lens, **kw)
    side.synchronize()
    assert torch.equal(got, want)


def test_empty_batches():
    import paper_2603_12707_amd as hs
    cache = hs.PagedCache(R.blocks(1, 1, 2, 16, 64, "f16", 1), torch.zeros(1, 1, dtype=torch.int64, device="cuda"))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    q = torch.empty(0, 4, 64, dtype=torch.float16, device="cuda")
    assert cache.attention(0, q, none).shape == q.shape
    k = torch.empty(0, 2, 64, dtype=torch.float16, device="cuda")
    assert cache.append(0, k, k, none, q=q).shape == q.shape


def test_a_step_of_answers_to_one_prompt():
    """Rows stored and then attended to, several answers to one prompt, step by step: as one sequence of its own each."""
    import paper_2603_12707_amd as hs
    g, n, kv, heads, hd, block, prompt = gen(6), 6, 2, 8, 64, 16, 70
    width = 8
    # the prompt's whole blocks are the first row's; the block that it ends in is copied for each answer
    table = torch.arange(n * width).reshape(n, width)
    table[:, : prompt // block] = table[0, : prompt // block].clone()
    blocks = R.blocks(n * width, 1, kv, block, hd, "bf16", fill=math.nan)
    cache = hs.PagedCache(blocks, table.cuda())
    rope = hs.Rope(hs.rope_frequencies(1e4, hd // 2))
    rand = lambda m, h: torch.randn(m, h, hd, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    at = torch.arange(prompt, dtype=torch.int32, device="cuda")
    cache.append(0, rand(prompt, kv), rand(prompt, kv), at, seqs=torch.zeros_like(at), rope=rope)
    last = table[:, prompt // block]
    blocks[last[1:].cuda()] = blocks[int(last[0])].clone()
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    shared = torch.tensor([prompt // block * block], dtype=torch.int32, device="cuda")
    for step in range(12):
        pos = torch.full((n,), prompt + step, dtype=torch.int32, device="cuda")
        q = cache.append(0, rand(n, kv), rand(n, kv), pos, q=rand(n, heads), rope=rope)
        out = cache.attention(0, q, pos + 1, group_starts=starts, shared=shared, max_len=128, max_shared=96)
        want, off = R.attention(q.cpu(), blocks.cpu(), table, 0, (pos + 1).cpu(), torch.arange(n))
        close(out, want, off, "bf16")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("own,heads", [(True, 1), (False, 1), (False, 2), (False, 4)])
def test_weights_of_24_bits(hd, own, heads):
    """Of weights 1, 1 and w, times -(w's first 8 bits), -(its next 8) and 1, what is left is w's last bits.  Row and
    channel i: w = e^-q_i, with little in common with any sum of two bf16 numbers."""
    import paper_2603_12707_amd as hs
    bf = torch.bfloat16
    q = torch.cat([torch.arange(128, 256) / 2.0 ** e for e in (8, 9, 10, 11)]).to(bf)  # each of 8 bits
    w = torch.exp(-q.double())
    one = w.to(bf).double()
    two = (w - one).to(bf).double()
    left = w - one - two
    pick = left.abs().argsort(descending=True)[:64]
    q, w, one, two, left = (t[pick] for t in (q, w, one, two, left))
    assert float(left.abs().min()) > 1.2e-6
    blocks = torch.zeros(1, 1, 2, 1, 16, hd, dtype=bf)
    blocks[0, 0, 0, 0, 2, 0] = -1.0
    blocks[0, 0, 1, 0, 0, :64], blocks[0, 0, 1, 0, 1, :64], blocks[0, 0, 1, 0, 2, :64] = (-one).to(bf), (-two).to(bf), 1.0
    queries = torch.zeros(64, heads, hd, dtype=bf)
    queries[:, :, 0] = q[:, None]
    cache = hs.PagedCache(blocks.cuda(), torch.zeros(1, 1, dtype=torch.int64, device="cuda"))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    kw = {} if own else dict(group_starts=i32(0, 64), shared=i32(3))
    got = cache.attention(0, queries.cuda(), i32(*[3] * 64), seqs=i32(*[0] * 64), scale=1.0, max_len=16, **kw)
    got = torch.diagonal(got.double().cpu()[:, :, :64], dim1=0, dim2=2).T  # [row][head], channel = row
    want = (left / (2 + w))[:, None].expand(-1, heads)
    # the score in base 2 (at most 1.44) is off by 2^-23 of itself, the exponential by 2^-23, a third part by 2^-25 and
    # nine sums of at most 1 by 2^-24 each
    off = (1.0 * 2.0 ** -23 + 2.0 ** -23 + 2.0 ** -25 + 9 * 2.0 ** -24) / 2.0
    bound = off + R.half_step(want, "bf16")
    assert ((got - want).abs() <= bound).all(), float(((got - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("at", [0, 4100, 8000])
@pytest.mark.parametrize("nats", [11.0, 13.5, 15.5, 17.5, 19.0])
@pytest.mark.parametrize("n,group", [(1, 1), (5, 4), (40, 2), (90, 4)])
def test_a_position_far_above_all_others(dtype, at, nats, n, group):
    """Its value is 0, as of positions that take the weight which nothing else wants: what comes out is the others', some
    2^-16 to 2^-28 of it each, of rows by themselves and of groups in tiles of every width."""
    import paper_2603_12707_amd as hs
    length, hd, dt = 8001, 64, R.DT[dtype]
    width = -(-length // 256)
    blocks = torch.zeros(width, 1, 2, 1, 256, hd, dtype=dt)
    blocks[at // 256, 0, 0, 0, at % 256, 0] = nats
    blocks[:, 0, 1, 0] = (1.0 + torch.arange(hd) / hd).to(dt)
    blocks[at // 256, 0, 1, 0, at % 256] = 0.0
    table = torch.randperm(width, generator=gen(2))[None]
    placed = torch.empty_like(blocks)
    placed[table[0]] = blocks
    q = torch.zeros(n, group, hd, dtype=dt)
    q[:, :, 0] = 1.0
    own = torch.zeros(n, dtype=torch.int32)
    lengths = torch.full((n,), length, dtype=torch.int32)
    want, off = R.attention(q[:1, :1], placed, table, 0, lengths[:1], own[:1], scale=1.0)  # every row and head alike
    cache = hs.PagedCache(placed.cuda(), table.cuda())
    for shared in (0, 8000, length) if n > 1 else (0,):
        kw = {}
        if shared:
            kw = dict(group_starts=torch.tensor([0, n], dtype=torch.int32).cuda(), max_shared=shared,
                      shared=torch.tensor([shared], dtype=torch.int32).cuda())
        got = cache.attention(0, q.cuda(), lengths.cuda(), seqs=own.cuda(), scale=1.0, **kw)
        close(got, want.expand(n, group, -1), off.expand(n, group, -1), dtype)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("order", ["falling", "rising", "steps"])
def test_scores_that_fall_and_rise_along_a_row(hd, order):
    """f16 weights over 60 bits and more, in either order, so that no one scale holds them all."""
    import paper_2603_12707_amd as hs
    length, g = 3300, gen(hd)
    table = torch.randperm(13, generator=g)[None]
    score = {"falling": torch.linspace(45, 0, 3328), "rising": torch.linspace(0, 45, 3328),
             "steps": torch.tensor([0.0, 14.0, 3.0, 44.0, 20.0, 0.0]).repeat_interleave(555)[:3328]}[order]
    k = torch.zeros(13, 256, hd)
    k[..., 0] = score.reshape(13, 256)
    v = torch.randn(13, 256, hd, generator=g)
    blocks = torch.zeros(13, 1, 2, 1, 256, hd, dtype=torch.float16)
    blocks[table[0], 0, 0, 0], blocks[table[0], 0, 1, 0] = k.half(), v.half()
    for n, group in ((3, 1), (33, 2), (49, 4)):
        q = torch.zeros(n, group, hd)
        q[..., 0] = torch.linspace(-1, 1, n * group).reshape(n, group)
        q[..., 1:] = torch.randn(n, group, hd - 1, generator=g)
        kw = dict(seqs=torch.zeros(n, dtype=torch.int32), scale=1.0, layers=1, blocks=blocks.cuda(), q=q.half())
        lengths = torch.randint(1, length, (n,), generator=g, dtype=torch.int32)
        attend_case(hs, "f16", hd, 1, group, lengths, table, 13, 256, **kw)
        lengths = torch.full((n,), length, dtype=torch.int32)
        attend_case(hs, "f16", hd, 1, group, lengths, table, 13, 256, torch.tensor([0, n], dtype=torch.int32),
                    torch.tensor([3200], dtype=torch.int32), **kw)


@pytest.mark.parametrize("loud", [30.0, 300.0])
def test_loud_scores_in_half_precision(loud):
    import paper_2603_12707_amd as hs
    for n, groups, kv, hd in ((60, 1, 1, 128), (20, 2, 2, 64)):
        lengths, table, starts, shared, total = grouped(n, groups, [200], [1, 70], 16, 7)
        attend_case(hs, "f16", hd, kv, 4, lengths, table, total, 16, starts, shared, loud=loud)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n,group", [(6, 2), (50, 2), (50, 5)])
def test_nan_and_immense_queries_are_their_own(dtype, n, group):
    """A NaN query gives NaN; scores of 10^9, whose differences to a maximum are rounded, give finite outputs, and other
    rows are as without them."""
    import paper_2603_12707_amd as hs
    lengths, table, starts, shared, total = grouped(n, 1, [320], [20, 90], 16, 8)
    blocks = R.blocks(total, 1, 1, 16, 64, dtype, 4)
    cache = hs.PagedCache(blocks, table.cuda())
    q = torch.randn(n, group, 64, generator=gen(2)).to(R.DT[dtype])
    call = lambda q, **kw: cache.attention(0, q.cuda(), lengths.cuda(), scale=1000.0, **kw)  # noqa: E731
    kw = dict(group_starts=starts.cuda(), shared=shared.cuda())
    q[3] = 60000.0 * torch.sign(q[3])
    first = [call(q), call(q, **kw)]
    q[2, 1, 3] = math.nan
    for got, before in zip((call(q), call(q, **kw)), first):
        assert bool(torch.isfinite(before).all())
        assert bool(torch.isnan(got[2, 1]).all())
        rest = torch.ones(n, group, dtype=torch.bool)
        rest[2, 1] = False
        assert torch.equal(got[rest.cuda()], before[rest.cuda()])
