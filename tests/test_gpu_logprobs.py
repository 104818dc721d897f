"""Token log probabilities, entropies and alternatives on the GPU against a plain 64-bit form."""
from __future__ import annotations

import math
import os
import re

import pytest
import torch

import kvq_ref as R

pytestmark = pytest.mark.gpu


def check(hs, x, tokens, top, workspace=None):
    tk = tokens.to(torch.int32).cuda()
    lp, ent, ids, tops = hs.token_logprobs(x, tk, top=top, workspace=workspace)
    want = R.logprobs(x.float().cpu(), tokens, top)
    for got, ref in ((lp, want[0]), (ent, want[1])) + (((tops, want[3]),) if top else ()):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        inf = torch.isinf(ref)
        assert torch.equal(got[inf], ref[inf])
        fine = torch.isfinite(ref)
        err = (got[fine] - ref[fine]).abs()
        assert (err <= R.logprob_tolerance(ref[fine])).all(), float(err.max())
    if top:
        assert torch.equal(ids.long().cpu(), want[2])
    return lp, ent, ids, tops


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 63), (2, 64), (2, 65), (5, 997), (1, 4096), (2, 8191),
                                        (2, 8192), (2, 8193), (3, 16385), (3, 32000), (2, 152064), (1, 200001)])
def test_logprobs_of_every_size(dtype, rows, vocab):
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3).to(R.DT[dtype]).cuda()
    tokens = torch.randint(0, vocab, (rows,), generator=g)
    for top in sorted({0, 1, min(5, vocab), min(20, vocab), min(64, vocab)}):
        check(hs, x, tokens, top)


@pytest.mark.parametrize("vocab", [3, 100, 4099, 40000, 300000])
def test_equal_logits_come_by_index(vocab):
    """Ties everywhere: rows of one value, of two values, of zeros of both signs."""
    import paper_2603_12707_amd as hs
    x = torch.zeros(5, vocab)
    x[1] = -2.5
    x[2, 1::2] = 1.0
    x[3, ::2] = -0.0
    x[4] = torch.arange(vocab) // 7
    top = min(vocab, 64)
    for dtype in ("f32", "bf16"):
        check(hs, x.to(R.DT[dtype]).cuda(), torch.tensor([0, vocab - 1, 1, 2, vocab // 2]), top)


@pytest.mark.parametrize("vocab", [4097, 40000])
def test_sorted_rows(vocab):
    """The largest logits side by side at the start, at the end, and a stride apart."""
    import paper_2603_12707_amd as hs
    up = torch.linspace(-8, 8, vocab)
    x = torch.stack([up, up.flip(0), up.reshape(-1)[torch.arange(vocab) * 64 % vocab] if vocab % 2 else up])
    check(hs, x.cuda(), torch.tensor([0, 1, 2]), 64)


@pytest.mark.parametrize("vocab", [5, 9001, 33000])
def test_banned_words_and_rows_without_a_distribution(vocab):
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(1)
    x = torch.randn(12, vocab, generator=g)
    x[0, torch.rand(vocab, generator=g) < 0.9] = -math.inf
    x[0, 2] = 0.0
    x[1] = -math.inf
    x[1, vocab - 1] = -300.0  # one word left
    x[2] = -math.inf          # none
    x[3, 1] = math.nan
    x[4, vocab - 1] = math.inf
    x[5] = torch.finfo(torch.float32).min  # the lowest number, everywhere: an even distribution
    x[6] = torch.finfo(torch.float32).min
    x[6, 3] = 0.0
    x[7, vocab // 2] = -math.nan
    x[8] = math.inf
    x[9] = -math.inf
    x[9, :2] = torch.tensor([1.0, 1.0])
    x[10, 0] = 80.0
    x[11] *= 1e30
    tokens = torch.tensor([2, vocab - 1, 0, 0, 0, 1, 0, -1, 4, 3, 0, 0])
    check(hs, x.cuda(), tokens, 5)
    check(hs, x.cuda(), torch.full((12,), -1), 3)
    check(hs, x.cuda(), torch.tensor([vocab, vocab + 5, 2 ** 31 - 1, -2 ** 31] * 3), 1)


@pytest.mark.parametrize("dtype,vocab", [("f32", 600001), ("f32", 1100003), ("bf16", 2200007)])
def test_rows_of_more_parts_than_a_wave_has_lanes(dtype, vocab):
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(3, vocab, generator=g).to(R.DT[dtype])
    x[1] = torch.tensor([0.5, -0.25])[torch.randint(0, 2, (vocab,), generator=g)].to(x.dtype)  # ties everywhere
    x[2] = -math.inf
    x[2, vocab - 3 :] = torch.tensor([1.0, 2.0, 1.0]).to(x.dtype)
    for top in (0, 1, 20, 64):
        check(hs, x.cuda(), torch.tensor([vocab - 1, 5, vocab - 2]), top)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [700, 40000])
def test_nan_among_banned_words(dtype, vocab):
    """A NaN counts too where the numbers about it are all -inf, or where there are none."""
    import paper_2603_12707_amd as hs
    x = torch.full((6, vocab), -math.inf)
    x[:, vocab - 1] = 1.0
    x[0, :] = math.nan
    x[1, 3] = math.nan
    x[2, :vocab // 2] = math.nan
    x[3, vocab // 2:] = math.nan
    x[4, :vocab - 1] = math.nan
    for top in (0, 1, 5):
        check(hs, x.to(R.DT[dtype]).cuda(), torch.tensor([vocab - 1, 0, vocab - 1, 0, vocab - 1, vocab - 1]), top)


def test_nearly_certain_tokens_keep_their_digits():
    """log Z of a row with one likely word: as small as e^-40, and within a few 2^-22 of itself."""
    import paper_2603_12707_amd as hs
    x = torch.zeros(3, 20000)
    for r, gap in enumerate((20.0, 30.0, 50.0)):
        x[r, 12345] = gap
    lp, ent, ids, tops = hs.token_logprobs(x.cuda(), torch.full((3,), 12345, dtype=torch.int32).cuda(), top=1)
    want = R.logprobs(x, torch.full((3,), 12345), 1)
    assert ids.flatten().tolist() == [12345] * 3
    assert ((lp.double().cpu() - want[0]).abs() <= 2.0 ** -18 * want[0].abs()).all()
    assert ((ent.double().cpu() - want[1]).abs() <= 2.0 ** -18 * want[1].abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_and_unaligned_rows(dtype):
    """Rows inside a wider matrix, from every offset of a 16-byte chunk."""
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(2)
    base = (torch.randn(4, 9100, generator=g) * 2).to(R.DT[dtype])
    for off in range(0, 9):
        for vocab in (8192, 9000 + off, 3 + off):
            x = base.cuda()[:, off : off + vocab]
            check(hs, x, torch.tensor([0, vocab - 1, 1, -1]), min(vocab, 7))


@pytest.mark.parametrize("rows", [511, 513])
def test_rows_of_several_parts_on_both_sides_of_the_one_launch_limit(rows):
    import paper_2603_12707_amd as hs
    g = torch.Generator(device="cuda").manual_seed(9)
    x = (torch.randn(rows, 8200, device="cuda", generator=g) * 2).bfloat16()
    x[::3, 8192:] = 30.0  # the largest, and equal, in the short part
    x[1::7, :8192] = -math.inf
    tokens = torch.randint(-1, 8200, (rows,), device="cuda", generator=g)
    lp, ent, ids, tops = hs.token_logprobs(x, tokens.int(), top=3)
    ref = torch.log_softmax(x.double(), -1)
    want = torch.where(tokens >= 0, ref.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isneginf(lp), torch.isneginf(want))
    assert ((lp.double() - want).abs()[fine] <= R.logprob_tolerance(want)[fine]).all()
    assert ((ent.double() + torch.where(ref > -math.inf, ref.exp() * ref, 0.0).sum(-1)).abs() <= 2.0 ** -16).all()
    order = torch.sort(x.float(), descending=True, stable=True)
    assert torch.equal(ids.long(), order.indices[:, :3])
    assert ((tops.double() - ref.gather(1, order.indices[:, :3])).abs() <= 2.0 ** -16).all()


def _constant(name):
    """An integer constant of the library's sources, or a product of two."""
    src = os.path.join(os.path.dirname(__file__), "..", "paper_2603_12707_amd", "csrc", "hs_internal.h")
    with open(src) as f:
        value = re.search(rf"constexpr int {name} = ([0-9* ]+);", f.read()).group(1)
    return math.prod(int(x) for x in value.split("*"))


@pytest.mark.parametrize("dtype,vocab,rows,one", [("f32", 8200, 511, True), ("f32", 8200, 513, False),
                                                  ("bf16", 16400, 512, True), ("bf16", 16400, 513, False),
                                                  ("f16", 40000, 426, True), ("f16", 40000, 427, False),
                                                  ("f32", 152064, 67, True), ("f32", 152064, 68, False),
                                                  ("bf16", 32003, 700, False)])
def test_rows_of_several_parts_joined_in_the_launch_and_after_it(dtype, vocab, rows, one):
    """Both sides of the limits up to which one launch does, with rows whose parts hold ties, nothing but -inf, a NaN or
    +inf in one part alone, and the largest value in the last elements."""
    import paper_2603_12707_amd as hs
    part = _constant("LOGPROB_PART") * (1 if dtype == "f32" else 2)
    parts = -(-vocab // part)
    assert parts > 1
    assert one == (rows * parts <= _constant("LOGPROB_ONE_LAUNCH") and rows <= _constant("LOGPROB_COUNTERS"))
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, vocab, device="cuda", generator=g) * 2).to(R.DT[dtype])
    tail = part * (parts - 1)
    x[::3, tail:] = 30.0            # the largest, and equal, in the last part
    x[1::7, :tail] = -math.inf      # parts of nothing else
    x[2::11, tail:] = -math.inf
    x[3::13] = x[3::13].round()     # ties across parts
    for r, (at, bad) in enumerate(((3, math.nan), (vocab - 1, math.nan), (part, math.inf), (tail - 1, math.nan))):
        x[5 + 9 * r, at] = bad
    x[50] = -math.inf
    x[51] = -math.inf
    x[51, vocab - 2] = 1.5
    none = torch.isnan(x).any(1) | (x == math.inf).any(1) | (x == -math.inf).all(1)
    assert none.sum() >= 5
    tokens = torch.randint(-1, vocab, (rows,), device="cuda", generator=g)
    tokens[51] = vocab - 2
    ref = torch.log_softmax(x.double(), -1)
    want = torch.where(tokens >= 0, ref.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    want[none & (tokens >= 0)] = math.nan
    ent = -torch.where(ref > -math.inf, ref.exp() * ref, 0.0).sum(-1)
    order = torch.sort(x.float() + 0.0, descending=True, stable=True).indices
    for top in (0, 1, 20):
        lp, e, ids, tops = hs.token_logprobs(x, tokens.int(), top=top)
        assert torch.equal(torch.isnan(lp), torch.isnan(want)) and torch.equal(torch.isinf(lp), torch.isinf(want))
        fine = torch.isfinite(want)
        assert ((lp.double() - want).abs()[fine] <= R.logprob_tolerance(want)[fine]).all()
        assert torch.equal(torch.isnan(e), none)
        assert ((e.double() - ent).abs()[~none] <= 2.0 ** -16).all()
        if not top:
            continue
        assert (ids[none] == -1).all() and torch.isnan(tops[none]).all()
        assert torch.equal(ids.long()[~none], order[~none][:, :top])
        t = ref.gather(1, order[:, :top])[~none]
        got = tops.double()[~none]
        assert torch.equal(torch.isinf(got), torch.isinf(t))
        assert ((got - t).abs()[torch.isfinite(t)] <= R.logprob_tolerance(t)[torch.isfinite(t)]).all()


def test_many_rows():
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(70000, 17, generator=g) * 2).cuda()  # more rows than a grid's second dimension takes
    tokens = torch.randint(-1, 17, (70000,), generator=g)
    lp, ent, ids, tops = hs.token_logprobs(x, tokens.int().cuda(), top=2)
    ref = torch.log_softmax(x.double(), -1).cpu()
    want = torch.where(tokens >= 0, ref.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    assert ((lp.double().cpu() - want).abs() <= R.logprob_tolerance(want)).all()
    assert ((ent.double().cpu() + (ref.exp() * ref).sum(-1)).abs() <= 2.0 ** -16).all()
    order = torch.sort(x.cpu(), descending=True, stable=True)
    assert torch.equal(ids.long().cpu(), order.indices[:, :2])


def test_outputs_are_optional():
    import paper_2603_12707_amd as hs
    x = torch.randn(3, 5000, device="cuda")
    tk = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    lp, ent, ids, tops = hs.token_logprobs(x, tk, top=4)
    a = hs.token_logprobs(x)
    assert a[0] is None and a[2] is None and a[3] is None and torch.equal(a[1], ent)
    b = hs.token_logprobs(x, top=4)
    assert b[0] is None and torch.equal(b[2], ids) and torch.equal(b[3], tops)
    empty = hs.token_logprobs(x[:0], tk[:0], top=4)
    assert empty[0].shape == (0,) and empty[2].shape == (0, 4)
    L = hs.lib()
    need = hs.token_logprobs_workspace(3, 5000, 4)
    lp2 = torch.empty_like(lp)
    P = lambda t: t.data_ptr() or None  # noqa: E731
    st = torch.cuda.current_stream().cuda_stream
    rc = L.hs_token_logprobs(0, P(x), 3, 5000, 5000, P(tk), 4, P(lp2), None, None, None, P(need), need.numel(), st)
    assert rc == hs.HS_OK and torch.equal(lp2, lp)
    rc = L.hs_token_logprobs(0, P(x), 3, 5000, 5000, None, 4, None, None, None, None, P(need), need.numel(), st)
    assert rc == hs.HS_OK


def test_deterministic_and_replayed_in_a_graph():
    import paper_2603_12707_amd as hs
    x = torch.randn(6, 40001, device="cuda")
    tk = torch.arange(6, dtype=torch.int32, device="cuda")
    ws = hs.token_logprobs_workspace(6, 40001, 20)
    ws[2048:].fill_(0xFF)  # only the first 2048 bytes are kept between calls
    first = [t.clone() for t in hs.token_logprobs(x, tk, top=20, workspace=ws)]
    again = hs.token_logprobs(x, tk, top=20, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and not ws[:2048].any()
    # the same workspace serves another shape, and the first one again
    g = torch.Generator().manual_seed(5)
    check(hs, torch.randn(3, 70000, generator=g).half().cuda(), torch.tensor([1, 2, 69999]), 7, workspace=ws)
    again = hs.token_logprobs(x, tk, top=20, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        outs = hs.token_logprobs(x, tk, top=20, workspace=ws)
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        want = [t.clone() for t in hs.token_logprobs(x, tk, top=20)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
