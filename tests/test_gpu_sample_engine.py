"""Decode steps that draw their tokens, on the GPU: against the definition applied to the step's own logits, in every
kind of cache, in replayed graphs, and a run of them together with the log probabilities."""
from __future__ import annotations

import pytest
import torch

import paged_ref as R
from helpers import small_cfg
from workload import synth

pytestmark = pytest.mark.gpu

GQA = dict(n_heads=8, n_kv_heads=2, head_dim=64, rope_kind=1, mrope_section=(8, 12, 12), dtype="bf16", qkv_bias=1)


def numbers(n, g, greedy=False):
    pick = lambda *v: torch.tensor(v)[torch.randint(0, len(v), (n,), generator=g)]  # noqa: E731
    t = 0.5 + torch.rand(n, generator=g)
    if greedy:
        t[0] = 0.0
    return dict(u=torch.rand(n, generator=g).cuda(), temperature=t.cuda(), top_k=pick(0, 5, 100).int().cuda(),
                top_p=pick(1.0, 0.9).cuda(), min_p=pick(0.0, 0.05).cuda())


def drawn(logits, kw, at):
    p = {k: v.cpu()[at] for k, v in kw.items()}
    return R.draw(logits.cpu(), p["u"], p["temperature"], p["top_k"], p["top_p"], p["min_p"])


def same(lp, want):
    return bool(((lp.double().cpu() - want).abs() <= want.abs() * 2.0 ** -24 + 1e-12).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_contiguous_caches(dtype):
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(1)
    cfg = small_cfg(n_layers=1, dtype=dtype, vocab=9001)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 3, 64)
    kvs = [hs.KVCache(model, [0] * 3, [64] * 3) for _ in range(2)]
    for kv in kvs:
        for r in range(3):
            kv.prefill(r, None, synth.text_ids(cfg, r, 5 + r).cuda())
    tin = torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(tin), torch.empty_like(tin)
    logits, plain = torch.empty(3, cfg["vocab"], device="cuda"), torch.empty(3, cfg["vocab"], device="cuda")
    for step in range(6):
        kw = numbers(3, g, greedy=True)
        lp = kvs[0].decode_sample(tin, a, **kw, logits=logits)
        kvs[1].decode(tin, b, plain)
        assert torch.equal(plain, logits) and int(a[0]) == int(b[0])
        want = drawn(logits, kw, slice(None))
        assert torch.equal(a.cpu(), want[0]) and same(lp, want[1])
        again = hs.sample_tokens(logits, **kw)
        assert torch.equal(again[0], a) and torch.equal(again[1], lp)
        tin = a.clone()
    assert kvs[0].lengths() == kvs[1].lengths() == [11, 12, 13]
    # without a place for the logits, and with every default
    u = torch.rand(3, generator=g).cuda()
    kvs[0].decode_sample(tin, a, u)
    kvs[1].decode(tin, b, plain)
    assert torch.equal(a, hs.sample_tokens(plain, u)[0])


@pytest.mark.parametrize("kind", ["KVPool", "QuantKVPool"])
def test_pools_index_by_slot(kind):
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(2)
    cfg = small_cfg(**GQA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 4, 300)
    pool = getattr(hs, kind)(model, 6, 256, 6)
    slots = [1, 3, 4]
    for s in slots:
        pool.admit(s, 0, 60)
        pool.prefill(s, None, synth.text_ids(cfg, s, 9).cuda(), synth.mrope_positions(0, 9).cuda())
    tin = torch.zeros(6, dtype=torch.int32, device="cuda")
    logits = torch.empty(3, cfg["vocab"], device="cuda")
    for step in range(4):
        kw = numbers(6, g)
        tout = torch.full((6,), -9, dtype=torch.int32, device="cuda")
        lp = pool.decode_sample(tin, tout, **kw, logits=logits)
        want = drawn(logits, kw, slots)
        assert torch.equal(tout[slots].cpu(), want[0]) and same(lp[:3], want[1])
        assert tout[[0, 2, 5]].tolist() == [-9] * 3 and bool(torch.isnan(lp[3:]).all())
        tin[slots] = tout[slots]


def test_replayed_steps_read_new_numbers():
    import paper_2603_12707_amd as hs
    g = torch.Generator().manual_seed(3)
    cfg = small_cfg(n_layers=1, vocab=20000)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 2, 64)
    kvs = [hs.KVCache(model, [0] * 2, [64] * 2) for _ in range(2)]
    for kv in kvs:
        for r in range(2):
            kv.prefill(r, None, synth.text_ids(cfg, r, 5).cuda())
    tin = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    tout, held = torch.empty_like(tin), numbers(2, g)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        lp = kvs[0].decode_sample(tin, tout, **held)
    kvs[0].sync()
    for step in range(6):
        for k, v in numbers(2, g).items():
            held[k].copy_(v)
        graph.replay()
        other = torch.empty_like(tin)
        want = kvs[1].decode_sample(tin, other, **held)
        torch.cuda.synchronize()
        assert torch.equal(tout, other) and torch.equal(lp, want)
        tin.copy_(other)
    kvs[0].sync()
    assert kvs[0].lengths() == kvs[1].lengths() == [11, 11]


def test_refusals():
    import paper_2603_12707_amd as hs
    headless = small_cfg(n_layers=1, lm_head=False)
    model = hs.Model(headless, synth.make_weights(headless, device="cuda"), 1, 64)
    kv = hs.KVCache(model, [0], [64])
    kv.set_length(0, 3, 3)
    t, u = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    with pytest.raises(hs.HsError) as e:
        kv.decode_sample(t, t.clone(), u)
    assert e.value.code == hs.HS_E_STATE
    cfg = small_cfg(n_layers=1)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 1, 64)
    kv = hs.KVCache(model, [0], [8])
    with pytest.raises(hs.HsError) as e:  # nothing prefilled
        kv.decode_sample(t, t.clone(), u)
    assert e.value.code == hs.HS_E_STATE
    kv.prefill(0, None, synth.text_ids(cfg, 0, 7).cuda())
    for kw in (dict(u=None), dict(u=u.double()), dict(u=u.cpu()), dict(u=u, top_k=u), dict(u=u, min_p=torch.zeros(2)),
               dict(u=u, temperature=t)):
        with pytest.raises(ValueError):
            kv.decode_sample(t, t.clone(), **kw)
    with pytest.raises(hs.HsError) as e:  # the tokens would be written over
        kv.decode_sample(t, t, u)
    assert e.value.code == hs.HS_E_INVALID
    kv.decode_sample(t, t.clone(), u)
    with pytest.raises(hs.HsError) as e:
        kv.decode_sample(t, t.clone(), u)
    assert e.value.code == hs.HS_E_CAPACITY
