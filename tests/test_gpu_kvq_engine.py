"""Prefill and decode over a pool held in 4 bits (hs_kvq_pool_create), and decode steps with log probabilities.

The reference is a plain decoder in 64 bits with the engine's rounding points.  Rounding to 4 bits is a step function,
so that a last-place difference of a key may become a whole step; the reference therefore attends over the values that
the cache holds (read back), and the stored rows are checked against its own rows apart."""
from __future__ import annotations

import pytest
import torch

import kvq_ref as R
from helpers import KV_ROWS_DEEP_TOL, LOGIT_TOL, rel_err, small_cfg
from workload import synth

pytestmark = pytest.mark.gpu


class Plain:
    def __init__(self, cfg, w):
        self.cfg, self.w = cfg, {k: v.double() for k, v in w.items()}
        self.dt = R.DT[cfg["dtype"]]

    def r(self, x):
        return x.to(self.dt).double()

    def norm(self, x, g):
        return self.r(x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.cfg["rms_eps"]) * self.w[g])

    def rope(self, x, pos3):
        """x [T, heads, hd], pos3 [3, T]."""
        c, half = self.cfg, self.cfg["head_dim"] // 2
        i = torch.arange(half)
        s = c["mrope_section"]
        sec = (i >= s[0]).long() + (i >= s[0] + s[1]).long() if c["rope_kind"] else torch.zeros(half, dtype=torch.long)
        ang = pos3[sec].double().T * c["rope_theta"] ** (-2.0 * i.double() / c["head_dim"])
        co, si = ang.cos()[:, None], ang.sin()[:, None]
        a, b = x[..., :half], x[..., half:]
        return torch.cat((a * co - b * si, b * co + a * si), -1)

    def rows(self, x, pos3, first, stored):
        """Rows x [T, d] at positions first.. of a request whose cache holds stored(layer) -> (K, V) [n_kv, len, hd];
        returns the logits of every row, and each layer's own (K, V) rows before they were stored."""
        c, w = self.cfg, self.w
        nh, nk, hd, T = c["n_heads"], c["n_kv_heads"], c["head_dim"], x.shape[0]
        x, own = x.double(), []
        for l in range(c["n_layers"]):
            p = f"layers.{l}."
            h = self.norm(x, p + "attn_norm")
            q, k, v = (h @ w[p + n].T + (w[p + b] if c["qkv_bias"] else 0.0)
                       for n, b in (("wq", "bq"), ("wk", "bk"), ("wv", "bv")))
            q = self.r(self.rope(q.reshape(T, nh, hd), pos3))
            own.append((self.r(self.rope(k.reshape(T, nk, hd), pos3)), self.r(v.reshape(T, nk, hd))))
            K, V = stored(l)
            n = first + T
            s = torch.einsum("tjgd,jpd->jgtp", q.reshape(T, nk, nh // nk, hd), K[:, :n]) * hd ** -0.5
            s = s.masked_fill(torch.arange(n)[None] > first + torch.arange(T)[:, None], -torch.inf)
            o = torch.einsum("jgtp,jpd->tjgd", torch.softmax(s, -1), V[:, :n]).reshape(T, nh * hd)
            x = x + self.r(o) @ w[p + "wo"].T
            h = self.norm(x, p + "mlp_norm")
            g, u = h @ w[p + "w_gate"].T, h @ w[p + "w_up"].T
            x = x + self.r(g / (1 + torch.exp(-g)) * u) @ w[p + "w_down"].T
        return self.norm(x, "final_norm") @ w["lm_head"].T, own


class Run:
    """A 4-bit pool on the GPU and the plain decoder over what it holds."""

    def __init__(self, cfg, slots, n_blocks, bt=256, max_ctx=600, max_batch=None):
        import paper_2603_12707_amd as hs
        self.hs, self.cfg = hs, cfg
        w = synth.make_weights(cfg)
        self.plain = Plain(cfg, w)
        self.embed = w["embed"]
        self.model = hs.Model(cfg, {k: v.cuda() for k, v in w.items()}, max_batch or slots, max_ctx)
        self.pool = hs.QuantKVPool(self.model, slots, bt, n_blocks)
        self.slots, self.len, self.pos = slots, {}, {}

    def stored(self, slot, n):
        c = self.cfg

        def get(layer):
            out = torch.empty(2, c["n_kv_heads"], n, c["head_dim"], dtype=R.DT[c["dtype"]])
            for sel in range(2):
                for j in range(c["n_kv_heads"]):
                    self.pool.read(slot, layer, sel, j, 0, n, out[sel, j])
            return out[0].double(), out[1].double()

        return get

    def check_rows(self, slot, first, own, where):
        """The stored rows are this side's rows rounded to 4 bits: half a step off at most, a whole one where a border
        lies between the two sides' numbers, and twice that where the group's power differs."""
        n = first + own[0][0].shape[0]
        get = self.stored(slot, n)
        for l, pair in enumerate(own):
            for got, x in zip(get(l), pair):
                got = got[:, first:].transpose(0, 1)
                a = x.reshape(*x.shape[:2], -1, 32).abs().amax(-1)
                e = torch.frexp(a).exponent - 2
                room = 2.0 * 2.0 ** e.double() + KV_ROWS_DEEP_TOL * float(x.abs().max())
                off = (got - x).abs().reshape(*x.shape[:2], -1, 32).amax(-1)
                assert (off <= room).all(), (where, l)
                # and mostly the nearest value exactly
                val = R.quantize(x.to(R.DT[self.cfg["dtype"]]), self.cfg["dtype"])[2]
                assert float((got == val).double().mean()) > 0.9, (where, l)

    def prefill(self, entries, key=0):
        """entries: [(slot, n_v, s_text, capacity)]"""
        c, embs, idss, poss = self.cfg, [], [], []
        for slot, n_v, s_text, cap in entries:
            self.pool.admit(slot, n_v, cap)
            embs.append(synth.vision_rows(c, key + slot, n_v))
            idss.append(synth.text_ids(c, key + slot, s_text))
            poss.append(synth.mrope_positions(n_v, s_text) if c["rope_kind"]
                        else torch.arange(n_v + s_text, dtype=torch.int32).repeat(3, 1))
        logits = torch.empty(len(entries), c["vocab"], device="cuda")
        emb = torch.cat(embs)
        self.pool.prefill_batch([e[0] for e in entries], emb.cuda() if emb.numel() else None, torch.cat(idss).cuda(),
                                [e[2] for e in entries], torch.cat(poss, 1).cuda() if c["rope_kind"] else None,
                                last_logits=logits)
        for i, (slot, n_v, s_text, _) in enumerate(entries):
            n = n_v + s_text
            x = torch.cat((embs[i].double(), self.embed[idss[i].long()].double()))
            want, own = self.plain.rows(x, poss[i], 0, self.stored(slot, n))
            assert rel_err(logits[i].cpu(), want[-1]) <= LOGIT_TOL, (slot, rel_err(logits[i].cpu(), want[-1]))
            self.check_rows(slot, 0, own, ("prefill", slot))
            self.len[slot], self.pos[slot] = n, int(poss[i].max()) + 1

    def release(self, slot):
        self.pool.release(slot)
        del self.len[slot], self.pos[slot]

    def decode(self, steps, key=0, check=True):
        c, live = self.cfg, sorted(self.len)
        logits = torch.empty(len(live), c["vocab"], device="cuda")
        tout = torch.full((self.slots,), -7, dtype=torch.int32, device="cuda")
        g = torch.Generator().manual_seed(key)
        for step in range(steps):
            tin = torch.randint(0, c["vocab"], (self.slots,), generator=g, dtype=torch.int32)
            self.pool.decode(tin.cuda(), tout, logits)
            for k, slot in enumerate(live):
                if check:
                    want, own = self.plain.rows(self.embed[int(tin[slot])][None].double(),
                                                torch.full((3, 1), self.pos[slot]), self.len[slot],
                                                self.stored(slot, self.len[slot] + 1))
                    err = rel_err(logits[k].cpu(), want[0])
                    assert err <= LOGIT_TOL, (step, slot, err)
                    self.check_rows(slot, self.len[slot], own, (step, slot))
                assert int(tout[slot]) == int(logits[k].argmax())
                self.len[slot] += 1
                self.pos[slot] += 1
            assert all(int(tout[s]) == -7 for s in range(self.slots) if s not in self.len)

    def close(self):
        assert self.model.status() == 0
        self.pool.close()
        self.model.close()


GQA = dict(n_layers=2, d_model=512, n_heads=14, n_kv_heads=2, head_dim=64, ffn_dim=1000, dtype="bf16", qkv_bias=1,
           rope_kind=1, mrope_section=(8, 12, 12), rope_theta=1e6)
MHA = dict(n_layers=2, d_model=512, n_heads=4, n_kv_heads=4, head_dim=128, ffn_dim=1000, dtype="f16")


@pytest.mark.parametrize("kind", [GQA, MHA, dict(GQA, n_heads=8, n_kv_heads=1, head_dim=128, mrope_section=(16, 24, 24),
                                                 dtype="f16"), dict(MHA, n_heads=8, n_kv_heads=4, head_dim=64, dtype="bf16")],
                         ids=["gqa7", "mha", "gqa8", "gqa2"])
def test_prefill_and_decode_across_blocks(kind):
    """Three requests whose steps cross block borders; a slot released and filled anew in between."""
    run = Run(small_cfg(**kind), slots=5, n_blocks=14)
    run.prefill([(3, 200, 99, 340), (0, 40, 214, 300), (2, 0, 256, 300)])
    assert run.pool.lengths() == [254, 0, 256, 299, 0]
    assert run.pool.blocks() == (14 - 1 - 1 - 2, 14)
    run.decode(4)
    run.release(2)
    run.prefill([(2, 17, 1, 300), (4, 1, 0, 20)] if kind["n_heads"] == 14 else [(2, 17, 240, 300)], key=50)
    run.decode(3, key=1)
    run.close()


def test_single_prefills_of_one_row_and_a_long_prompt():
    run = Run(small_cfg(**GQA), slots=2, n_blocks=6)
    run.prefill([(1, 0, 1, 40)])
    run.prefill([(0, 500, 77, 600)])
    run.decode(2)
    run.close()


def test_batches_of_more_than_32_columns():
    """40 requests: activations in the packed layout, one split per request, the many-column GEMMs in prefill."""
    run = Run(small_cfg(**dict(GQA, d_model=1024, n_heads=8, n_kv_heads=2, head_dim=128, mrope_section=(16, 24, 24),
                               n_layers=1)), slots=42, n_blocks=44, max_ctx=300)
    run.prefill([(s, s % 5, 3 + (7 * s) % 23, 60) for s in range(1, 41)])
    run.decode(2)
    run.close()


def test_passes_are_bounded_by_what_the_handle_stages():
    """The model's row workspaces grow after the handle is made: its passes stay within its own room."""
    run = Run(small_cfg(**MHA), slots=4, n_blocks=8, max_ctx=300)
    run.model.reserve_rows(2000)
    run.prefill([(s, 100, 50 + s, 200) for s in range(4)])
    run.decode(1)
    run.close()


def _filled(cfg, slots=3, max_ctx=600):
    """Two identical 4-bit pools of one model, filled by hand."""
    import paper_2603_12707_amd as hs
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), slots, max_ctx)
    # the same bytes where nothing is stored, so that whole buffers can be compared
    need = (2 * slots + 2) * hs.kvq_block_bytes(cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"], 256)
    pools = [hs.QuantKVPool(model, slots, 256, 2 * slots + 2, torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"))
             for _ in range(2)]
    lens = [255, 130, 400][:slots]
    for p in pools:
        for r, n in enumerate(lens):
            p.admit(r, 0, 590)
            p.set_length(r, n, n)
            for l in range(cfg["n_layers"]):
                for sel in range(2):
                    for j in range(cfg["n_kv_heads"]):
                        p.write(r, l, sel, j, 0, synth.kv_block(cfg, r, l, sel, j, n, device="cuda"))
    return model, pools


@pytest.mark.parametrize("length", [2600, 6000])
def test_long_requests_in_several_splits(length):
    """Splits joined in the output projection (up to eight) and by the combine kernel."""
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**GQA)
    run = Run(cfg, slots=2, n_blocks=-(-(length + 40) // 256) + 2, max_ctx=length + 40)
    for slot, n in ((0, length), (1, 300)):
        run.pool.admit(slot, 0, n + 20)
        run.pool.set_length(slot, n, n)
        for l in range(cfg["n_layers"]):
            for sel in range(2):
                for j in range(cfg["n_kv_heads"]):
                    run.pool.write(slot, l, sel, j, 0, synth.kv_block(cfg, slot, l, sel, j, n, device="cuda"))
        run.len[slot], run.pos[slot] = n, n
    run.decode(2)
    run.close()


def test_static_step_equals_the_step():
    cfg = small_cfg(**GQA)
    model, (a, b) = _filled(cfg)
    tok = synth.uniform_int(1, "t", 3, 0, cfg["vocab"] - 1, device="cuda")
    for _ in range(3):
        outs = []
        for p, step in ((a, "decode"), (b, "decode_static")):
            o, lg = torch.empty_like(tok), torch.empty(3, cfg["vocab"], device="cuda")
            hidden = torch.empty(3, cfg["d_model"], device="cuda")
            getattr(p, step)(tok, o, lg, hidden)
            outs.append((o, lg, hidden))
        assert all(torch.equal(x, y) for x, y in zip(*outs))
        tok = outs[0][0]
    assert torch.equal(a.buf, b.buf)
    assert model.status() == 0


def test_replayed_steps_take_blocks_and_equal_eager_ones():
    cfg = small_cfg(**GQA)
    model, (a, b) = _filled(cfg)
    tin, tout = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    target = torch.zeros(3, dtype=torch.int32, device="cuda")
    logits = torch.empty(3, cfg["vocab"], device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        lp = a.decode_logprobs(tin, tout, target, top=5, logits=logits)
    a.sync()  # the capture advanced the host's mirrors only
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(5):
        tin.copy_(torch.randint(0, cfg["vocab"], (3,), device="cuda", generator=g))
        target.copy_(torch.randint(0, cfg["vocab"], (3,), device="cuda", generator=g))
        o, lg = torch.empty_like(tout), torch.empty_like(logits)
        want = b.decode_logprobs(tin, o, target, top=5, logits=lg)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tout, o) and torch.equal(logits, lg), i
        assert all(torch.equal(x, y) for x, y in zip(lp, want)), i
    a.sync()
    assert a.lengths() == b.lengths() and a.blocks() == b.blocks()
    assert torch.equal(a.buf, b.buf)
    assert model.status() == 0


def test_a_replayed_step_serves_a_longer_request_than_at_its_capture():
    """A slot released and filled with a request of a larger capacity than any at the capture: the replayed step attends
    over all of its positions, in one split and in several."""
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**GQA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 1, 5200)
    for first, later in ((300, 1500), (2600, 5100)):
        pools = [hs.QuantKVPool(model, 1, 256, 21) for _ in range(2)]

        def fill(p, n, cap):
            p.admit(0, 0, cap)
            p.set_length(0, n, n)
            for l in range(cfg["n_layers"]):
                for sel in range(2):
                    for j in range(cfg["n_kv_heads"]):
                        p.write(0, l, sel, j, 0, synth.kv_block(cfg, 0, l, sel, j, n, device="cuda"))

        fill(pools[0], first - 10, first)
        tin, tout = torch.tensor([5], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        logits, want = (torch.empty(1, cfg["vocab"], device="cuda") for _ in range(2))
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            pools[0].decode(tin, tout, logits)
        pools[0].sync()
        pools[0].release(0)
        for p in pools:
            fill(p, later - 40, later)
        for i in range(3):
            pools[1].decode(tin, torch.empty_like(tout), want)
            graph.replay()
            torch.cuda.synchronize()
            assert rel_err(logits[0].cpu(), want[0].cpu()) <= 2.0 ** -6, (first, i)
        pools[0].sync()
        assert pools[0].lengths() == pools[1].lengths() == [later - 37]
    assert model.status() == 0


def test_a_pool_that_runs_dry_inside_replays():
    """Request 0 enters a block that is not there: the step says so, keeps its new rows unstored and masks their places,
    in one split and where they are all that a split holds; request 1 goes on as in a pool with room."""
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**GQA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 2, 2700)
    for first, cap in ((250, 400), (2558, 2700)):
        blocks = -(-first // 256) + 1
        pools = [hs.QuantKVPool(model, 2, 256, blocks + room) for room in (0, 1)]
        for p in pools:
            for r, n in ((0, first), (1, 100)):
                p.admit(r, 0, cap)
                p.set_length(r, n, n)
                for l in range(cfg["n_layers"]):
                    for sel in range(2):
                        for j in range(cfg["n_kv_heads"]):
                            p.write(r, l, sel, j, 0, synth.kv_block(cfg, r, l, sel, j, n, device="cuda"))
        assert pools[0].blocks() == (0, blocks)
        tin, tout = torch.tensor([3, 4], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        logits, want = (torch.empty(2, cfg["vocab"], device="cuda") for _ in range(2))
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            pools[0].decode(tin, tout, logits)
        pools[0].sync()
        steps = 256 - first % 256
        for i in range(steps + 3):
            pools[1].decode(tin, torch.empty_like(tout), want)
            graph.replay()
            torch.cuda.synchronize()
            assert model.status() == (4 if i >= steps else 0), i
            assert torch.isfinite(logits).all()
            assert torch.equal(logits[1], want[1]), i
            assert (i >= steps) or torch.equal(logits[0], want[0]), i
        pools[0].sync()
        assert pools[0].lengths() == [first + steps + 3, 100 + steps + 3]
        with pytest.raises(hs.HsError):
            pools[0].decode(tin, tout)


def test_write_and_read_round_and_give_stored_values():
    cfg = small_cfg(**MHA)
    import paper_2603_12707_amd as hs
    model, (p, _) = _filled(cfg)
    rows = synth.kv_block(cfg, 7, 0, 0, 0, 300)
    want = R.quantize(rows, "f16")[2]
    p.write(2, 1, 1, 3, 50, rows.cuda())  # across a block border
    for out in (torch.empty(300, 128, dtype=torch.float16), torch.empty(300, 128, dtype=torch.float16, device="cuda")):
        p.read(2, 1, 1, 3, 50, 300, out)
        assert torch.equal(out.double().cpu(), want)
    p.write(2, 1, 0, 0, 7, rows[:9])      # from the host
    loose = torch.empty(9 * 128 + 1, dtype=torch.float16, device="cuda")[1:].reshape(9, 128)  # not 16-byte aligned
    p.read(2, 1, 0, 0, 7, 9, loose)
    assert torch.equal(loose.double().cpu(), want[:9])
    loose.copy_(rows[9:18])
    p.write(2, 1, 0, 0, 7, loose)
    out = torch.empty(9, 128, dtype=torch.float16)
    p.read(2, 1, 0, 0, 7, 9, out)
    assert torch.equal(out.double(), want[9:18])
    for bad in ((3, 0, 0, 0, 0), (0, 2, 0, 0, 0), (0, 0, 2, 0, 0), (0, 0, 0, 4, 0), (0, 0, 0, 0, 590)):
        with pytest.raises(hs.HsError) as e:
            p.read(*bad, 1, out)
        assert e.value.code == hs.HS_E_INVALID
    with pytest.raises(hs.HsError):  # no block there yet
        p.write(1, 0, 0, 0, 300, rows[:9])


def test_refusals_of_the_pool_and_of_steps():
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**MHA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 2, 300)
    bb = hs.kvq_block_bytes(cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"], 256)

    def refused(code, fn, *a, **kw):
        with pytest.raises(hs.HsError) as e:
            fn(*a, **kw)
        assert e.value.code == code

    refused(hs.HS_E_INVALID, hs.QuantKVPool, model, 0, 256, 4)
    refused(hs.HS_E_INVALID, hs.QuantKVPool, model, 2, 128, 4)
    refused(hs.HS_E_INVALID, hs.QuantKVPool, model, 2, 384, 4)
    refused(hs.HS_E_BUFFER, hs.QuantKVPool, model, 2, 256, 1, torch.empty(bb - 1, dtype=torch.uint8, device="cuda"))
    refused(hs.HS_E_INVALID, hs.QuantKVPool, model, 2, 256, 1, torch.empty(bb + 8, dtype=torch.uint8, device="cuda")[8:])
    f32 = small_cfg(**dict(MHA, dtype="f32"))
    wide = hs.Model(f32, synth.make_weights(f32, device="cuda"), 2, 300)
    refused(hs.HS_E_INVALID, hs.QuantKVPool, wide, 2, 256, 4)
    # exactly the bytes of two blocks
    pool = hs.QuantKVPool(model, 2, 256, 2, torch.empty(2 * bb + 100, dtype=torch.uint8, device="cuda"))
    assert pool.blocks() == (2, 2)
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    refused(hs.HS_E_STATE, pool.decode, t, t.clone())
    refused(hs.HS_E_STATE, pool.decode_logprobs, t, t.clone())
    pool.admit(0, 0, 300)
    ids = torch.zeros(299, dtype=torch.int32, device="cuda")
    pool.prefill(0, None, ids)
    refused(hs.HS_E_INVALID, pool.decode_logprobs, t, t.clone(), top=65)
    refused(hs.HS_E_INVALID, pool.decode_logprobs, t, t.clone(), top=-1)
    refused(hs.HS_E_INVALID, pool.decode_logprobs, t, t)
    pool.admit(1, 0, 10)
    refused(hs.HS_E_CAPACITY, pool.prefill, 1, None, ids[:5])  # no block left
    pool.decode_logprobs(t, t.clone())
    refused(hs.HS_E_CAPACITY, pool.decode_logprobs, t, t.clone())
    assert pool.lengths() == [300, 0]


@pytest.mark.parametrize("quant", [True, False], ids=["quant", "plain"])
def test_scoring_a_text_with_log_probabilities(quant):
    """Texts of several lengths scored token by token over either cache: a request's prompt is prefilled, then its
    given tokens are fed one a step and each next one's log probability asked for; -1 where a text has ended."""
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**GQA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 3, 400)
    pool = (hs.QuantKVPool if quant else hs.KVPool)(model, 4, 256, 8)
    prompts, texts = [5, 250, 33], [9, 12, 4]
    slots = [3, 0, 1]
    for s, n in zip(slots, prompts):
        pool.admit(s, 0, 300)
    ids = [synth.text_ids(cfg, s, n) for s, n in zip(slots, prompts)]
    pos = torch.cat([synth.mrope_positions(0, n) for n in prompts], 1).cuda()
    pool.prefill_batch(slots, None, torch.cat(ids).cuda(), prompts, pos)
    given = {s: synth.decode_tokens(cfg, s, n) for s, n in zip(slots, texts)}
    total = torch.zeros(3, dtype=torch.float64)
    want = torch.zeros(3, dtype=torch.float64)
    tout = torch.empty(4, dtype=torch.int32, device="cuda")
    logits = torch.empty(3, cfg["vocab"], device="cuda")
    for step in range(max(texts) - 1):
        at = lambda k: torch.tensor([int(given[s][k]) if s in given and k < len(given[s]) else -1  # noqa: E731
                                     for s in range(4)], dtype=torch.int32)
        tin, target = at(step).clamp(min=0), at(step + 1)
        lp, ent, top_ids, tops = pool.decode_logprobs(tin.cuda(), tout, target.cuda(), top=7, logits=logits)
        rows = target[sorted(slots)]
        ref = R.logprobs(logits.cpu(), rows, 7)
        for got, r in zip((lp, ent, tops), (ref[0], ref[1], ref[3])):
            assert ((got.double().cpu() - r).abs() <= R.logprob_tolerance(r)).all(), step
        assert torch.equal(top_ids.long().cpu(), ref[2])
        assert torch.equal(top_ids[:, 0], tout[sorted(slots)])
        # the same from the logits apart, and of the chosen tokens
        again = hs.token_logprobs(logits, rows.cuda(), top=7)
        assert all(torch.equal(x, y) for x, y in zip(again, (lp, ent, top_ids, tops)))
        total += lp.double().cpu()
        want += ref[0]
    assert ((total - want).abs() <= 16 * 2.0 ** -15).all()
    lp, ent, ids, tops = pool.decode_logprobs(tin.cuda(), tout, top=1)
    assert torch.equal(lp, tops[:, 0]) and torch.equal(ids[:, 0], tout[sorted(slots)])
    assert model.status() == 0


def test_log_probabilities_of_a_partly_filled_pool():
    """Rows past the decoded requests say so: NaN, and -1 for tokens."""
    import paper_2603_12707_amd as hs
    cfg = small_cfg(**GQA)
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 4, 300)
    pool = hs.KVPool(model, 5, 256, 5)
    for s in (1, 3):
        pool.admit(s, 0, 60)
        pool.prefill(s, None, synth.text_ids(cfg, s, 9).cuda(), synth.mrope_positions(0, 9).cuda())
    tin, tout = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    junk = [torch.full((64,), 7.0, device="cuda") for _ in range(8)]  # what new memory may hold
    del junk
    for top in (0, 1, 3):
        lp, ent, ids, tops = pool.decode_logprobs(tin, tout, top=top)
        assert lp.shape == ent.shape == (4,) and torch.isfinite(lp[:2]).all() and torch.isfinite(ent[:2]).all()
        assert torch.isnan(lp[2:]).all() and torch.isnan(ent[2:]).all()
        if top:
            assert ids.shape == tops.shape == (4, top) and (ids[:2] >= 0).all() and (ids[2:] == -1).all()
            assert torch.isfinite(tops[:2]).all() and torch.isnan(tops[2:]).all()
    assert model.status() == 0


def test_contiguous_caches_have_log_probabilities_too():
    import paper_2603_12707_amd as hs
    cfg = small_cfg(n_layers=1, dtype="f32")
    model = hs.Model(cfg, synth.make_weights(cfg, device="cuda"), 2, 64)
    kvs = [hs.KVCache(model, [0, 0], [64, 64]) for _ in range(2)]
    for kv in kvs:
        for r in range(2):
            kv.prefill(r, None, synth.text_ids(cfg, r, 5 + r).cuda())
    tin = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(tin), torch.empty_like(tin)
    logits = torch.empty(2, cfg["vocab"], device="cuda")
    lp, ent, ids, tops = kvs[0].decode_logprobs(tin, a, top=3, logits=logits)
    plain = torch.empty_like(logits)
    kvs[1].decode(tin, b, plain)
    assert torch.equal(a, b) and torch.equal(plain, logits)
    assert torch.equal(ids[:, 0], a) and torch.equal(lp, tops[:, 0])
    headless = small_cfg(n_layers=1, dtype="f16", lm_head=False)
    m2 = hs.Model(headless, synth.make_weights(headless, device="cuda"), 1, 64)
    kv = hs.KVCache(m2, [0], [64])
    kv.set_length(0, 3, 3)
    with pytest.raises(hs.HsError) as e:
        kv.decode_logprobs(tin[:1], a[:1])
    assert e.value.code == hs.HS_E_STATE
