"""Host-side checks of the paged cache's and the token draw's entry points (no GPU needed): sizes and refusals.  Every
refused call returns before anything is launched."""
import ctypes

import pytest

import paper_2603_12707_amd as hs
from paper_2603_12707_amd import hs as H

BUF = (ctypes.c_char * 65536)()
AT = (ctypes.addressof(BUF) + 63) // 64 * 64  # an aligned address that is never dereferenced


def cache(**kw):
    c = dict(blocks=AT, bytes=1 << 20, table=AT, n_seqs=2, table_ld=3, n_layers=2, n_kv_heads=2, head_dim=64,
             block_tokens=32, dtype=H.HS_BF16)
    c.update(kw)
    return H.hs_paged_cache(**c)


def append(c, layer=0, n=4, heads=4, q=AT, ld_q=256, ldh_q=64, q_out=AT, ld_qo=256, ldh_qo=64, k=AT, v=AT, ld=128,
           ld_head=64, seqs=None, pos=AT, rope=None, at=None, q_gain=None, k_gain=None, eps=1e-6):
    r = None if rope is None else ctypes.byref(H.hs_rope(**dict(dict(frequencies=AT, axes=None, n_pairs=32, n_axes=1,
                                                                    adjacent=0), **rope)))
    return hs.lib().hs_paged_append(ctypes.byref(c), layer, n, heads, q, ld_q, ldh_q, q_out, ld_qo, ldh_qo, k, v, ld,
                                    ld_head, seqs, pos, r, at, q_gain, k_gain, eps, None)


def attend(c, layer=0, n=2, heads=4, q=AT, ld_q=256, lens=AT, groups=0, starts=None, shared=None, max_len=96,
           max_shared=0, out=AT, ld_out=256, ws=AT, ws_bytes=1 << 30):
    return hs.lib().hs_paged_attention(ctypes.byref(c), layer, n, heads, q, ld_q, None, lens, groups, starts, shared,
                                       max_len, max_shared, 0.125, out, ld_out, ws, ws_bytes, None)


def sample(dtype=H.HS_F32, logits=AT, rows=2, vocab=100, ld=100, u=AT, tokens=AT, lp=AT, ws=AT, ws_bytes=1 << 40):
    return hs.lib().hs_sample_tokens(dtype, logits, rows, vocab, ld, u, None, None, None, None, tokens, lp, ws, ws_bytes,
                                     None)


def test_block_bytes():
    import torch
    for dtype, b in ((torch.float32, 4), (torch.float16, 2), (torch.bfloat16, 2)):
        for layers, kv, hd, bt in ((1, 1, 64, 16), (28, 4, 128, 256), (32, 32, 128, 16384)):
            assert hs.paged_block_bytes(dtype, layers, kv, hd, bt) == 2 * layers * kv * bt * hd * b


@pytest.mark.parametrize("bad", [(0, 1, 64, 16), (1, 0, 64, 16), (1, 1, 96, 16), (1, 1, 32, 16), (1, 1, 64, 8),
                                 (1, 1, 64, 48), (1, 1, 64, 32768), (1, 4097, 64, 16), (-1, 1, 64, 16),
                                 (2 ** 31 - 1, 2 ** 31 - 1, 128, 16384)])
def test_block_bytes_refuses(bad):
    import torch
    with pytest.raises(hs.HsError) as e:
        hs.paged_block_bytes(torch.bfloat16, *bad)
    assert e.value.code == H.HS_E_INVALID


CACHE_FAULTS = [dict(blocks=None), dict(table=None), dict(blocks=AT + 8), dict(table=AT + 4), dict(n_seqs=0),
                dict(table_ld=0), dict(n_layers=0), dict(n_kv_heads=0), dict(head_dim=80), dict(block_tokens=24),
                dict(dtype=3), dict(dtype=-1)]


@pytest.mark.parametrize("fault", CACHE_FAULTS, ids=lambda f: "-".join(f))
@pytest.mark.parametrize("call", [append, attend], ids=["append", "attend"])
def test_a_faulty_cache_is_refused(call, fault):
    assert call(cache(**fault)) == H.HS_E_INVALID


@pytest.mark.parametrize("call", [append, attend], ids=["append", "attend"])
def test_cache_arguments_every_call_checks(call):
    assert call(cache(bytes=100)) == H.HS_E_BUFFER  # less than one block
    assert call(cache(), layer=2) == H.HS_E_INVALID
    assert call(cache(), layer=-1) == H.HS_E_INVALID
    assert call(cache(), n=-1) == H.HS_E_INVALID
    assert call(cache(), n=0) == H.HS_OK


def test_rows_refused():
    for fault in (dict(k=None), dict(v=None), dict(pos=None), dict(k=AT + 8), dict(v=AT + 4), dict(ld=132),
                  dict(ld_head=68), dict(ld=-128), dict(ld_head=-64), dict(ld=64), dict(ld=0), dict(ld_head=32),
                  dict(ld=96, ld_head=64), dict(ld=1 << 50), dict(n=2 ** 31 - 1), dict(n=1 << 26, ld=1 << 40),
                  dict(q=None), dict(q_out=None), dict(q=AT + 8), dict(q_out=AT + 8), dict(ld_q=192), dict(ld_qo=192),
                  dict(ldh_q=32), dict(ldh_qo=32), dict(ld_q=260), dict(ld_q=512), dict(heads=-1), dict(heads=1 << 20),
                  dict(q_gain=AT + 8), dict(k_gain=AT + 2), dict(eps=-1.0), dict(eps=float("nan")),
                  dict(eps=float("inf"))):
        assert append(cache(), **fault) == H.HS_E_INVALID, fault
    # fp32 rows are aligned to 4 elements
    assert append(cache(dtype=H.HS_F32), ld=130) == H.HS_E_INVALID


def test_ropes_refused():
    for fault in (dict(n_pairs=4), dict(n_pairs=40), dict(n_pairs=-8), dict(n_axes=0), dict(n_axes=9),
                  dict(frequencies=None), dict(frequencies=AT + 4)):
        assert append(cache(), rope=fault) == H.HS_E_INVALID, fault
    assert append(cache(), rope=dict(n_axes=3, axes=AT)) == H.HS_E_INVALID  # three axes and no angles_at


def test_attention_refused():
    for fault in (dict(q=None), dict(out=None), dict(lens=None), dict(q=AT + 8), dict(out=AT + 2), dict(ws=AT + 4),
                  dict(heads=0), dict(heads=3), dict(heads=34), dict(heads=-2), dict(max_len=0), dict(max_len=-5),
                  dict(max_len=2 ** 30 + 1), dict(ld_q=255), dict(ld_q=128), dict(ld_out=128), dict(n=2 ** 30),
                  dict(groups=-1), dict(groups=3), dict(groups=1), dict(groups=1, starts=AT),
                  dict(groups=1, shared=AT), dict(max_shared=-1), dict(max_shared=97)):
        assert attend(cache(), **fault) == H.HS_E_INVALID, fault
    assert attend(cache(), n=1 << 20, ld_q=1 << 40) == H.HS_E_INVALID
    assert attend(cache(), n=1 << 20, heads=4) == H.HS_E_INVALID


def test_attention_workspace_too_small():
    c = cache(table_ld=1000)
    need = ctypes.c_uint64()
    assert hs.lib().hs_paged_attention_workspace(ctypes.byref(c), 2, 4, 32000, 1, 16000, ctypes.byref(need)) == H.HS_OK
    assert need.value > 0
    more = dict(groups=1, starts=AT, shared=AT, max_len=32000, max_shared=16000)
    assert attend(c, ws_bytes=need.value - 1, **more) == H.HS_E_BUFFER
    assert attend(c, ws=None, **more) == H.HS_E_BUFFER
    # what a few positions of ungrouped rows need is nothing
    assert hs.lib().hs_paged_attention_workspace(ctypes.byref(c), 2, 4, 100, 0, 0, ctypes.byref(need)) == H.HS_OK
    assert need.value == 0


def test_sample_refused():
    for fault in (dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(u=None), dict(tokens=None), dict(rows=-1),
                  dict(vocab=0), dict(vocab=-4), dict(vocab=(1 << 30) + 1), dict(ld=99), dict(ld=1 << 50),
                  dict(logits=AT + 2), dict(rows=1 << 26, ld=1 << 40), dict(rows=1 << 24), dict(ws=AT + 8)):
        assert sample(**fault) == H.HS_E_INVALID, fault
    assert sample(rows=0) == H.HS_OK


def test_sample_workspace_too_small():
    need = ctypes.c_uint64()
    assert hs.lib().hs_sample_tokens_workspace(3, 152064, ctypes.byref(need)) == H.HS_OK
    if need.value:
        assert sample(rows=3, vocab=152064, ld=152064, ws_bytes=need.value - 1) == H.HS_E_BUFFER
        assert sample(rows=3, vocab=152064, ld=152064, ws=None) == H.HS_E_BUFFER


def test_the_binding_refuses():
    """Tensors that are not what the calls take (on the CPU, where nothing can be launched)."""
    import torch
    blocks = torch.zeros(2, 1, 2, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(2, 1, dtype=torch.int64)
    for b, t in ((blocks[0], table), (blocks.transpose(3, 4), table), (blocks.int(), table), (blocks, table.int()),
                 (blocks, table[0]), (blocks[:, :, :1], table)):
        with pytest.raises(ValueError):
            hs.PagedCache(b, t)
    with pytest.raises(hs.HsError):
        hs.PagedCache(torch.zeros(2, 1, 2, 2, 16, 48, dtype=torch.bfloat16), table)
    c = hs.PagedCache(blocks, table)
    k, pos = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    f = hs.rope_frequencies(1e4, 32, device="cpu")
    for args in ((k, k, pos), (k.float(), k.float(), pos), (k, k[:2], pos), (k, k, pos.long()), (k[:, :1], k[:, :1], pos)):
        with pytest.raises(ValueError):
            c.append(0, *args)
    for kw in (dict(q_out=q), dict(q=q[:2]), dict(q=q, q_gain=k[0, 0].float()), dict(k_gain=k[0, 0, :32]),
               dict(angles_at=pos), dict(q=q, rope=hs.Rope(f), angles_at=torch.zeros(2, 3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.append(0, k, k, pos, **kw)
    for bad in (f.float(), f[None], f[::2]):
        with pytest.raises(ValueError):
            hs.Rope(bad)
    with pytest.raises(ValueError):
        hs.Rope(f, axes=torch.zeros(31, dtype=torch.int32))
    lens = torch.ones(3, dtype=torch.int32)
    for kw in (dict(group_starts=pos), dict(shared=pos), dict(out=q.float()), dict(workspace=blocks.transpose(0, 1)),
               dict(seqs=lens.long())):
        with pytest.raises(ValueError):
            c.attention(0, q, lens, **kw)
    x, u = torch.zeros(2, 10), torch.zeros(2)
    for kw in (dict(u=None), dict(u=u.double()), dict(u=u, top_k=u), dict(u=u, temperature=torch.zeros(3)),
               dict(u=u, tokens=torch.zeros(2, dtype=torch.int64)), dict(u=u)):
        with pytest.raises(ValueError):
            hs.sample_tokens(x, **kw)
    for bad in (x[0], x.T, x.int()):
        with pytest.raises(ValueError):
            hs.sample_tokens(bad, u)


@pytest.mark.parametrize("kv,heads", [(1, 0), (1, 1), (1, 2)])
def test_more_rows_than_a_launch_takes_are_refused(kv, heads):
    """Of few heads: a work group takes four rows at most, however few they hold."""
    rows = dict(heads=heads, ld=2 * 64, ld_q=2 * 64, ld_qo=2 * 64)
    assert append(cache(n_kv_heads=kv), n=1 << 26, **rows) == H.HS_E_INVALID


def test_sample_workspaces_of_every_length():
    """Rows up to 32768 logits need none, longer ones some; a call says so before it writes anything."""
    need = ctypes.c_uint64()
    for vocab in (1, 64, 257, 32000, 32768):
        assert hs.lib().hs_sample_tokens_workspace(5, vocab, ctypes.byref(need)) == H.HS_OK
        assert need.value == 0
    last = 0
    for vocab in (32769, 65536, 152064, 200001):
        assert hs.lib().hs_sample_tokens_workspace(3, vocab, ctypes.byref(need)) == H.HS_OK
        assert need.value >= max(1, last) and need.value % 3 == 0
        last = need.value
        for dtype in (H.HS_F32, H.HS_F16, H.HS_BF16):
            long = dict(dtype=dtype, rows=3, vocab=vocab, ld=vocab)
            assert sample(ws_bytes=need.value - 1, **long) == H.HS_E_BUFFER
            assert sample(ws=None, **long) == H.HS_E_BUFFER


def test_more_groups_than_a_work_group_looks_through_are_refused():
    """Their time grows with their square: 16384 groups of one row and 8 KV heads take 23 ms, 4 million would take minutes."""
    need = ctypes.c_uint64()
    c = cache()
    size = lambda n, groups: hs.lib().hs_paged_attention_workspace(  # noqa: E731
        ctypes.byref(c), n, 2, 96, groups, 32, ctypes.byref(need))
    assert size(65537, 65537) == H.HS_E_INVALID
    assert size(1 << 20, 1 << 20) == H.HS_E_INVALID
    assert size(1 << 20, 65536) == H.HS_OK
    assert attend(c, n=1 << 20, heads=2, ld_q=128, ld_out=128, groups=1 << 20, starts=AT, shared=AT,
                  max_shared=32) == H.HS_E_INVALID
