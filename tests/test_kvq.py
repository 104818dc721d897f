"""Host-side checks of the 4-bit cache's and the log probabilities' entry points (no GPU needed): sizes and refusals.
Every refused call returns before anything is launched."""
import ctypes

import pytest

import paper_2603_12707_amd as hs
from paper_2603_12707_amd import hs as H

BUF = (ctypes.c_char * 65536)()
AT = (ctypes.addressof(BUF) + 63) // 64 * 64  # an aligned address that is never dereferenced


def cache(**kw):
    c = dict(blocks=AT, bytes=1 << 20, table=AT, n_seqs=2, table_ld=3, n_layers=2, n_kv_heads=2, head_dim=64,
             block_tokens=32)
    c.update(kw)
    return H.hs_kvq_cache(**c)


def append(c, layer=0, dtype=H.HS_BF16, n=4, k=AT, v=AT, ld=128, ld_head=64, seqs=None, pos=AT, kv=None, vv=None):
    return hs.lib().hs_kvq_append(ctypes.byref(c), layer, dtype, n, k, v, ld, ld_head, seqs, pos, kv, vv, None)


def read(c, layer=0, dtype=H.HS_BF16, n=4, k=AT, v=AT, ld=128, ld_head=64, seqs=None, pos=AT):
    return hs.lib().hs_kvq_read(ctypes.byref(c), layer, dtype, n, k, v, ld, ld_head, seqs, pos, None)


def attend(c, layer=0, dtype=H.HS_BF16, n=2, heads=4, q=AT, ld_q=256, lens=AT, max_len=96, out=AT, ld_out=256, ws=AT,
           ws_bytes=1 << 30):
    return hs.lib().hs_kvq_attention(ctypes.byref(c), layer, dtype, n, heads, q, ld_q, None, lens, max_len,
                                     0.125, out, ld_out, ws, ws_bytes, None)


def logprobs(dtype=H.HS_F32, logits=AT, rows=2, vocab=100, ld=100, tokens=AT, top=3, lp=AT, ws=AT, ws_bytes=1 << 30):
    return hs.lib().hs_token_logprobs(dtype, logits, rows, vocab, ld, tokens, top, lp, AT, AT, AT, ws, ws_bytes, None)


def test_block_bytes():
    for layers, kv, hd, bt in ((1, 1, 64, 16), (28, 4, 128, 256), (32, 32, 128, 16384)):
        assert hs.kvq_block_bytes(layers, kv, hd, bt) == 2 * layers * kv * bt * (hd // 2 + hd // 32)
    # 17/64 of the 16-bit cache's bytes
    cfg = dict(n_layers=28, d_model=3584, n_heads=28, n_kv_heads=4, head_dim=128, ffn_dim=18944, vocab=152064,
               rope_theta=1e6, rms_eps=1e-6, rope_kind=0, mrope_section=(0, 0, 0), qkv_bias=1, dtype="bf16")
    assert hs.kvq_block_bytes(28, 4, 128, 256) * 64 == hs.hs_kv_bytes(cfg, 0, 256)[0] * 17


@pytest.mark.parametrize("bad", [(0, 1, 64, 16), (1, 0, 64, 16), (1, 1, 96, 16), (1, 1, 32, 16), (1, 1, 64, 8),
                                 (1, 1, 64, 48), (1, 1, 64, 32768), (1, 4097, 64, 16), (-1, 1, 64, 16), (2 ** 31 - 1, 2 ** 31 - 1, 128, 16384)])
def test_block_bytes_refuses(bad):
    with pytest.raises(hs.HsError) as e:
        hs.kvq_block_bytes(*bad)
    assert e.value.code == H.HS_E_INVALID


CACHE_FAULTS = [dict(blocks=None), dict(table=None), dict(blocks=AT + 8), dict(table=AT + 4), dict(n_seqs=0),
                dict(table_ld=0), dict(n_layers=0), dict(n_kv_heads=0), dict(head_dim=80), dict(block_tokens=24)]


@pytest.mark.parametrize("fault", CACHE_FAULTS, ids=lambda f: "-".join(f))
@pytest.mark.parametrize("call", [append, read, attend], ids=["append", "read", "attend"])
def test_a_faulty_cache_is_refused(call, fault):
    assert call(cache(**fault)) == H.HS_E_INVALID


@pytest.mark.parametrize("call", [append, read, attend], ids=["append", "read", "attend"])
def test_cache_arguments_every_call_checks(call):
    assert call(cache(bytes=100)) == H.HS_E_BUFFER  # less than one block
    assert call(cache(), layer=2) == H.HS_E_INVALID
    assert call(cache(), layer=-1) == H.HS_E_INVALID
    assert call(cache(), dtype=3) == H.HS_E_INVALID
    assert call(cache(), dtype=-1) == H.HS_E_INVALID
    assert call(cache(), n=-1) == H.HS_E_INVALID
    assert call(cache(), n=0) == H.HS_OK
    assert hs.lib().hs_kvq_append(None, 0, 2, 1, AT, AT, 128, 64, None, AT, None, None, None) == H.HS_E_INVALID


@pytest.mark.parametrize("call", [append, read], ids=["append", "read"])
def test_rows_refused(call):
    for fault in (dict(k=None), dict(v=None), dict(pos=None), dict(k=AT + 8), dict(v=AT + 4), dict(ld=132),
                  dict(ld_head=68), dict(ld=-128), dict(ld_head=-64), dict(ld=64), dict(ld=0), dict(ld_head=32),
                  dict(ld=96, ld_head=64), dict(ld=1 << 50), dict(n=2 ** 31 - 1)):
        assert call(cache(), **fault) == H.HS_E_INVALID, fault
    # fp32 rows are aligned to 4 elements
    assert call(cache(), dtype=H.HS_F32, ld=130) == H.HS_E_INVALID


def test_append_values_come_in_pairs_and_aligned():
    assert append(cache(), kv=AT) == H.HS_E_INVALID
    assert append(cache(), vv=AT) == H.HS_E_INVALID
    assert append(cache(), kv=AT + 8, vv=AT) == H.HS_E_INVALID


def test_attention_refused():
    for fault in (dict(q=None), dict(out=None), dict(lens=None), dict(q=AT + 8), dict(out=AT + 2), dict(ws=AT + 4),
                  dict(heads=0), dict(heads=3), dict(heads=34), dict(heads=-2), dict(max_len=0), dict(max_len=-5),
                  dict(max_len=2 ** 30 + 1),
                  dict(ld_q=255), dict(ld_q=128), dict(ld_out=128), dict(n=2 ** 30)):
        assert attend(cache(), **fault) == H.HS_E_INVALID, fault


def test_strides_whose_last_row_lies_past_64_bits_are_refused():
    far, n = 1 << 40, 1 << 26
    assert append(cache(), n=n, ld=far) == H.HS_E_INVALID
    assert read(cache(), n=n, ld=far) == H.HS_E_INVALID
    assert read(cache(n_kv_heads=4096, bytes=1 << 40), n=2, ld=64, ld_head=1 << 50) == H.HS_E_INVALID
    c = cache(n_seqs=1 << 30)
    assert attend(c, n=n, ld_q=far) == H.HS_E_INVALID
    assert attend(c, n=n, ld_out=far) == H.HS_E_INVALID
    assert logprobs(rows=n, ld=far) == H.HS_E_INVALID


def test_more_rows_than_a_launch_takes_are_refused():
    """A launch has less than 2^32 threads in a dimension; what would need more is refused before it."""
    one = cache(n_kv_heads=1, n_seqs=1 << 30)
    for call in (append, read):
        assert call(one, n=1 << 28, ld=64) == H.HS_E_INVALID
        assert call(cache(n_kv_heads=4096, bytes=1 << 40), n=1 << 16, ld=4096 * 64) == H.HS_E_INVALID
    assert attend(one, n=1 << 24, heads=1, ld_q=64, ld_out=64) == H.HS_E_INVALID
    assert logprobs(rows=1 << 24) == H.HS_E_INVALID
    assert logprobs(rows=1 << 20, vocab=16 * 8192, ld=16 * 8192) == H.HS_E_INVALID


def test_attention_workspace_is_checked():
    c, need = cache(n_seqs=1, table_ld=1 << 16), ctypes.c_uint64()
    ask = hs.lib().hs_kvq_attention_workspace
    assert ask(ctypes.byref(c), H.HS_BF16, 1, 4, 1 << 20, ctypes.byref(need)) == H.HS_OK
    if need.value:
        assert attend(c, n=1, max_len=1 << 20, ws=None) == H.HS_E_BUFFER
        assert attend(c, n=1, max_len=1 << 20, ws_bytes=need.value - 1) == H.HS_E_BUFFER
    assert ask(ctypes.byref(c), H.HS_BF16, 1, 4, 1 << 20, None) == H.HS_E_INVALID
    assert ask(None, H.HS_BF16, 1, 4, 1 << 20, ctypes.byref(need)) == H.HS_E_INVALID
    assert ask(ctypes.byref(c), 7, 1, 4, 1 << 20, ctypes.byref(need)) == H.HS_E_INVALID
    assert ask(ctypes.byref(c), H.HS_BF16, 1, 5, 1 << 20, ctypes.byref(need)) == H.HS_E_INVALID


def test_logprobs_refused():
    for fault in (dict(dtype=3), dict(logits=None), dict(logits=AT + 2), dict(rows=-1), dict(rows=1 << 40),
                  dict(vocab=0), dict(vocab=-7), dict(ld=99), dict(ld=1 << 50), dict(tokens=None), dict(top=-1),
                  dict(top=65), dict(vocab=2), dict(ws=AT + 4), dict(vocab=2 ** 30 + 1, ld=2 ** 31)):
        assert logprobs(**fault) == H.HS_E_INVALID, fault
    assert logprobs(dtype=H.HS_F16, logits=AT + 1) == H.HS_E_INVALID
    assert logprobs(rows=0) == H.HS_OK


def test_logprobs_workspace_is_checked():
    need = ctypes.c_uint64()
    ask = hs.lib().hs_token_logprobs_workspace
    assert ask(16, 152064, 20, ctypes.byref(need)) == H.HS_OK
    if need.value:
        assert logprobs(rows=16, vocab=152064, ld=152064, top=20, ws=None) == H.HS_E_BUFFER
        assert logprobs(rows=16, vocab=152064, ld=152064, top=20, ws_bytes=need.value - 1) == H.HS_E_BUFFER
    assert ask(16, 152064, 20, None) == H.HS_E_INVALID


def test_pool_and_step_refuse_what_is_missing():
    """(What needs a model is refused in the GPU tests.)"""
    out = ctypes.c_void_p(7)
    L = hs.lib()
    assert L.hs_kvq_pool_create(None, 1, 256, AT, 1 << 20, ctypes.byref(out)) == H.HS_E_INVALID and not out.value
    assert L.hs_kvq_pool_create(None, 1, 256, AT, 1 << 20, None) == H.HS_E_INVALID
    assert L.hs_decode_step_logprobs(None, None, AT, AT, None, 1, None, None, AT, AT, AT, AT, None) == H.HS_E_INVALID


def test_binding_refuses_wrong_tensors():
    """Shapes, types and devices that the binding looks at before it calls the library."""
    import torch
    blocks, table = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.int64)
    q = hs.QuantCache(blocks, table, 2, 2, 64, 32)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        hs.QuantCache(blocks.int(), table, 2, 2, 64, 32)
    with pytest.raises(ValueError):
        hs.QuantCache(blocks, table.int(), 2, 2, 64, 32)
    with pytest.raises(hs.HsError):
        hs.QuantCache(blocks, table, 2, 2, 80, 32)
    for bad in (dict(k=k[:, :1]), dict(v=k.half()), dict(k=k[..., :32]), dict(positions=pos[:3]),
                dict(positions=pos.long()), dict(seqs=pos.long()), dict(k_values=k), dict(k_values=k, v_values=k.half()),
                dict(k=k.double(), v=k.double())):
        with pytest.raises(ValueError):
            q.append(**{**dict(layer=0, k=k, v=k, positions=pos), **bad})
    with pytest.raises(ValueError):  # not on the GPU
        q.append(0, k, k, pos)
    with pytest.raises(ValueError):
        q.read(0, pos.long(), torch.bfloat16)
    qq = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        q.attention(0, qq[..., :32], pos[:2])
    with pytest.raises(ValueError):
        q.attention(0, qq, pos)
    with pytest.raises(ValueError):
        q.attention(0, qq, pos[:2], out=qq.half())
    x = torch.zeros(2, 10)
    with pytest.raises(ValueError):
        hs.token_logprobs(x[0])
    with pytest.raises(ValueError):
        hs.token_logprobs(x.t())
    with pytest.raises(ValueError):
        hs.token_logprobs(x.double())
    with pytest.raises(ValueError):
        hs.token_logprobs(x, torch.zeros(2, dtype=torch.int64))


class _Tokens:
    """What the binding looks at of a token tensor on a GPU."""

    def __init__(self, n, dtype=None, index=0, contiguous=True):
        import torch
        self.n, self.dtype, self.index, self.contiguous, self.device = n, dtype or torch.int32, index, contiguous, "cuda"

    def numel(self):
        return self.n

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 0


def test_steps_with_log_probabilities_refuse_wrong_tokens():
    """One int32 token for each request of the handle, on the GPU: the kernels read by request number."""
    import types

    import torch
    pool = object.__new__(hs.KVPool)
    pool.batch, pool.handle, pool.model = 4, None, types.SimpleNamespace(max_batch=2, handle=None)
    good = dict(tokens_in=_Tokens(4), tokens_out=_Tokens(4))
    for bad in (_Tokens(4, torch.int64), _Tokens(2), _Tokens(5), _Tokens(4, index=-1), _Tokens(4, index=1),
                _Tokens(4, contiguous=False), torch.zeros(4, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)):
        for name in ("targets", "tokens_in", "tokens_out"):
            with pytest.raises(ValueError):
                pool.decode_logprobs(**{**good, name: bad})
    with pytest.raises(ValueError):
        pool.decode_logprobs(None, _Tokens(4))
