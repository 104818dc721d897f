"""Thin ctypes binding of libhs (include/hs.h).

Argument marshalling only: every step of prefill and decode runs in the HIP
kernels of libhs.so.  torch tensors supply device memory and the current HIP
stream.  The library is loaded from this package directory; if it is missing
the import fails loudly (there is no fallback path).
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
# HS_LIBRARY names another build of the same library (the host-sanitizer
# build of the tests); by default the in-tree libhs.so
LIB_PATH = os.environ.get("HS_LIBRARY") or os.path.join(HERE, "libhs.so")

HS_OK, HS_E_INVALID, HS_E_CAPACITY, HS_E_BUFFER, HS_E_STATE, HS_E_DEVICE = 0, -1, -2, -3, -4, -5
HS_F32, HS_F16, HS_BF16 = 0, 1, 2
HS_ROPE_1D, HS_ROPE_M3 = 0, 1

# every symbol include/hs.h declares
EXPORTS = ("hs_last_error", "hs_kv_bytes", "hs_model_create", "hs_model_free", "hs_kv_alloc", "hs_kv_free",
           "hs_prefill_embeddings", "hs_decode_step", "hs_model_status", "hs_kv_lengths", "hs_kv_write",
           "hs_kv_read", "hs_kv_set_length", "hs_replay_kernels", "hs_packed_bytes", "hs_pack_matrix", "hs_pack_matrix_heads", "hs_kv_sync",
           "hs_prefill_batch", "hs_model_reserve_rows", "hs_kv_pool_create", "hs_kv_admit", "hs_kv_release",
           "hs_kv_pool_blocks", "hs_handoff_create", "hs_handoff_free", "hs_handoff_push", "hs_handoff_pop",
           "hs_handoff_pending", "hs_stream_read", "hs_decode_step_static", "hs_kvq_block_bytes", "hs_kvq_append",
           "hs_kvq_read", "hs_kvq_attention_workspace", "hs_kvq_attention", "hs_token_logprobs_workspace",
           "hs_token_logprobs", "hs_kvq_pool_create", "hs_decode_step_logprobs", "hs_paged_block_bytes",
           "hs_paged_append", "hs_paged_attention_workspace", "hs_paged_attention", "hs_sample_tokens_workspace",
           "hs_sample_tokens", "hs_decode_step_sample")

# projection matrices the library reads in its packed layout
PACKED = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "lm_head")

HS_K_NAMES = ("embed", "qkv", "attn", "combine", "oproj", "gateup", "down", "head", "argmax")


class HsError(RuntimeError):
    def __init__(self, func: str, code: int, msg: str):
        super().__init__(f"{func} failed with status {code}: {msg}")
        self.code = code


class hs_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("rope_kind", ctypes.c_int32), ("mrope_section", ctypes.c_int32 * 3),
                ("qkv_bias", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class hs_layer_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "mlp_norm",
                                                 "w_gate", "w_up", "w_down")]


class hs_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p), ("lm_head", ctypes.c_void_p),
                ("layers", ctypes.POINTER(hs_layer_weights))]


class hs_kvq_cache(ctypes.Structure):
    _fields_ = [("blocks", ctypes.c_void_p), ("bytes", ctypes.c_uint64), ("table", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("table_ld", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32)]


class hs_paged_cache(ctypes.Structure):
    _fields_ = hs_kvq_cache._fields_ + [("dtype", ctypes.c_int32)]


class hs_rope(ctypes.Structure):
    _fields_ = [("frequencies", ctypes.c_void_p), ("axes", ctypes.c_void_p), ("n_pairs", ctypes.c_int32),
                ("n_axes", ctypes.c_int32), ("adjacent", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libhs.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    # torch ships its own HIP runtime under the same soname as the system one;
    # importing it first makes libhs.so bind to that runtime instead of
    # loading a second copy into the process
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2603_12707_amd/build.py "
                          "(or __graft_entry__.build()); there is no fallback implementation")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64, U64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64
    L.hs_last_error.restype = ctypes.c_char_p
    L.hs_last_error.argtypes = []
    sig = {
        "hs_kv_bytes": [ctypes.POINTER(hs_config), I64, I64, ctypes.POINTER(U64), ctypes.POINTER(U64)],
        "hs_model_create": [ctypes.POINTER(hs_config), ctypes.POINTER(hs_weights), I32, I32, ctypes.POINTER(P)],
        "hs_model_free": [P],
        "hs_kv_alloc": [P, I32, P, P, P, U64, ctypes.POINTER(P)],
        "hs_kv_free": [P],
        "hs_prefill_embeddings": [P, P, I32, P, P, I32, P, P, P, P],
        "hs_prefill_batch": [P, P, I32, P, P, P, P, P, P, P, P],
        "hs_model_reserve_rows": [P, I64],
        "hs_kv_pool_create": [P, I32, I32, P, U64, ctypes.POINTER(P)],
        "hs_kv_admit": [P, I32, I32, I32, P],
        "hs_kv_release": [P, I32, P],
        "hs_kv_pool_blocks": [P, ctypes.POINTER(I32), ctypes.POINTER(I32)],
        "hs_handoff_create": [I32, I64, I32, ctypes.c_double, ctypes.POINTER(P)],
        "hs_handoff_free": [P],
        "hs_handoff_push": [P, I32, I32, ctypes.c_double],
        "hs_handoff_pop": [P, ctypes.c_double, P, I32, ctypes.POINTER(I32), ctypes.POINTER(I64),
                           ctypes.POINTER(ctypes.c_double)],
        "hs_handoff_pending": [P, ctypes.POINTER(I32)],
        "hs_stream_read": [P, U64, P, I32, P],
        "hs_decode_step": [P, P, P, P, P, P, P],
        "hs_decode_step_static": [P, P, P, P, P, P, P],
        "hs_model_status": [P, ctypes.POINTER(I32)],
        "hs_kv_lengths": [P, P],
        "hs_kv_sync": [P],
        "hs_kv_write": [P, I32, I32, I32, I32, I32, I32, P, I32],
        "hs_kv_read": [P, I32, I32, I32, I32, I32, I32, P, I32],
        "hs_kv_set_length": [P, I32, I32, I32],
        "hs_replay_kernels": [P, P, I32, I32, P],
        "hs_packed_bytes": [I32, I64, I64, ctypes.POINTER(U64)],
        "hs_pack_matrix": [I32, P, I64, I64, P, P],
        "hs_pack_matrix_heads": [I32, P, I64, I64, I32, P, P],
        "hs_kvq_block_bytes": [I32, I32, I32, I32, ctypes.POINTER(U64)],
        "hs_kvq_append": [P, I32, I32, I32, P, P, I64, I64, P, P, P, P, P],
        "hs_kvq_read": [P, I32, I32, I32, P, P, I64, I64, P, P, P],
        "hs_kvq_attention_workspace": [P, I32, I32, I32, I32, ctypes.POINTER(U64)],
        "hs_kvq_attention": [P, I32, I32, I32, I32, P, I64, P, P, I32, ctypes.c_float, P, I64, P, U64, P],
        "hs_token_logprobs_workspace": [I64, I32, I32, ctypes.POINTER(U64)],
        "hs_kvq_pool_create": [P, I32, I32, P, U64, ctypes.POINTER(P)],
        "hs_decode_step_logprobs": [P, P, P, P, P, I32, P, P, P, P, P, P, P],
        "hs_paged_block_bytes": [I32, I32, I32, I32, I32, ctypes.POINTER(U64)],
        "hs_paged_append": [P, I32, I32, I32, P, I64, I64, P, I64, I64, P, P, I64, I64, P, P, P, P, P, P,
                            ctypes.c_float, P],
        "hs_paged_attention_workspace": [P, I32, I32, I32, I32, I32, ctypes.POINTER(U64)],
        "hs_paged_attention": [P, I32, I32, I32, P, I64, P, P, I32, P, P, I32, I32, ctypes.c_float, P, I64, P, U64, P],
        "hs_sample_tokens_workspace": [I64, I32, ctypes.POINTER(U64)],
        "hs_sample_tokens": [I32, P, I64, I32, I64, P, P, P, P, P, P, P, P, U64, P],
        "hs_decode_step_sample": [P, P, P, P, P, P, P, P, P, P, P, P, P],
        "hs_token_logprobs": [I32, P, I64, I32, I64, P, I32, P, P, P, P, P, U64, P],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    _lib = L
    return L


def check(func: str, rc: int) -> None:
    if rc != HS_OK:
        raise HsError(func, rc, lib().hs_last_error().decode())


def _call(func: str, *args) -> None:
    check(func, getattr(lib(), func)(*args))


def make_config(cfg: dict) -> hs_config:
    c = hs_config()
    for k in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn_dim", "vocab", "rope_kind",
              "qkv_bias"):
        setattr(c, k, int(cfg[k]))
    c.rope_theta = float(cfg["rope_theta"])
    c.rms_eps = float(cfg["rms_eps"])
    c.mrope_section[:] = [int(v) for v in cfg["mrope_section"]]
    c.dtype = {"f32": HS_F32, "f16": HS_F16, "bf16": HS_BF16}[cfg["dtype"]]
    return c


def hs_kv_bytes(cfg: dict, n_v: int, s_text: int) -> tuple:
    kv, emb = ctypes.c_uint64(), ctypes.c_uint64()
    _call("hs_kv_bytes", ctypes.byref(make_config(cfg)), n_v, s_text, ctypes.byref(kv), ctypes.byref(emb))
    return kv.value, emb.value


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def stream_read(buf, sink, blocks: int) -> None:
    """Plain streaming read of a device tensor (measurement)."""
    _call("hs_stream_read", _ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), blocks, _stream())


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


_DT = {"f32": HS_F32, "f16": HS_F16, "bf16": HS_BF16}


def _is_packed(name: str) -> bool:
    return name.split(".")[-1] in PACKED


def hs_packed_bytes(dtype: str, rows: int, cols: int) -> int:
    out = ctypes.c_uint64()
    _call("hs_packed_bytes", _DT[dtype], rows, cols, ctypes.byref(out))
    return out.value


def pack_matrix(t, dtype: str, head_dim: int = 0):
    """Packed copy (uint8 device tensor) of a row-major [rows, cols] device
    matrix, written on the current stream by hs_pack_matrix, or with head_dim
    by hs_pack_matrix_heads (the q/k/v projections)."""
    import torch
    assert t.is_cuda and t.dim() == 2 and t.is_contiguous()
    rows, cols = t.shape
    out = torch.empty(hs_packed_bytes(dtype, rows, cols), dtype=torch.uint8, device=t.device)
    if head_dim:
        _call("hs_pack_matrix_heads", _DT[dtype], _ptr(t), rows, cols, head_dim, _ptr(out), _stream())
    else:
        _call("hs_pack_matrix", _DT[dtype], _ptr(t), rows, cols, _ptr(out), _stream())
    return out


HEAD_PAIRED = ("wq", "wk", "wv")


def pack_weight(cfg: dict, name: str, t):
    """The tensor the model takes for weight `name`: projection matrices
    packed (q/k/v head-paired), everything else as it is."""
    leaf = name.split(".")[-1]
    if leaf not in PACKED:
        return t
    return pack_matrix(t, cfg["dtype"], cfg["head_dim"] if leaf in HEAD_PAIRED else 0)


def pack_weights(cfg: dict, weights: dict, free_source: bool = False) -> dict:
    """Returns the weight dict with every projection matrix packed; vectors
    and the embedding table pass through.  With free_source the row-major
    matrices are removed from `weights` as they are packed."""
    out = {}
    for name in list(weights):
        out[name] = pack_weight(cfg, name, weights[name])
        if free_source and _is_packed(name):
            del weights[name]
    return out


class Model:
    """A model over device weight tensors named as in the workload generator
    (embed, layers.{i}.wq, ..., final_norm, lm_head).  Row-major projection
    matrices are packed on construction unless packed=True says they already
    are."""

    def __init__(self, cfg: dict, weights: dict, max_batch: int, max_ctx: int, packed: bool = False):
        self.cfg = cfg
        if not packed:
            weights = pack_weights(cfg, weights)
        self._w = weights  # keeps the tensors alive
        L = cfg["n_layers"]
        self._layers = (hs_layer_weights * L)()
        for i in range(L):
            p = f"layers.{i}."
            for n in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down"):
                setattr(self._layers[i], n, weights[p + n].data_ptr())
            if cfg["qkv_bias"]:
                for n in ("bq", "bk", "bv"):
                    setattr(self._layers[i], n, weights[p + n].data_ptr())
        hw = hs_weights()
        hw.embed = weights["embed"].data_ptr()
        if cfg.get("lm_head", True):
            hw.final_norm = weights["final_norm"].data_ptr()
            hw.lm_head = weights["lm_head"].data_ptr()
        hw.layers = self._layers
        self._hw = hw
        self._cfg_c = make_config(cfg)
        h = ctypes.c_void_p()
        _call("hs_model_create", ctypes.byref(self._cfg_c), ctypes.byref(hw), max_batch, max_ctx, ctypes.byref(h))
        self.handle = h
        self.max_batch, self.max_ctx = max_batch, max_ctx

    def reserve_rows(self, rows: int) -> None:
        """Room for `rows` packed prefill rows per pass (grows only)."""
        _call("hs_model_reserve_rows", self.handle, rows)

    def status(self) -> int:
        f = ctypes.c_int32()
        _call("hs_model_status", self.handle, ctypes.byref(f))
        return f.value

    def close(self) -> None:
        if self.handle:
            _call("hs_model_free", self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVCache:
    """Per-request contiguous KV cache over a caller-owned uint8 device tensor."""

    def __init__(self, model: Model, n_v, capacity, buf=None):
        import torch
        self.model = model
        self.batch = len(capacity)
        self.n_v = [int(v) for v in n_v]
        self.capacity = [int(c) for c in capacity]
        cfg = model.cfg
        need = sum(hs_kv_bytes(cfg, 0, c)[0] for c in self.capacity)
        if buf is None:
            buf = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.buf = buf
        nv = (ctypes.c_int32 * self.batch)(*self.n_v)
        cap = (ctypes.c_int32 * self.batch)(*self.capacity)
        h = ctypes.c_void_p()
        _call("hs_kv_alloc", model.handle, self.batch, nv, cap, _ptr(buf), buf.numel() * buf.element_size(),
              ctypes.byref(h))
        self.handle = h

    def prefill(self, req: int, emb, text_ids, pos_thw=None, last_logits=None, first_token=None):
        import torch
        if first_token is None:
            first_token = torch.empty(1, dtype=torch.int32, device="cuda")
        _call("hs_prefill_embeddings", self.model.handle, self.handle, req, _ptr(emb), _ptr(text_ids),
              0 if text_ids is None else text_ids.numel(), _ptr(pos_thw), _ptr(last_logits), _ptr(first_token),
              _stream())
        return first_token

    def prefill_batch(self, reqs, emb, text_ids, s_text, pos_thw=None, last_logits=None, first_tokens=None):
        """Prefill of several requests with their rows packed request by
        request: emb holds their vision rows back to back, text_ids their
        text ids, pos_thw (M-RoPE) [3][rows]; returns first_tokens [n]."""
        import torch
        n = len(reqs)
        if first_tokens is None:
            first_tokens = torch.empty(n, dtype=torch.int32, device="cuda")
        r = (ctypes.c_int32 * n)(*reqs)
        t = (ctypes.c_int32 * n)(*s_text)
        _call("hs_prefill_batch", self.model.handle, self.handle, n, r, _ptr(emb), _ptr(text_ids), t, _ptr(pos_thw),
              _ptr(last_logits), _ptr(first_tokens), _stream())
        return first_tokens

    def decode(self, tokens_in, tokens_out, logits=None, hidden_out=None, model=None) -> None:
        """One greedy step; `model` (default: the handle's) may be any model of the same configuration."""
        _call("hs_decode_step", (model or self.model).handle, self.handle, _ptr(tokens_in), _ptr(tokens_out),
              _ptr(logits), _ptr(hidden_out), _stream())

    def decode_static(self, tokens_in, tokens_out, logits=None, hidden_out=None, model=None) -> None:
        """The same step with its scratch in the library's static device array
        (hs_decode_step_static: allocates nothing)."""
        _call("hs_decode_step_static", (model or self.model).handle, self.handle, _ptr(tokens_in), _ptr(tokens_out),
              _ptr(logits), _ptr(hidden_out), _stream())

    def decode_logprobs(self, tokens_in, tokens_out, targets=None, top: int = 0, logits=None, hidden_out=None,
                        model=None):
        """The same step, and of its logits (logprob, entropy, top_ids, top_logprobs) as token_logprobs gives them,
        a row for each decoded request: of the tokens in targets (int32, one for each request of the handle, like
        tokens_in; None: the chosen ones), with `top` alternatives (None without).  The rows come first; a pool that
        decodes fewer requests than it could (slots, max_batch) has NaN, and -1 for tokens, in the others."""
        import torch
        func = "decode_logprobs"
        index = -1 if tokens_in is None else tokens_in.get_device()
        if index < 0:
            raise ValueError(f"{func}: tokens_in must be on the GPU")
        # the kernels read and write an entry for every request of the handle
        for name, t in (("tokens_in", tokens_in), ("tokens_out", tokens_out), ("targets", targets)):
            _int32(func, name, t, self.batch, index)
        m = model or self.model
        device = tokens_in.device
        # as many rows as requests can be decoded; those that a pool decodes fewer keep NaN and -1
        rows, alts = min(self.batch, m.max_batch), max(top, 0)
        if isinstance(self, KVPool):
            numbers = torch.full((rows * (2 + alts),), float("nan"), dtype=torch.float32, device=device)
            ids = torch.full((rows, alts), -1, dtype=torch.int32, device=device) if alts else None
        else:
            numbers = torch.empty(rows * (2 + alts), dtype=torch.float32, device=device)
            ids = torch.empty(rows, alts, dtype=torch.int32, device=device) if alts else None
        lp, entropy = numbers[:rows], numbers[rows : 2 * rows]
        tops = numbers[2 * rows :].view(rows, alts) if alts else None
        _call("hs_decode_step_logprobs", m.handle, self.handle, _ptr(tokens_in), _ptr(tokens_out), _ptr(targets), top,
              _ptr(logits), _ptr(hidden_out), _ptr(lp), _ptr(entropy), _ptr(ids), _ptr(tops), _stream())
        return lp, entropy, ids, tops

    def decode_sample(self, tokens_in, tokens_out, u, temperature=None, top_k=None, top_p=None, min_p=None,
                      logits=None, hidden_out=None, model=None):
        """The same step with its tokens drawn as sample_tokens draws them, instead of the largest logit; u, temperature,
        top_p, min_p (float32) and top_k (int32) have an entry for each request of the handle, like tokens_in.  Returns
        the log probabilities of the drawn tokens, a row for each decoded request (the rows come first; a pool that
        decodes fewer than it could has NaN in the others)."""
        import torch
        func = "decode_sample"
        index = -1 if tokens_in is None else tokens_in.get_device()
        if index < 0:
            raise ValueError(f"{func}: tokens_in must be on the GPU")
        if u is None:
            raise ValueError(f"{func}: u must be {self.batch} contiguous float32 values")
        for name, t in (("tokens_in", tokens_in), ("tokens_out", tokens_out), ("top_k", top_k)):
            _int32(func, name, t, self.batch, index)
        for name, t in (("u", u), ("temperature", temperature), ("top_p", top_p), ("min_p", min_p)):
            _float32(func, name, t, self.batch, index)
        m = model or self.model
        rows = min(self.batch, m.max_batch)
        lp = torch.full((rows,), float("nan"), dtype=torch.float32, device=tokens_in.device)
        _call("hs_decode_step_sample", m.handle, self.handle, _ptr(tokens_in), _ptr(tokens_out), _ptr(u),
              _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(logits), _ptr(hidden_out), _ptr(lp),
              _stream())
        return lp

    def sync(self) -> None:
        """Host mirrors of the lengths from the device (after graph replays)."""
        _call("hs_kv_sync", self.handle)

    def lengths(self) -> list:
        out = (ctypes.c_int32 * self.batch)()
        _call("hs_kv_lengths", self.handle, out)
        return list(out)

    def write(self, req: int, layer: int, kv_sel: int, head: int, pos0: int, rows) -> None:
        n = rows.shape[0]
        _call("hs_kv_write", self.handle, req, layer, kv_sel, head, pos0, n, _ptr(rows), int(rows.is_cuda))

    def read(self, req: int, layer: int, kv_sel: int, head: int, pos0: int, n: int, out) -> None:
        _call("hs_kv_read", self.handle, req, layer, kv_sel, head, pos0, n, _ptr(out), int(out.is_cuda))

    def replay(self, kind: str, count: int, model: "Model | None" = None) -> None:
        """Launches `count` kernels of one kind back to back (measurement)."""
        _call("hs_replay_kernels", (model or self.model).handle, self.handle, HS_K_NAMES.index(kind), count, _stream())

    def set_length(self, req: int, length: int, rope_pos: int) -> None:
        _call("hs_kv_set_length", self.handle, req, length, rope_pos)

    def close(self) -> None:
        if self.handle:
            _call("hs_kv_free", self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVPool(KVCache):
    """Block-granular KV cache: `slots` request slots over n_blocks blocks of
    block_tokens positions in a caller-owned (or fresh) uint8 device tensor.
    Requests are admitted into empty slots, prefilled and decoded like
    KVCache requests (slot = request number) and released when done."""

    _create = "hs_kv_pool_create"

    def __init__(self, model: Model, slots: int, block_tokens: int, n_blocks: int, buf=None):
        import torch
        self.model = model
        self.batch = slots
        self.block_tokens = block_tokens
        if buf is None:
            buf = torch.empty(n_blocks * self._block_bytes(), dtype=torch.uint8, device="cuda")
        self.buf = buf
        h = ctypes.c_void_p()
        _call(self._create, model.handle, slots, block_tokens, _ptr(buf), buf.numel() * buf.element_size(),
              ctypes.byref(h))
        self.handle = h

    def _block_bytes(self) -> int:
        return hs_kv_bytes(self.model.cfg, 0, self.block_tokens)[0]

    def admit(self, slot: int, n_v: int, capacity: int) -> None:
        _call("hs_kv_admit", self.handle, slot, n_v, capacity, _stream())

    def release(self, slot: int) -> None:
        _call("hs_kv_release", self.handle, slot, _stream())

    def blocks(self) -> tuple:
        """(free, total) blocks."""
        f, n = ctypes.c_int32(), ctypes.c_int32()
        _call("hs_kv_pool_blocks", self.handle, ctypes.byref(f), ctypes.byref(n))
        return f.value, n.value


class QuantKVPool(KVPool):
    """A KVPool held in 4 bits (hs_kvq_pool_create): 17/64 of its bytes, the
    rows rounded as they are stored, read and written through the same calls."""

    _create = "hs_kvq_pool_create"

    def _block_bytes(self) -> int:
        cfg = self.model.cfg
        return kvq_block_bytes(cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"], self.block_tokens)


def _dtype_code(func: str, t) -> int:
    import torch
    if t.dtype is torch.bfloat16:
        return HS_BF16
    if t.dtype is torch.float16:
        return HS_F16
    if t.dtype is torch.float32:
        return HS_F32
    raise ValueError(f"{func}: {t.dtype} is none of float32, float16, bfloat16")


def _int32(func: str, name: str, t, n: int, index: int):
    """Address of a contiguous int32 tensor of n values on GPU `index` (None: NULL)."""
    import torch
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != index:
        raise ValueError(f"{func}: {name} must be {n} contiguous int32 values on GPU {index}")
    return t.data_ptr()


def _float32(func: str, name: str, t, n: int, index: int):
    """Address of a contiguous float32 tensor of n values on GPU `index` (None: NULL)."""
    import torch
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != index:
        raise ValueError(f"{func}: {name} must be {n} contiguous float32 values on GPU {index}")
    return t.data_ptr()


def _on_device(func: str, name: str, index: int, *args) -> None:
    """Calls the library's function `name` with args and the current stream of GPU `index`, that GPU current."""
    import torch
    if index < 0:
        raise ValueError(f"{func}: tensors must be on the GPU")
    stream = torch._C._cuda_getCurrentRawStream(index)
    if index == torch.cuda.current_device():
        rc = getattr(_lib, name)(*args, stream)
    else:
        with torch.cuda.device(index):
            rc = getattr(_lib, name)(*args, stream)
    if rc != HS_OK:
        check(name, rc)


def kvq_block_bytes(n_layers: int, n_kv_heads: int, head_dim: int, block_tokens: int) -> int:
    """Bytes of one block of a cache held in 4 bits."""
    out = ctypes.c_uint64()
    _call("hs_kvq_block_bytes", n_layers, n_kv_heads, head_dim, block_tokens, ctypes.byref(out))
    return out.value


class QuantCache:
    """A KV cache held in 4 bits (hs_kvq_cache) over caller-owned tensors:
    blocks, a contiguous uint8 tensor of whole blocks (kvq_block_bytes each),
    and table, a contiguous int64 tensor [sequences][blocks per sequence] of
    block numbers, negative where there is none.  The table may be rewritten
    between calls."""

    def __init__(self, blocks, table, n_layers: int, n_kv_heads: int, head_dim: int, block_tokens: int):
        import torch
        if blocks.dtype is not torch.uint8 or not blocks.is_contiguous():
            raise ValueError("QuantCache: blocks must be a contiguous uint8 tensor")
        if table.dtype is not torch.int64 or table.dim() != 2 or not table.is_contiguous() or \
                table.device != blocks.device:
            raise ValueError("QuantCache: table must be a contiguous int64 matrix on the blocks' device")
        kvq_block_bytes(n_layers, n_kv_heads, head_dim, block_tokens)  # checks the sizes
        self.blocks, self.table = blocks, table  # keeps the tensors alive
        self.n_layers, self.n_kv_heads, self.head_dim, self.block_tokens = n_layers, n_kv_heads, head_dim, block_tokens
        self._index = blocks.get_device()
        self._c = hs_kvq_cache(blocks.data_ptr(), blocks.numel(), table.data_ptr(), table.shape[0], table.shape[1],
                               n_layers, n_kv_heads, head_dim, block_tokens)
        self._ref = ctypes.addressof(self._c)

    def _check_rows(self, func: str, k, v):
        """k, v: [n][n_kv_heads][head_dim], equal strides, channels contiguous; returns (n, strides), the strides of
        a single row or head, which nothing uses, as 0."""
        shape, stride = k.shape, k.stride()
        if len(shape) != 3 or shape[1] != self.n_kv_heads or shape[2] != self.head_dim or v.shape != shape or \
                v.dtype != k.dtype or stride[2] != 1 or v.stride(2) != 1 or \
                (shape[0] > 1 and v.stride(0) != stride[0]) or (shape[1] > 1 and v.stride(1) != stride[1]) or \
                k.get_device() != self._index or v.get_device() != self._index:
            raise ValueError(f"{func}: k and v must be [n][{self.n_kv_heads}][{self.head_dim}] on {self.blocks.device}, "
                             "of one type and equal strides, channels contiguous")
        return shape[0], (stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0)

    def append(self, layer: int, k, v, positions, seqs=None, k_values=None, v_values=None) -> None:
        """Stores rows of K and V ([n][n_kv_heads][head_dim]) at positions (int32 [n]) of sequences seqs (int32 [n];
        None: row i is sequence i).  k_values / v_values (of k's strides; may be k and v) receive the stored values."""
        func = "QuantCache.append"
        n, stride = self._check_rows(func, k, v)
        kv = vv = None
        if k_values is not None or v_values is not None:
            if k_values is None or v_values is None:
                raise ValueError(f"{func}: k_values and v_values are given together")
            if self._check_rows(func, k_values, v_values) != (n, stride) or k_values.dtype != k.dtype:
                raise ValueError(f"{func}: k_values and v_values must be laid out as k")
            kv, vv = k_values.data_ptr(), v_values.data_ptr()
        index = self._index
        _on_device(func, "hs_kvq_append", index, self._ref, layer, _dtype_code(func, k), n, k.data_ptr(), v.data_ptr(),
                   stride[0], stride[1], _int32(func, "seqs", seqs, n, index),
                   _int32(func, "positions", positions, n, index), kv, vv)

    def read(self, layer: int, positions, dtype, seqs=None, k=None, v=None):
        """The rows at positions of sequences seqs, as (k, v) of a torch dtype (or into k and v)."""
        import torch
        func = "QuantCache.read"
        n, index = positions.numel(), self._index
        if k is None:
            k = torch.empty((n, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.blocks.device)
        if v is None:
            v = torch.empty_like(k) if k.is_contiguous() else torch.empty_strided(k.shape, k.stride(), dtype=k.dtype,
                                                                                 device=k.device)
        rows, stride = self._check_rows(func, k, v)
        if rows != n or k.dtype != dtype:
            raise ValueError(f"{func}: k and v must hold {n} rows of {dtype}")
        _on_device(func, "hs_kvq_read", index, self._ref, layer, _dtype_code(func, k), n, k.data_ptr(), v.data_ptr(),
                   stride[0], stride[1], _int32(func, "seqs", seqs, n, index),
                   _int32(func, "positions", positions, n, index))
        return k, v

    def _workspace_bytes(self, dt: int, n: int, n_heads: int, max_len: int) -> int:
        out = ctypes.c_uint64()
        _call("hs_kvq_attention_workspace", self._ref, dt, n, n_heads, max_len, ctypes.byref(out))
        return out.value

    def attention_workspace(self, n: int, n_heads: int, max_len: int, dtype=None):
        """A workspace for attention over n rows of n_heads heads and max_len positions (dtype None: of any type)."""
        import torch
        codes = range(HS_F32, HS_BF16 + 1) if dtype is None else (_dtype_code("QuantCache.attention_workspace",
                                                                              torch.empty(0, dtype=dtype)),)
        most = max(self._workspace_bytes(dt, n, n_heads, max_len) for dt in codes)
        return torch.zeros(most, dtype=torch.uint8, device=self.blocks.device)

    def attention(self, layer: int, q, lengths, seqs=None, max_len=None, scale=None, out=None, workspace=None):
        """Decode attention of q ([n][n_heads][head_dim]) over the first lengths (int32 [n]) positions of sequences
        seqs; max_len bounds the lengths (None: what the table holds), scale None: head_dim ** -0.5.  A workspace
        (attention_workspace) may be kept from call to call, which saves clearing a new one; calls on several streams
        do not share one."""
        import torch
        func = "QuantCache.attention"
        index, hd, shape, stride = self._index, self.head_dim, q.shape, q.stride()
        if len(shape) != 3 or shape[2] != hd or stride[2] != 1 or (shape[1] > 1 and stride[1] != hd) or \
                q.get_device() != index:
            raise ValueError(f"{func}: q must be [n][n_heads][{hd}] on {self.blocks.device}, each row contiguous")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != shape or out.dtype != q.dtype or out.get_device() != index or out.stride(2) != 1 or \
                (shape[1] > 1 and out.stride(1) != hd):
            raise ValueError(f"{func}: out must be of q's shape and type, each row contiguous")
        n, heads, dt = shape[0], shape[1], _dtype_code(func, q)
        if max_len is None:
            max_len = min(self.table.shape[1] * self.block_tokens, 1 << 30)
        if workspace is None:
            workspace = torch.empty(self._workspace_bytes(dt, n, heads, max_len), dtype=torch.uint8,
                                    device=self.blocks.device)
            if workspace.numel():
                workspace[:2048].zero_()
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError(f"{func}: workspace must be contiguous on {self.blocks.device}")
        _on_device(func, "hs_kvq_attention", index, self._ref, layer, dt, n, heads, q.data_ptr(), stride[0],
                   _int32(func, "seqs", seqs, n, index), _int32(func, "lengths", lengths, n, index), max_len,
                   hd ** -0.5 if scale is None else scale, out.data_ptr(), out.stride(0), workspace.data_ptr(),
                   workspace.nbytes)
        return out


def rope_frequencies(theta: float, n_pairs: int, device="cuda"):
    """theta^(-i / n_pairs) for the n_pairs pairs of a rotation, in float64."""
    import torch
    return theta ** (-torch.arange(n_pairs, dtype=torch.float64, device=device) / n_pairs)


class Rope:
    """A rotation by position (hs_rope): pair i of a head's channels, (i, i + pairs) or, with adjacent, (2 i, 2 i + 1),
    is turned by position[axes[i]] * frequencies[i].  frequencies: contiguous float64 [pairs], pairs a multiple of 8;
    axes: contiguous int32 [pairs] (None: one axis); n_axes: how many axes there are (None: what axes names, which is
    looked up once, here)."""

    def __init__(self, frequencies, axes=None, adjacent: bool = False, n_axes=None):
        import torch
        if frequencies.dtype is not torch.float64 or frequencies.dim() != 1 or not frequencies.is_contiguous():
            raise ValueError("Rope: frequencies must be a contiguous float64 vector")
        self._index, pairs = frequencies.get_device(), frequencies.numel()
        at = _int32("Rope", "axes", axes, pairs, self._index)
        if n_axes is None:
            n_axes = 1 if axes is None else int(axes.max()) + 1
        self.frequencies, self.axes, self.n_axes = frequencies, axes, n_axes  # keeps the tensors alive
        self._c = hs_rope(frequencies.data_ptr(), at, pairs, n_axes, int(adjacent))
        self._ref = ctypes.addressof(self._c)


def paged_block_bytes(dtype, n_layers: int, n_kv_heads: int, head_dim: int, block_tokens: int) -> int:
    """Bytes of one block of a paged cache of a torch dtype."""
    import torch
    out = ctypes.c_uint64()
    _call("hs_paged_block_bytes", _dtype_code("paged_block_bytes", torch.empty(0, dtype=dtype)), n_layers, n_kv_heads,
          head_dim, block_tokens, ctypes.byref(out))
    return out.value


class PagedCache:
    """A paged KV cache in the model's own type (hs_paged_cache) over caller-owned tensors: blocks, contiguous
    [blocks][layers][2][n_kv_heads][block_tokens][head_dim] of float32, float16 or bfloat16, and table, a contiguous
    int64 tensor [sequences][blocks per sequence] of block numbers, negative where there is none.  The table may be
    rewritten between calls, and sequences may share blocks."""

    def __init__(self, blocks, table):
        import torch
        if blocks.dim() != 6 or blocks.shape[2] != 2 or not blocks.is_contiguous():
            raise ValueError("PagedCache: blocks must be contiguous [blocks][layers][2][n_kv_heads][block_tokens]"
                             "[head_dim]")
        if table.dtype is not torch.int64 or table.dim() != 2 or not table.is_contiguous() or \
                table.device != blocks.device:
            raise ValueError("PagedCache: table must be a contiguous int64 matrix on the blocks' device")
        self.dtype = blocks.dtype
        _, self.n_layers, _, self.n_kv_heads, self.block_tokens, self.head_dim = blocks.shape
        paged_block_bytes(self.dtype, self.n_layers, self.n_kv_heads, self.head_dim, self.block_tokens)  # checks
        self.blocks, self.table = blocks, table  # keeps the tensors alive
        self._index, self._align = blocks.get_device(), 16 // blocks.element_size()
        self._c = hs_paged_cache(blocks.data_ptr(), blocks.nbytes, table.data_ptr(), table.shape[0], table.shape[1],
                                 self.n_layers, self.n_kv_heads, self.head_dim, self.block_tokens,
                                 _dtype_code("PagedCache", blocks))
        self._ref = ctypes.addressof(self._c)

    def _rows(self, func: str, name: str, t, n, heads):
        """Strides of t ([n][heads][head_dim], channels contiguous); those of a single row or head, which nothing
        uses, as 0."""
        shape, stride = t.shape, t.stride()
        if len(shape) != 3 or (n is not None and shape[0] != n) or (heads is not None and shape[1] != heads) or \
                shape[2] != self.head_dim or stride[2] != 1 or t.dtype is not self.dtype or \
                t.get_device() != self._index:
            raise ValueError(f"{func}: {name} must be [{'n' if n is None else n}][{heads or 'heads'}]"
                             f"[{self.head_dim}] of {self.dtype} on {self.blocks.device}, channels contiguous")
        return stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0

    def append(self, layer: int, k, v, positions, seqs=None, q=None, rope=None, angles_at=None, q_gain=None,
               k_gain=None, eps: float = 1e-6, q_out=None):
        """Stores rows of K and V ([n][n_kv_heads][head_dim]) at positions (int32 [n]) of sequences seqs (int32 [n];
        None: row i is sequence i), K normalised with k_gain ([head_dim]; None: not) and turned by rope (None: not) at
        angles_at (int32 [axes][n]; None: positions).  Queries q ([n][heads][head_dim]) are normalised and turned
        alike into q_out (None: a new tensor; may be q), which is returned."""
        import torch
        func = "PagedCache.append"
        n, index = k.shape[0], self._index
        ld, ldh = self._rows(func, "k", k, None, self.n_kv_heads)
        if self._rows(func, "v", v, n, self.n_kv_heads) != (ld, ldh):
            raise ValueError(f"{func}: k and v must have equal strides")
        heads = lq = lqh = lo = loh = 0
        if q is not None:
            lq, lqh = self._rows(func, "q", q, n, None)
            heads = q.shape[1]
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            lo, loh = self._rows(func, "q_out", q_out, n, heads)
        elif q_out is not None or q_gain is not None:
            raise ValueError(f"{func}: q_out and q_gain are given with q")
        for name, t in (("q_gain", q_gain), ("k_gain", k_gain)):
            if t is not None and (t.dtype is not self.dtype or t.shape != (self.head_dim,) or not t.is_contiguous() or
                                  t.get_device() != index):
                raise ValueError(f"{func}: {name} must be {self.head_dim} contiguous values of {self.dtype}")
        ref = None
        if rope is not None:
            if rope._index != index:
                raise ValueError(f"{func}: the rope's tensors must be on {self.blocks.device}")
            ref = rope._ref
        elif angles_at is not None:
            raise ValueError(f"{func}: angles_at is given with a rope")
        _on_device(func, "hs_paged_append", index, self._ref, layer, n, heads, None if q is None else q.data_ptr(), lq,
                   lqh, None if q_out is None else q_out.data_ptr(), lo, loh, k.data_ptr(), v.data_ptr(), ld, ldh,
                   _int32(func, "seqs", seqs, n, index), _int32(func, "positions", positions, n, index), ref,
                   None if rope is None else _int32(func, "angles_at", angles_at, rope.n_axes * n, index),
                   None if q_gain is None else q_gain.data_ptr(), None if k_gain is None else k_gain.data_ptr(), eps)
        return q_out

    def _workspace_bytes(self, n: int, n_heads: int, max_len: int, n_groups: int, max_shared: int) -> int:
        out = ctypes.c_uint64()
        _call("hs_paged_attention_workspace", self._ref, n, n_heads, max_len, n_groups, max_shared, ctypes.byref(out))
        return out.value

    def attention_workspace(self, n: int, n_heads: int, max_len: int, n_groups: int = 0, max_shared: int = 0):
        """A workspace for attention over n rows of n_heads heads, max_len positions, n_groups groups of rows and
        max_shared shared positions."""
        import torch
        return torch.empty(self._workspace_bytes(n, n_heads, max_len, n_groups, max_shared), dtype=torch.uint8,
                           device=self.blocks.device)

    def attention(self, layer: int, q, lengths, seqs=None, group_starts=None, shared=None, max_len=None,
                  max_shared=None, scale=None, out=None, workspace=None):
        """Attention of q ([n][n_heads][head_dim]) over the first lengths (int32 [n]) positions of sequences seqs.
        Rows group_starts[g] .. group_starts[g + 1] - 1 (int32 [groups + 1], not falling) have their first shared[g]
        (int32 [groups]) positions in common, which are read once, through the first row's sequence.  max_len bounds
        the lengths (None: what the table holds), max_shared the shared positions (None: max_len; near what is shared it
        is faster, as rows' own positions are split by max_len - max_shared); scale None:
        head_dim ** -0.5.  A workspace (attention_workspace) may be kept from call to call; calls on several streams
        do not share one."""
        import torch
        func = "PagedCache.attention"
        index, hd = self._index, self.head_dim
        ld, ldh = self._rows(func, "q", q, None, None)
        n, heads = q.shape[0], q.shape[1]
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lo, loh = self._rows(func, "out", out, n, heads)
        if heads > 1 and (ldh != hd or loh != hd):
            raise ValueError(f"{func}: each row of q and out must be contiguous")
        groups = 0
        if group_starts is not None or shared is not None:
            if group_starts is None or shared is None:
                raise ValueError(f"{func}: group_starts and shared are given together")
            groups = shared.numel()
        if max_len is None:
            max_len = min(self.table.shape[1] * self.block_tokens, 1 << 30)
        if max_shared is None:
            max_shared = max_len if groups else 0
        if workspace is None:
            workspace = torch.empty(self._workspace_bytes(n, heads, max_len, groups, max_shared), dtype=torch.uint8,
                                    device=self.blocks.device)
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError(f"{func}: workspace must be contiguous on {self.blocks.device}")
        _on_device(func, "hs_paged_attention", index, self._ref, layer, n, heads, q.data_ptr(), ld,
                   _int32(func, "seqs", seqs, n, index), _int32(func, "lengths", lengths, n, index), groups,
                   _int32(func, "group_starts", group_starts, groups + 1, index),
                   _int32(func, "shared", shared, groups, index), max_len, max_shared,
                   hd ** -0.5 if scale is None else scale, out.data_ptr(), lo, workspace.data_ptr(), workspace.nbytes)
        return out


def _sample_bytes(rows: int, vocab: int) -> int:
    out = ctypes.c_uint64()
    _call("hs_sample_tokens_workspace", rows, vocab, ctypes.byref(out))
    return out.value


def sample_tokens_workspace(rows: int, vocab: int, device="cuda"):
    """A workspace for sample_tokens over rows of vocab logits, which may be kept from call to call."""
    import torch
    return torch.empty(_sample_bytes(rows, vocab), dtype=torch.uint8, device=device)


def sample_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, workspace=None):
    """(tokens, logprob) of rows of logits ([rows][vocab]; float32, float16 or bfloat16): a token (int32) for each row,
    drawn with the row's uniform number u (float32 [rows], in [0, 1)), and its log probability among the tokens that the
    row's temperature, top_p, min_p (float32 [rows]) and top_k (int32 [rows]) leave, each None for none.  Of the logits
    in falling order the first top_k stay, of these the shortest beginning with top_p of their weight, of these the
    ones with at least min_p of the largest weight; temperature 0 takes the largest logit.  A row without a distribution
    has token -1 and logprob NaN.  tokens: written there (None: a new tensor)."""
    import torch
    func = "sample_tokens"
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"{func}: logits must be [rows][vocab], each row contiguous")
    rows, vocab = logits.shape
    index, dt = logits.get_device(), _dtype_code(func, logits)
    if u is None:
        raise ValueError(f"{func}: u must be {rows} contiguous float32 values")
    at = [_float32(func, name, t, rows, index) for name, t in
          (("u", u), ("temperature", temperature), ("top_p", top_p), ("min_p", min_p))]
    tk = _int32(func, "top_k", top_k, rows, index)
    if tokens is None:
        tokens = logits.new_empty((rows,), dtype=torch.int32)
    out = _int32(func, "tokens", tokens, rows, index)
    logprob = torch.empty_like(u)
    if workspace is None:
        workspace = logits.new_empty((_sample_bytes(rows, vocab),), dtype=torch.uint8)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"{func}: workspace must be contiguous on the logits' device")
    _on_device(func, "hs_sample_tokens", index, dt, logits.data_ptr(), rows, vocab, logits.stride(0), at[0], at[1], tk,
               at[2], at[3], out, logprob.data_ptr(), workspace.data_ptr(), workspace.nbytes)
    return tokens, logprob


def _logprobs_bytes(rows: int, vocab: int, top: int) -> int:
    out = ctypes.c_uint64()
    _call("hs_token_logprobs_workspace", rows, vocab, top, ctypes.byref(out))
    return out.value


def token_logprobs_workspace(rows: int, vocab: int, top: int = 0, device="cuda"):
    """A workspace for token_logprobs over rows of vocab logits, which may be kept from call to call."""
    import torch
    return torch.zeros(_logprobs_bytes(rows, vocab, top), dtype=torch.uint8, device=device)


def token_logprobs(logits, tokens=None, top: int = 0, workspace=None):
    """(logprob, entropy, top_ids, top_logprobs) of rows of logits ([rows][vocab]; float32, float16 or bfloat16):
    the log probability of each row's given token (int32 [rows]; a negative one asks for none and gives 0; None: no
    logprob), the row's entropy in nats, and its `top` most probable tokens with their log probabilities
    ([rows][top]; None without)."""
    import torch
    func = "token_logprobs"
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"{func}: logits must be [rows][vocab], each row contiguous")
    rows, vocab = logits.shape
    index, dt = logits.get_device(), _dtype_code(func, logits)
    tk = _int32(func, "tokens", tokens, rows, index)
    lp = None if tokens is None else torch.empty_like(tokens, dtype=torch.float32)
    entropy = logits.new_empty((rows,), dtype=torch.float32) if lp is None else torch.empty_like(lp)
    ids = tops = None
    if top > 0:
        tops = logits.new_empty((rows, top), dtype=torch.float32)
        ids = torch.empty_like(tops, dtype=torch.int32)
    if workspace is None:
        workspace = logits.new_empty((_logprobs_bytes(rows, vocab, top),), dtype=torch.uint8)
        if workspace.numel():
            workspace[:2048].zero_()
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"{func}: workspace must be contiguous on the logits' device")
    _on_device(func, "hs_token_logprobs", index, dt, logits.data_ptr(), rows, vocab, logits.stride(0), tk, top,
               None if lp is None else lp.data_ptr(), entropy.data_ptr(), None if ids is None else ids.data_ptr(),
               None if tops is None else tops.data_ptr(), workspace.data_ptr(), workspace.nbytes)
    return lp, entropy, ids, tops


class Handoff:
    """Aligned batch handoff: requests whose embeddings have arrived wait in
    arrival order until a batch of `align` requests (or the row budget, or
    the oldest request's timeout) is due for prefill."""

    def __init__(self, align: int = 32, max_rows: int = 0, max_pending: int = 4096, timeout_ms: float = 500.0):
        self.align = align
        h = ctypes.c_void_p()
        _call("hs_handoff_create", align, max_rows, max_pending, timeout_ms, ctypes.byref(h))
        self.handle = h

    def push(self, req: int, rows: int, now_ms: float) -> None:
        _call("hs_handoff_push", self.handle, req, rows, now_ms)

    def pop(self, now_ms: float):
        """(requests of the due batch or [], their rows, ms until the next timeout or -1)."""
        out = (ctypes.c_int32 * self.align)()
        n, rows, wait = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_double()
        _call("hs_handoff_pop", self.handle, now_ms, out, self.align, ctypes.byref(n), ctypes.byref(rows),
              ctypes.byref(wait))
        return list(out[:n.value]), rows.value, wait.value

    def pending(self) -> int:
        n = ctypes.c_int32()
        _call("hs_handoff_pending", self.handle, ctypes.byref(n))
        return n.value

    def close(self) -> None:
        if self.handle:
            _call("hs_handoff_free", self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
