"""ctypes binding of the cache and attention entry points of libgorgo.so: the paged key-value cache of a replica's layer, and
the attention of prompts and of single tokens over it.  Argument marshalling only; torch tensors are device memory."""
from __future__ import annotations

import ctypes as C
from typing import Optional

from .binding import GorgoError, _check, lib


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("type", C.c_int32),
                ("pages", C.c_int32), ("page_tokens", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("_pad", C.c_int32),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


class _Batch(C.Structure):
    _fields_ = [("sequences", C.c_int32), ("tokens", C.c_int32), ("table_columns", C.c_int32), ("_pad", C.c_int32),
                ("page_table", C.c_void_p), ("lengths", C.c_void_p), ("token_offsets", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Attention(C.Structure):
    _fields_ = [("q_heads", C.c_int32), ("window", C.c_int32), ("scale", C.c_float), ("_pad", C.c_int32)]


_COUNTS = 2048                       # bytes of a workspace that have to be zero before its first call
_declared = None


def _lib():
    global _declared
    if _declared is None:
        L, vp, p = lib(), C.c_void_p, C.POINTER
        for f in (L.gorgo_kv_write, L.gorgo_kv_read):
            f.argtypes, f.restype = [p(_Cache), p(_Batch), p(_Rows), p(_Rows), vp], C.c_int
        for f in (L.gorgo_attend_prompt, L.gorgo_attend_token):
            f.argtypes, f.restype = [p(_Cache), p(_Batch), p(_Attention), p(_Rows), p(_Rows), vp, vp, C.c_size_t, vp], C.c_int
        L.gorgo_attend_workspace_bytes.argtypes, L.gorgo_attend_workspace_bytes.restype = [p(_Cache), p(_Batch), C.c_int32, p(C.c_size_t)], C.c_int
        _declared = L
    return _declared


def _invalid(msg: str):
    raise GorgoError(-1, msg)


def _strides(t):
    """Strides, 0 for dimensions of one element: theirs may be any number, and none of them is taken."""
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape, t.stride()))


def _no_gradient(t, name: str):
    """Refuses a tensor through which somebody waits for a gradient: there is no backward pass, and results would not say so."""
    if t.requires_grad:
        import torch
        if torch.is_grad_enabled():
            _invalid(f"{name} requires a gradient, and nothing here has a backward pass: detach it, or call under torch.no_grad()")


class KvCache:
    """A layer's paged cache over the caller's tensors (gorgo_kv_cache): k and v [pages, kv_heads, page_tokens, head_dim] in
    bfloat16, float16 or 8 bits (float8_e4m3fn or uint8, with k_scale and v_scale uint8 [pages, kv_heads, page_tokens]), any
    strides whose last is 1, the same for both.  The tensors are kept alive by the object."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        import torch
        types = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2, torch.uint8: 2}
        if k.dim() != 4 or k.shape != v.shape or _strides(k) != _strides(v) or k.dtype != v.dtype or k.device != v.device:
            _invalid("k and v must be [pages, kv_heads, page_tokens, head_dim] tensors of one shape, type, device and layout")
        if k.dtype not in types:
            _invalid("the cache must be bfloat16, float16, float8_e4m3fn or uint8 (e4m3)")
        for t, name in ((k, "k"), (v, "v")):
            _no_gradient(t, name)
        if k.device.type != "cuda":
            _invalid("the cache must be on the GPU")
        if k.stride(3) != 1 and k.shape[3] > 1:
            _invalid("the values of a row must lie side by side")
        self.type = types[k.dtype]
        if self.type == 2:
            for s in (k_scale, v_scale):
                if s is None or s.dtype != torch.uint8 or s.shape != k.shape[:3] or not s.is_contiguous() or s.device != k.device:
                    _invalid("an e4m3 cache needs k_scale and v_scale, contiguous uint8 [pages, kv_heads, page_tokens]")
        elif k_scale is not None or v_scale is not None:
            _invalid("only an e4m3 cache has scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = torch.device("cuda", k.device.index)
        self.pages, self.kv_heads, self.page_tokens, self.head_dim = k.shape
        self.row_dtype = torch.float16 if self.type == 1 else torch.bfloat16
        self._c = _Cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if self.type == 2 else None,
                         v_scale.data_ptr() if self.type == 2 else None, self.type, self.pages, self.page_tokens, self.kv_heads, self.head_dim, 0,
                         *_strides(k)[:3])
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page_tokens: int = 512, dtype: str = "bf16", device="cuda:0") -> "KvCache":
        """A cache of its own: "bf16", "fp16" or "e4m3"; a page is a cache block of the traces (512 tokens)."""
        import torch
        types = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
        if dtype not in types:
            _invalid("dtype must be bf16, fp16 or e4m3")
        k, v = (torch.empty((pages, kv_heads, page_tokens, head_dim), dtype=types[dtype], device=device) for _ in range(2))
        if dtype != "e4m3":
            return cls(k, v)
        scales = (torch.ones((pages, kv_heads, page_tokens), dtype=torch.uint8, device=device) for _ in range(2))
        return cls(k, v, *scales)


class KvBatch:
    """The sequences of a call (gorgo_kv_batch): page_table int32 [sequences, columns], lengths int32 [sequences] (tokens with the
    new ones), token_offsets int32 [sequences + 1] of the packed new tokens, or None for one token each.  `tokens` is the number of
    packed rows, token_offsets[-1]; max_tokens, if known, the most new tokens of a sequence, which `tokens` is checked against and
    nothing else (the kernels find their work from the offsets alone).  The tensors are read when a call runs: refill them in place for the next step, or replay a
    captured graph with them."""

    def __init__(self, page_table, lengths, token_offsets=None, tokens: Optional[int] = None, max_tokens: Optional[int] = None):
        import torch
        if page_table.dim() != 2 or lengths.dim() != 1 or page_table.shape[0] != lengths.shape[0]:
            _invalid("page_table must be [sequences, columns] and lengths [sequences]")
        S = lengths.shape[0]
        if token_offsets is not None and tuple(token_offsets.shape) != (S + 1,):
            _invalid("token_offsets must be [sequences + 1]")
        for t in (page_table, lengths, token_offsets):
            if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or t.device.type != "cuda" or t.device != lengths.device):
                _invalid("page_table, lengths and token_offsets must be contiguous int32 tensors on one GPU")
        if token_offsets is None:
            tokens = S if tokens is None else tokens
        elif tokens is None:
            _invalid("tokens (token_offsets[-1]) must be given with token_offsets")
        if max_tokens is not None and not 0 <= int(tokens) <= S * int(max_tokens):
            _invalid("tokens must be in 0 .. sequences * max_tokens")
        self.page_table, self.lengths, self.token_offsets, self.tokens, self.sequences = page_table, lengths, token_offsets, int(tokens), S
        self.max_tokens = self.tokens if max_tokens is None else int(max_tokens)
        self.device = lengths.device
        self._c = _Batch(S, self.tokens, page_table.shape[1], 0, page_table.data_ptr(), lengths.data_ptr(),
                         None if token_offsets is None else token_offsets.data_ptr())
        self._ref = C.byref(self._c)


def _rows(t, heads: int, cache: KvCache, batch: KvBatch, name: str) -> _Rows:
    if t.shape != (batch.tokens, heads, cache.head_dim):
        _invalid(f"{name} must be [{batch.tokens}, {heads}, {cache.head_dim}]")
    if t.dtype != cache.row_dtype or t.device != cache.device:
        _invalid(f"{name} must be {cache.row_dtype} on {cache.device}")
    _no_gradient(t, name)
    stride = t.stride()
    if stride[2] != 1:
        _invalid(f"the values of a row of {name} must lie side by side")
    return _Rows(t.data_ptr(), stride[0] if batch.tokens > 1 else 0, stride[1] if heads > 1 else 0)


def _new_rows(heads: int, cache: KvCache, batch: KvBatch, stream):
    """A tensor of rows, and what describes it."""
    t = _empty((batch.tokens, heads, cache.head_dim), cache.row_dtype, cache.device, stream)
    return t, _Rows(t.data_ptr(), heads * cache.head_dim, cache.head_dim)


def _call(device, f, args, stream):
    """Runs f on `stream`, or on the device's current one."""
    import torch
    index = device.index
    s = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        _check(f(*args, s))
    else:
        with torch.cuda.device(index):
            _check(f(*args, s))


def _empty(shape, dtype, device, stream):
    """A tensor of the stream that is going to write it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _same_device(cache: KvCache, batch: KvBatch):
    if cache.device != batch.device:
        _invalid("cache and batch must be on one GPU")


def kv_write(cache: KvCache, batch: KvBatch, k, v, stream=None) -> None:
    """gorgo_kv_write: the new tokens' keys and values [tokens, kv_heads, head_dim] into their pages."""
    _same_device(cache, batch)
    rk, rv = _rows(k, cache.kv_heads, cache, batch, "k"), _rows(v, cache.kv_heads, cache, batch, "v")
    _call(cache.device, _lib().gorgo_kv_write, (cache._ref, batch._ref, C.byref(rk), C.byref(rv)), stream)


def kv_read(cache: KvCache, batch: KvBatch, out=None, stream=None):
    """gorgo_kv_read: the batch's tokens as (k, v), [tokens, kv_heads, head_dim] each, in the cache's type (bf16 of an e4m3 cache).
    out: a pair of tensors to write to."""
    _same_device(cache, batch)
    if out is None:
        k, rk = _new_rows(cache.kv_heads, cache, batch, stream)
        v, rv = _new_rows(cache.kv_heads, cache, batch, stream)
        out = (k, v)
    else:
        rk, rv = _rows(out[0], cache.kv_heads, cache, batch, "out[0]"), _rows(out[1], cache.kv_heads, cache, batch, "out[1]")
    _call(cache.device, _lib().gorgo_kv_read, (cache._ref, batch._ref, C.byref(rk), C.byref(rv)), stream)
    return out


def attend_workspace_bytes(cache: KvCache, batch: KvBatch, q_heads: int) -> int:
    n = C.c_size_t()
    _check(_lib().gorgo_attend_workspace_bytes(cache._ref, batch._ref, q_heads, C.byref(n)))
    return n.value


def attend_workspace(cache: KvCache, batch: KvBatch, q_heads: int):
    """A workspace that fits every attention call with this cache and q_heads and batches of at most this one's sequences, tokens and
    columns, its counts zero as the first call wants them; keep it for the calls of one stream."""
    import torch
    workspace = torch.empty((attend_workspace_bytes(cache, batch, q_heads),), dtype=torch.uint8, device=cache.device)
    workspace[:_COUNTS].zero_()
    return workspace


def _attend(f, cache, batch, q, scale, window, lse, out, workspace, stream):
    import torch
    _same_device(cache, batch)
    if q.dim() != 3 or q.shape[1] % cache.kv_heads:
        _invalid("q must be [tokens, q_heads, head_dim], q_heads a multiple of the cache's heads")
    heads = q.shape[1]
    rq = _rows(q, heads, cache, batch, "q")
    if out is None:
        out, ro = _new_rows(heads, cache, batch, stream)
    else:
        ro = _rows(out, heads, cache, batch, "out")
    if lse is True:
        lse = _empty((batch.tokens, heads), torch.float32, cache.device, stream)
    elif lse is False:
        lse = None
    if lse is not None and (tuple(lse.shape) != (batch.tokens, heads) or lse.dtype != torch.float32 or not lse.is_contiguous()
                            or lse.device != cache.device):
        _invalid("lse must be a contiguous float32 tensor [tokens, q_heads]")
    if lse is not None:
        _no_gradient(lse, "lse")
    if workspace is None:
        with torch.cuda.stream(stream):
            workspace = attend_workspace(cache, batch, heads)
    elif workspace.device != cache.device or not workspace.is_contiguous():
        _invalid("workspace must be a contiguous tensor on the cache's GPU")
    how = _Attention(heads, window, cache.head_dim ** -0.5 if scale is None else scale, 0)
    _call(cache.device, f, (cache._ref, batch._ref, C.byref(how), C.byref(rq), C.byref(ro), None if lse is None else lse.data_ptr(),
                            workspace.data_ptr(), workspace.nbytes), stream)
    return out if lse is None else (out, lse)


def attend_prompt(cache: KvCache, batch: KvBatch, q, *, scale: Optional[float] = None, window: int = 0, lse=False, out=None,
                  workspace=None, stream=None):
    """gorgo_attend_prompt: causal attention of the new tokens' queries [tokens, q_heads, head_dim] over their sequences in the
    cache (keys and values written before, their own included).  scale: head_dim ** -0.5 if None.  lse: True (or a tensor) for
    the rows' log of sums as well.  Asynchronous on `stream` (default: torch's current stream)."""
    return _attend(_lib().gorgo_attend_prompt, cache, batch, q, scale, window, lse, out, workspace, stream)


def attend_token(cache: KvCache, batch: KvBatch, q, *, scale: Optional[float] = None, window: int = 0, lse=False, out=None,
                 workspace=None, stream=None):
    """gorgo_attend_token: attend_prompt for one new token of each sequence (a batch without token_offsets)."""
    return _attend(_lib().gorgo_attend_token, cache, batch, q, scale, window, lse, out, workspace, stream)
