"""ctypes binding of the cache and attention entry points of libgorgo.so: the paged key-value cache of a replica's layer, the norms and
the rotation of heads on their way into it, and the attention of prompts and of single tokens over it.  Argument marshalling only; torch tensors are device memory."""
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
    _fields_ = [("q_heads", C.c_int32), ("window", C.c_int32), ("scale", C.c_float), ("sinks", C.c_int32)]


class _Rotation(C.Structure):
    _fields_ = [("frequencies", C.c_void_p), ("positions", C.c_void_p), ("axis_stride", C.c_int64), ("pairs", C.c_int32), ("layout", C.c_int32),
                ("axes", C.c_int32), ("magnitude", C.c_float), ("axis_of_pair", C.c_uint8 * 64)]


class _Norm(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("head_stride", C.c_int64), ("eps", C.c_float), ("_pad", C.c_int32)]


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
        L.gorgo_kv_append.argtypes = [p(_Cache), p(_Batch), p(_Rotation), p(_Norm), p(_Norm), C.c_int32] + [p(_Rows)] * 4 + [vp]
        L.gorgo_rotate_heads.argtypes = [p(_Batch), p(_Rotation), p(_Norm)] + [C.c_int32] * 3 + [p(_Rows)] * 2 + [vp]
        L.gorgo_kv_append.restype = L.gorgo_rotate_heads.restype = C.c_int
        L.gorgo_attend_workspace_bytes.argtypes, L.gorgo_attend_workspace_bytes.restype = [p(_Cache), p(_Batch), C.c_int32, p(C.c_size_t)], C.c_int
        _declared = L
    return _declared


def _invalid(msg: str):
    raise GorgoError(-1, msg)


def _int32(n, name: str) -> int:
    """A count for the library, which takes 32 bits: one that they do not hold is refused, not cut off."""
    if not -2 ** 31 <= n < 2 ** 31:
        _invalid(f"{name} must fit 32 bits")
    return n


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
        _int32(int(tokens), "tokens")
        if max_tokens is not None and not 0 <= int(tokens) <= S * int(max_tokens):
            _invalid("tokens must be in 0 .. sequences * max_tokens")
        self.page_table, self.lengths, self.token_offsets, self.tokens, self.sequences = page_table, lengths, token_offsets, int(tokens), S
        self.max_tokens = self.tokens if max_tokens is None else int(max_tokens)
        self.device = lengths.device
        self._c = _Batch(S, self.tokens, page_table.shape[1], 0, page_table.data_ptr(), lengths.data_ptr(),
                         None if token_offsets is None else token_offsets.data_ptr())
        self._ref = C.byref(self._c)


class Rotation:
    """Rotation of heads by positions (gorgo_rotation).  frequencies: float64 [pairs] on the GPU, radians from a position to the next
    (Rotation.of_base computes the usual ones).  positions: int32 [tokens], or [axes, tokens] with axis_of_pair, a list of which axis turns each
    pair; None: a token's place in its sequence.  layout: pair i is the values i and i + pairs ("halves") or 2 i and 2 i + 1
    ("neighbours").  magnitude multiplies the rotated values.  The tensors are kept alive by the object and read when a call runs:
    refill the positions in place for the next step, or replay a captured graph with them."""

    def __init__(self, frequencies, positions=None, *, axis_of_pair=None, layout: str = "halves", magnitude: float = 1.0):
        import torch
        layouts = {"halves": 0, "neighbours": 1}
        if layout not in layouts:
            _invalid("layout must be halves or neighbours")
        if frequencies.dim() != 1 or frequencies.dtype != torch.float64 or not frequencies.is_contiguous() or frequencies.device.type != "cuda":
            _invalid("frequencies must be a contiguous float64 tensor [pairs] on the GPU")
        pairs = frequencies.shape[0]
        if not 1 <= pairs <= 64:
            _invalid("there must be 1 to 64 frequencies")
        _no_gradient(frequencies, "frequencies")
        axes, stride = 1, 0
        if positions is not None:
            if positions.dim() not in (1, 2) or positions.dtype != torch.int32 or positions.device != frequencies.device:
                _invalid("positions must be int32 [tokens] or [axes, tokens] on the frequencies' GPU")
            if positions.shape[-1] > 1 and positions.stride(-1) != 1:
                _invalid("an axis's positions must lie side by side")
            if positions.dim() == 2:
                axes, stride = positions.shape[0], positions.stride(0) if positions.shape[0] > 1 else 0
        if not 1 <= axes <= 4:
            _invalid("positions must have 1 to 4 axes")
        axis_of_pair = [0] * pairs if axis_of_pair is None else [int(i) for i in axis_of_pair]
        if len(axis_of_pair) != pairs or not all(0 <= i < axes for i in axis_of_pair):
            _invalid("axis_of_pair must name one of the positions' axes for each pair")
        self.frequencies, self.positions, self.pairs, self.axes, self.layout, self.magnitude = frequencies, positions, pairs, axes, layout, float(magnitude)
        self.device = torch.device("cuda", frequencies.device.index)
        self.tokens = None if positions is None else positions.shape[-1]
        self._c = _Rotation(frequencies.data_ptr(), None if positions is None else positions.data_ptr(), stride, pairs, layouts[layout], axes, self.magnitude,
                            (C.c_uint8 * 64)(*axis_of_pair))
        self._ref = C.byref(self._c)

    @classmethod
    def of_base(cls, pairs: int, base: float = 10000.0, positions=None, *, device="cuda:0", **how) -> "Rotation":
        """Frequencies base ** (-i / pairs)."""
        import torch
        return cls(base ** (-torch.arange(pairs, dtype=torch.float64, device=device) / pairs), positions, **how)


class HeadNorm:
    """Norm of each head's row by its root mean square (gorgo_norm).  weight: float32 [head_dim], or [heads, head_dim] for a row of each
    head's own (a model's 16-bit weights, converted once), None for ones."""

    def __init__(self, weight=None, eps: float = 1e-6):
        import torch
        if weight is not None:
            if weight.dim() not in (1, 2) or weight.dtype != torch.float32 or not weight.is_contiguous() or weight.device.type != "cuda":
                _invalid("the weight of a norm must be a contiguous float32 tensor [head_dim] or [heads, head_dim] on the GPU")
            _no_gradient(weight, "the weight of a norm")
        self.weight, self.eps = weight, float(eps)
        self.device = None if weight is None else torch.device("cuda", weight.device.index)
        own = weight is not None and weight.dim() == 2
        self._c = _Norm(None if weight is None else weight.data_ptr(), weight.shape[1] if own else 0, self.eps, 0)
        self._ref = C.byref(self._c)

    def _check(self, heads: int, head_dim: int, device, name: str):
        if self.weight is None:
            return
        shape = self.weight.shape
        if shape[-1] != head_dim or (len(shape) == 2 and shape[0] != heads):
            _invalid(f"the weight of {name} must be [{head_dim}] or [{heads}, {head_dim}]")
        if self.device != device:
            _invalid(f"the weight of {name} must be on {device}")


def _rows(t, heads: int, cache: KvCache, batch: KvBatch, name: str) -> _Rows:
    if t.shape != (batch.tokens, heads, cache.head_dim):
        _invalid(f"{name} must be [{batch.tokens}, {heads}, {cache.head_dim}]")
    if t.dtype != cache.row_dtype or t.device != cache.device:
        _invalid(f"{name} must be {cache.row_dtype} on {cache.device}")
    if t.requires_grad:
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


def _taken(rotation, tokens: int, head_dim: int, device):
    """Checks of a rotation for rows of these sizes."""
    if rotation is None:
        return
    if rotation.device != device:
        _invalid(f"the rotation must be on {device}")
    if rotation.tokens is not None and rotation.tokens != tokens:
        _invalid(f"there must be positions of {tokens} tokens")
    if 2 * rotation.pairs > head_dim:
        _invalid(f"heads of {head_dim} values have at most {head_dim // 2} pairs")


def _ref(x):
    return None if x is None else x._ref


def _near(x: int, step: int, lo: int, hi: int, width: int) -> bool:
    """Whether |x + n * step| < width for some whole n of lo .. hi."""
    n = -x // step if step else lo
    return any(abs(x + max(lo, min(hi, i)) * step) < width for i in (n, n + 1))


def _folds(rows, tokens: int, width: int) -> bool:
    """Whether rows (address, bytes from token to token, from head to head, heads) of `width` bytes overlap each other."""
    _, t, h, heads = rows
    if h >= width and (tokens == 1 or t >= (heads - 1) * h + width):
        return False                                  # (token by token, as nearly always)
    if (tokens > 1 and t < width) or (heads > 1 and h < width):
        return True
    return tokens > 1 and any(_near(n * h, t, 1 - tokens, tokens - 1, width) for n in range(1, heads))


def _touch(a, b, tokens: int, width: int) -> bool:
    """Whether rows a and rows b, each as above, have a byte in common."""
    (at, ta, ha, na), (to, tb, hb, nb) = a, b
    x, span_a, span_b = to - at, (na - 1) * ha + width, (nb - 1) * hb + width          # (spans of a token)
    if x >= (tokens - 1) * ta + span_a or -x >= (tokens - 1) * tb + span_b:
        return False

    if ta == tb:
        if ta > 0 and x % ta >= span_a and x % ta + span_b <= ta:
            return False                              # (parts of one row of heads: queries, keys and values of one product)
        apart = (n * ha for n in range(1 - na, nb)) if ha == hb else (j * hb - i * ha for i in range(na) for j in range(nb))
        return any(_near(x + n, ta, 1 - tokens, tokens - 1, width) for n in apart)
    for i in range(tokens):
        y = x - i * ta                                # tokens j of b that reach token i of a: -span_b < y + j * tb < span_a
        first, last = (0, 0) if tb == 0 else (max(0, (-span_b - y) // tb + 1), min(tokens - 1, (span_a - 1 - y) // tb))
        if any(_near(y + j * tb - n * ha, hb, 0, nb - 1, width) for j in range(first, last + 1) for n in range(na)):
            return True
    return False


def _no_overlap(out, x, others, tokens: int) -> None:
    """Refuses an `out` whose rows overlap each other or, but for x's own in place, rows that the call reads: its workgroups run side by side."""
    if tokens == 0:
        return

    def rows(t):
        stride = t.stride()
        return t.data_ptr(), stride[0] * 2 if tokens > 1 else 0, stride[1] * 2 if t.shape[1] > 1 else 0, t.shape[1]
    width, to = 2 * out.shape[2], rows(out)
    if _folds(to, tokens, width):
        _invalid("rows of out overlap each other")
    for t, name in others:
        of = rows(t)
        if _touch(to, of, tokens, width) and not (t is x and of == to):
            _invalid(f"out overlaps {name}" + (", and is not in its place" if t is x else ""))


def kv_append(cache: KvCache, batch: KvBatch, k, v, q=None, *, rotation: Optional[Rotation] = None, q_norm: Optional[HeadNorm] = None,
              k_norm: Optional[HeadNorm] = None, out=None, stream=None):
    """gorgo_kv_append: kv_write with keys that are normed and rotated on the way.  With q [tokens, q_heads, head_dim] the queries of the same tokens,
    normed and rotated, are returned, in `out` or a new tensor.  `out` may be q, row for row; otherwise its rows share no memory with q, k, v or each
    other (parts of one tensor that lie side by side do not).  Rows of tokens that belong to no sequence are not written: what they hold in a new
    tensor is undefined.  Asynchronous on `stream` (default: torch's current stream)."""
    _same_device(cache, batch)
    rk, rv = _rows(k, cache.kv_heads, cache, batch, "k"), _rows(v, cache.kv_heads, cache, batch, "v")
    heads, rq, ro = 0, None, None
    if q is not None:
        if q.dim() != 3 or q.shape[1] < 1:
            _invalid("q must be [tokens, q_heads, head_dim]")
        heads = _int32(q.shape[1], "q_heads")
        rq = _rows(q, heads, cache, batch, "q")
        if out is None:
            out = q.new_empty((batch.tokens, heads, cache.head_dim)) if stream is None else _empty(q.shape, q.dtype, q.device, stream)
            ro = _Rows(out.data_ptr(), heads * cache.head_dim, cache.head_dim)
        else:
            ro = _rows(out, heads, cache, batch, "out")
            _no_overlap(out, q, ((q, "q"), (k, "k"), (v, "v")), batch.tokens)
        rq, ro = C.byref(rq), C.byref(ro)
    elif out is not None or q_norm is not None:
        _invalid("out and q_norm are of queries, and q is None")
    _taken(rotation, batch.tokens, cache.head_dim, cache.device)
    if q_norm is not None:
        q_norm._check(heads, cache.head_dim, cache.device, "q_norm")
    if k_norm is not None:
        k_norm._check(cache.kv_heads, cache.head_dim, cache.device, "k_norm")
    _call(cache.device, _lib().gorgo_kv_append, (cache._ref, batch._ref, _ref(rotation), _ref(q_norm), _ref(k_norm), heads, rq, ro, C.byref(rk), C.byref(rv)), stream)
    return out


def rotate_heads(x, *, rotation: Optional[Rotation] = None, norm: Optional[HeadNorm] = None, batch: Optional[KvBatch] = None, out=None, stream=None):
    """gorgo_rotate_heads: rows x [tokens, heads, head_dim] in bfloat16 or float16, normed and rotated, to `out` or a new tensor.  `out` may
    be x, row for row; otherwise its rows share no memory with x's or each other.  batch: the tokens' sequences, by which they are rotated where the
    rotation has no positions; rows of tokens that belong to none are not written, and undefined in a new tensor.  Without a batch all rows
    count.  Asynchronous on `stream` (default: torch's current stream)."""
    import torch
    half = x.dtype == torch.float16
    device = x.device
    if x.dim() != 3 or not (half or x.dtype == torch.bfloat16) or device.type != "cuda":
        _invalid("x must be a bfloat16 or float16 tensor [tokens, heads, head_dim] on the GPU")
    tokens, heads, d = x.shape
    _int32(tokens, "tokens")
    _int32(heads, "heads")
    if batch is not None:
        if batch.device != device or batch.tokens != tokens:
            _invalid(f"batch must have {tokens} tokens, on {device}")
    elif rotation is not None and rotation.positions is None:
        _invalid("a rotation without positions needs a batch")
    if rotation is None and norm is None:
        _invalid("neither rotation nor norm is given")
    out_given = out is not None
    if not out_given:
        out = x.new_empty((tokens, heads, d)) if stream is None else _empty((tokens, heads, d), x.dtype, device, stream)
    elif out.shape != x.shape or out.dtype != x.dtype or out.device != device:
        _invalid("out must be of x's shape and type, on its GPU")
    rows = []
    for t, name in ((x, "x"), (out, "out")):
        _no_gradient(t, name)
        stride = t.stride()
        if stride[2] != 1 and d > 1:
            _invalid(f"the values of a row of {name} must lie side by side")
        rows.append(_Rows(t.data_ptr(), stride[0] if tokens > 1 else 0, stride[1] if heads > 1 else 0))
    if out_given and heads > 0 and d > 0:
        _no_overlap(out, x, ((x, "x"),), tokens)
    _taken(rotation, tokens, d, device)
    if norm is not None:
        norm._check(heads, d, device, "norm")
    of = batch._ref if batch is not None else C.byref(_Batch(0, tokens, 0, 0, None, None, None))
    _call(device, _lib().gorgo_rotate_heads, (of, _ref(rotation), _ref(norm), 1 if half else 0, heads, d, C.byref(rows[0]), C.byref(rows[1])), stream)
    return out


def attend_workspace_bytes(cache: KvCache, batch: KvBatch, q_heads: int) -> int:
    n = C.c_size_t()
    _check(_lib().gorgo_attend_workspace_bytes(cache._ref, batch._ref, _int32(q_heads, "q_heads"), C.byref(n)))
    return n.value


def attend_workspace(cache: KvCache, batch: KvBatch, q_heads: int):
    """A workspace that fits every attention call with this cache and q_heads and batches of at most this one's sequences, tokens and
    columns, its counts zero as the first call wants them; keep it for the calls of one stream."""
    import torch
    workspace = torch.empty((attend_workspace_bytes(cache, batch, q_heads),), dtype=torch.uint8, device=cache.device)
    workspace[:_COUNTS].zero_()
    return workspace


def _attend(f, cache, batch, q, scale, window, sinks, lse, out, workspace, stream):
    import torch
    _int32(window, "window")
    _int32(sinks, "sinks")
    _same_device(cache, batch)
    if q.dim() != 3 or q.shape[1] % cache.kv_heads:
        _invalid("q must be [tokens, q_heads, head_dim], q_heads a multiple of the cache's heads")
    heads = _int32(q.shape[1], "q_heads")
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
    how = _Attention(heads, window, cache.head_dim ** -0.5 if scale is None else scale, sinks)
    _call(cache.device, f, (cache._ref, batch._ref, C.byref(how), C.byref(rq), C.byref(ro), None if lse is None else lse.data_ptr(),
                            workspace.data_ptr(), workspace.nbytes), stream)
    return out if lse is None else (out, lse)


def attend_prompt(cache: KvCache, batch: KvBatch, q, *, scale: Optional[float] = None, window: int = 0, sinks: int = 0, lse=False, out=None,
                  workspace=None, stream=None):
    """gorgo_attend_prompt: causal attention of the new tokens' queries [tokens, q_heads, head_dim] over their sequences in the
    cache (keys and values written before, their own included).  scale: head_dim ** -0.5 if None.  window > 0: a token sees the last
    `window` positions, and the first `sinks` ones.  lse: True (or a tensor) for the rows' log of sums as well.  Asynchronous on `stream` (default: torch's current stream)."""
    return _attend(_lib().gorgo_attend_prompt, cache, batch, q, scale, window, sinks, lse, out, workspace, stream)


def attend_token(cache: KvCache, batch: KvBatch, q, *, scale: Optional[float] = None, window: int = 0, sinks: int = 0, lse=False, out=None,
                 workspace=None, stream=None):
    """gorgo_attend_token: attend_prompt for one new token of each sequence (a batch without token_offsets)."""
    return _attend(_lib().gorgo_attend_token, cache, batch, q, scale, window, sinks, lse, out, workspace, stream)
