"""Refusals of the cache and attention entry points, and their workspace sizes: nothing here touches a device."""
import ctypes as C

import pytest

import paper_2602_11688_amd as g
from paper_2602_11688_amd import attention as ga

FAKE = 4096                                              # an aligned address that no refused call looks at


def _cache(**kw):
    c = ga._Cache(FAKE, FAKE, None, None, 0, 10, 16, 2, 64, 0, 2 * 16 * 64, 16 * 64, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(**kw):
    b = ga._Batch(3, 7, 5, 0, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _rows(**kw):
    r = ga._Rows(FAKE, 8 * 64, 64)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _how(**kw):
    h = ga._Attention(8, 0, 0.125, 0)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def _ref(x):
    return None if x is None else C.byref(x)


def _write(cache=_cache(), batch=_batch(), k=_rows(), v=_rows()):
    L = ga._lib()
    a, b = (f(_ref(cache), _ref(batch), _ref(k), _ref(v), None) for f in (L.gorgo_kv_write, L.gorgo_kv_read))
    assert a == b
    return a


def _attend(cache=_cache(), batch=_batch(), how=_how(), q=_rows(), out=_rows(), ws=FAKE, nbytes=1 << 40, token=False):
    L = ga._lib()
    f = L.gorgo_attend_token if token else L.gorgo_attend_prompt
    return f(_ref(cache), _ref(batch), _ref(how), _ref(q), _ref(out), None, ws, nbytes, None)


BAD_CACHES = [dict(type=3), dict(type=-1), dict(pages=0), dict(page_tokens=0), dict(page_tokens=32768), dict(kv_heads=0), dict(kv_heads=1025),
              dict(head_dim=0), dict(head_dim=68), dict(head_dim=136), dict(type=2), dict(type=2, k_scale=FAKE), dict(type=2, k_scale=FAKE, v_scale=FAKE, head_dim=72),
              dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(page_stride=-8), dict(head_stride=12), dict(token_stride=4),
              dict(page_stride=2 ** 40 + 8), dict(type=2, k_scale=FAKE, v_scale=FAKE, token_stride=8)]
BAD_BATCHES = [dict(sequences=-1), dict(sequences=2 ** 16 + 1), dict(tokens=-1), dict(tokens=2 ** 24 + 1), dict(token_offsets=None), dict(table_columns=0),
               dict(table_columns=2 ** 27), dict(page_table=None), dict(lengths=None)]
BAD_ROWS = [dict(data=None), dict(data=FAKE + 8), dict(token_stride=4), dict(head_stride=12), dict(token_stride=-8), dict(head_stride=2 ** 40 + 8)]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_caches_refused(kw):
    assert _write(cache=_cache(**kw)) == -1 and b"cache" in ga._lib().gorgo_last_error()
    assert _attend(cache=_cache(**kw)) == -1 and _attend(cache=_cache(**kw), token=True) == -1
    assert ga._lib().gorgo_attend_workspace_bytes(C.byref(_cache(**kw)), C.byref(_batch()), 8, C.byref(C.c_size_t())) == -1


@pytest.mark.parametrize("kw", BAD_BATCHES)
def test_batches_refused(kw):
    assert _write(batch=_batch(**kw)) == -1 and b"batch" in ga._lib().gorgo_last_error()
    assert _attend(batch=_batch(**kw)) == -1


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_rows_refused(kw):
    assert _write(k=_rows(**kw)) == -1 and _write(v=_rows(**kw)) == -1
    assert _attend(q=_rows(**kw)) == -1 and _attend(out=_rows(**kw)) == -1


def test_null_structures_refused():
    assert _write(cache=None) == -1 and _write(batch=None) == -1 and _write(k=None) == -1 and _write(v=None) == -1
    for name in ("cache", "batch", "how", "q", "out"):
        assert _attend(**{name: None}) == -1
    assert ga._lib().gorgo_attend_workspace_bytes(C.byref(_cache()), C.byref(_batch()), 8, None) == -1


@pytest.mark.parametrize("kw,code", [(dict(q_heads=0), -1), (dict(q_heads=7), -1), (dict(q_heads=4098), -1), (dict(window=-1), -1), (dict(scale=0.0), -6),
                                     (dict(scale=-1.0), -6), (dict(scale=float("nan")), -6), (dict(scale=float("inf")), -6)])
def test_attention_refused(kw, code):
    assert _attend(how=_how(**kw)) == code
    one = _batch(token_offsets=None, tokens=3)
    assert _attend(how=_how(**kw), batch=one, token=True) == code


def test_token_form_takes_no_offsets():
    assert _attend(token=True) == -1 and b"token_offsets" in ga._lib().gorgo_last_error()


def test_rows_beyond_31_bits_refused():
    big = _batch(tokens=2 ** 24)
    assert _attend(batch=big, how=_how(q_heads=256)) == -1 and b"2^31" in ga._lib().gorgo_last_error()


def test_launches_beyond_32_bits_of_threads_refused():
    assert _attend(batch=_batch(tokens=2 ** 24), how=_how(q_heads=128)) == -1 and b"split the batch" in ga._lib().gorgo_last_error()


def test_workspace_refused():
    one = _batch(token_offsets=None, tokens=3, table_columns=400)
    n = C.c_size_t()
    assert ga._lib().gorgo_attend_workspace_bytes(C.byref(_cache()), C.byref(one), 8, C.byref(n)) == 0 and n.value > 0
    assert _attend(batch=one, token=True, ws=None) == -7
    assert _attend(batch=one, token=True, ws=FAKE + 64) == -7
    assert _attend(batch=one, token=True, nbytes=64) == -7 and b"workspace" in ga._lib().gorgo_last_error()


def test_no_tokens_is_no_launch():
    none = _batch(tokens=0)
    assert _write(batch=none, k=_rows(data=None), v=_rows(data=None)) == 0
    assert _attend(batch=none, q=_rows(data=None), out=_rows(data=None)) == 0
    nobody = _batch(sequences=0, tokens=0, token_offsets=None, page_table=None, lengths=None)
    assert _attend(batch=nobody, q=_rows(data=None), out=_rows(data=None), token=True) == 0


def test_wrapper_refuses_tensors_before_the_library_sees_them():
    import torch
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(g.GorgoError, match="GPU"):
        g.KvCache(k, k.clone())
    with pytest.raises(g.GorgoError, match="one shape"):
        g.KvCache(k, k[:, :1])
    with pytest.raises(g.GorgoError, match="bfloat16"):
        g.KvCache(k.float(), k.float())
    with pytest.raises(g.GorgoError, match="int32"):
        g.KvBatch(torch.zeros((2, 3), dtype=torch.int64), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(g.GorgoError, match="columns"):
        g.KvBatch(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(g.GorgoError, match="bf16"):
        g.KvCache.empty(2, 2, 64, dtype="fp64")


@pytest.mark.parametrize("type,stride", [(0, 2 ** 25 + 8), (2, 2 ** 26 + 16)])
def test_token_strides_beyond_32_bits_of_a_tile_refused(type, stride):
    kw = dict(type=type, token_stride=stride, **(dict(k_scale=FAKE, v_scale=FAKE) if type == 2 else {}))
    assert _write(cache=_cache(**kw)) == -1 and b"token_stride" in ga._lib().gorgo_last_error()


def test_workspace_holds_the_counts_whatever_the_batch():
    """The counts' place does not depend on the batch, and a prompt's pieces leave it alone: one workspace serves calls of all sizes."""
    n = C.c_size_t()
    for batch in (_batch(token_offsets=None, tokens=3, table_columns=400), _batch(token_offsets=None, sequences=1, tokens=1, table_columns=2)):
        assert ga._lib().gorgo_attend_workspace_bytes(C.byref(_cache()), C.byref(batch), 8, C.byref(n)) == 0 and n.value > 2048


def test_tokens_of_no_sequence_refused():
    """No sequence has offsets, lengths or a row of the table that a kernel could look at."""
    for tokens in (1, 5, 100000):
        nobody = _batch(sequences=0, tokens=tokens, page_table=None, lengths=None)
        assert _write(batch=nobody) == -1 and b"without sequences" in ga._lib().gorgo_last_error()
        assert _attend(batch=nobody) == -1
        assert ga._lib().gorgo_attend_workspace_bytes(C.byref(_cache()), C.byref(nobody), 8, C.byref(C.c_size_t())) == -1
