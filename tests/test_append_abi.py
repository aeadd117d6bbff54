"""Refusals of the entry points that norm, rotate and append heads: nothing here touches a device."""
import ctypes as C

import pytest
import torch

import paper_2602_11688_amd as g
from paper_2602_11688_amd import attention as ga
from tests.test_attention_abi import BAD_BATCHES, BAD_CACHES, BAD_ROWS, FAKE, _batch, _cache, _ref, _rows


def _rotation(**kw):
    r = ga._Rotation(FAKE, None, 0, 32, 0, 1, 1.0)
    for k, v in kw.items():
        if k == "axis_of_pair":
            v = (C.c_uint8 * 64)(*v)
        setattr(r, k, v)
    return r


def _norm(**kw):
    n = ga._Norm(FAKE, 64, 1e-6, 0)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _append(cache=_cache(), batch=_batch(), rotation=_rotation(), q_norm=_norm(), k_norm=_norm(), heads=8, q=_rows(), out=_rows(), k=_rows(), v=_rows()):
    return ga._lib().gorgo_kv_append(_ref(cache), _ref(batch), _ref(rotation), _ref(q_norm), _ref(k_norm), heads, _ref(q), _ref(out), _ref(k), _ref(v), None)


def _rotate(batch=_batch(), rotation=_rotation(), norm=_norm(), type=0, heads=8, d=64, x=_rows(), out=_rows()):
    return ga._lib().gorgo_rotate_heads(_ref(batch), _ref(rotation), _ref(norm), type, heads, d, _ref(x), _ref(out), None)


BAD_ROTATIONS = [(dict(pairs=0), -1), (dict(pairs=33), -1), (dict(pairs=-1), -1), (dict(layout=2), -1), (dict(layout=-1), -1), (dict(axes=0), -1), (dict(axes=5), -1),
                 (dict(axes=2), -1), (dict(frequencies=None), -1), (dict(frequencies=FAKE + 4), -1), (dict(positions=FAKE + 2), -1), (dict(positions=FAKE, axis_stride=-1), -1),
                 (dict(positions=FAKE, axis_stride=2 ** 40 + 1), -1), (dict(axis_of_pair=[0] * 31 + [1]), -1), (dict(positions=FAKE, axes=3, axis_of_pair=[0, 1, 2, 3]), -1),
                 (dict(magnitude=float("nan")), -6), (dict(magnitude=float("inf")), -6)]
BAD_NORMS = [(dict(eps=0.0), -6), (dict(eps=-1.0), -6), (dict(eps=float("nan")), -6), (dict(eps=float("inf")), -6), (dict(weight=FAKE + 8), -1), (dict(head_stride=-4), -1),
             (dict(head_stride=2), -1), (dict(head_stride=2 ** 40 + 4), -1)]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_caches_refused(kw):
    assert _append(cache=_cache(**kw)) == -1 and b"cache" in ga._lib().gorgo_last_error()


@pytest.mark.parametrize("kw", BAD_BATCHES)
def test_batches_refused(kw):
    assert _append(batch=_batch(**kw)) == -1 and b"batch" in ga._lib().gorgo_last_error()
    if "table_columns" not in kw and "page_table" not in kw:
        assert _rotate(batch=_batch(**kw)) == -1 and b"batch" in ga._lib().gorgo_last_error()


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_rows_refused(kw):
    for name in ("q", "out", "k", "v"):
        assert _append(**{name: _rows(**kw)}) == -1
    assert _rotate(x=_rows(**kw)) == -1 and _rotate(out=_rows(**kw)) == -1


@pytest.mark.parametrize("kw,code", BAD_ROTATIONS)
def test_rotations_refused(kw, code):
    assert _append(rotation=_rotation(**kw)) == code and b"rotation" in ga._lib().gorgo_last_error()
    assert _rotate(rotation=_rotation(**kw)) == code


@pytest.mark.parametrize("kw,code", BAD_NORMS)
def test_norms_refused(kw, code):
    assert _append(q_norm=_norm(**kw)) == code and b"q_norm" in ga._lib().gorgo_last_error()
    assert _append(k_norm=_norm(**kw)) == code and b"k_norm" in ga._lib().gorgo_last_error()
    assert _rotate(norm=_norm(**kw)) == code


def test_null_structures_refused():
    for name in ("cache", "batch", "q", "out", "k", "v"):
        assert _append(**{name: None}) == -1
    for name in ("batch", "x", "out"):
        assert _rotate(**{name: None}) == -1
    assert _rotate(rotation=None, norm=None) == -1


@pytest.mark.parametrize("kw", [dict(type=2), dict(type=-1), dict(heads=0), dict(heads=4097), dict(d=0), dict(d=68), dict(d=136)])
def test_rows_alone_refused(kw):
    assert _rotate(**kw) == -1


def test_heads_refused():
    assert _append(heads=-1) == -1 and _append(heads=4097) == -1


def test_tokens_of_no_sequence_need_positions():
    nobody = _batch(sequences=0, tokens=5, page_table=None, lengths=None, token_offsets=None)
    assert _rotate(batch=nobody) == -1 and b"positions" in ga._lib().gorgo_last_error()
    assert _append(batch=nobody) == -1


def test_no_tokens_is_no_launch():
    none, rows = _batch(tokens=0), _rows(data=None)
    assert _append(batch=none, q=rows, out=rows, k=rows, v=rows) == 0 and _rotate(batch=none, x=rows, out=rows) == 0
    assert _append(batch=none, heads=0, q=None, out=None, k=rows, v=rows) == 0


def test_wrapper_refuses_tensors_before_the_library_sees_them():
    f = torch.ones(32, dtype=torch.float64)
    with pytest.raises(g.GorgoError, match="float64"):
        g.Rotation(f)
    with pytest.raises(g.GorgoError, match="float64"):
        g.Rotation(f.float())
    with pytest.raises(g.GorgoError, match="halves"):
        g.Rotation(f, layout="quarters")
    with pytest.raises(g.GorgoError, match="float32"):
        g.HeadNorm(torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(g.GorgoError, match="on the GPU"):
        g.rotate_heads(torch.ones((2, 2, 64), dtype=torch.bfloat16), norm=g.HeadNorm())


def test_sinks_refused():
    from tests.test_attention_abi import _attend, _how
    how = _how(window=5)
    how.sinks = -1
    assert _attend(how=how) == -1 and b"sinks" in ga._lib().gorgo_last_error()
    assert _attend(how=how, batch=_batch(token_offsets=None, tokens=3), token=True) == -1
