"""Results of norms, rotations and appends that share memory with what the same call reads: refused, but for rows in their own place; parts of one
tensor that lie side by side are not meant."""
import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case

pytestmark = pytest.mark.gpu


def _how():
    return dict(rotation=g.Rotation.of_base(32, device=DEVICE)), dict(q_norm=g.HeadNorm(), k_norm=g.HeadNorm())


def test_rows_alone():
    c = Case([(5, 5), (2, 9)], d=64, q_heads=4, kv_heads=2, seed=1)
    rotation, _ = _how()
    how = dict(**rotation, norm=g.HeadNorm(), batch=c.batch)
    wide = torch.zeros((9, 8, 64), dtype=c.q.dtype, device=DEVICE)
    wide[:7, :4] = c.q
    before = wide.clone()
    x = wide[:7, :4]
    want = g.rotate_heads(c.q, **how)
    for out in (wide[:7, 2:6], wide[1:8, :4], wide[2:9, 3:7], wide[:7, ::2], wide.view(-1, 4, 64)[:7], c.q.new_empty((1, 4, 64)).expand(7, 4, 64),
                c.q.new_empty((7, 1, 64)).expand(7, 4, 64), c.q.new_empty(7 * 128 + 256).as_strided((7, 4, 64), (128, 64, 1))):
        with pytest.raises(g.GorgoError, match="out"):
            g.rotate_heads(x, out=out, **how)
    assert torch.equal(wide, before)
    assert torch.equal(g.rotate_heads(x, out=wide[:7, 4:], **how), want)
    assert torch.equal(wide[:, :4], before[:, :4]) and not wide[7:].any()
    assert torch.equal(g.rotate_heads(x, out=wide.as_strided((7, 4, 64), (512, 64, 1)), **how), want)
    # heads first in memory, an input that all tokens share, a single token between others
    turned = torch.zeros((4, 7, 64), dtype=c.q.dtype, device=DEVICE).transpose(0, 1)
    assert torch.equal(g.rotate_heads(c.q, out=turned, **how), want)
    same = c.q[:1].expand(7, 4, 64)
    assert torch.equal(g.rotate_heads(same, out=turned, **how), g.rotate_heads(same.contiguous(), **how))


def test_appends():
    c = Case([(5, 5), (2, 9)], d=64, q_heads=4, kv_heads=2, seed=1)
    rotation, norms = _how()
    product = torch.cat((c.q, c.new_k, c.new_v), 1)
    q, k, v = product[:, :4], product[:, 4:6], product[:, 6:]
    want = g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, **rotation, **norms)
    cache = c.k.clone(), c.v.clone()
    before = product.clone()
    for out in (product[:, 1:5], product[:, 2:6], product[:, 4:], product[:, ::2], q[:1].expand(7, 4, 64), q[:, :1].expand(7, 4, 64)):
        with pytest.raises(g.GorgoError, match="out"):
            g.kv_append(c.cache, c.batch, k, v, q, out=out, **rotation, **norms)
    assert torch.equal(product, before) and torch.equal(c.k, cache[0]) and torch.equal(c.v, cache[1])
    c.k.zero_()
    c.v.zero_()
    assert torch.equal(g.kv_append(c.cache, c.batch, k, v, q, out=q, **rotation, **norms), want)
    held = c.cache, c.batch
    got_k, got_v = g.kv_read(*held)
    assert torch.equal(got_v, c.new_v) and torch.equal(product[:, 4:], before[:, 4:])
    g.kv_append(*held, c.new_k, c.new_v, c.q, out=torch.empty_like(c.q), **rotation, **norms)
    assert torch.equal(g.kv_read(*held)[0], got_k)


def test_no_tokens():
    x = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEVICE)
    assert g.rotate_heads(x, norm=g.HeadNorm(), out=x).shape == (0, 4, 64)
