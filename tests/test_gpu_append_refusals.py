"""What the binding of norms, rotations and appends refuses of tensors on the GPU: nothing is launched for these."""
import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case

pytestmark = pytest.mark.gpu


def _f():
    return torch.ones(32, dtype=torch.float64, device=DEVICE)


def _positions(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEVICE)


@pytest.mark.parametrize("make,match", [
    (lambda: g.Rotation(_f().float()), "float64"), (lambda: g.Rotation(_f()[None]), "float64"), (lambda: g.Rotation(torch.ones(64, dtype=torch.float64, device=DEVICE)[::2]), "contiguous"),
    (lambda: g.Rotation(torch.ones(65, dtype=torch.float64, device=DEVICE)), "1 to 64"), (lambda: g.Rotation(_f()[:0]), "1 to 64"),
    (lambda: g.Rotation(_f(), _positions(5).long()), "int32"), (lambda: g.Rotation(_f(), _positions(5).cpu()), "GPU"), (lambda: g.Rotation(_f(), _positions(2, 2, 5)), "axes, tokens"),
    (lambda: g.Rotation(_f(), _positions(5, 7)), "1 to 4"), (lambda: g.Rotation(_f(), _positions(5, 3).T), "side by side"), (lambda: g.Rotation(_f(), _positions(2, 5), axis_of_pair=[0, 1]), "each pair"),
    (lambda: g.Rotation(_f(), _positions(2, 5), axis_of_pair=[2] * 32), "each pair"), (lambda: g.Rotation(_f(), axis_of_pair=[1] * 32), "each pair"),
    (lambda: g.Rotation(_f().clone().requires_grad_()), "gradient"), (lambda: g.HeadNorm(torch.ones(64, device=DEVICE).requires_grad_()), "gradient"),
    (lambda: g.HeadNorm(torch.ones((2, 2, 64), device=DEVICE)), "float32"), (lambda: g.HeadNorm(torch.ones((64, 2), device=DEVICE).T), "contiguous")])
def test_plans(make, match):
    with pytest.raises(g.GorgoError, match=match):
        make()


def test_rows():
    c = Case([(5, 5), (2, 9)], d=64, q_heads=4, kv_heads=2, seed=1)
    r, n = g.Rotation(_f()), g.HeadNorm(torch.ones(64, device=DEVICE))
    x = c.q
    leaf = x.clone().requires_grad_()
    for bad, match in ((dict(x=x.float()), "bfloat16"), (dict(x=x[0]), "bfloat16"), (dict(x=x, batch=None), "needs a batch"), (dict(x=x, rotation=None), "neither"),
                       (dict(x=x[:3]), "tokens"), (dict(x=x, out=x[:3]), "shape"), (dict(x=x, out=x.to(torch.float16)), "shape"), (dict(x=leaf), "x requires a gradient"),
                       (dict(x=x, out=leaf), "out requires a gradient"), (dict(x=x.transpose(1, 2).contiguous().transpose(1, 2)), "side by side"),
                       (dict(x=x, rotation=g.Rotation(_f(), _positions(8))), "positions of 7"), (dict(x=x[..., :32], rotation=g.Rotation(_f())), "at most 16 pairs"),
                       (dict(x=x, norm=g.HeadNorm(torch.ones(32, device=DEVICE))), r"\[64\] or \[4, 64\]"), (dict(x=x, norm=g.HeadNorm(torch.ones((2, 64), device=DEVICE))), r"\[4, 64\]"),
                       (dict(x=x[..., 4:60].contiguous()[..., :36], rotation=None, norm=g.HeadNorm()), "head_dim")):
        with pytest.raises(g.GorgoError, match=match):
            how = dict(rotation=r, batch=c.batch)
            how.update({k: v for k, v in bad.items() if k != "x"})
            g.rotate_heads(bad["x"], **how)
    with torch.no_grad():
        assert torch.equal(g.rotate_heads(leaf, rotation=r, norm=n, batch=c.batch), g.rotate_heads(x, rotation=r, norm=n, batch=c.batch))


def test_appends():
    c = Case([(5, 5), (2, 9)], d=64, q_heads=4, kv_heads=2, seed=1)
    before = c.k.clone()
    good = dict(k=c.new_k, v=c.new_v, q=c.q)
    for bad, match in ((dict(k=c.new_k[:3]), "k must be"), (dict(v=c.new_v.to(torch.float16)), "v must be"), (dict(q=c.q[..., :32]), "q must be"), (dict(q=c.q[0]), "q must be"),
                       (dict(out=c.q[:3]), "out must be"), (dict(q=None, out=c.q), "q is None"), (dict(q=None, q_norm=g.HeadNorm()), "q is None"),
                       (dict(k=c.new_k.clone().requires_grad_()), "k requires a gradient"), (dict(rotation=g.Rotation(_f(), _positions(8))), "positions of 7"),
                       (dict(k_norm=g.HeadNorm(torch.ones((4, 64), device=DEVICE))), r"k_norm must be \[64\] or \[2, 64\]"),
                       (dict(q_norm=g.HeadNorm(torch.ones((2, 64), device=DEVICE))), r"q_norm must be \[64\] or \[4, 64\]"),
                       (dict(k_norm=g.HeadNorm(eps=0.0)), "eps"), (dict(rotation=g.Rotation(_f(), magnitude=float("inf"))), "magnitude"),
                       (dict(k_norm=g.HeadNorm(torch.ones(65, device=DEVICE)[1:])), "16-byte")):
        with pytest.raises(g.GorgoError, match=match):
            how = {**good, **bad}
            g.kv_append(c.cache, c.batch, how.pop("k"), how.pop("v"), how.pop("q"), **how)
    assert torch.equal(before, c.k)
    with pytest.raises(g.GorgoError, match="sinks"):
        g.attend_prompt(c.cache, c.batch, c.q, window=4, sinks=-1)
