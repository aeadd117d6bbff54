"""Writing tokens into the paged cache and reading them back: 16 bits as they are, 8 bits by the definition in 64 bits."""
import math

import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case

pytestmark = pytest.mark.gpu


def _quantised(x):
    """Codes' values times powers of two, and the scale bytes, of rows x in 64 bits."""
    x = x.double()
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1, keepdim=True)
    k = torch.full_like(a, -126.0)
    for e in range(-126, 119):                           # least exponent that holds the row, 119 at most
        k = torch.where(a > 448.0 * 2.0 ** e, torch.full_like(k, e + 1.0), k)
    y = torch.where(torch.isfinite(x), (x * torch.exp2(-k)).clamp(-448.0, 448.0), x)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.where(torch.isfinite(x), torch.round(y / step) * step, torch.full_like(y, math.nan))
    return y * torch.exp2(k), (k[..., 0] + 127).to(torch.uint8)


def _positions(c):
    for s, (n, L) in enumerate(c.spec):
        for i in range(n):
            pos = L - n + i
            if 0 <= pos < c.table.shape[1] * c.page:
                page = int(c.table[s, pos // c.page])
                if 0 <= page < c.k.shape[0]:
                    yield c.first[s] + i, page, pos % c.page


def _check(c):
    before = [x.clone() for x in (c.k.view(torch.uint8) if c.type == "e4m3" else c.k, c.v.view(torch.uint8) if c.type == "e4m3" else c.v, *c.scales)]
    g.kv_write(c.cache, c.batch, c.new_k, c.new_v)
    got = g.kv_read(c.cache, c.batch)
    rows = list(_positions(c))
    t = torch.tensor([r[0] for r in rows], dtype=torch.long, device=DEVICE)
    page, slot = (torch.tensor([r[i] for r in rows], dtype=torch.long, device=DEVICE) for i in (1, 2))
    for i, x in enumerate((c.new_k, c.new_v)):
        want = torch.zeros(x.shape, dtype=torch.float64, device=DEVICE)
        if c.type == "e4m3":
            values, bytes_ = _quantised(x)
            want[t] = values[t]
            want_scale = before[2 + i].clone()
            want_scale[page, :, slot] = bytes_[t]
            assert torch.equal(c.scales[i], want_scale)
        else:
            want[t] = x[t].double()
            expect = before[i].clone()
            expect[page, :, slot] = x[t]
            assert torch.equal((c.k, c.v)[i], expect)
        same = (got[i].double() == want) | (torch.isnan(got[i]) & torch.isnan(want))
        assert same.all(), (c.type, i, int((~same).sum()))
    if c.type == "e4m3":                                 # nothing else was written
        for i, x in enumerate((c.k, c.v)):
            now, then = x.view(torch.uint8).clone(), before[i].clone()
            now[page, :, slot] = 0
            then[page, :, slot] = 0
            assert torch.equal(now, then)


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d", [16, 64, 80, 128])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_written_and_read_back(type, d, page):
    _check(Case([(1, 1), (0, 5), (30, 77), (200, 200)], type=type, d=d, page=page, kv_heads=3, q_heads=3))


@pytest.mark.parametrize("type", ["fp16", "e4m3"])
def test_one_token_each(type):
    _check(Case([(1, L) for L in (1, 16, 17, 0, 900)], type=type, d=128, page=16, kv_heads=8, token=True))


@pytest.mark.parametrize("order", ["pthd", "hptd", "tphd"])
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_other_orders(order, type):
    _check(Case([(30, 77), (5, 200)], type=type, d=64, page=48, order=order))


def test_magnitudes():
    """Rows of zeros, of the least and the largest values, of powers of two around the borders between two exponents."""
    c = Case([(64, 64)], type="e4m3", d=64, page=16, kv_heads=2, q_heads=2)
    x = c.new_k
    x[0] = 0
    x[1] = torch.finfo(torch.bfloat16).max
    x[2] = torch.finfo(torch.bfloat16).tiny
    x[3] = 2.0 ** -133                                   # least bf16 value
    x[4, :, 1:] = 0
    x[5, 0, 0], x[5, 1, 0] = 448.0, 450.0
    for i in range(6, 30):
        x[i] *= 2.0 ** (10 * (i - 18))
    x[30, :, 0], x[30, :, 1:] = 1.0, 2.0 ** -20
    x[31] = -x[31].abs()
    x[32, 0, 3], x[32, 1, 4], x[33, 0, 5] = math.inf, -math.inf, math.nan
    x[34] = math.nan
    # ties: halfway between two codes
    x[35, :, 0], x[35, :, 1:9] = 448.0, torch.tensor([17.0, 19.0, 21.0, 23.0, 272.0, 304.0, -17.0, -19.0], device=DEVICE, dtype=torch.bfloat16)
    _check(c)


def test_missing_pages_and_lengths_that_do_not_fit():
    for type in ("bf16", "e4m3"):
        c = Case([(100, 500), (10, 4), (3, 0), (5, -7), (40, 40)], page=16, type=type)
        c.table[0, 27] = -1
        c.table[0, 29] = c.k.shape[0]
        c.table[4, :] = -2 ** 31
        _check(c)
        c = Case([(6, 90), (4, 33)], page=16, columns=3, type=type)
        _check(c)


def test_strided_rows():
    c = Case([(30, 77), (5, 200)], d=64, page=48)
    qkv = torch.randn((c.T, 8, c.d), device=DEVICE).to(c.rows)
    c.new_k, c.new_v = qkv[:, 4:6], qkv[:, 6:8]
    _check(c)
    out = torch.full((c.T, 4, c.d), float("nan"), dtype=c.rows, device=DEVICE)
    g.kv_read(c.cache, c.batch, out=(out[:, 0:2], out[:, 2:4]))
    assert torch.equal(out[:, 0:2], c.new_k) and torch.equal(out[:, 2:4], c.new_v)


def test_many_sequences():
    _check(Case([(i % 7, 11 * i % 50 + i % 7) for i in range(300)], d=64, page=16))
