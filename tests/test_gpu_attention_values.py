"""Values and scores at the ends of their ranges in the attention over the paged cache, against the plain 64-bit implementation:
what lies in slots that nobody sees, scores far beyond 2^24, weights far below the largest, values near the end of bf16."""
import math

import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case, check

pytestmark = pytest.mark.gpu


def _attend(case, **kw):
    return (g.attend_token if case.batch.token_offsets is None else g.attend_prompt)(case.cache, case.batch, case.q, lse=True, **kw)


def _unseen(c, window):
    """[pages, slots]: those that no new token of any sequence sees."""
    unseen = torch.ones((c.k.shape[0], c.page), dtype=torch.bool, device=DEVICE)
    for s, (n, L) in enumerate(c.spec):
        first = max(0, L - max(n, 1) + 1 - window) if window else 0
        for j in range(first, min(L, c.table.shape[1] * c.page)):
            page = int(c.table[s, j // c.page])
            if 0 <= page < len(unseen):
                unseen[page, j % c.page] = False
    return unseen


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("heads", [(4, 2, 64), (24, 1, 128)])
@pytest.mark.parametrize("token", [False, True])
def test_scale_bytes_of_slots_that_nobody_sees(token, heads, page, window):
    """Beyond the lengths, before the windows, in pages of nobody and in the first page, beside sequences whose pages are missing:
    255, which as an exponent is an infinity."""
    c = Case([(1, 100), (1, 70), (1, 529), (1, 1)] if token else [(30, 100), (70, 70), (1, 129), (5, 529)], page=page, type="e4m3", token=token,
             q_heads=heads[0], kv_heads=heads[1], d=heads[2])
    c.table[c.table == 0] = -1
    c.table[2, 1] = -1
    unseen = _unseen(c, window)
    assert bool(unseen[0].all()) and int(unseen.sum()) > c.page
    for x in c.scales:
        x.copy_(torch.where(unseen[:, None], torch.full_like(x, 255), x))
    check(c, _attend(c, window=window), window)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 48), (128, 16)])
@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("token", [False, True])
def test_scores_of_thousands_of_millions(token, type, d, page, sign):
    """32 bits hold such scores in steps of hundreds: the largest one's weight is 1 all the same."""
    for spec in ([(1, 500), (1, 300)], [(1, 20000)]) if token else ([(100, 500), (300, 300)], [(2, 20000)]):
        c = Case(spec, d=d, page=page, type=type, token=token, q_heads=2, kv_heads=1)
        c.q.zero_()
        c.q[..., 0] = 60000.0
        c.k.zero_()
        # 8 .. 15 times a power of two, which every type holds exactly (several keys share the largest)
        c.k[..., 0] = (sign * (8 + torch.randint(0, 8, c.k.shape[:-1], device=DEVICE)) * (16 if type == "e4m3" else 4096)).to(c.k.dtype)
        if type == "e4m3":
            c.scales[0].fill_(127 + 8)
        out, lse = _attend(c, scale=1.0)
        check(c, (out, None), scale=1.0)
        _, want, _ = c.attend(1.0)
        # (log2(e) and the product with it, in 32 bits, the way back, and the logarithm of at most 20,000, which is less than a step)
        assert ((lse.double() - want).abs() <= 2.0 ** -21 * want.abs()).all()


def _score(c, s, j, x):
    """Gives key j of sequence s the score x in powers of two: of every query, whose first value is 1 and whose others are 0."""
    c.k[int(c.table[s, j // c.page]), :, j % c.page] = 0
    c.k[int(c.table[s, j // c.page]), :, j % c.page, 0] = x


LN2 = math.log(2.0)


@pytest.mark.parametrize("below", [18, 21, 24])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 48), (128, 16)])
@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("token", [False, True])
def test_small_weights_beside_a_key_that_has_nearly_all(token, type, d, page, below):
    """A key whose value is 0 (the first one, or one in the middle) and others that weigh 2^-below of it: they are the whole result."""
    for spec in ([(1, 2000), (1, 300)], [(1, 30000)]) if token else ([(100, 2000), (300, 300)], [(2, 30000)]):
        c = Case(spec, d=d, page=page, type=type, token=token, q_heads=2, kv_heads=1)
        c.q.zero_()
        c.q[..., 0] = 1.0
        c.k.zero_()
        c.k[..., 0] = -below - 0.3 * torch.rand(c.k.shape[:-1], device=DEVICE)
        for s, (_, L) in enumerate(spec):
            for j in (0, L - 1) if L == 300 else (0,):
                _score(c, s, j, 0.0)
                c.v[int(c.table[s, j // page]), :, j % page] = 0
        check(c, _attend(c, scale=LN2), scale=LN2)


@pytest.mark.parametrize("rise", [0.0, 7.0])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 48), (128, 16)])
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("token", [False, True])
def test_values_near_the_end_of_bf16(token, type, d, page, rise):
    """All values within a factor of two of the largest finite one, of either sign: so is what they are averaged to.  With scores that are
    equal, or that rise by 2^7 after a sequence's first tiles, which no renewed maximum takes notice of."""
    for spec in ([(1, 3000), (1, 300)], [(1, 30000)]) if token else ([(100, 3000), (300, 300)], [(2, 30000)]):
        c = Case(spec, d=d, page=page, type=type, token=token, q_heads=2, kv_heads=1)
        c.q.zero_()
        c.q[..., 0] = 1.0
        c.k.zero_()
        if type == "e4m3":
            for x in c.scales:
                x.fill_(127)
            c.scales[1].fill_(119 + 127)
        sign = torch.where(torch.arange(d, device=DEVICE) % 2 == 0, 1.0, -1.0)
        most = 448.0 if type == "e4m3" else torch.finfo(torch.bfloat16).max
        c.v.copy_(((0.5 + 0.5 * torch.rand(c.v.shape, device=DEVICE)) * sign * most).to(c.v.dtype))
        for s, (_, L) in enumerate(spec):
            _score(c, s, 0, 0.0)
        if rise:
            later = torch.zeros((len(c.k), page), device=DEVICE)
            for s, (_, L) in enumerate(spec):
                j = torch.arange(256, L, device=DEVICE)
                later[c.table[s, j // page].long(), j % page] = rise
            c.k[..., 0] = later[:, None].to(c.k.dtype)
        check(c, _attend(c, scale=LN2), scale=LN2)


@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 48), (128, 16)])
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("token", [False, True])
def test_values_of_2_to_the_minus_40(token, type, d, page):
    """The room that large values need is not taken from small ones: down to there they keep all their bits."""
    for spec in ([(1, 3000), (1, 300)], [(1, 30000)]) if token else ([(100, 3000), (300, 300)], [(2, 30000)]):
        c = Case(spec, d=d, page=page, type=type, token=token, q_heads=2, kv_heads=1)
        if type == "e4m3":
            c.scales[1].sub_(33)                         # (codes of hundreds times 2^-42 .. 2^-39)
        else:
            c.v.mul_(2.0 ** -40)
        check(c, _attend(c))
