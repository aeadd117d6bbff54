"""Values that lie exactly between two codes of 8 bits go to the even one, wherever they are written from; the powers of two that tests compare with."""
import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE

pytestmark = pytest.mark.gpu


def _two_to(k):
    """2^k in 64 bits, from its bits."""
    return ((torch.as_tensor(k, dtype=torch.int64) + 1023) << 52).view(torch.float64)


def _codes(x):
    """Codes and scale bytes of rows x (on the CPU, in 64 bits, every step exact)."""
    top = x.abs().amax(-1)
    k = torch.full(top.shape, -126, dtype=torch.int64)
    for _ in range(246):
        k = torch.where((top > 448 * _two_to(k)) & (k < 119), k + 1, k)
    y = x * _two_to(-k)[..., None]
    step = _two_to(torch.frexp(y.abs())[1].long().clamp(min=-5) - 4)       # 2^-3 of the power of two at or below it, 2^-9 at least
    y = torch.round(y / step) * step
    return y.float().to(torch.float8_e4m3fn).view(torch.uint8), (k + 127).to(torch.uint8)


def _rows(d):
    """Rows of values between two codes: each code's odd half step of every power of two, both signs, below tops that give every scale."""
    half = (torch.arange(8, 16, dtype=torch.float64) + 0.5) / 8             # 1.0625 to 1.9375: between codes
    low = (torch.arange(0, 8, dtype=torch.float64) + 0.5) / 512              # below 2^-6 the codes' steps are 2^-9
    y = torch.cat([half * float(_two_to(e)) for e in range(-6, 8)] + [low])
    y = torch.cat((y, -y))
    y = y[: len(y) // (d - 1) * (d - 1)].view(-1, d - 1)
    rows = []
    for k in (-100, -9, -7, 0, 3, 60):
        rows.append(torch.cat((y, torch.full((len(y), 1), 440.0, dtype=torch.float64)), 1) * _two_to(k))
    return torch.cat(rows)


@pytest.mark.parametrize("d", [16, 64, 128])
def test_ties(d):
    x = _rows(d)
    assert torch.equal(x.to(torch.bfloat16).double(), x)
    first = torch.zeros((1, d), dtype=torch.float64)
    first[0, 0], first[0, 1] = -0.007080078125, 2.9375                       # 14.5 steps of 2^-11
    x = torch.cat((x, first))
    n = len(x)
    codes, scale = _codes(x)
    assert codes[-1, 0] == (-14.0 / 16 * torch.ones(())).to(torch.float8_e4m3fn).view(torch.uint8)
    rows = x.to(torch.bfloat16).to(DEVICE)[:, None]
    batch = g.KvBatch(torch.arange(-(-n // 16), dtype=torch.int32, device=DEVICE)[None], torch.tensor([n], dtype=torch.int32, device=DEVICE),
                      torch.tensor([0, n], dtype=torch.int32, device=DEVICE), tokens=n)
    for write in (g.kv_write, g.kv_append, lambda *a: g.kv_append(*a, rotation=g.Rotation(torch.zeros(d // 2, dtype=torch.float64, device=DEVICE)))):
        cache = g.KvCache.empty(-(-n // 16), 1, d, 16, "e4m3")
        write(cache, batch, rows, rows)
        for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            assert torch.equal(t.view(torch.uint8).view(-1, d)[:n].cpu(), codes)
            assert torch.equal(s.view(-1)[:n].cpu(), scale)


def test_powers_of_two_on_the_gpu():
    """Other tests take their powers from torch.exp2 in 64 bits."""
    k = torch.arange(-127, 128)
    assert torch.equal(torch.exp2(k.double().to(DEVICE)).cpu(), _two_to(k))
