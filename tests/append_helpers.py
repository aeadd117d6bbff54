"""A plain 64-bit implementation of norms and rotations of heads, for the tests of what runs them."""
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE


class How:
    """A rotation and norms, as the library and as the plain implementation take them."""

    def __init__(self, d, *, pairs=0, layout="halves", positions=None, axis_of_pair=None, base=10000.0, magnitude=1.0, norm="", eps=1e-6, heads=(8, 2), seed=0):
        gen = torch.Generator(device=DEVICE)
        gen.manual_seed(seed + 1000)
        self.d, self.pairs, self.layout, self.positions, self.magnitude, self.eps = d, pairs, layout, positions, magnitude, eps
        self.axis_of_pair = [0] * pairs if axis_of_pair is None else axis_of_pair
        self.frequencies = base ** (-torch.arange(max(1, pairs), dtype=torch.float64, device=DEVICE) / max(1, pairs))
        self.rotation = g.Rotation(self.frequencies, positions, axis_of_pair=axis_of_pair, layout=layout, magnitude=magnitude) if pairs else None
        self.weights, self.norms = [None, None], [None, None]
        for i, h in enumerate(heads):
            if norm in ("shared", "each"):
                self.weights[i] = 1 + 0.4 * torch.randn((h, d) if norm == "each" else (d,), generator=gen, device=DEVICE)
            if norm:
                self.norms[i] = g.HeadNorm(self.weights[i], eps)

    def turned(self, x, pos, which=0):
        """Rows [tokens, heads, d] in 64 bits, and the sums of the sizes of what each value is added up from."""
        x = x.double()
        if self.norms[which] is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.norms[which].eps)
            if self.weights[which] is not None:
                x = x * self.weights[which].double()
        size, P = x.abs(), self.pairs
        if not P:
            return x, size
        where = pos[:, None] if self.positions is None else self.positions.view(-1, self.positions.shape[-1])[self.axis_of_pair].T
        angle = where.double() * self.frequencies
        c, s = (self.magnitude * f(angle)[:, None] for f in (torch.cos, torch.sin))
        a, b = (slice(0, P), slice(P, 2 * P)) if self.layout == "halves" else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
        out, parts = x.clone(), size.clone()
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        parts[..., a], parts[..., b] = (x[..., a] * c).abs() + (x[..., b] * s).abs(), (x[..., b] * c).abs() + (x[..., a] * s).abs()
        return out, parts


def near(got, want, size, rows):
    """Tolerances.  The result's rounding is off by at most eps / 2 of it.  Before it, in 32 bits: the sum of d <= 128 squares by d roundings of
    2^-24 at most, half of that in its root, whose instruction is off by one unit, 2^-23; a row's factor, a weight, a cosine or sine, a
    product and a sum are a rounding each: (128 / 2 + 2 + 5) * 2^-24 of the sizes of what is added up, less than 2^-17."""
    half = torch.finfo(rows).eps / 2
    least = 2.0 ** -25 if rows == torch.float16 else 2.0 ** -134          # (half the least 16-bit step below the normal range)
    assert got.dtype == rows and torch.equal(torch.isnan(got), torch.isnan(want))
    most = float(torch.finfo(rows).max)
    fine = torch.isfinite(want) & (want.abs() < most)
    off = (got.double() - want).abs()
    allowed = half * want.abs() + 2.0 ** -17 * (1 + half) * size + least
    bad = fine & ~(off <= allowed)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off, first {torch.nonzero(bad)[0].tolist()}, by {float((off / allowed)[fine].max()):.2f} of the bound"
    wild = torch.isinf(want)
    assert torch.equal(got[wild].double(), want[wild])


def positions_of(case):
    """Position of each packed token, and whether it belongs to a sequence."""
    pos = torch.zeros(case.T, dtype=torch.long)
    for s, (n, L) in enumerate(case.spec):
        pos[case.first[s]:case.first[s] + n] = torch.arange(max(L, 0) - n, max(L, 0))
    return pos.to(DEVICE)
