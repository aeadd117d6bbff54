"""Cases and a plain 64-bit implementation for the tests of the paged cache and the attention over it."""
import math

import torch

import paper_2602_11688_amd as g

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


class Case:
    """Sequences in a paged cache of random contents: `spec` has a pair (new tokens, tokens in the cache with them) for each."""

    def __init__(self, spec, *, type="bf16", q_heads=8, kv_heads=2, d=64, page=16, seed=0, token=False, spare=3, columns=None, order="phtd"):
        gen = torch.Generator(device=DEVICE)
        gen.manual_seed(seed)
        self.spec, self.type, self.q_heads, self.kv_heads, self.d, self.page = spec, type, q_heads, kv_heads, d, page
        S = len(spec)
        pages = [-(-max(L, 0) // page) for _, L in spec]
        n = sum(pages) + spare
        perm = torch.randperm(n, generator=gen, device=DEVICE).to(torch.int32)
        columns = max([1] + pages) if columns is None else columns
        self.table = torch.full((S, columns), -1, dtype=torch.int32, device=DEVICE)
        at = 0
        for s, p in enumerate(pages):
            p = min(p, columns)
            self.table[s, :p] = perm[at:at + p]
            at += p
        self.rows = torch.float16 if type == "fp16" else torch.bfloat16

        def normal(*shape):
            return torch.randn(shape, generator=gen, device=DEVICE)
        # (order of the cache's dimensions in memory: pages, heads, tokens, values)
        size = dict(p=n, h=kv_heads, t=page, d=d)
        store = [size[c] for c in order]
        back = [order.index(c) for c in "phtd"]

        def cache():
            x = normal(*store)
            if type == "e4m3":
                x = (x * 100).clamp(-448, 448)
            return x.to(TYPES[type]).permute(back)
        self.k, self.v = cache(), cache()
        self.scales = ()
        if type == "e4m3":
            self.scales = tuple(torch.randint(118, 122, (n, kv_heads, page), generator=gen, device=DEVICE, dtype=torch.uint8) for _ in range(2))
        self.cache = g.KvCache(self.k, self.v, *self.scales)
        first = [0]
        for new, _ in spec:
            first.append(first[-1] + new)
        self.first, self.T = first, first[-1]
        self.lengths = torch.tensor([L for _, L in spec], dtype=torch.int32, device=DEVICE)
        self.offsets = torch.tensor(first, dtype=torch.int32, device=DEVICE)
        self.batch = g.KvBatch(self.table, self.lengths, None if token else self.offsets, tokens=self.T)
        self.q = (1.5 * normal(self.T, q_heads, d)).to(self.rows)
        self.new_k, self.new_v = normal(self.T, kv_heads, d).to(self.rows), normal(self.T, kv_heads, d).to(self.rows)

    def dense(self, name, s):
        """[positions, kv_heads, d] of a sequence in 64 bits, and which positions exist."""
        L = min(max(self.spec[s][1], 0), self.table.shape[1] * self.page)
        x = getattr(self, name)
        if L == 0:
            return torch.zeros((0, self.kv_heads, self.d), dtype=torch.float64, device=DEVICE), torch.zeros(0, dtype=torch.bool, device=DEVICE)
        pos = torch.arange(L, device=DEVICE)
        page = self.table[s, pos // self.page].long()
        held = (page >= 0) & (page < x.shape[0])
        page, slot = torch.where(held, page, torch.zeros_like(page)), pos % self.page
        if self.type == "e4m3":
            rows = x.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).double()
            rows = rows * torch.exp2(self.scales[name == "v"][page, :, slot].double() - 127)[..., None]
        else:
            rows = x[page, :, slot].double()
        return rows, held

    def attend(self, scale=None, window=0):
        """out, lse and the sums of weights times |v| in 64 bits."""
        scale = self.d ** -0.5 if scale is None else scale
        G = self.q_heads // self.kv_heads
        out = torch.zeros((self.T, self.q_heads, self.d), dtype=torch.float64, device=DEVICE)
        size = torch.zeros_like(out)
        lse = torch.full((self.T, self.q_heads), -math.inf, dtype=torch.float64, device=DEVICE)
        for s, (n, L) in enumerate(self.spec):
            k, held = self.dense("k", s)
            v, _ = self.dense("v", s)
            if n == 0 or len(k) == 0:
                continue
            at = slice(self.first[s], self.first[s] + n)
            pos = torch.arange(L - n, L, device=DEVICE)[:, None]
            key = torch.arange(len(k), device=DEVICE)
            seen = (key <= pos) & held
            if window:
                seen &= key > pos - window
            for h in range(self.q_heads):
                score = (self.q[at, h].double() @ k[:, h // G].T.contiguous()) * scale
                score = torch.where(seen, score, torch.full_like(score, -math.inf))
                top = score.amax(-1, keepdim=True).clamp(min=-1e300)
                e = torch.where(seen, torch.exp(score - top), torch.zeros_like(score))
                total = e.sum(-1, keepdim=True)
                w = torch.where(total > 0, e / total, torch.zeros_like(e))
                # (a value that is not finite reaches the rows that see it and no others)
                x = v[:, h // G]
                tame = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
                o = w @ tame
                for kind in (math.inf, -math.inf, math.nan):
                    is_kind = (torch.isnan(x) if math.isnan(kind) else x == kind).double()
                    if bool(is_kind.any()):
                        o = o + torch.where(seen.double() @ is_kind > 0, kind, 0.0)
                out[at, h], size[at, h] = o, w @ tame.abs()
                lse[at, h] = (top + total.log())[:, 0]
        return out, lse, size


def check(case, got, window=0, scale=None):
    """Tolerances.  A rounding to the rows' type is off by at most eps / 2 of the value: once for every weight (its share of the
    sum of weights times |v|), once for the result.  Scores and sums are 32-bit: a dot product of d terms is off by
    d * 2^-24 of its terms' sizes at most, which for these inputs (scores below 100) moves a weight by less than 2^-12."""
    out, lse = got
    want, want_lse, size = case.attend(scale, window)
    half = torch.finfo(case.rows).eps / 2
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out[torch.isinf(want)].double(), want[torch.isinf(want)])
    assert torch.isfinite(out[fine]).all()
    off = (out.double() - want).abs()
    # (half the least 16-bit step below the normal range)
    least = 2.0 ** -25 if case.rows == torch.float16 else 2.0 ** -134
    allowed = half * want.abs() + (half + 2.0 ** -12) * size + least
    bad = fine & (off > allowed)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off, first {torch.nonzero(bad)[0].tolist()}, by {float((off / allowed)[fine].max()):.2f} of the bound"
    if lse is not None:
        assert torch.equal(torch.isinf(lse), torch.isinf(want_lse))
        fine = torch.isfinite(want_lse)
        assert ((lse.double() - want_lse).abs()[fine] <= 2.0 ** -12).all()
