"""Which rows share memory, by the binding's rule and by looking at every byte."""
import random

import pytest

from paper_2602_11688_amd import attention as ga


def _bytes(rows, tokens, width):
    at, t, h, heads = rows
    return [set(range(at + i * t + n * h, at + i * t + n * h + width)) for i in range(tokens) for n in range(heads)]


def _shares(a, b, tokens, width):
    return bool(set().union(*_bytes(a, tokens, width)) & set().union(*_bytes(b, tokens, width)))


def _folded(rows, tokens, width):
    each = _bytes(rows, tokens, width)
    return len(set().union(*each)) < sum(map(len, each))


@pytest.mark.parametrize("seed", range(6))
def test_every_layout(seed):
    """Strides and distances of any kind, in units that make rows meet, miss by one step, and lie between each other."""
    rng, width = random.Random(seed), 8
    seen = {}
    for _ in range(4000):
        tokens = rng.randint(1, 6)

        def rows(at):
            heads = rng.randint(1, 4)
            t, h = rng.choice((0, 4, 8, 12, 16, 24, 32, 40, 64, 96)), rng.choice((0, 4, 8, 12, 16, 24, 48))
            return at, t if tokens > 1 else 0, h if heads > 1 else 0, heads
        a, b = rows(400), rows(400 + 4 * rng.randint(-60, 60))
        if rng.random() < 0.5:
            b = (b[0], a[1], *b[2:])
        if rng.random() < 0.3 and b[3] > 1 and a[3] > 1:
            b = (*b[:2], a[2], b[3])
        folded = _folded(a, tokens, width)
        assert ga._folds(a, tokens, width) == folded, (a, tokens)
        if not folded:                                # (out's rows are looked at first)
            shares = _shares(a, b, tokens, width)
            assert ga._touch(a, b, tokens, width) == shares, (a, b, tokens)
            seen[a[1] == b[1], shares] = seen.get((a[1] == b[1], shares), 0) + 1
    assert len(seen) == 4 and min(seen.values()) > 50


def test_usual_layouts():
    """Queries, keys and values side by side in one product's rows of 8, 2 and 2 heads of 64; the halves of a wider tensor; a head too far."""
    width, token = 128, 12 * 128
    q, k, v = (0, token, 128, 8), (8 * 128, token, 128, 2), (10 * 128, token, 128, 2)
    for tokens in (1, 2, 1000, 1 << 24):
        assert not ga._folds(q, tokens, width)
        assert not ga._touch(q, k, tokens, width) and not ga._touch(q, v, tokens, width)
        assert ga._touch(q, (128, token, 128, 8), tokens, width) and ga._touch(q, q, tokens, width)
        assert not ga._touch(q, (token * tokens, token, 128, 8), tokens, width)
        assert ga._touch(q, (token * (tokens - 1) + 7 * 128, token, 128, 8), tokens, width)
    # heads first, tokens within: [heads][tokens][64]
    assert not ga._folds((0, 128, 128 * 50, 8), 50, width) and ga._folds((0, 128, 128 * 49, 8), 50, width)
    assert ga._folds((0, 0, 128, 8), 2, width) and ga._folds((0, 1024, 0, 8), 2, width)
