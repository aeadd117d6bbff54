"""Counts that 32 bits do not hold: refused by the binding, where ctypes would cut them off and another call would run."""
import pytest
import torch

import paper_2602_11688_amd as g
from paper_2602_11688_amd import attention as ga


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, 2 ** 70, -2 ** 31 - 1])
def test_windows_and_sinks(n):
    for attend in (g.attend_prompt, g.attend_token):
        for how in (dict(window=n), dict(window=4, sinks=n)):
            with pytest.raises(g.GorgoError, match="32 bits"):
                attend(None, None, None, **how)           # (refused before anything is looked at)
    with pytest.raises(g.GorgoError, match="32 bits"):
        ga._int32(n, "tokens")
    assert ga._int32(2 ** 31 - 1, "tokens") == 2 ** 31 - 1


@pytest.mark.gpu
def test_tokens():
    import tests.attention_helpers as h
    table, lengths, offsets = (torch.zeros(shape, dtype=torch.int32, device=h.DEVICE) for shape in ((1, 1), (1,), (2,)))
    with pytest.raises(g.GorgoError, match="32 bits"):
        g.KvBatch(table, lengths, offsets, tokens=2 ** 32 + 5)
    wide = torch.zeros((1, 1, 8), dtype=torch.bfloat16, device=h.DEVICE)
    for x in (wide.expand(2 ** 32 + 5, 1, 8), wide.expand(1, 2 ** 32 + 5, 8)):
        with pytest.raises(g.GorgoError, match="32 bits"):
            g.rotate_heads(x, norm=g.HeadNorm(), out=x)
    c = h.Case([(1, 5)], token=True)
    many = c.q[:, :1].expand(1, 2 ** 32 + 8, 64)
    for call in (lambda: g.kv_append(c.cache, c.batch, c.new_k, c.new_v, many, out=many), lambda: g.attend_token(c.cache, c.batch, many, out=many)):
        with pytest.raises(g.GorgoError, match="32 bits"):
            call()
