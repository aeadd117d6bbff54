"""Workspaces, offsets and lengths of any content in the attention over the paged cache and in the cache itself."""
import copy

import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type,d,page", [("bf16", 128, 64), ("e4m3", 64, 48)])
def test_a_workspace_of_a_large_batch_serves_every_smaller_one(type, d, page):
    """Sized once, for many tokens of many sequences that need no pieces, and then used for few, which do, and for single tokens."""
    large = Case([(3000, 9000)] * 4, q_heads=4, kv_heads=1, d=d, page=page, type=type, columns=20000 // page + 1)
    ws = g.attend_workspace(large.cache, large.batch, 4)
    check(large, g.attend_prompt(large.cache, large.batch, large.q, lse=True, workspace=ws))
    for spec, token in (([(3, 20000)], False), ([(1, 20000), (1, 3), (1, 777)], True), ([(500, 7000), (1, 9)], False), ([(1, 20000)], True)):
        c = Case(spec, q_heads=4, kv_heads=1, d=d, page=page, type=type, token=token)
        check(c, (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, c.q, lse=True, workspace=ws))


def test_lengths_at_both_ends_of_32_bits():
    """2^31 - 1 tokens over a table of a few pages: the new tokens see all that it holds.  -2^31: they see nothing, and are not written."""
    for page in (16, 64):
        for token in (False, True):
            n = 1 if token else 70
            c = Case([(n, 200), (n, 200)], page=page, token=token, columns=4 * 64 // page)
            lengths = [2 ** 31 - 1, -2 ** 31]
            c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
            out, lse = (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, c.q, lse=True)
            assert not out[n:].any() and torch.isinf(lse[n:]).all()
            before = (c.k.clone(), c.v.clone())
            g.kv_write(c.cache, c.batch, c.new_k, c.new_v)
            assert torch.equal(before[0], c.k) and torch.equal(before[1], c.v)
            assert not any(x.any() for x in g.kv_read(c.cache, c.batch))
            for i in (0, n - 1):                         # (each sees what a single token at the table's end does)
                one = copy.copy(c)
                one.spec, one.first, one.T, one.q = [(1, c.table.shape[1] * page)], [0, 1], 1, c.q[i:i + 1]
                check(one, (out[i:i + 1], lse[i:i + 1]))
