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


WRONG = ([0, 40, 2 ** 31 - 1], [-5, 40, 130], [130, 40, 0], [2 ** 31 - 1] * 3, [-2 ** 31, 0, 0], [7, 50, 120], [60, 20, 100])


def _spans(offsets, T):
    """New rows of each sequence, whatever stands in the offsets: within the packed rows, an end no earlier than its beginning."""
    for s in range(len(offsets) - 1):
        begin = min(max(offsets[s], 0), T)
        yield s, begin, min(max(offsets[s + 1], begin), T)


@pytest.mark.parametrize("type,page", [("bf16", 48), ("e4m3", 48), ("bf16", 64), ("e4m3", 64)])
@pytest.mark.parametrize("wrong", WRONG)
def test_offsets_that_are_not_offsets_reach_no_other_memory(wrong, type, page):
    """Rows before and behind the results stay what they were, rows of no sequence do or become zero, and the cache changes only in
    slots that rows of some sequence have."""
    c = Case([(40, 100), (90, 257)], page=page, type=type)
    c.offsets.copy_(torch.tensor(wrong, dtype=torch.int32))
    spans = list(_spans(wrong, c.T))
    nobodys = torch.ones(c.T, dtype=torch.bool, device=DEVICE)
    slots = torch.zeros((c.k.shape[0], page), dtype=torch.bool, device=DEVICE)
    for s, begin, end in spans:
        nobodys[begin:end] = False
        for pos in range(max(0, c.spec[s][1] - (end - begin)), c.spec[s][1]):
            slots[int(c.table[s, pos // page]), pos % page] = True

    def inside(*shape, dtype):
        """Results amid 64 rows of 7 on either side."""
        whole = torch.full((c.T + 128, *shape), 7.0, dtype=dtype, device=DEVICE)
        return whole, whole[64:64 + c.T]

    def untouched(whole):
        return bool((whole[:64] == 7).all() and (whole[64 + c.T:] == 7).all())

    wide, out = inside(c.q_heads, c.d, dtype=c.rows)
    wide_lse, lse = inside(c.q_heads, dtype=torch.float32)
    g.attend_prompt(c.cache, c.batch, c.q, out=out, lse=lse)
    assert untouched(wide) and untouched(wide_lse)
    assert ((out[nobodys] == 7) | (out[nobodys] == 0)).all()

    (wide_k, k), (wide_v, v) = inside(c.kv_heads, c.d, dtype=c.rows), inside(c.kv_heads, c.d, dtype=c.rows)
    g.kv_read(c.cache, c.batch, out=(k, v))
    assert untouched(wide_k) and untouched(wide_v)
    assert not k[nobodys].any() and not v[nobodys].any()

    stores = [x.view(torch.uint8) if type == "e4m3" else x for x in (c.k, c.v)] + list(c.scales)
    before = [x.clone() for x in stores]
    g.kv_write(c.cache, c.batch, c.new_k, c.new_v)
    for x, then in zip(stores, before):
        at = slots[:, None, :].expand(x.shape[:3])
        assert torch.equal(x[~at], then[~at])


@pytest.mark.parametrize("type,d,page", [("bf16", 128, 64), ("e4m3", 128, 512), ("fp16", 64, 48), ("e4m3", 64, 16)])
def test_sequences_that_share_the_pages_of_a_prefix(type, d, page):
    """A long prefix in common, pages of their own behind it: written, then read by prompts and by single tokens, in any order of pages."""
    shared = 1536 // page * page
    for token in (False, True):
        spec = [(1, shared + n) for n in (1, 700, 33, 64, 5)] if token else [(n, shared + n) for n in (1, 700, 33, 64, 0)]
        c = Case(spec, d=d, page=page, type=type, token=token)
        c.table[1:, :shared // page] = c.table[0, :shared // page]
        g.kv_write(c.cache, c.batch, c.new_k, c.new_v)
        check(c, (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, c.q, lse=True))
        whole = g.KvBatch(c.table[:2].contiguous(), c.lengths[:2].contiguous(), torch.tensor([0, spec[0][1], spec[0][1] + spec[1][1]], dtype=torch.int32, device=DEVICE),
                          tokens=spec[0][1] + spec[1][1])
        k, v = g.kv_read(c.cache, whole)
        for x in (k, v):                                 # (both sequences begin with the same rows, and end with the first one's and the second one's new one)
            assert torch.equal(x[:shared], x[spec[0][1]:spec[0][1] + shared])
        if type != "e4m3":
            assert torch.equal(k[spec[0][1] - 1], c.new_k[0]) and torch.equal(v[-1], c.new_v[c.first[2] - 1])
