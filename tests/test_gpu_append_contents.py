"""Offsets, lengths, pages, positions and frequencies of any content: calls that norm, rotate and append, and attention with sinks, write what is
theirs and nothing else."""
import copy

import pytest
import torch

import paper_2602_11688_amd as g
from tests.append_helpers import How, near
from tests.attention_helpers import DEVICE, check
from tests.test_gpu_attention_contents import WRONG, _spans
from tests.test_gpu_sinks import SinkCase

pytestmark = pytest.mark.gpu


def _amid(c, heads):
    """Results amid 64 rows of 7 on either side."""
    whole = torch.full((c.T + 128, heads, c.d), 7.0, dtype=c.rows, device=DEVICE)
    return whole, whole[64:64 + c.T]


def _untouched(c, whole):
    return bool((whole[:64] == 7).all() and (whole[64 + c.T:] == 7).all())


@pytest.mark.parametrize("type,page", [("bf16", 48), ("e4m3", 48), ("e4m3", 64)])
@pytest.mark.parametrize("wrong", WRONG)
def test_offsets_that_are_not_offsets(wrong, type, page):
    """Rows of no sequence stay as they were, the others are rotated by the place that their sequence gives them, and the cache changes only in their slots."""
    c = SinkCase([(40, 100), (90, 257)], 5, 50, page=page, type=type)
    c.offsets.copy_(torch.tensor(wrong, dtype=torch.int32))
    how = How(c.d, pairs=32, norm="shared")
    places = [[] for _ in range(c.T)]
    slots = torch.zeros((c.k.shape[0], page), dtype=torch.bool, device=DEVICE)
    for s, begin, end in _spans(wrong, c.T):
        for i in range(begin, end):
            places[i].append(c.spec[s][1] - (end - i))
        for pos in range(max(0, c.spec[s][1] - (end - begin)), c.spec[s][1]):
            slots[int(c.table[s, pos // page]), pos % page] = True
    before = [x.clone() for x in ([c.k.view(torch.uint8), c.v.view(torch.uint8), *c.scales] if type == "e4m3" else [c.k, c.v])]
    wide, out = _amid(c, c.q_heads)
    g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1], out=out)
    assert _untouched(c, wide)
    # (offsets that fall back let spans overlap: then any of them may be taken, or none that the search comes by)
    nobodys = torch.tensor([not p for p in places], device=DEVICE)
    assert (out[nobodys] == 7).all()
    if all(len(p) <= 1 for p in places) and list(wrong) == sorted(wrong):
        mine = ~nobodys
        pos = torch.tensor([p[0] if p else 0 for p in places], device=DEVICE)
        want, size = how.turned(c.q, pos, 0)
        near(out[mine], want[mine], size[mine], c.rows)
    for now, then in zip([c.k.view(torch.uint8), c.v.view(torch.uint8), *c.scales] if type == "e4m3" else [c.k, c.v], before):
        changed = (now != then) if now.dim() == 3 else (now != then).any(-1)
        assert not (changed.any(1) & ~slots).any()

    wide, out = _amid(c, c.q_heads)
    g.rotate_heads(c.q, rotation=how.rotation, norm=how.norms[0], batch=c.batch, out=out)
    assert _untouched(c, wide) and (out[nobodys] == 7).all()
    wide, out = _amid(c, c.q_heads)
    g.attend_prompt(c.cache, c.batch, c.q, window=50, sinks=5, out=out)
    assert _untouched(c, wide) and ((out[nobodys] == 7) | (out[nobodys] == 0)).all()


def test_lengths_at_both_ends_of_32_bits():
    """2^31 - 1 tokens over a table of a few pages: its sinks alone are seen, nothing is written, queries are rotated all the same.  -2^31: as if there were none before."""
    for page in (16, 64):
        for token in (False, True):
            n = 1 if token else 70
            c = SinkCase([(n, 200), (n, 200)], 20, 30, page=page, token=token, columns=4 * 64 // page)
            c.lengths.copy_(torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
            out, lse = (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, c.q, window=30, sinks=20, lse=True)
            assert not out[n:].any() and torch.isinf(lse[n:]).all()
            for i in (0, n - 1):
                one = copy.copy(c)
                # (what a token sees whose table ends behind the sinks, and whose window sees the last of them)
                one.spec, one.first, one.T, one.q, one.sinks = [(1, 20)], [0, 1], 1, c.q[i:i + 1], 20
                check(one, (out[i:i + 1], lse[i:i + 1]), 30)
            before = (c.k.clone(), c.v.clone())
            how = How(c.d, pairs=32)
            q = g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, rotation=how.rotation)
            assert torch.equal(before[0], c.k) and torch.equal(before[1], c.v)
            pos = torch.cat([torch.arange(2 ** 31 - 1 - n, 2 ** 31 - 1, device=DEVICE), torch.arange(-n, 0, device=DEVICE)])
            near(q, *how.turned(c.q, pos, 0), c.rows)


def test_frequencies_and_magnitudes_of_any_content():
    """What a pair is turned by reaches that pair alone; frequencies that are not finite make it NaN."""
    c = SinkCase([(9, 30)], 0, 1, d=64)
    how = How(64, pairs=32)
    how.frequencies[3], how.frequencies[7], how.frequencies[20] = float("nan"), float("inf"), 1e300
    got = g.rotate_heads(c.q, rotation=how.rotation, batch=c.batch)
    spared = [i for i in range(64) if i % 32 not in (3, 7, 20)]
    want, size = how.turned(c.q, torch.arange(21, 30, device=DEVICE))
    near(got[..., spared], want[..., spared], size[..., spared], c.rows)
    assert torch.isnan(got[..., [3, 7, 35, 39]]).all()
    none = g.Rotation.of_base(32, magnitude=0.0)
    assert not g.rotate_heads(c.q, rotation=none, batch=c.batch).any()
