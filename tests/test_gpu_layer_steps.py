"""A layer's steps as they are run one after the other: prompts normed, rotated and appended, attention over a window and the first tokens, then
captured decode steps while pages between the two are taken away; the cache and every result against the definition in 64 bits."""
import pytest
import torch

import paper_2602_11688_amd as g
from tests.append_helpers import How, near
from tests.attention_helpers import DEVICE, check
from tests.test_gpu_kv_cache import _quantised
from tests.test_gpu_sinks import SinkCase

pytestmark = pytest.mark.gpu

WINDOW, SINKS, STEPS, PAGE = 100, 20, 40, 16


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,pairs,layout,norm", [(128, 64, "halves", "shared"), (64, 20, "neighbours", "each"), (80, 36, "halves", "")])
def test_prompts_and_steps(type, d, pairs, layout, norm):
    c = SinkCase([(70, 70), (9, 300), (1, 1)], SINKS, WINDOW, type=type, d=d, page=PAGE, q_heads=8, kv_heads=2, columns=30, spare=80, seed=pairs)
    free = iter(sorted(set(range(c.k.shape[0])) - set(c.table[c.table >= 0].tolist())))
    for s in range(3):
        for i in range(30):
            if c.table[s, i] < 0:
                c.table[s, i] = next(free)
    how = How(d, pairs=pairs, layout=layout, norm=norm, heads=(8, 2))
    calls = dict(rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1])
    workspace = g.attend_workspace(c.cache, c.batch, 8)

    def held(pos, k):
        """What the cache holds of the sequences' keys at `pos` is what the definition gives of k."""
        got = c.k.view(torch.uint8) if type == "e4m3" else c.k
        page, slot = c.table[torch.arange(3, device=DEVICE), pos // PAGE].long(), pos % PAGE
        want, size = how.turned(k, pos, 1)
        if type != "e4m3":
            return near(got[page, :, slot], want, size, c.rows)
        values, bytes_ = _quantised(want)
        assert torch.equal(c.scales[0][page, :, slot], bytes_)
        assert torch.equal(got[page, :, slot].view(torch.float8_e4m3fn).double() * torch.exp2(bytes_.double() - 127)[..., None], values)

    # the prompts
    last = torch.tensor([69, 78, 79], device=DEVICE)
    c.q = g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, **calls)
    check(c, g.attend_prompt(c.cache, c.batch, c.q, window=WINDOW, sinks=SINKS, lse=True, workspace=workspace), WINDOW)
    held(torch.tensor([69, 299, 0], device=DEVICE), c.new_k[last])

    # the steps: one captured, replayed with other rows and longer sequences
    one = g.KvBatch(c.table, c.lengths)
    k, v, q = (torch.empty((3, h, d), dtype=c.rows, device=DEVICE) for h in (2, 2, 8))
    turned, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((3, 8), device=DEVICE)

    def step():
        c.lengths.add_(1)
        g.kv_append(c.cache, one, k, v, q, out=turned, **calls)
        g.attend_token(c.cache, one, turned, window=WINDOW, sinks=SINKS, out=out, lse=lse, workspace=workspace)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1)
    c.first, c.T = [0, 1, 2, 3], 3
    graph = None
    for i in range(STEPS):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=gen, device=DEVICE))
        if i == 1:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        step() if graph is None else graph.replay()
        c.spec = [(1, int(L)) for L in c.lengths]
        pos = c.lengths.long() - 1
        near(turned, *how.turned(q, pos), c.rows)
        held(pos, k)
        c.q = turned
        check(c, (out, lse), WINDOW)
        # pages that no coming step sees
        for s, (_, L) in enumerate(c.spec):
            for j in range((L + 1 - WINDOW) // PAGE):
                if j * PAGE >= SINKS:
                    c.table[s, j] = -1
    assert [L for _, L in c.spec] == [70 + STEPS, 300 + STEPS, 1 + STEPS]
