"""Single tokens with 17 to 32 query heads of a cache head: two blocks of rows a wavefront, in every width, page and type, with windows and sinks."""
import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, check
from tests.test_gpu_sinks import SinkCase

pytestmark = pytest.mark.gpu

LENGTHS = (3, 700, 1900, 0, 64, 129)


@pytest.mark.parametrize("heads", [(17, 1), (32, 1), (48, 2)])
@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("page", [16, 48, 64, 128])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_heads(d, page, type, heads):
    c = SinkCase([(1, L) for L in LENGTHS], 70, 300, type=type, d=d, page=page, q_heads=heads[0], kv_heads=heads[1], seed=1, token=True)
    c.step()
    check(c, g.attend_token(c.cache, c.batch, c.q, lse=True), 2 ** 30)


@pytest.mark.parametrize("sinks,window", [(1, 1), (4, 7), (200, 100), (130, 63), (128, 256)])
@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64])
def test_windows(page, type, sinks, window):
    """Sinks and windows that begin and end anywhere, pages between them gone."""
    SinkCase([(1, L) for L in (1, 40, 65, 1500, 2100, 777)], sinks, window, type=type, d=128, page=page, q_heads=24, kv_heads=1, seed=sinks + window, token=True,
             evicted=window % 2 == 0).step()


@pytest.mark.parametrize("page", (16, 24, 64, 128))
@pytest.mark.parametrize("type", ("bf16", "fp16", "e4m3"))
def test_many_runs_give_the_same_bits(type, page):
    c = SinkCase([(1, L) for L in (1, 700, 64, 5000, 129)], 0, 0, type=type, d=128, page=page, q_heads=32, kv_heads=1, seed=9, token=True)
    workspace = g.attend_workspace(c.cache, c.batch, c.q_heads)
    for window, sinks in ((0, 0), (64, 0), (64, 4), (300, 130)):
        def run():
            return g.attend_token(c.cache, c.batch, c.q, window=window, sinks=sinks, lse=True, workspace=workspace)
        out, lse = run()
        differ = torch.zeros((), dtype=torch.int64, device=DEVICE)
        for _ in range(500):
            o, l = run()
            differ += (o.view(torch.int16) != out.view(torch.int16)).any() | (l.view(torch.int32) != lse.view(torch.int32)).any()
        assert int(differ) == 0, (window, sinks)
