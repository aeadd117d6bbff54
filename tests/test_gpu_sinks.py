"""Attention over a sliding window and the first tokens of a sequence, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case, check

pytestmark = pytest.mark.gpu


class SinkCase(Case):
    """A case whose tokens see their first positions beside a window; `evicted`: pages that no new token sees are not there, and what
    the cache holds in other sequences' or nobody's pages is infinite."""

    def __init__(self, spec, sinks, window, *, evicted=False, **how):
        super().__init__(spec, **how)
        self.sinks, self.window = sinks, window
        if evicted:
            for s, (n, L) in enumerate(spec):
                for i in range(self.table.shape[1]):
                    if (i + 1) * self.page <= L - n + 1 - window and i * self.page >= sinks and self.table[s, i] >= 0:
                        if self.type != "e4m3":
                            self.k[self.table[s, i]] = math.inf
                            self.v[self.table[s, i]] = math.nan
                        else:
                            for x, y in zip((self.k, self.v), self.scales):
                                x.view(torch.uint8)[self.table[s, i]] = 0x7f
                                y[self.table[s, i]] = 255
                        self.table[s, i] = -1 if i % 2 else self.k.shape[0] + i

    def attend(self, scale=None, window=0):
        scale, G = self.d ** -0.5 if scale is None else scale, self.q_heads // self.kv_heads
        out = torch.zeros((self.T, self.q_heads, self.d), dtype=torch.float64, device=DEVICE)
        size, lse = torch.zeros_like(out), torch.full((self.T, self.q_heads), -math.inf, dtype=torch.float64, device=DEVICE)
        for s, (n, L) in enumerate(self.spec):
            (k, held), (v, _) = self.dense("k", s), self.dense("v", s)
            if n == 0 or len(k) == 0:
                continue
            me = torch.arange(max(L, 0) - n, max(L, 0), device=DEVICE)[:, None]
            key = torch.arange(len(k), device=DEVICE)
            seen = held & (key <= me) & ((me - key < window) | (key < self.sinks) if window else key >= 0)
            # (only keys that somebody sees: others may hold anything)
            some = seen.any(0)
            k, v, seen = k[some], v[some], seen[:, some]
            for h in range(self.q_heads):
                at = slice(self.first[s], self.first[s] + n)
                score = (self.q[at, h].double() @ k[:, h // G].T.contiguous() * scale).masked_fill(~seen, -math.inf)
                lse[at, h] = torch.logsumexp(score, -1)
                w = torch.where(seen, torch.exp(score - lse[at, h, None]), torch.zeros_like(score))
                x = v[:, h // G]
                tame = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
                o = w @ tame
                for kind in (math.inf, -math.inf, math.nan):
                    is_kind = (torch.isnan(x) if math.isnan(kind) else x == kind).double()
                    o = o + torch.where(seen.double() @ is_kind > 0, kind, 0.0)
                out[at, h], size[at, h] = o, w @ tame.abs()
        return out, lse, size

    def prompt(self, **how):
        check(self, g.attend_prompt(self.cache, self.batch, self.q, window=self.window, sinks=self.sinks, lse=True, **how), self.window)

    def step(self, **how):
        check(self, g.attend_token(self.cache, self.batch, self.q, window=self.window, sinks=self.sinks, lse=True, **how), self.window)


RAGGED = [(5, 5), (0, 9), (1, 40), (33, 500), (170, 300), (0, 0), (64, 64), (7, 1500), (200, 901)]
SEEN = [(1, 1), (4, 7), (64, 64), (200, 100), (1000, 300), (3, 5000), (130, 63), (63, 129), (128, 256), (5, 320)]


@pytest.mark.parametrize("sinks,window", SEEN)
@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 128), (64, 16), (128, 48), (80, 512)])
def test_prompts(type, d, page, sinks, window):
    SinkCase(RAGGED, sinks, window, type=type, d=d, page=page, q_heads=8, kv_heads=2, seed=sinks + window, evicted=window % 2 == 0).prompt()


@pytest.mark.parametrize("sinks,window", SEEN + [(600, 50), (257, 513)])
@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 128), (64, 16), (128, 48), (80, 512)])
def test_single_tokens(type, d, page, sinks, window):
    spec = [(1, L) for L in (1, 5, 40, 64, 65, 300, 1500, 777, 2100, 0, 129)]
    SinkCase(spec, sinks, window, type=type, d=d, page=page, q_heads=8, kv_heads=2, seed=sinks + window, token=True, evicted=window % 2 == 0).step()


@pytest.mark.parametrize("heads", [(1, 1), (12, 12), (17, 1), (32, 1), (40, 1), (71, 1)])
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_heads(heads, type):
    SinkCase([(1, L) for L in (3, 700, 1900)], 70, 300, type=type, d=64, page=64, q_heads=heads[0], kv_heads=heads[1], seed=1, token=True).step()
    SinkCase([(40, 40), (9, 1100)], 70, 300, type=type, d=64, page=64, q_heads=heads[0], kv_heads=heads[1], seed=1).prompt()


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("sinks,window", [(4, 6000), (3000, 3000), (9000, 100), (64, 2000)])
def test_few_rows_in_pieces(type, page, sinks, window):
    """Keys split over workgroups, pieces that end inside the sinks, at their end and in the window."""
    SinkCase([(3, 12000), (9, 2500)], sinks, window, type=type, d=128, page=page, q_heads=4, kv_heads=1, seed=3, evicted=True).prompt()
    SinkCase([(1, 12000), (1, 2500)], sinks, window, type=type, d=128, page=page, q_heads=4, kv_heads=1, seed=3, token=True, evicted=True).step()


@pytest.mark.parametrize("sinks,window", [(4, 100), (130, 50)])
def test_lengths_and_pages_that_are_not_there(sinks, window):
    """Lengths beyond the table, shorter than the new tokens, tables whose window lies behind their end, sinks whose pages are gone."""
    for token in (False, True):
        spec = [(1, 400), (1, 130), (1, 200), (1, 0), (1, 160), (1, 60)] if token else [(20, 12), (9, 400), (30, 200), (4, 0), (50, 160), (3, 170)]
        c = SinkCase(spec, sinks, window, d=64, page=16, columns=10, token=token, seed=2)
        c.table[2, 0] = -1
        c.table[2, 9] = c.k.shape[0] + 3
        c.table[4, :] = -1
        c.step() if token else c.prompt()


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
def test_values_that_are_not_finite(type, d, page):
    """In the sinks they reach every row that sees them, in the window the rows whose window it is, between the two nobody."""
    for token in (False, True):
        spec = [(1, 900), (1, 60)] if token else [(300, 900), (60, 60)]
        for at, kind in ((2, math.inf), (9, math.nan), (40, -math.inf), (200, math.nan), (610, math.inf), (700, math.nan), (899, -math.inf)):
            c = SinkCase(spec, 10, 100, type=type, d=d, page=page, q_heads=4, kv_heads=2, token=token, seed=at)
            c.v[c.table[0, at // page], 1, at % page, 5] = math.nan if type == "e4m3" else kind
            c.step() if token else c.prompt()


def test_without_a_window_there_are_no_sinks():
    c = Case(RAGGED, d=64, seed=5)
    a, b = (g.attend_prompt(c.cache, c.batch, c.q, sinks=sinks, lse=True) for sinks in (0, 50))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_window_that_reaches_the_sinks_sees_all():
    """Nothing lies between: what a call without a window says, up to the order of sums."""
    c = SinkCase(RAGGED, 1000, 700, d=128, page=64, seed=6)
    c.prompt()
    check(c, g.attend_prompt(c.cache, c.batch, c.q, window=700, sinks=2 ** 31 - 1, lse=True))


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [32767, 32704])
def test_positions_near_the_end_of_31_bits(type, page):
    """A conversation of 2^31 tokens of which a few pages are left: single tokens and a prompt, against the same keys side by side."""
    columns = (2 ** 31 - 1024) // page
    cache = g.KvCache.empty(3, 1, 64, page, type)
    k, v = (torch.randn((3 * page, 1, 64), device=DEVICE, generator=torch.Generator(DEVICE).manual_seed(i)).to(torch.bfloat16) for i in (1, 2))
    whole = g.KvBatch(torch.arange(3, device=DEVICE, dtype=torch.int32)[None], torch.tensor([3 * page], dtype=torch.int32, device=DEVICE),
                      torch.tensor([0, 3 * page], dtype=torch.int32, device=DEVICE), tokens=3 * page)
    g.kv_write(cache, whole, k, v)
    table = torch.full((1, columns), -1, dtype=torch.int32, device=DEVICE)
    table[0, 0], table[0, -2], table[0, -1] = 0, 1, 2
    near = torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEVICE)
    q = torch.randn((9, 2, 64), device=DEVICE).to(torch.bfloat16)
    for L_near, sinks, window in ((3 * page, 70, page + 100), (3 * page - 5, 5, 300), (2 * page + 9, 200, 4000)):
        far = columns * page - (3 * page - L_near)
        for n in (1, 9):
            def batch(table, L):
                return g.KvBatch(table, torch.tensor([L], dtype=torch.int32, device=DEVICE), torch.tensor([0, n], dtype=torch.int32, device=DEVICE) if n > 1 else None, tokens=n)
            f = g.attend_token if n == 1 else g.attend_prompt
            a = f(cache, batch(table, far), q[:n], window=window, sinks=sinks, lse=True)
            # (the sinks' page and the window's, with the same distances between new tokens and window)
            b = f(cache, batch(near, L_near), q[:n], window=window, sinks=sinks, lse=True)
            # each is off by a rounding of weights and one of the result: see check()
            assert ((a[0].double() - b[0].double()).abs() <= 2 * (2 * 2.0 ** -8 + 2.0 ** -12) * 6).all() and ((a[1] - b[1]).abs() <= 2.0 ** -11).all()


def test_a_step_captured_and_replayed():
    """Lengths that grow past the window while a graph is replayed, pages between sinks and window taken away, two graphs on one workspace."""
    c = SinkCase([(1, 40), (1, 90), (1, 500)], 5, 64, d=128, page=16, q_heads=8, kv_heads=2, columns=40, spare=90, token=True, seed=7)
    free = iter(sorted(set(range(c.k.shape[0])) - set(c.table[c.table >= 0].tolist())))
    for s in range(3):
        for i in range(40):
            if c.table[s, i] < 0:
                c.table[s, i] = next(free, -1)
    workspace = g.attend_workspace(c.cache, c.batch, 8)
    prompt = g.KvBatch(c.table, c.lengths, torch.arange(4, dtype=torch.int32, device=DEVICE), tokens=3)
    outs, graphs = [], []
    for f, b in ((g.attend_token, c.batch), (g.attend_prompt, prompt)):
        f(c.cache, b, c.q, window=64, sinks=5, lse=True, workspace=workspace)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f(c.cache, b, c.q, window=64, sinks=5, lse=True, workspace=workspace))
        graphs.append(graph)
    for step in range(4):
        c.lengths.add_(13)
        c.spec = [(1, int(L)) for L in c.lengths]
        c.table[2, 1 + step] = -1
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            check(c, out, 64)
        c.step(workspace=workspace)


def test_results_do_not_depend_on_the_run():
    c = SinkCase([(3, 12000), (9, 2500), (300, 4000)], 100, 2000, type="e4m3", d=128, page=64, q_heads=8, kv_heads=2, seed=8)
    a = [g.attend_prompt(c.cache, c.batch, c.q, window=2000, sinks=100, lse=True) for _ in range(3)]
    assert all(torch.equal(a[0][0], x[0]) and torch.equal(a[0][1], x[1]) for x in a)
    c = SinkCase([(1, L) for L in (12000, 2500, 40, 4000)], 100, 2000, type="bf16", d=128, page=64, q_heads=8, kv_heads=2, seed=8, token=True)
    a = [g.attend_token(c.cache, c.batch, c.q, window=2000, sinks=100, lse=True) for _ in range(3)]
    assert all(torch.equal(a[0][0], x[0]) and torch.equal(a[0][1], x[1]) for x in a)


@pytest.mark.parametrize("page", (16, 24, 64))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("type", ("bf16", "fp16", "e4m3"))
def test_many_runs_give_the_same_bits(type, d, page):
    """What goes wrong in one run of a hundred shows here and in no comparison of single results."""
    prompt = SinkCase([(1, 1), (300, 300), (70, 900), (1, 640)], 0, 0, type=type, d=d, page=page, seed=9)
    step = SinkCase([(1, L) for L in (1, 700, 64, 5000, 129)], 0, 0, type=type, d=d, page=page, seed=9, token=True)
    for c, attend in ((prompt, g.attend_prompt), (step, g.attend_token)):
        workspace = g.attend_workspace(c.cache, c.batch, c.q_heads)
        for window, sinks in ((64, 0), (200, 0), (64, 4), (300, 130)):
            def run():
                return attend(c.cache, c.batch, c.q, window=window, sinks=sinks, lse=True, workspace=workspace)
            out, lse = run()
            differ = torch.zeros((), dtype=torch.int64, device=DEVICE)
            for _ in range(500):
                o, l = run()
                differ += (o.view(torch.int16) != out.view(torch.int16)).any() | (l.view(torch.int32) != lse.view(torch.int32)).any()
            assert int(differ) == 0, (attend.__name__, window, sinks)
