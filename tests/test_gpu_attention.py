"""The attention of prompts and single tokens over the paged cache, against a plain 64-bit implementation."""
import math

import pytest
import torch

import paper_2602_11688_amd as g
from tests.attention_helpers import DEVICE, Case, check

pytestmark = pytest.mark.gpu


def _prompt(case, **kw):
    return g.attend_prompt(case.cache, case.batch, case.q, lse=True, **kw)


def _token(case, **kw):
    return g.attend_token(case.cache, case.batch, case.q, lse=True, **kw)


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 48])
def test_prompts_of_all_lengths(type, d, page):
    check(c := Case([(1, 1), (5, 5), (63, 63), (64, 64), (65, 130), (200, 777), (0, 40), (257, 257), (7, 1000)], type=type, d=d, page=page), _prompt(c))


@pytest.mark.parametrize("heads", [(1, 1), (3, 1), (7, 7), (28, 4), (40, 8), (71, 1), (160, 1)])
def test_prompts_of_all_groups(heads):
    check(c := Case([(30, 30), (1, 200), (100, 333)], q_heads=heads[0], kv_heads=heads[1], d=128, page=64), _prompt(c))


@pytest.mark.parametrize("d,type", [(8, "bf16"), (40, "fp16"), (72, "bf16"), (80, "e4m3"), (96, "bf16"), (112, "e4m3"), (120, "fp16"), (16, "e4m3")])
def test_odd_head_sizes(d, type):
    check(c := Case([(30, 30), (1, 200), (100, 333)], d=d, type=type, page=32), _prompt(c))
    check(c := Case([(1, 1), (1, 33), (1, 1000)], d=d, type=type, page=32, token=True), _token(c))


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 100000])
@pytest.mark.parametrize("page", [24, 128])
def test_windows(window, page):
    check(c := Case([(1, 1), (300, 300), (70, 900), (1, 640)], page=page), _prompt(c, window=window), window)
    check(c := Case([(1, 1), (1, 300), (1, 901), (1, 640)], page=page, token=True), _token(c, window=window), window)


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 512, 24])
def test_single_tokens_of_all_lengths(type, d, page):
    check(c := Case([(1, L) for L in (1, 2, 31, 32, 33, 127, 128, 129, 1000, 4097, 0, 9000)], type=type, d=d, page=page, token=True), _token(c))


@pytest.mark.parametrize("heads", [(1, 1), (7, 7), (12, 2), (40, 8), (16, 1), (17, 1), (32, 1), (33, 1), (71, 1)])
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_single_tokens_of_all_groups(heads, type):
    check(c := Case([(1, 5), (1, 200), (1, 3001)], q_heads=heads[0], kv_heads=heads[1], d=128, page=64, type=type, token=True), _token(c))


@pytest.mark.parametrize("S", [1, 2, 63, 64, 65, 200])
def test_many_sequences(S):
    lengths = [(37 * i * i + 11 * i) % 1500 for i in range(S)]
    check(c := Case([(1, L) for L in lengths], token=True, page=32), _token(c))
    check(c := Case([(min(L, i % 9), L) for i, L in enumerate(lengths)], page=64), _prompt(c))


def test_long_prefix_is_split():
    """Few rows over many keys: pieces of the keys in workgroups of their own, joined afterwards."""
    for spec in ([(3, 20000)], [(64, 9000), (1, 3)], [(200, 5000)]):
        for type in ("bf16", "e4m3"):
            check(c := Case(spec, q_heads=4, kv_heads=1, d=128, page=64, type=type), _prompt(c))
            assert g.attend_workspace_bytes(c.cache, c.batch, 4) > 0


def test_scale_and_results_given():
    c = Case([(33, 70), (5, 300)], d=128, page=16)
    out, lse = torch.empty_like(c.q), torch.empty((c.T, c.q_heads), device=DEVICE)
    got = _prompt(c, scale=0.03125, out=out)
    assert got[0] is out
    check(c, got, scale=0.03125)
    got = g.attend_prompt(c.cache, c.batch, c.q, lse=lse)
    assert got[1] is lse
    check(c, got)


@pytest.mark.parametrize("order", ["phtd", "pthd", "hptd", "tphd"])
def test_orders_and_strides_of_the_cache_and_rows(order):
    for token in (False, True):
        c = Case([(1, 100), (1, 257)] if token else [(40, 100), (90, 257)], page=48, order=order, token=token, type="e4m3" if order == "pthd" else "bf16")
        wide = torch.full((c.T, c.q_heads * 3, c.d), float("nan"), dtype=c.rows, device=DEVICE)
        q, out = wide[:, 1::3], wide[:, 2::3]
        q.copy_(c.q)
        got = (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, q, lse=True, out=out)
        check(c, got)
        assert torch.isnan(wide[:, 0::3]).all() and torch.equal(q, c.q)


def test_missing_pages_hold_no_keys():
    for token in (False, True):
        for page in (16, 64):
            c = Case([(1, 500), (1, 130), (1, 40)] if token else [(100, 500), (130, 130), (40, 40)], page=page, token=token)
            c.table[0, 0] = -1
            c.table[0, 3] = c.k.shape[0]
            c.table[0, 5] = 2 ** 31 - 1
            c.table[1, 1] = -2 ** 31
            c.table[2, :] = -1
            got = (_token if token else _prompt)(c)
            check(c, got)
            assert torch.isinf(got[1][c.first[2]:]).all() and not got[0][c.first[2]:].any()


def test_lengths_that_do_not_fit():
    """Lengths below the new tokens (rows at negative positions see nothing), negative ones, ones beyond the table."""
    check(c := Case([(10, 4), (3, 0), (5, -7), (20, 100)], page=16), _prompt(c))
    check(c := Case([(1, 0), (1, -5), (1, 100)], page=16, token=True), _token(c))
    c = Case([(6, 90), (4, 33)], page=16, columns=3)
    check(c, _prompt(c))
    c = Case([(1, 90), (1, 33)], page=16, columns=3, token=True)
    check(c, _token(c))


def test_offsets_that_are_not_offsets():
    """Whatever stands in the offsets: rows that belong to no sequence are left alone or zero, nothing else is touched."""
    c = Case([(40, 100), (90, 257)], page=48)
    good = _prompt(c)
    for wrong in ([0, 40, 2 ** 31 - 1], [-5, 40, 130], [130, 40, 0], [2 ** 31 - 1] * 3, [-2 ** 31, 0, 0]):
        c.offsets.copy_(torch.tensor(wrong, dtype=torch.int32))
        _prompt(c)
        g.kv_read(c.cache, c.batch)
    c.offsets.copy_(torch.tensor([0, 40, 130], dtype=torch.int32))
    again = _prompt(c)
    assert torch.equal(good[0], again[0]) and torch.equal(good[1], again[1])


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
def test_infinities_and_nan_beyond_what_is_seen(type):
    """Cache rows beyond a sequence's length and rows that a window leaves out hold NaN: nothing of it arrives."""
    def poison(c, upto, before=0):
        for x in (c.k, c.v):
            for s, (_, L) in enumerate(c.spec):
                for j in list(range(L, -(-L // c.page) * c.page)) + list(range(0, max(0, min(before, L)))):
                    x[int(c.table[s, j // c.page]), :, j % c.page] = float("nan") if type == "e4m3" or j % 2 else float("inf")
            used = set(c.table.flatten().tolist())
            for p in range(x.shape[0]):
                if p not in used:
                    x[p] = float("nan")
    for page in (16, 64):
        c = Case([(30, 100), (70, 70), (1, 129)], page=page, type=type)
        want = _prompt(c)
        poison(c, 0)
        got = _prompt(c)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        check(c, got)
        c = Case([(1, 100), (1, 70), (1, 529)], page=page, type=type, token=True)
        want = _token(c, window=40)
        poison(c, 0, before=30)
        got = _token(c, window=40)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        check(c, got, 40)


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("window", [0, 50])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(type, window):
    """V holds an infinity or NaN at positions in the middle: earlier tokens stay clean, later ones get it."""
    for page in (16, 64):
        c = Case([(200, 300), (90, 90)], page=page, type=type, d=128)
        for s, j, kv, d, x in ((0, 150, 0, 3, math.inf), (0, 210, 1, 77, -math.inf), (0, 290, 0, 3, -math.inf), (1, 40, 1, 5, math.nan), (1, 89, 0, 127, math.inf)):
            c.v[int(c.table[s, j // page]), kv, j % page, d] = math.nan if type == "e4m3" else x
        check(c, _prompt(c, window=window), window)


def test_keys_of_the_lowest_value_and_equal_scores():
    c = Case([(40, 80)], d=64, page=16)
    c.q.zero_()
    check(c, _prompt(c))
    lowest = torch.finfo(torch.bfloat16).min
    c = Case([(1, 80)], d=64, page=16, token=True)
    c.q.fill_(1.0)
    c.k[int(c.table[0, 2])] = lowest                     # scores overflow to -infinity
    out, lse = _token(c)
    c.table[0, 2] = -1                                   # which weighs as much as a page that is not there
    again = _token(c)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_rows_of_infinite_scores_are_nan_and_others_are_not():
    c = Case([(1, 80), (1, 50)], d=64, page=16, token=True)
    c.k[int(c.table[0, 2]), 0, 3, 5] = float("nan")
    out, _ = _token(c)
    G = c.q_heads // c.kv_heads
    assert torch.isnan(out[0, :G]).all() and torch.isfinite(out[0, G:]).all() and torch.isfinite(out[1]).all()


def test_a_cache_of_more_than_32_bits_of_elements():
    """Pages beyond 2^31 elements and 2^32 bytes."""
    H, D, page = 8, 128, 512
    pages = 2 ** 32 // (H * D * page) + 40
    k = torch.empty((pages, H, page, D), dtype=torch.bfloat16, device=DEVICE)
    v = torch.empty_like(k)
    cache = g.KvCache(k, v)
    c = Case([(700, 1500)], q_heads=16, kv_heads=H, d=D, page=page)
    for n, far in enumerate((pages - 1, pages - 30, pages // 2 + 3)):
        k[far], v[far] = c.k[int(c.table[0, n])], c.v[int(c.table[0, n])]
    table = torch.tensor([[pages - 1, pages - 30, pages // 2 + 3]], dtype=torch.int32, device=DEVICE)
    batch = g.KvBatch(table, c.lengths, c.offsets, tokens=c.T)
    want, got = _prompt(c), g.attend_prompt(cache, batch, c.q, lse=True)
    assert torch.equal(want[0], got[0])
    one = g.KvBatch(table, c.lengths)
    t = Case([(1, 1500)], q_heads=16, kv_heads=H, d=D, page=page, token=True)
    got = g.attend_token(cache, one, c.q[-1:], lse=True)
    check_last = g.attend_prompt(cache, g.KvBatch(table, c.lengths, torch.tensor([0, 1], dtype=torch.int32, device=DEVICE), tokens=1), c.q[-1:], lse=True)
    assert torch.allclose(got[0].float(), check_last[0].float(), atol=2 ** -7, rtol=2 ** -6) and torch.allclose(got[1], check_last[1], atol=2 ** -12)
    g.kv_write(cache, batch, c.new_k, c.new_v)
    back = g.kv_read(cache, batch)
    assert torch.equal(back[0], c.new_k) and torch.equal(back[1], c.new_v)
    assert t.T == 1


def test_the_same_twice_and_on_another_stream():
    for token in (False, True):
        c = Case([(1, 3000), (1, 1234)] if token else [(300, 3000), (100, 1234)], d=128, page=64, token=token)
        f = _token if token else _prompt
        want = f(c)
        for _ in range(3):
            got = f(c)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = f(c, stream=s)
        s.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_captured_into_a_graph_and_replayed_with_new_contents():
    """A decode step (write, then attend) captured once; lengths, pages, queries and cache change between the replays."""
    c = Case([(1, 900), (1, 70), (1, 2000)], d=128, page=64, token=True, type="e4m3", columns=40, spare=40)
    ws = g.attend_workspace(c.cache, c.batch, c.q_heads)
    out, lse = torch.empty_like(c.q), torch.empty((c.T, c.q_heads), device=DEVICE)

    def step():
        g.kv_write(c.cache, c.batch, c.new_k, c.new_v)
        g.attend_token(c.cache, c.batch, c.q, out=out, lse=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([900, 70, 2000], [901, 71, 1999], [64, 1, 2048], [0, 65, 640]):
        c.spec = [(1, L) for L in lengths]
        c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.q.normal_()
        c.new_v.normal_()
        graph.replay()
        torch.cuda.synchronize()
        check(c, (out, lse))
        want = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_one_workspace_for_calls_of_all_batches():
    """Prompts and single tokens of batches of different sizes take turns on one workspace."""
    prompt = Case([(3, 20000)], q_heads=4, kv_heads=1, d=128, page=64)
    tokens = [Case([(1, 5000 + 777 * i) for i in range(S)], q_heads=4, kv_heads=1, d=128, page=64, token=True, seed=S) for S in (1, 9, 3)]
    size = max(g.attend_workspace_bytes(c.cache, c.batch, 4) for c in [prompt] + tokens)
    ws = torch.zeros(size, dtype=torch.uint8, device=DEVICE)
    for c in tokens + tokens[::-1]:
        check(prompt, _prompt(prompt, workspace=ws))
        check(c, _token(c, workspace=ws))
        check(c, g.attend_prompt(c.cache, c.batch, c.q, lse=True, workspace=ws))     # (a prompt of one token each)
        check(c, _token(c, workspace=ws))


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30])
def test_the_widest_windows(window):
    """Rows before position 0, and positions near the window's end of 32 bits."""
    check(c := Case([(40, 20), (300, 200), (7, 600)], page=16), _prompt(c, window=window), window)
    check(c := Case([(40, 20), (300, 200), (7, 600)], page=64), _prompt(c, window=window), window)
    check(c := Case([(1, 0), (1, -3), (1, 100)], page=16, token=True), _token(c, window=window), window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("type", ["fp16", "e4m3"])
def test_windows_over_pieces_and_many_tiles(d, type):
    """Long windows in whole tiles, begun and ended inside one, in one piece and in several."""
    for spec, window in (([(900, 5000), (3, 4000)], 1000), ([(5, 20000)], 7001), ([(1500, 1500)], 333)):
        for page in (64, 80, 512):
            check(c := Case(spec, q_heads=2, kv_heads=2, d=d, page=page, type=type), _prompt(c, window=window), window)


def test_missing_pages_of_whole_tiles_and_of_many_rows():
    """Pages of several tiles that are not there, the first and the last among them."""
    for type in ("bf16", "e4m3"):
        for d in (64, 128):
            c = Case([(700, 2000), (300, 300)], page=128, d=d, type=type)
            for s, i in ((0, 0), (0, 1), (0, 7), (0, 11), (0, 15), (1, 0), (1, 2)):
                c.table[s, i] = -1 if i % 2 else c.k.shape[0] + i
            check(c, _prompt(c))


def test_scores_near_the_end_of_32_bits():
    """All scores of a row about -3.3e38 in powers of two: no finite score counts as none."""
    for token in (False, True):
        c = Case([(1, 40), (1, 100)], d=64, page=64, token=token)
        c.k.fill_(-2.0 ** 100)
        c.q.fill_(2.0 ** 20)
        # (64 * 2^120 = 2^126, times the scale, times log2(e) = -3.3e38)
        scale = 3.3e38 / 2.0 ** 126 / 1.4426950408889634
        out, lse = (_token if token else _prompt)(c, scale=scale)
        want = torch.stack([c.dense("v", s)[0].mean(0) for s in range(2)]).repeat_interleave(c.q_heads // c.kv_heads, 1)
        # (equal weights: the mean, a rounding of the result and one of each weight's)
        assert ((out.double() - want).abs() <= 2.0 ** -7).all() and torch.isfinite(lse).all()


def test_dimensions_of_one_element_have_any_stride():
    c = Case([(1, 50)], q_heads=4, kv_heads=1, d=64, page=64, token=True)
    want = _token(c)
    k, v = (torch.as_strided(x, x.shape, (x.stride(0), 3, x.stride(2), 1)) for x in (c.k, c.v))
    q = torch.as_strided(c.q, c.q.shape, (5, c.q.stride(1), 1))
    got = g.attend_token(g.KvCache(k, c.v), c.batch, q, lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g.kv_write(g.KvCache(k, v), c.batch, torch.as_strided(c.new_k, c.new_k.shape, (1, 7, 1)), c.new_v)


@pytest.mark.parametrize("d,page", [(64, 64), (64, 48), (128, 512), (128, 80)])
def test_the_most_pieces(d, page):
    """Few rows over very many keys: as many pieces as there can be, rows of several sequences, some with few pieces."""
    for spec in ([(30, 30000), (3, 500)], [(1, 40000)], [(100, 12000), (1, 1), (40, 5000)]):
        check(c := Case(spec, q_heads=8, kv_heads=1, d=d, page=page), _prompt(c))
        check(c, _prompt(c, window=9999), 9999)
