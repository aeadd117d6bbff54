"""Heads normed, rotated and appended to the paged cache, or rotated alone, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2602_11688_amd as g
from tests.append_helpers import How, near, positions_of
from tests.attention_helpers import DEVICE, Case
from tests.test_gpu_kv_cache import _positions, _quantised

pytestmark = pytest.mark.gpu

RAGGED = [(5, 5), (0, 9), (1, 40), (33, 50), (17, 300), (0, 0), (64, 64)]
# d, pairs, layout: halves that begin at a whole load, at half of one and anywhere; whole heads and parts of them
SHAPES = [(64, 32, "halves"), (128, 64, "halves"), (128, 64, "neighbours"), (128, 32, "halves"), (64, 5, "neighbours"), (72, 36, "halves"), (80, 40, "halves"),
          (80, 13, "halves"), (80, 13, "neighbours"), (8, 4, "halves"), (8, 4, "neighbours"), (16, 8, "halves"), (120, 60, "halves"), (96, 48, "neighbours"),
          (128, 1, "halves"), (112, 24, "halves"), (128, 63, "halves"), (128, 0, "halves"), (40, 0, "halves"), (8, 3, "halves"), (16, 3, "halves"), (16, 7, "halves"),
          (96, 44, "halves"), (64, 31, "halves"), (80, 9, "halves"), (128, 2, "neighbours"), (24, 11, "halves"), (48, 20, "halves"), (96, 36, "halves")]


def _append(c, how, q=None, k=None, v=None, out=None, **more):
    """Runs kv_append and checks all that it wrote, and that nothing else changed."""
    q, k, v = c.q if q is None else q, c.new_k if k is None else k, c.new_v if v is None else v
    pos = positions_of(c)
    want_q, size_q = how.turned(q, pos, 0)
    want_k, size_k = how.turned(k, pos, 1)
    before = [x.clone() for x in (c.k.view(torch.uint8) if c.type == "e4m3" else c.k, c.v.view(torch.uint8) if c.type == "e4m3" else c.v, *c.scales)]
    got = g.kv_append(c.cache, c.batch, k, v, q, rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1], out=out, **more)
    torch.cuda.synchronize()
    near(got, want_q, size_q, c.rows)
    rows = list(_positions(c))
    t, page, slot = (torch.tensor([r[i] for r in rows], dtype=torch.long, device=DEVICE) for i in range(3))
    for i, (want, size) in enumerate(((want_k, size_k), (v.double(), None))):
        held = (c.k, c.v)[i]
        if c.type == "e4m3":
            # (the definition's codes: 64 bits leave no value that lies on another side of a border)
            values, bytes_ = _quantised(want)
            now = before[2 + i].clone()
            now[page, :, slot] = bytes_[t]
            assert torch.equal(c.scales[i], now)
            codes = held.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).double()
            codes = codes * torch.exp2(bytes_[t].double() - 127)[..., None]
            same = (codes == values[t]) | (torch.isnan(codes) & torch.isnan(values[t]))
            assert same.all(), (i, int((~same).sum()))
            held = held.view(torch.uint8).clone()
            held[page, :, slot] = before[i][page, :, slot]
            assert torch.equal(held, before[i])
        else:
            if i == 0:
                near(held[page, :, slot], want[t], size[t], c.rows)
            else:
                assert torch.equal(held[page, :, slot].view(torch.int16), v[t].view(torch.int16))
            held = held.clone()
            held[page, :, slot] = before[i][page, :, slot]
            assert torch.equal(held.view(torch.int16), before[i].view(torch.int16))
    return got


@pytest.mark.parametrize("type,d,pairs,layout", [(type, *shape) for type in ("bf16", "fp16", "e4m3") for shape in SHAPES if type != "e4m3" or shape[0] % 16 == 0])
def test_shapes(type, d, pairs, layout):
    norm = ["shared", "each", "ones", ""][(d + pairs) % 4]
    c = Case(RAGGED, type=type, d=d, q_heads=6, kv_heads=3, page=16, seed=d + pairs)
    _append(c, How(d, pairs=pairs, layout=layout, norm=norm if pairs else "shared", heads=(6, 3), seed=pairs))


@pytest.mark.parametrize("type", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("norm", ["", "ones", "shared", "each"])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_norms(type, norm, layout):
    c = Case([(40, 90), (1, 700)], type=type, d=128, q_heads=32, kv_heads=8, page=48, seed=3)
    _append(c, How(128, pairs=64, layout=layout, norm=norm, eps=1e-2 if norm == "ones" else 1e-6, heads=(32, 8), base=1e6, magnitude=1.25))


@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (5, 5), (64, 2), (96, 48)])
@pytest.mark.parametrize("token", [False, True])
def test_heads(heads, token):
    spec = [(1, L) for L in (1, 2, 65, 1000, 17)] if token else [(300, 300), (1, 1), (3, 77)]
    c = Case(spec, d=64, q_heads=heads[0], kv_heads=heads[1], page=32, token=token, seed=9)
    _append(c, How(64, pairs=32, norm="shared", heads=heads))


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_missing_pages_and_lengths(type):
    """Pages that are not there, lengths shorter than the new tokens, lengths beyond the table: dropped; the queries are rotated all the same."""
    c = Case([(20, 12), (9, 100), (30, 64), (4, 0)], type=type, d=64, page=16, columns=4, seed=2)
    c.table[2, 2] = -1
    c.table[2, 3] = c.k.shape[0] + 5
    _append(c, How(64, pairs=32, norm="shared"))


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_axes(axes, layout):
    c = Case(RAGGED, type="bf16", d=128, q_heads=4, kv_heads=2, page=16, seed=axes)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(axes)
    positions = torch.randint(-50, 100000, (axes + 2, c.T), generator=gen, device=DEVICE, dtype=torch.int32)[1:axes + 1]
    how = How(128, pairs=60 if layout == "neighbours" else 64, layout=layout, positions=positions, axis_of_pair=[i * 7 % axes for i in range(60 if layout == "neighbours" else 64)],
              heads=(4, 2), norm="each")
    _append(c, how)


def test_positions_without_axes():
    c = Case(RAGGED, d=64, seed=4)
    positions = torch.arange(c.T, device=DEVICE, dtype=torch.int32) * 3 - 100
    _append(c, How(64, pairs=32, positions=positions))


@pytest.mark.parametrize("base", [10000.0, 1.0])
def test_far_positions(base):
    """Angles up to 2^31 radians: 32 bits would hold none of their turns."""
    c = Case([(6, 6)], type="fp16", d=64, seed=5)
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 123456789, -1, 0], device=DEVICE, dtype=torch.int32)
    _append(c, How(64, pairs=32, positions=positions, base=base))


def test_far_places():
    """A token at the end of a table of 2^31 - 1024 positions whose other pages are not there."""
    page = 32767
    columns = (2 ** 31 - 1024) // page
    table = torch.full((1, columns), -1, dtype=torch.int32, device=DEVICE)
    table[0, -1] = 0
    cache = g.KvCache.empty(1, 1, 64, page, "bf16")
    L = columns * page
    batch = g.KvBatch(table, torch.tensor([L], dtype=torch.int32, device=DEVICE))
    how = How(64, pairs=32, heads=(2, 1))
    k, q = (torch.randn((1, h, 64), device=DEVICE).to(torch.bfloat16) for h in (1, 2))
    got = g.kv_append(cache, batch, k, k, q, rotation=how.rotation)
    pos = torch.tensor([L - 1], device=DEVICE)
    near(got, *how.turned(q, pos), torch.bfloat16)
    want, size = how.turned(k, pos)
    near(cache.k[0, :, (L - 1) % page][None], want, size, torch.bfloat16)


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_rows_that_32_bits_do_not_norm(type):
    """Squares beyond 32 bits, squares that underflow beside a tiny eps, rows of zeros, the end of the type's range."""
    c = Case([(8, 8)], type=type, d=64, q_heads=2, kv_heads=2, seed=6)
    by = torch.tensor([1.0, 1e30, 3e37, 1e-25, 1e-38, 0.0, 1e19, 1e-13], device=DEVICE)[:, None, None]
    q, k = ((torch.randn((8, 2, 64), device=DEVICE, generator=torch.Generator(DEVICE).manual_seed(i)) * by).to(torch.bfloat16) for i in (1, 2))
    for eps in (1e-6, 1e-30, 1e-38):
        _append(c, How(64, pairs=32, norm="shared", eps=eps, heads=(2, 2)), q=q, k=k)


def test_rows_of_zeros_and_tiny_eps():
    """A root of a number below the normal range of 32 bits."""
    x = torch.zeros((3, 2, 64), dtype=torch.float16, device=DEVICE)
    x[1, 0, 3] = 2.0 ** -24
    x[2] = 1.0
    for dtype in (torch.float16, torch.bfloat16):
        for eps in (1e-6, 1e-20, 1e-40):
            how = How(64, norm="ones", eps=eps, heads=(2, 1))
            y = x.to(dtype)
            near(g.rotate_heads(y, norm=how.norms[0]), *how.turned(y, None), dtype)


def test_no_tokens():
    c = Case(RAGGED, d=64, seed=1)
    none = g.KvBatch(c.table, c.lengths, torch.zeros_like(c.offsets), tokens=0)
    positions = torch.zeros((3, 0), dtype=torch.int32, device=DEVICE)
    rotation = g.Rotation.of_base(32, positions=positions, axis_of_pair=[i % 3 for i in range(32)])
    assert g.kv_append(c.cache, none, c.new_k[:0], c.new_v[:0], c.q[:0], rotation=rotation).shape == (0, 8, 64)
    assert g.rotate_heads(c.q[:0], rotation=rotation).shape == (0, 8, 64)


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("normed", [False, True])
def test_not_finite_rows(type, normed):
    """What is not finite stays in its row, and without a norm in its pair (each of which the definition gives)."""
    c = Case([(6, 6)], type=type, d=128, q_heads=2, kv_heads=2, seed=7)
    q, k = c.q.clone(), c.new_k.clone()
    for x in (q, k):
        x[1, 0, 5] = math.inf
        x[2, 1, 70] = -math.inf
        x[3, 0, 127] = math.nan
        x[4, 0, 100] = math.inf
        x[4, 0, 36] = math.inf
    _append(c, How(128, pairs=40, norm="shared" if normed else "", heads=(2, 2)), q=q, k=k)


def test_strides_orders_and_in_place():
    """Rows inside wider ones, a cache in another order of dimensions, results over their own queries."""
    for order in ("pthd", "htpd"):
        c = Case(RAGGED, type="fp16", d=64, q_heads=4, kv_heads=2, seed=8, order=order)
        wide = torch.zeros((c.T, 8, 64), dtype=c.rows, device=DEVICE)
        wide[:, :4], wide[:, 4:6], wide[:, 6:] = c.q, c.new_k, c.new_v
        how = How(64, pairs=32, norm="each", heads=(4, 2))
        want, size = how.turned(c.q, positions_of(c))
        got = g.kv_append(c.cache, c.batch, wide[:, 4:6], wide[:, 6:], wide[:, :4], rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1], out=wide[:, :4])
        assert got.data_ptr() == wide.data_ptr() and torch.equal(wide[:, 4:6], c.new_k) and torch.equal(wide[:, 6:], c.new_v)
        near(got, want, size, c.rows)
        _append(c, how)


@pytest.mark.parametrize("S", [65, 300, 5000])
def test_many_sequences(S):
    """More sequences than a wavefront looks at at once, many of them without a token, tokens behind the last one."""
    gen = torch.Generator()
    gen.manual_seed(S)
    new = torch.randint(0, 3, (S,), generator=gen) * (torch.rand(S, generator=gen) < 0.4)
    new[S // 2:S // 2 + 200] = 0
    spec = [(int(n), int(n) + s % 37) for s, n in enumerate(new)]
    c = Case(spec, d=16, q_heads=2, kv_heads=1, page=16, seed=S)
    how = How(16, pairs=8, heads=(2, 1))
    _append(c, how)
    # rows behind the last sequence
    more = g.KvBatch(c.table, c.lengths, c.offsets, tokens=c.T + 40)
    x = torch.randn((c.T + 40, 3, 16), device=DEVICE).to(torch.bfloat16)
    out = torch.full_like(x, 7.0)
    g.rotate_heads(x, rotation=how.rotation, batch=more, out=out)
    assert (out[c.T:] == 7.0).all()
    near(out[:c.T], *how.turned(x[:c.T], positions_of(c)), torch.bfloat16)


def test_keys_alone_and_nothing_to_do():
    c = Case(RAGGED, type="e4m3", d=64, seed=10)
    other = Case(RAGGED, type="e4m3", d=64, seed=10)
    assert g.kv_append(c.cache, c.batch, c.new_k, c.new_v) is None              # neither norm nor rotation: kv_write
    g.kv_write(other.cache, other.batch, c.new_k, c.new_v)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((c.k, c.v, *c.scales), (other.k, other.v, *other.scales)))
    none = g.KvBatch(c.table, c.lengths, torch.zeros_like(c.offsets), tokens=0)
    assert g.kv_append(c.cache, none, c.new_k[:0], c.new_v[:0], c.q[:0], k_norm=g.HeadNorm()).shape == (0, 8, 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,pairs,layout", SHAPES)
def test_rows_alone(dtype, d, pairs, layout):
    T, H = 333, 5
    x = (3 * torch.randn((T, H, d), device=DEVICE, generator=torch.Generator(DEVICE).manual_seed(d))).to(dtype)
    positions = torch.stack([torch.arange(T, device=DEVICE) // 18, torch.arange(T, device=DEVICE) % 18]).to(torch.int32)
    for norm in ("", "each"):
        if not pairs and not norm:
            continue
        how = How(d, pairs=pairs, layout=layout, positions=positions if pairs else None, axis_of_pair=[i % 2 for i in range(pairs)] if pairs else None, norm=norm, heads=(H, 1))
        near(g.rotate_heads(x, rotation=how.rotation, norm=how.norms[0]), *how.turned(x, None), dtype)
        y = x.clone()
        assert g.rotate_heads(y, rotation=how.rotation, norm=how.norms[0], out=y) is y
        near(y, *how.turned(x, None), dtype)


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 200, 257, 1023, 1024, 3001, 9001])
def test_batches(tokens):
    """From one token to more than a block for each compute unit; one sequence, and one for each token."""
    for type, token in (("bf16", False), ("e4m3", True)):
        c = Case([(1, 3 + i % 9) for i in range(tokens)] if token else [(tokens, tokens + 5)], type=type, d=32, q_heads=3, kv_heads=1, page=16, token=token, seed=tokens)
        _append(c, How(32, pairs=16, norm="shared", heads=(3, 1)))


def test_turning_back():
    """A rotation and the one of the opposite angles leave what was there: off by a rounding of the parts for each of the two."""
    x = torch.randn((50, 3, 64), device=DEVICE).to(torch.float16)
    pos = torch.arange(50, device=DEVICE, dtype=torch.int32) * 1001
    one, back = g.Rotation.of_base(32, positions=pos), g.Rotation.of_base(32, positions=-pos)
    y = g.rotate_heads(g.rotate_heads(x, rotation=one), rotation=back)
    size = x[..., :32].float().abs() + x[..., 32:].float().abs()
    size = torch.cat([size, size], -1)
    assert ((y.float() - x.float()).abs() <= 4 * 2.0 ** -11 * size + 2.0 ** -24).all()


def test_streams_and_graphs():
    """Another stream, and a captured step whose lengths, positions and rows change between replays."""
    c = Case([(1, L) for L in (3, 50, 700)], type="e4m3", d=128, q_heads=4, kv_heads=2, page=16, token=True, columns=60, seed=11)
    positions = torch.tensor([[2, 49, 699], [5, 6, 7]], dtype=torch.int32, device=DEVICE)
    how = How(128, pairs=64, positions=positions, axis_of_pair=[i % 2 for i in range(64)], norm="shared", heads=(4, 2))
    out = torch.empty_like(c.q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _append(c, how, out=out, stream=side)
    step = dict(rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1], out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, **step)
    for i in range(4):
        c.lengths.add_(1)
        positions.add_(3)
        c.q.copy_(torch.randn_like(c.q, dtype=torch.float32))
        c.spec = [(1, int(L)) for L in c.lengths]
        graph.replay()
        torch.cuda.synchronize()
        got, k = out.clone(), c.k.view(torch.uint8).clone()
        _append(c, how, out=out)
        assert torch.equal(got, out) and torch.equal(k, c.k.view(torch.uint8))


def test_append_then_attend():
    """A layer's step as it is run: append a prompt and attend, append a token and attend, against attention over what the cache holds."""
    c = Case([(70, 70), (9, 130)], d=128, q_heads=8, kv_heads=2, page=16, columns=20, spare=20, seed=12)
    free = iter(sorted(set(range(c.k.shape[0])) - set(c.table[c.table >= 0].tolist())))
    for s in range(2):
        for i in range(10):
            if c.table[s, i] < 0:
                c.table[s, i] = next(free)
    how = How(128, pairs=64, norm="shared", heads=(8, 2))
    q = g.kv_append(c.cache, c.batch, c.new_k, c.new_v, c.q, rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1])
    from tests.attention_helpers import check
    c.q = q
    check(c, g.attend_prompt(c.cache, c.batch, q, lse=True))
    c.lengths.add_(1)
    one = g.KvBatch(c.table, c.lengths)
    k1, v1 = (torch.randn((2, 2, 128), device=DEVICE).to(torch.bfloat16) for _ in range(2))
    q1 = torch.randn((2, 8, 128), device=DEVICE).to(torch.bfloat16)
    c.q = g.kv_append(c.cache, one, k1, v1, q1, rotation=how.rotation, q_norm=how.norms[0], k_norm=how.norms[1])
    near(c.q, *how.turned(q1, torch.tensor([70, 130], device=DEVICE)), torch.bfloat16)
    c.spec, c.first, c.T = [(1, 71), (1, 131)], [0, 1, 2], 2
    check(c, g.attend_token(c.cache, one, c.q, lse=True))
