"""What a layer does between its projections and its attention, and attention that forgets the middle of a sequence, as timed on one
GPU: heads of queries and keys are normed and rotated by their positions, keys and values go into the paged cache on the way, and
prompts and single tokens attend over a sliding window and the first few tokens.

A case says which operator runs: "append" (norms, rotation and cache in one call, read back where the cache has 8 bits), "rotate" (rows
alone), "prompt" or "token" (attention with `window` and `sinks`).  Sequences are as many as "S"; how many tokens of each are new, and
how many come before them, lies between a low and a high end, evenly over the logarithm, drawn from the case's own "shape".  Where
"evicted" is true the pages that no token sees any more are not there.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
E4M3_MOST = 448.0
EPS = 1e-6
CHUNK = 1024                      # query tokens that the plain form of a prompt holds scores of at a time


def _case(name, op, type, heads, d, page, S, new, before, *, pairs=0, layout="halves", axes=1, base=10000.0, magnitude=1.0, norm="",
          window=0, sinks=0, evicted=False, lse=False, shape=1):
    c = dict(op=op, type=type, q_heads=heads[0], kv_heads=heads[1], d=d, page=page, S=S, new_lo=new[0], new_hi=new[1], before_lo=before[0],
             before_hi=before[1], pairs=pairs, layout=layout, axes=axes, base=base, magnitude=magnitude, norm=norm, window=window, sinks=sinks,
             evicted=evicted, lse=lse, shape=shape)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a decode step of a replica's eight slots: everything between projections and attention for one token of each
        _case("append_step_8bit", "append", "e4m3", (32, 8), 128, 512, 8, (1, 1), (1000, 60000), pairs=64, base=1e6, norm="shared"),
        # the uncached suffixes of a batch of requests, quantised as they are written
        _case("append_suffixes_8bit", "append", "e4m3", (32, 8), 128, 512, 8, (500, 12000), (512, 30000), pairs=64, base=1e6, norm="shared"),
        # whole prompts of a smaller model that rotates neighbours, half of each head; pages that are no multiple of anything
        _case("append_prompts_16bit", "append", "fp16", (16, 4), 64, 48, 3, (17, 40000), (0, 0), pairs=16, layout="neighbours"),
        # prompts with images in them: time, height and width have pairs of their own
        _case("append_axes", "append", "bf16", (28, 4), 128, 16, 5, (200, 9000), (0, 3000), pairs=64, axes=3, base=1e6),
        # an image encoder's patches, by row and column; no cache, heads that are no power of two
        _case("rotate_patches", "rotate", "bf16", (16, 16), 80, 64, 1, (50000, 50000), (0, 0), pairs=40, axes=2),
        # queries of a decode step over a cache that another layer wrote, a norm of its own for each head
        _case("rotate_step", "rotate", "fp16", (32, 32), 128, 512, 48, (1, 1), (500, 500000), pairs=64, layout="neighbours", norm="each", magnitude=1.2),
        # ragged prompts, heads whose halves do not begin at a whole load
        _case("rotate_odd", "rotate", "bf16", (12, 12), 72, 64, 4, (1, 9000), (0, 1000), pairs=36, norm="shared"),
        # short turns of a few conversations, small pages: a launch of little work
        _case("sinks_short", "prompt", "bf16", (32, 8), 128, 16, 5, (1, 130), (1, 2000), window=256, sinks=4),
        # one long prompt of a model with a sliding window
        _case("sinks_prompt", "prompt", "bf16", (32, 8), 128, 512, 1, (60000, 60000), (0, 0), window=4096, sinks=4),
        # suffixes of long conversations whose middle is gone from the 8-bit cache
        _case("sinks_suffixes_8bit", "prompt", "e4m3", (16, 2), 64, 64, 6, (500, 2500), (10000, 120000), window=2048, sinks=128, evicted=True, lse=True),
        # one conversation that has run for long: latency
        _case("sinks_step", "token", "bf16", (32, 8), 128, 16, 1, (1, 1), (300000, 300000), window=1024, sinks=4, evicted=True),
        # a busy replica: slots of all lengths, most beyond the window
        _case("sinks_batch_8bit", "token", "e4m3", (32, 8), 128, 512, 48, (1, 1), (500, 1000000), window=8192, sinks=64, evicted=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "rotate", "rotate", "prompt", "prompt", "token", "token"])
    type = rng.choice(["bf16", "fp16"] if op == "rotate" else ["bf16", "fp16", "e4m3", "e4m3"])
    heads = rng.choice([(32, 8), (32, 8), (28, 4), (16, 16), (8, 1), (12, 2), (40, 8)])
    d = rng.choice([64, 80, 96, 128, 128, 128] if op != "rotate" else [64, 72, 80, 104, 128, 128])
    page = rng.choice([16, 48, 64, 128, 512, 512])
    shape = rng.randrange(1 << 30)
    if op == "token":
        S = _log(rng, 1, 64)
        top = min(1000000, (1 << 22) // S)
        lo = _log(rng, 1, top // 2)
        return _case(None, op, type, heads, d, page, S, (1, 1), (lo, _log(rng, lo + 1, top)), shape=shape, window=_log(rng, 64, 8192),
                     sinks=_log(rng, 1, 256), evicted=True, lse=rng.random() < 0.3)
    if op == "prompt":
        S = _log(rng, 1, 16)
        top = max(16, 16000 // S)
        lo = _log(rng, 1, top // 2)
        before = (0, 0) if rng.random() < 0.4 else (1, _log(rng, 100, 100000))
        return _case(None, op, type, heads, d, page, S, (lo, _log(rng, lo + 1, top)), before, shape=shape, window=_log(rng, 64, 5000),
                     sinks=_log(rng, 1, 256), evicted=rng.random() < 0.5, lse=rng.random() < 0.3)
    S = _log(rng, 1, 64)
    top = max(4, 40000 // S)
    lo = _log(rng, 1, top // 2)
    layout = rng.choice(["halves", "halves", "neighbours"])
    return _case(None, op, type, heads, d, page, S, (lo, _log(rng, lo + 1, top)), (0, _log(rng, 1, 200000 // S)), shape=shape, layout=layout,
                 pairs=rng.choice([d // 2, d // 2, d // 4, rng.randint(1, d // 2)]), axes=rng.choice([1, 1, 2, 3]), base=rng.choice([1e4, 5e5, 1e6]),
                 norm=rng.choice(["", "shared", "each"]))


def _lengths(c):
    """New tokens of each sequence, and its tokens with them."""
    r = random.Random(c["shape"])

    def some(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1
    new = [max(1, some(c["new_lo"], c["new_hi"])) for _ in range(c["S"])]
    return new, [n + some(c["before_lo"], c["before_hi"]) for n in new]


def _seen(c, n, L):
    """Keys of a sequence that its last n of L tokens see: how many some token sees, and those of each added up."""
    w, k = c["window"], c["sinks"]
    lo = max(0, L - n - w + 1)                               # of the first new token's window
    some = L - lo + min(k, lo)

    def upto(m):                                             # sums over positions 0 .. m - 1, of min(p + 1, w) + min(k, max(0, p + 1 - w))
        a, b = min(m, w), max(0, m - w)
        e = min(b, k)
        return a * (a + 1) // 2 + b * w + e * (e + 1) // 2 + (b - e) * k
    return some, upto(L) - upto(L - n)


def _cache_bytes(c):
    return 2 * c["d"] * (1 if c["type"] == "e4m3" else 2) + (2 if c["type"] == "e4m3" else 0)     # of a token and head


def work(c):
    new, lengths = _lengths(c)
    T, H, Hq, D = sum(new), c["kv_heads"], c["q_heads"], c["d"]
    turned = (4 * D if c["norm"] else 0) + 6 * c["pairs"]    # operations of a row
    if c["op"] == "rotate":
        return {"bytes": T * (Hq * 4 * D + (4 * c["axes"] if c["axes"] > 1 else 0)), "flops": T * Hq * turned}
    if c["op"] == "append":
        back = H * (4 * D + _cache_bytes(c)) if c["type"] == "e4m3" else 0
        return {"bytes": T * (Hq * 4 * D + H * (4 * D + _cache_bytes(c)) + back + (4 * c["axes"] if c["axes"] > 1 else 0)), "flops": T * (Hq + H) * turned}
    seen = [_seen(c, n, L) for n, L in zip(new, lengths)]
    return {"bytes": T * Hq * D * 4 + sum(s for s, _ in seen) * H * _cache_bytes(c) + (T * Hq * 4 if c["lse"] else 0),
            "flops": 4 * D * Hq * sum(p for _, p in seen)}


def _grid(c, T):
    """Positions [axes, T]: lines of text, each followed by an image of 32 x 32 patches (two axes: patches alone)."""
    i = torch.arange(T, device=DEVICE)
    text = 0 if c["axes"] == 2 else 300
    at, nth = i % (text + 1024), i // (text + 1024)
    patch = (at - text).clamp(min=0)
    begin = nth * (text + 32)
    time = torch.where(at < text, begin + at, begin + text)
    row, column = torch.where(at < text, time, begin + text + patch // 32), torch.where(at < text, time, begin + text + patch % 32)
    return torch.stack([row, column] if c["axes"] == 2 else [time, row, column]).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    new, lengths = _lengths(c)
    S, H, Hq, D, p, T = c["S"], c["kv_heads"], c["q_heads"], c["d"], c["page"], sum(new)
    x16 = torch.float16 if c["type"] == "fp16" else torch.bfloat16
    attends, holds = c["op"] in ("prompt", "token"), c["op"] != "rotate"

    # pages of each sequence: of the sinks, and from the first one that a new token's window reaches
    parts = []
    for n, L in zip(new, lengths):
        every = list(range(-(-L // p)))
        if c["evicted"]:
            lo = max(0, L - n - c["window"] + 1)
            every = [i for i in every if i * p < c["sinks"] or (i + 1) * p > lo]
        parts.append(every)
    columns = max(1, max(-(-L // p) for L in lengths))
    n_pages = sum(len(e) for e in parts) + 3 if holds else 1
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((S, columns), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for s in range(S if holds else 0):
        table[s, torch.tensor(parts[s], device=DEVICE)] = order[at:at + len(parts[s])]
        at += len(parts[s])

    def normal(*size):
        return torch.randn(size, generator=g, device=DEVICE, dtype=torch.bfloat16)

    # keys have some channels that are much larger than the others
    channel = torch.exp(0.5 * torch.randn((1, H, 1, D), generator=g, device=DEVICE))
    st = {"case": c, "table": table, "new": new, "lengths": lengths, "parts": parts}
    st["lengths_t"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
    first = [0]
    for n in new:
        first.append(first[-1] + n)
    st["first_t"] = torch.tensor(first, dtype=torch.int32, device=DEVICE)
    shape = (n_pages, H, p, D)
    scales = ()
    if not attends:
        st["frequencies"] = c["base"] ** (-torch.arange(c["pairs"], dtype=torch.float64, device=DEVICE) / c["pairs"])
        # runs of pairs for each axis, the first one's a little shorter
        st["axis_of_pair"] = [min(c["axes"] - 1, (i + c["pairs"] // 16) * c["axes"] // c["pairs"]) for i in range(c["pairs"])]
        st["positions"] = _grid(c, T) if c["axes"] > 1 else None
        for name, heads in (("q", Hq), ("k", H)):
            size = (heads, D) if c["norm"] == "each" else (D,)
            st[name + "_weight"] = (1 + 0.3 * normal(*size).float()).to(torch.bfloat16).float() if c["norm"] else None
        st["new_q"] = (1.5 * normal(T, Hq, D).float()).to(x16)
        if holds:
            st["new_k"] = (normal(T, H, D).float() * channel[0, :, 0]).to(x16)
            st["new_v"] = normal(T, H, D).to(x16)
            st["k"], st["v"] = (torch.zeros(shape, dtype=TYPES[c["type"]], device=DEVICE) for _ in range(2))
            scales = [torch.ones((n_pages, H, p), dtype=torch.uint8, device=DEVICE) for _ in range(2)]
    else:
        k, v = normal(*shape), normal(*shape)
        k.mul_(channel.to(torch.bfloat16))
        if c["type"] == "e4m3":
            # what quantising leaves of such rows: codes up to 448, and exponents about 2^-7
            k, v = k.mul_(60.0).clamp_(-E4M3_MOST, E4M3_MOST), v.mul_(120.0).clamp_(-E4M3_MOST, E4M3_MOST)
        st["k"], st["v"] = k.to(TYPES[c["type"]]), v.to(TYPES[c["type"]])
        del k, v
        scales = [torch.randint(119, 122, (n_pages, H, p), generator=g, device=DEVICE, dtype=torch.uint8) for _ in range(2)]
        st["q"] = (1.5 * normal(T, Hq, D).float()).to(x16)
    if holds and c["type"] == "e4m3":
        st["k_scale"], st["v_scale"] = scales
    if own:
        import paper_2602_11688_amd as lib
        st["batch"] = lib.KvBatch(table, st["lengths_t"], None if c["op"] == "token" or c["new_hi"] == 1 else st["first_t"], tokens=T)
        if holds:
            st["cache"] = lib.KvCache(st["k"], st["v"], st.get("k_scale"), st.get("v_scale"))
        if attends:
            st["workspace"] = lib.attend_workspace(st["cache"], st["batch"], Hq)
        else:
            st["rotation"] = lib.Rotation(st["frequencies"], st["positions"], axis_of_pair=st["axis_of_pair"], layout=c["layout"], magnitude=c["magnitude"])
            for name in ("q", "k"):
                st[name + "_norm"] = lib.HeadNorm(st[name + "_weight"], eps=EPS) if c["norm"] else None
    return st


# -------------------------------------------------------------------------------------- plain forms, in 32 bits

def _power(byte, type):
    return torch.ldexp(torch.ones((), device=DEVICE, dtype=type), byte.to(torch.int32) - 127)


def _places(st):
    """Position of every new token, and its page and slot."""
    new = torch.diff(st["first_t"])
    s = torch.repeat_interleave(torch.arange(len(new), device=DEVICE), new, output_size=sum(st["new"]))
    pos = torch.arange(len(s), device=DEVICE) - st["first_t"][s] + (st["lengths_t"] - new)[s]
    p = st["case"]["page"]
    return pos, st["table"][s, pos // p].long(), pos % p


def _turned(st, name, pos, type):
    """Rows, normed and rotated, in `type`; the angles always in 64 bits."""
    c, P, w = st["case"], st["case"]["pairs"], st[name + "_weight"]
    x = st["new_" + name].to(type)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(type)
    else:
        x = x.clone()
    at = pos[:, None] if st["positions"] is None else st["positions"].T[:, st["axis_of_pair"]]
    angle = at.double() * st["frequencies"]
    cos, sin = ((c["magnitude"] * f(angle)).to(type)[:, None] for f in (torch.cos, torch.sin))
    first, second = (slice(0, P), slice(P, 2 * P)) if c["layout"] == "halves" else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    a, b = x[..., first].clone(), x[..., second].clone()
    x[..., first] = a * cos - b * sin
    x[..., second] = b * cos + a * sin
    return x


def _plain_rotate(st):
    return _turned(st, "q", _places(st)[0], torch.float32).to(st["new_q"].dtype)


def _plain_append(st):
    c = st["case"]
    pos, page, slot = _places(st)
    q = _turned(st, "q", pos, torch.float32).to(st["new_q"].dtype)
    if c["type"] != "e4m3":
        st["k"][page, :, slot] = _turned(st, "k", pos, torch.float32).to(st["k"].dtype)
        st["v"][page, :, slot] = st["new_v"]
        return q, st["k"], st["v"]
    out = [q]
    # (in 64 bits: which side of a code's border a value lies on)
    for name, x in (("k", _turned(st, "k", pos, torch.float64)), ("v", st["new_v"].double())):
        m, e = torch.frexp(x.abs().amax(-1))                # a = m * 2^e, m in [0.5, 1), 448 = 0.875 * 2^9
        byte = torch.where(m > 0, (e - 9 + (m > 0.875).to(torch.int32) + 127).clamp(1, 254), torch.ones_like(e)).to(torch.uint8)
        y = x / _power(byte, torch.float64)[..., None]
        step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
        st[name + "_scale"][page, :, slot] = byte
        st[name].view(torch.uint8)[page, :, slot] = (torch.round(y / step) * step).float().to(torch.float8_e4m3fn).view(torch.uint8)
    for name in ("k", "v"):
        x = st[name].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
        out.append((x * _power(st[name + "_scale"][page, :, slot], torch.float32)[..., None]).to(torch.bfloat16))
    return tuple(out)


def _gather(st, name, s, pos):
    """Rows of a sequence [B] at positions [B, n], as [B, kv_heads, n, d] in 32 bits; pages that are not there give any row."""
    c = st["case"]
    page, slot = st["table"][s[:, None], pos // c["page"]].clamp(min=0).long(), pos % c["page"]
    if c["type"] == "e4m3":
        x = st[name].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float() * _power(st[name + "_scale"][page, :, slot], torch.float32)[..., None]
    else:
        x = st[name][page, :, slot].float()
    return x.transpose(1, 2)


def _attend(q, k, v, scale, seen, type):
    """q [B, H, G, rows, d] over k, v [B, H, n, d]; seen [B, 1, 1, rows, n]."""
    B, H, G, R, D = q.shape
    s = torch.matmul(q.reshape(B, H, G * R, D), k.transpose(-1, -2).contiguous()).view(B, H, G, R, -1).mul_(scale)
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s.view(B, H, G * R, -1), v.contiguous()).view(B, H, G, R, D) / total
    return out.to(type), (top + total.log())[..., 0]


def _plain_prompt(st):
    c = st["case"]
    H, G, D, scale = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"], c["d"] ** -0.5
    out, lse, at = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], device=DEVICE), 0
    for s, (n, L) in enumerate(zip(st["new"], st["lengths"])):
        for i in range(0, n, CHUNK):
            # the sinks, and what the windows of these tokens reach
            m = min(n, i + CHUNK)
            lo = max(0, L - n + i + 1 - c["window"])
            key = torch.cat([torch.arange(min(c["sinks"], lo), device=DEVICE), torch.arange(lo, L - n + m, device=DEVICE)])
            k, v = (_gather(st, name, torch.tensor([s], device=DEVICE), key[None]) for name in ("k", "v"))
            pos = torch.arange(L - n + i, L - n + m, device=DEVICE)[:, None]
            seen = (key <= pos) & ((key > pos - c["window"]) | (key < c["sinks"]))
            q = st["q"][at + i:at + m]
            o, e = _attend(q.float().view(1, len(q), H, G, D).permute(0, 2, 3, 1, 4), k, v, scale, seen, q.dtype)
            out[at + i:at + m] = o[0].permute(2, 0, 1, 3).reshape(len(q), -1, D)
            lse[at + i:at + m] = e[0].permute(2, 0, 1).reshape(len(q), -1)
        at += n
    return (out, lse) if c["lse"] else out


def _plain_token(st):
    c = st["case"]
    S, H, G, D = c["S"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"]
    L = st["lengths_t"].long()[:, None]
    lo = (L - c["window"]).clamp(min=0)
    sink, near = torch.arange(c["sinks"], device=DEVICE), torch.arange(c["window"], device=DEVICE)
    key = torch.cat([sink.expand(S, -1), lo + near], 1)
    seen = torch.cat([sink < lo, lo + near < L], 1)
    key = torch.where(seen, key, torch.zeros_like(key))
    k, v = (_gather(st, name, torch.arange(S, device=DEVICE), key) for name in ("k", "v"))
    o, e = _attend(st["q"].float().view(S, H, G, 1, D), k, v, D ** -0.5, seen[:, None, None, None], st["q"].dtype)
    out, lse = o.reshape(S, H * G, D), e.reshape(S, H * G)
    return (out, lse) if c["lse"] else out


def run(state):
    st, c = state, state["case"]
    if own:
        import paper_2602_11688_amd as lib
        if c["op"] == "rotate":
            return lib.rotate_heads(st["new_q"], rotation=st["rotation"], norm=st["q_norm"], batch=st["batch"])
        if c["op"] == "append":
            q = lib.kv_append(st["cache"], st["batch"], st["new_k"], st["new_v"], st["new_q"], rotation=st["rotation"], q_norm=st["q_norm"], k_norm=st["k_norm"])
            return (q, *lib.kv_read(st["cache"], st["batch"])) if c["type"] == "e4m3" else (q, st["k"], st["v"])
        attend = lib.attend_prompt if c["op"] == "prompt" else lib.attend_token
        return attend(st["cache"], st["batch"], st["q"], window=c["window"], sinks=c["sinks"], lse=c["lse"], workspace=st["workspace"])
    return {"rotate": _plain_rotate, "append": _plain_append, "prompt": _plain_prompt, "token": _plain_token}[c["op"]](st)


# --------------------------------------------------------------------- the definitions in 64 bits, written apart

def _two_to(k):
    return torch.ldexp(torch.ones_like(k), k.to(torch.int32))         # (exp2 in 64 bits is a little off on the GPU)


def _e4m3_exact(x):
    """Rows of x in 64 bits, each value replaced by the nearest that 8 bits and the row's power of two hold."""
    a = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(a.clamp(min=1e-300) / E4M3_MOST))
    k = torch.where(a > E4M3_MOST * _two_to(k), k + 1, k)
    k = torch.where(a <= E4M3_MOST * _two_to(k - 1), k - 1, k)
    k = torch.where(a > 0, k.clamp(-126, 127), torch.full_like(k, -126.0))
    y = x * _two_to(-k)
    step = _two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * _two_to(k)


def _turned_exact(c, st, name, begin, new, L):
    """Normed and rotated rows of one sequence in 64 bits: pairs as complex numbers times powers of e."""
    x = st["new_" + name][begin:begin + new].double()
    if c["norm"]:
        x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["d"] + EPS) * st[name + "_weight"].double()
    P = c["pairs"]
    rotated, rest = x[..., :2 * P], x[..., 2 * P:]
    pairs = rotated.unflatten(-1, (2, P)).transpose(-1, -2) if c["layout"] == "halves" else rotated.unflatten(-1, (P, 2))
    angle = torch.empty((new, P), dtype=torch.float64, device=DEVICE)
    for i in range(P):
        where = torch.arange(L - new, L, device=DEVICE) if c["axes"] == 1 else st["positions"][st["axis_of_pair"][i], begin:begin + new]
        angle[:, i] = where.double() * c["base"] ** (-i / P)
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angle, c["magnitude"]), angle)[:, None])
    rotated = (pairs.transpose(-1, -2) if c["layout"] == "halves" else pairs).flatten(-2)
    return torch.cat([rotated, rest], -1)


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    new, lengths, p, table = st["new"], st["lengths"], c["page"], st["table"].tolist()
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"]
    begin = [sum(new[:s]) for s in range(len(new))]
    if c["op"] in ("rotate", "append"):
        q = torch.cat([_turned_exact(c, st, "q", b, n, L) for b, n, L in zip(begin, new, lengths)])
        if c["op"] == "rotate":
            return q
        k, v = torch.cat([_turned_exact(c, st, "k", b, n, L) for b, n, L in zip(begin, new, lengths)]), st["new_v"].double()
        if c["type"] == "e4m3":
            return q, _e4m3_exact(k), _e4m3_exact(v)
        out = [q]
        for name, x in (("k", k), ("v", v)):
            to = torch.zeros(st[name].shape, dtype=torch.float64, device=DEVICE)
            for s, (b, n, L) in enumerate(zip(begin, new, lengths)):
                pos = L - n
                while pos < L:
                    take = min(L, (pos // p + 1) * p) - pos
                    to[table[s][pos // p], :, pos % p:pos % p + take] = x[b + pos - L + n:b + pos - L + n + take].transpose(0, 1)
                    pos += take
            out.append(to)
        return tuple(out)
    if work(c)["flops"] > 2e13:
        return None

    out, lse = [], []
    for s, (b, n, L) in enumerate(zip(begin, new, lengths)):
        # the sequence's pages that are there, one after the other, and their positions
        pos = torch.cat([torch.arange(i * p, min(L, (i + 1) * p), device=DEVICE) for i in st["parts"][s]])
        k, v = (torch.cat([st[name][table[s][i]].double() * (torch.exp2(st[name + "_scale"][table[s][i]].double() - 127)[..., None] if c["type"] == "e4m3" else 1.0)
                           for i in st["parts"][s]], 1)[:, :len(pos)] for name in ("k", "v"))
        o, e = torch.empty((n, H * G, D), dtype=torch.float64, device=DEVICE), torch.empty((n, H * G), dtype=torch.float64, device=DEVICE)
        for i in range(0, n, 2048):
            m = min(n, i + 2048)
            me = torch.arange(L - n + i, L - n + m, device=DEVICE)[:, None]
            # (of the others no token of this part sees any)
            near = ((pos > L - n + i - c["window"]) | (pos < c["sinks"])) & (pos < L - n + m)
            hidden = (pos[near] > me) | ((pos[near] <= me - c["window"]) & (pos[near] >= c["sinks"]))
            for h in range(H * G):
                score = st["q"][b + i:b + m, h].double() @ k[h // G, near].T.contiguous() / math.sqrt(D)
                score[hidden] = -math.inf
                e[i:m, h] = torch.logsumexp(score, -1)
                o[i:m, h] = torch.exp(score - e[i:m, h, None]) @ v[h // G, near]
        out.append(o)
        lse.append(e)
    return (torch.cat(out), torch.cat(lse)) if c["lse"] else torch.cat(out)
