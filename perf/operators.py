"""What the cache and attention operators of a replica are timed on: a layer's paged key-value cache that is written as
tokens arrive, read back, and attended over by prompts and by single tokens.

A case says which operator runs ("write", "write_read", "read", "prompt", "token"), how the cache holds its values ("bf16",
"fp16", or "e4m3": 8 bits with a power of two for each token and head), the heads, the page size in tokens (a cache block of
the traces is 512) and the sequences: how many, how many tokens of each are new and how many the cache holds before them.
Those counts lie between a low and a high end, evenly over the logarithm, drawn from the case's own "shape".
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
E4M3_MOST = 448.0
CHUNK = 1024                      # query tokens that the plain form of a prompt holds scores of at a time


def _case(name, op, type, heads, d, page, S, new, cached, *, window=0, lse=False, shape=1):
    c = dict(op=op, type=type, q_heads=heads[0], kv_heads=heads[1], d=d, page=page, S=S, new_lo=new[0], new_hi=new[1],
             cached_lo=cached[0], cached_hi=cached[1], window=window, lse=lse, shape=shape)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a decode step of a replica's eight slots: every sequence's new token goes into the 8-bit cache (and is read back)
        _case("append_8bit", "write_read", "e4m3", (32, 8), 128, 512, 8, (1, 1), (1000, 60000)),
        # the uncached suffixes of a batch of requests, quantised as they are written, then as the model sees them
        _case("suffixes_8bit", "write_read", "e4m3", (32, 8), 128, 512, 8, (500, 12000), (512, 30000)),
        # whole prompts of a smaller model into a 16-bit cache whose pages are no multiple of anything
        _case("prompts_16bit", "write", "fp16", (16, 4), 64, 48, 3, (17, 40000), (0, 0)),
        # sequences that move to another replica: their 8-bit pages gathered into dense rows
        _case("gather_8bit", "read", "e4m3", (32, 8), 128, 512, 4, (9000, 30000), (0, 0)),
        # short prompts after a few cached pages, small pages: a launch of little work
        _case("prompt_short", "prompt", "bf16", (32, 8), 128, 16, 5, (1, 130), (1, 600)),
        # one prompt of the traces' median length, nothing cached
        _case("prompt_median", "prompt", "bf16", (32, 8), 128, 512, 1, (20000, 20000), (0, 0)),
        # what a prefix hit leaves to do: suffixes of a few blocks over long cached prefixes in 8 bits
        _case("prompt_suffixes", "prompt", "e4m3", (32, 8), 128, 512, 8, (500, 2500), (10000, 30000), lse=True),
        # a model with a sliding window, every head with keys of its own
        _case("prompt_window", "prompt", "fp16", (16, 16), 64, 64, 2, (11000, 24000), (0, 0), window=4096),
        # the longest prompt (256 blocks) on one of eight shards of the heads
        _case("prompt_longest", "prompt", "bf16", (4, 1), 128, 512, 1, (131072, 131072), (0, 0)),
        # one short conversation: latency
        _case("token_short", "token", "bf16", (32, 8), 128, 512, 1, (1, 1), (700, 700)),
        # a busy replica: slots of very different lengths over an 8-bit cache
        _case("token_batch", "token", "e4m3", (32, 8), 128, 512, 48, (1, 1), (500, 32000)),
        # eight slots at the longest length, 16 bits
        _case("token_longest", "token", "bf16", (32, 8), 128, 512, 8, (1, 1), (131071, 131071)),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["write", "write_read", "read", "prompt", "prompt", "prompt", "token", "token", "token"])
    type = "e4m3" if op == "write_read" else rng.choice(["bf16", "fp16"] if op == "write" else ["bf16", "fp16", "e4m3", "e4m3"])
    heads = rng.choice([(32, 8), (32, 8), (28, 4), (16, 16), (8, 1), (12, 2), (40, 8)])
    d = rng.choice([64, 80, 96, 128, 128, 128])
    page = rng.choice([16, 48, 64, 128, 512, 512])
    shape = rng.randrange(1 << 30)
    if op == "token":
        S = _log(rng, 1, 64)
        top = min(131071, (1 << 20) // S)
        lo = _log(rng, 1, top // 2)
        return _case(None, op, type, heads, d, page, S, (1, 1), (lo, _log(rng, lo + 1, top)), shape=shape,
                     window=rng.choice([0, 0, 0, _log(rng, 100, 5000)]), lse=rng.random() < 0.3)
    if op == "prompt":
        S = _log(rng, 1, 16)
        top = max(16, 16000 // S)
        lo = _log(rng, 1, top // 2)
        cached = (0, 0) if rng.random() < 0.4 else (1, _log(rng, 100, 32000))
        return _case(None, op, type, heads, d, page, S, (lo, _log(rng, lo + 1, top)), cached, shape=shape,
                     window=rng.choice([0, 0, 0, _log(rng, 100, 5000)]), lse=rng.random() < 0.3)
    S = _log(rng, 1, 64)
    top = max(4, 40000 // S)
    lo = _log(rng, 1, top // 2)
    return _case(None, op, type, heads, d, page, S, (lo, _log(rng, lo + 1, top)), (0, _log(rng, 1, 5000)), shape=shape)


def _lengths(c):
    """New tokens of each sequence, and the tokens in the cache with them."""
    r = random.Random(c["shape"])

    def some(lo, hi):
        v = int(round(math.exp(r.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1
        return v + 1 if v == 3072 else v
    new = [some(c["new_lo"], c["new_hi"]) for _ in range(c["S"])]
    return new, [n + some(c["cached_lo"], c["cached_hi"]) for n in new]


def _pairs(c, n, L):
    """Keys that the last n of L tokens see, added up."""
    w = c["window"]
    if not w:
        return n * (L - n) + n * (n + 1) // 2
    whole = max(0, L - max(w, L - n + 1) + 1)           # tokens that see a full window
    few = n - whole
    return whole * w + few * (L - n) + few * (few + 1) // 2


def _cache_bytes(c):
    return 2 * c["d"] * (1 if c["type"] == "e4m3" else 2) + (2 if c["type"] == "e4m3" else 0)     # of a token and head


def work(c):
    new, lengths = _lengths(c)
    T, H, Hq, D = sum(new), c["kv_heads"], c["q_heads"], c["d"]
    if c["op"] == "read" or c["op"] == "write":
        return {"bytes": T * H * (4 * D + _cache_bytes(c)), "flops": 0}
    if c["op"] == "write_read":
        return {"bytes": T * H * 2 * (4 * D + _cache_bytes(c)), "flops": 0}
    seen = sum(min(L, c["window"] + n - 1) if c["window"] else L for n, L in zip(new, lengths))
    return {"bytes": T * Hq * D * 4 + seen * H * _cache_bytes(c) + (T * Hq * 4 if c["lse"] else 0),
            "flops": 4 * D * Hq * sum(_pairs(c, n, L) for n, L in zip(new, lengths))}


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    new, lengths = _lengths(c)
    S, H, Hq, D, p, T = c["S"], c["kv_heads"], c["q_heads"], c["d"], c["page"], sum(new)
    pages = [-(-L // p) for L in lengths]
    n_pages, columns = sum(pages) + 3, max(1, max(pages))
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((S, columns), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for s in range(S):
        table[s, :pages[s]] = order[at:at + pages[s]]
        at += pages[s]
    x16 = torch.float16 if c["type"] == "fp16" else torch.bfloat16
    # keys have some channels that are much larger than the others
    channel = torch.exp(0.5 * torch.randn((1, H, 1, D), generator=g, device=DEVICE))

    def normal(*size):
        return torch.randn(size, generator=g, device=DEVICE, dtype=torch.bfloat16)

    st = {"case": c, "table": table, "new": new, "lengths": lengths}
    st["lengths_t"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
    first = [0]
    for n in new:
        first.append(first[-1] + n)
    st["first_t"] = torch.tensor(first, dtype=torch.int32, device=DEVICE)
    shape = (n_pages, H, p, D)
    if c["op"] in ("write", "write_read"):
        st["k"], st["v"] = (torch.zeros(shape, dtype=TYPES[c["type"]], device=DEVICE) for _ in range(2))
        st["new_k"] = (normal(T, H, D).float() * channel[0, :, 0]).to(x16)
        st["new_v"] = normal(T, H, D).to(x16)
        scales = (torch.ones((n_pages, H, p), dtype=torch.uint8, device=DEVICE) for _ in range(2))
    else:
        k, v = normal(*shape), normal(*shape)
        k.mul_(channel.to(torch.bfloat16))
        if c["type"] == "e4m3":
            # what quantising leaves of such rows: codes up to 448, and exponents about 2^-7
            k, v = k.mul_(60.0).clamp_(-E4M3_MOST, E4M3_MOST), v.mul_(120.0).clamp_(-E4M3_MOST, E4M3_MOST)
        st["k"], st["v"] = k.to(TYPES[c["type"]]), v.to(TYPES[c["type"]])
        del k, v
        scales = (torch.randint(119, 122, (n_pages, H, p), generator=g, device=DEVICE, dtype=torch.uint8) for _ in range(2))
        if c["op"] in ("prompt", "token"):
            st["q"] = (1.5 * normal(T, Hq, D).float()).to(x16)
    if c["type"] == "e4m3":
        st["k_scale"], st["v_scale"] = scales
    if own:
        import paper_2602_11688_amd as lib
        st["cache"] = lib.KvCache(st["k"], st["v"], st.get("k_scale"), st.get("v_scale"))
        st["batch"] = lib.KvBatch(table, st["lengths_t"], None if c["op"] == "token" else st["first_t"], tokens=T, max_tokens=max(new))
        if c["op"] in ("prompt", "token"):
            st["workspace"] = lib.attend_workspace(st["cache"], st["batch"], Hq)
    return st


# ------------------------------------------------------------------------------------------- plain forms, in 32 bits

def _exponent(a):
    """Least k with a <= 448 * 2^k, as the byte k + 127 (1 .. 254), of a >= 0."""
    m, e = torch.frexp(a)                              # a = m * 2^e, m in [0.5, 1), 448 = 0.875 * 2^9
    k = e - 9 + (m > 0.875).to(torch.int32)
    return torch.where(a > 0, (k + 127).clamp(1, 254), torch.ones_like(k))


def _power(byte):
    return torch.ldexp(torch.ones((), device=DEVICE), byte.to(torch.int32) - 127)


def _quantise(x):
    x = x.float()
    byte = _exponent(x.abs().amax(-1))
    return (x / _power(byte)[..., None]).to(torch.float8_e4m3fn), byte.to(torch.uint8)


def _rows(st):
    """Page and slot of every new token."""
    new = torch.diff(st["first_t"])
    s = torch.repeat_interleave(torch.arange(len(new), device=DEVICE), new, output_size=sum(st["new"]))
    pos = torch.arange(len(s), device=DEVICE) - st["first_t"][s] + (st["lengths_t"] - new)[s]
    p = st["k"].shape[2]
    return st["table"][s, pos // p].long(), pos % p


def _plain_write(st):
    page, slot = _rows(st)
    for name in ("k", "v"):
        x = st["new_" + name]
        if st["case"]["type"] == "e4m3":
            x, byte = _quantise(x)
            st[name + "_scale"][page, :, slot] = byte
            st[name].view(torch.uint8)[page, :, slot] = x.view(torch.uint8)
        else:
            st[name][page, :, slot] = x


def _plain_read(st):
    page, slot = _rows(st)
    out = []
    for name in ("k", "v"):
        if st["case"]["type"] == "e4m3":
            x = st[name].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
            out.append((x * _power(st[name + "_scale"][page, :, slot])[..., None]).to(torch.bfloat16))
        else:
            out.append(st[name][page, :, slot])
    return tuple(out)


def _dense(st, name, table):
    """Pages of a table [S, n] as rows [S, kv_heads, n * page, d] in 32 bits."""
    S, n = table.shape
    t = table.clamp(min=0).long()
    x = st[name]
    if st["case"]["type"] == "e4m3":
        x = x.view(torch.uint8)[t].view(torch.float8_e4m3fn).float() * _power(st[name + "_scale"][t])[..., None]
    else:
        x = x[t].float()
    return x.permute(0, 2, 1, 3, 4).reshape(S, x.shape[2], -1, x.shape[4])


def _attend(q, k, v, scale, seen, type):
    """q [B, H, G, rows, d] over k, v [B, H, L, d]; seen [B, 1, 1, rows, L]."""
    B, H, G, R, D = q.shape
    s = torch.matmul(q.reshape(B, H, G * R, D), k.transpose(-1, -2).contiguous()).view(B, H, G, R, -1).mul_(scale)
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s.view(B, H, G * R, -1), v).view(B, H, G, R, D) / total
    return out.to(type), (top + total.log())[..., 0]


def _plain_prompt(st):
    c = st["case"]
    H, G, D, scale = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"], c["d"] ** -0.5
    out, lse, at = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], device=DEVICE), 0
    for s, (n, L) in enumerate(zip(st["new"], st["lengths"])):
        table = st["table"][s:s + 1, :-(-L // c["page"])]
        k, v = (_dense(st, name, table)[:, :, :L] for name in ("k", "v"))
        key = torch.arange(L, device=DEVICE)
        for i in range(0, n, CHUNK):
            q = st["q"][at + i:at + min(n, i + CHUNK)]
            pos = torch.arange(L - n + i, L - n + i + len(q), device=DEVICE)[:, None]
            seen = key <= pos
            if c["window"]:
                seen &= key > pos - c["window"]
            o, e = _attend(q.float().view(1, len(q), H, G, D).permute(0, 2, 3, 1, 4), k, v, scale, seen, q.dtype)
            out[at + i:at + i + len(q)] = o[0].permute(2, 0, 1, 3).reshape(len(q), -1, D)
            lse[at + i:at + i + len(q)] = e[0].permute(2, 0, 1).reshape(len(q), -1)
        at += n
    return (out, lse) if c["lse"] else out


def _plain_token(st):
    c = st["case"]
    S, H, G, D = c["S"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"]
    k, v = (_dense(st, name, st["table"]) for name in ("k", "v"))
    key = torch.arange(k.shape[2], device=DEVICE)
    L = st["lengths_t"][:, None]
    seen = key < L
    if c["window"]:
        seen &= key >= L - c["window"]
    o, e = _attend(st["q"].float().view(S, H, G, 1, D), k, v, D ** -0.5, seen[:, None, None, None], st["q"].dtype)
    out, lse = o.reshape(S, H * G, D), e.reshape(S, H * G)
    return (out, lse) if c["lse"] else out


def run(state):
    st, op = state, state["case"]["op"]
    if own:
        import paper_2602_11688_amd as lib
        if op == "write":
            lib.kv_write(st["cache"], st["batch"], st["new_k"], st["new_v"])
            return st["k"], st["v"]
        if op == "write_read":
            lib.kv_write(st["cache"], st["batch"], st["new_k"], st["new_v"])
            return lib.kv_read(st["cache"], st["batch"])
        if op == "read":
            return lib.kv_read(st["cache"], st["batch"])
        attend = lib.attend_prompt if op == "prompt" else lib.attend_token
        out = attend(st["cache"], st["batch"], st["q"], window=st["case"]["window"], lse=st["case"]["lse"], workspace=st["workspace"])
        return out
    if op == "write":
        _plain_write(st)
        return st["k"], st["v"]
    if op == "write_read":
        _plain_write(st)
        return _plain_read(st)
    if op == "read":
        return _plain_read(st)
    return _plain_prompt(st) if op == "prompt" else _plain_token(st)


# --------------------------------------------------------------------------- the definition in 64 bits, written apart

def _e4m3_exact(x):
    """Rows of x in 64 bits, each value replaced by the nearest that 8 bits and the row's power of two hold."""
    a = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(a.clamp(min=1e-300) / E4M3_MOST))
    k = torch.where(a > E4M3_MOST * torch.exp2(k), k + 1, k)
    k = torch.where(a <= E4M3_MOST * torch.exp2(k - 1), k - 1, k)
    k = torch.where(a > 0, k.clamp(-126, 127), torch.full_like(k, -126.0))
    y = x * torch.exp2(-k)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(k)


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    new, lengths, p, table = st["new"], st["lengths"], c["page"], st["table"].tolist()

    def cached(name, s, lo, hi):
        """Rows lo .. hi of a sequence, [kv_heads, rows, d] in 64 bits."""
        pieces = []
        for i in range(lo // p, -(-hi // p)):
            a, b = max(lo - i * p, 0), min(hi - i * p, p)
            pieces.append((table[s][i], a, b))
        x = torch.cat([st[name][j][:, a:b].double() for j, a, b in pieces], 1)
        if c["type"] == "e4m3":
            x *= torch.cat([torch.exp2(st[name + "_scale"][j][:, a:b].double() - 127) for j, a, b in pieces], 1)[..., None]
        return x

    if c["op"] == "write_read":
        return _e4m3_exact(st["new_k"].double()), _e4m3_exact(st["new_v"].double())
    if c["op"] == "write":
        out = []
        for name in ("k", "v"):
            x, at = torch.zeros(st[name].shape, dtype=torch.float64, device=DEVICE), 0
            for s, (n, L) in enumerate(zip(new, lengths)):
                pos = L - n
                while pos < L:
                    take = min(L, (pos // p + 1) * p) - pos
                    x[table[s][pos // p], :, pos % p:pos % p + take] = st["new_" + name][at:at + take].double().transpose(0, 1)
                    pos, at = pos + take, at + take
            out.append(x)
        return tuple(out)
    if c["op"] == "read":
        return tuple(torch.cat([cached(name, s, L - n, L).transpose(0, 1) for s, (n, L) in enumerate(zip(new, lengths)) if n])
                     for name in ("k", "v"))
    if work(c)["flops"] > 2e13:
        return None
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"]
    out, lse, at = [], [], 0
    for s, (n, L) in enumerate(zip(new, lengths)):
        k, v = cached("k", s, 0, L), cached("v", s, 0, L)
        o, e = torch.empty((n, H * G, D), dtype=torch.float64, device=DEVICE), torch.empty((n, H * G), dtype=torch.float64, device=DEVICE)
        for h in range(H * G):
            for i in range(0, n, 2048):
                m = min(n, i + 2048)
                # only the keys that some of these tokens see
                lo = max(0, L - n + i + 1 - c["window"]) if c["window"] else 0
                hi = L - n + m
                score = st["q"][at + i:at + m, h].double() @ k[h // G, lo:hi].T.contiguous() / math.sqrt(D)
                ahead = torch.arange(lo, hi, device=DEVICE) - torch.arange(L - n + i, L - n + m, device=DEVICE)[:, None]
                score[(ahead > 0) | (ahead <= -c["window"] if c["window"] else ahead > L)] = -math.inf
                e[i:m, h] = torch.logsumexp(score, -1)
                o[i:m, h] = torch.exp(score - e[i:m, h, None]) @ v[h // G, lo:hi]
        out.append(o)
        lse.append(e)
        at += n
    return (torch.cat(out), torch.cat(lse)) if c["lse"] else torch.cat(out)
