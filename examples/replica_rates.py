"""Runs one replica's share of a routed trace through the cache and attention operators, and prints attention's share of the service
constants: what its times add to prefill_ms_per_token and decode_ms_per_token, beside the constants that the trace was replayed with.  The other
layers of a model, projections and feed-forward, are not run.

    python examples/replica_rates.py [--requests 4000] [--replica 0] [--layers 32] [--dtype e4m3]

The trace is replayed under a population of weight vectors first (eval_population); the best one says which requests the replica
gets and how many blocks of each it has cached by then.  The last of them are served in batches of the model's concurrent slots: what is not cached
is written (kv_write) and attends over the whole prompt (attend_prompt); then the batch decodes, one token of each sequence a step,
the step (kv_write, attend_token) captured once into a graph and replayed with longer lengths.  Keys, values and queries are
random, those of the cached blocks too; attention is one layer's, times `layers`.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2602_11688_amd as g  # noqa: E402
from synth import tracegen as tg  # noqa: E402

DEVICE = "cuda:0"


class Pages:
    """Pages of the prompt blocks that the replica holds, and of its slots' decoded tokens."""

    def __init__(self, count: int):
        self.count, self.of_block, self.free = count, {}, list(range(count))

    def prompt(self, ids):
        return [self.of_block[i] if i in self.of_block else self.of_block.setdefault(i, self.free.pop()) for i in ids]


def _seconds(f) -> float:
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    f()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) * 1e-3


def _worst(cache, table, length, q, out, heads):
    """Largest difference of a sequence's last row from the definition, in 64 bits."""
    offsets = torch.tensor([0, length], dtype=torch.int32, device=DEVICE)
    lengths = torch.tensor([length], dtype=torch.int32, device=DEVICE)
    k, v = (x.double() for x in g.kv_read(cache, g.KvBatch(table[None].contiguous(), lengths, offsets, tokens=length)))
    worst = 0.0
    for h in range(heads):
        s = k[:, h * cache.kv_heads // heads] @ q[h].double() * cache.head_dim ** -0.5
        want = torch.softmax(s, 0) @ v[:, h * cache.kv_heads // heads]
        worst = max(worst, float((want - out[h].double()).abs().max()))
    return worst


def run(requests: int = 4000, replica: int = 0, layers: int = 32, dtype: str = "e4m3", q_heads: int = 32, kv_heads: int = 8, head_dim: int = 128,
        steps: int = 64, batches: int = 4) -> dict:
    wl = tg.config(2, requests)
    t = wl.trace
    trace = g.Trace.from_arrays(t.ts_ms, t.in_len, t.out_len, t.blk_off, t.hash_ids)
    model = g.Model(wl.R, wl.batch, wl.cache_blocks, wl.prefill_ms_per_token, wl.decode_ms_per_token)
    routed = g.eval_population(trace, model, wl.rtt_ms, wl.params, wl.scale)
    best = int(routed.p95_ttft_ms.argmin())
    route, hit_blocks = routed.route[best].cpu().tolist(), routed.hit_blocks[best].cpu().tolist()
    mine = [r for r in range(requests) if route[r] == replica][-batches * wl.batch:]
    if not mine:
        raise SystemExit(f"replica {replica} gets none of {requests} requests")

    block, S = wl.block_tokens, wl.batch
    needed = len({int(i) for r in mine for i in t.ids_of(r)}) + S * (-(-steps // block) + 1)
    pages = Pages(needed)
    cache = g.KvCache.empty(needed, kv_heads, head_dim, block, dtype, DEVICE)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1)

    def rows(n, heads):
        return torch.randn((n, heads, head_dim), generator=gen, device=DEVICE, dtype=torch.float32).to(cache.row_dtype)

    for x in (cache.k, cache.v):
        for page in x:
            page.copy_(torch.randn(page.shape, generator=gen, device=DEVICE))
    if dtype == "e4m3":
        cache.k_scale.fill_(127)                                           # 2^0
        cache.v_scale.fill_(127)

    prefill = decode = 0.0
    new_tokens = hit_tokens = decoded = 0
    worst = 0.0
    for b in range(0, len(mine), S):
        batch = mine[b:b + S]
        found = [(pages.prompt([int(i) for i in t.ids_of(r)]), hit_blocks[r]) for r in batch]
        lengths = [len(p) * block for p, _ in found]                       # (prompts of whole blocks)
        new = [max(1, L - hit * block) for L, (_, hit) in zip(lengths, found)]
        own = [[pages.free.pop() for _ in range(-(-steps // block))] for _ in batch]     # for what is decoded
        columns = max(len(p) + len(o) for (p, _), o in zip(found, own))
        table = torch.tensor([p + o + [-1] * (columns - len(p) - len(o)) for (p, _), o in zip(found, own)], dtype=torch.int32, device=DEVICE)
        lengths_t = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
        offsets = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEVICE)

        prompts = g.KvBatch(table, lengths_t, offsets, tokens=sum(new), max_tokens=max(new))
        workspace = g.attend_workspace(cache, prompts, q_heads)
        k, v, q = rows(sum(new), kv_heads), rows(sum(new), kv_heads), rows(sum(new), q_heads)
        out = torch.empty_like(q)

        def serve():
            g.kv_write(cache, prompts, k, v)
            g.attend_prompt(cache, prompts, q, out=out, workspace=workspace)
        serve()                                                            # (the first launch of a kernel loads its code)
        prefill += _seconds(serve)
        new_tokens += sum(new)
        hit_tokens += sum(lengths) - sum(new)
        last = min(range(len(batch)), key=lambda i: lengths[i])
        worst = max(worst, _worst(cache, table[last], lengths[last], q[sum(new[:last + 1]) - 1], out[sum(new[:last + 1]) - 1], q_heads))

        one = g.KvBatch(table, lengths_t)
        workspace_1 = g.attend_workspace(cache, one, q_heads)
        k1, v1, q1 = rows(len(batch), kv_heads), rows(len(batch), kv_heads), rows(len(batch), q_heads)
        out1 = torch.empty_like(q1)

        def step():
            lengths_t.add_(1)
            g.kv_write(cache, one, k1, v1)
            g.attend_token(cache, one, q1, out=out1, workspace=workspace_1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        lengths_t.copy_(torch.tensor(lengths, dtype=torch.int32))
        decode += _seconds(lambda: [graph.replay() for _ in range(steps)])
        decoded += steps
        worst = max(worst, _worst(cache, table[last], lengths[last] + steps, q1[last], out1[last], q_heads))
        for o in own:
            pages.free += o
    return {"requests": len(mine), "new_tokens": new_tokens, "hit_tokens": hit_tokens, "worst": worst,
            "model_prefill": wl.prefill_ms_per_token, "model_decode": wl.decode_ms_per_token,
            "prefill_ms_per_token": layers * prefill * 1e3 / new_tokens, "decode_ms_per_token": layers * decode * 1e3 / decoded}


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--requests", type=int, default=4000)
    p.add_argument("--replica", type=int, default=0)
    p.add_argument("--layers", type=int, default=32)
    p.add_argument("--dtype", default="e4m3", choices=["bf16", "fp16", "e4m3"])
    a = p.parse_args()
    r = run(a.requests, a.replica, a.layers, a.dtype)
    print(f"replica {a.replica}: {r['requests']} requests, {r['new_tokens']} prompt tokens computed, {r['hit_tokens']} found in the cache")
    print(f"attention of {a.layers} layers, {a.dtype} cache: {r['prefill_ms_per_token']:.5f} of prefill_ms_per_token ({r['model_prefill']} replayed), "
          f"{r['decode_ms_per_token']:.4f} of decode_ms_per_token ({r['model_decode']} replayed; here a step of the batch)")
    print(f"largest difference of the rows looked at from the definition in 64 bits: {r['worst']:.2e}")


if __name__ == "__main__":
    main()
