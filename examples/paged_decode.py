"""Prompts and then decoding over the paged 4-bit key/value cache: the operators as a
serving loop runs them, for one attention layer with random queries, keys and values.

    python examples/paged_decode.py --requests 32 --prompt 4000 --steps 64

Every prompt is planned, written and attended to in one call each (prompts of different
lengths side by side). A decoding step is plan, append, select and attend; it is
captured once and replayed, with its inputs, the requests' lengths and the free
blocks in buffers that stay where they are. The last step is checked against fp64
over what the cache holds.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_08751_amd as ivf  # noqa: E402


def reference(ctx, cache, q, table, lengths, blocks, scale):
    """fp64 attention of one token a request over its selected blocks, on the host."""
    heads, bs = cache.heads, cache.block_size
    group = q.shape[1] // heads
    out = torch.zeros(q.shape, dtype=torch.float64)
    table, blocks, q = table.cpu(), blocks.cpu(), q.cpu().double()
    for b, n in enumerate(lengths):
        for h in range(heads):
            pos = [j * bs + i for j in blocks[b, h].tolist() if j >= 0 for i in range(bs) if j * bs + i < n]
            slots = [int(table[b, p // bs]) * bs + p % bs for p in pos]
            k, v, _ = ivf.ivf_kv_read(ctx, cache, torch.tensor(slots).cuda())
            k, v = k[:, h].cpu().double(), v[:, h].cpu().double()
            rows = slice(h * group, (h + 1) * group)
            out[b, rows] = torch.softmax(scale * (q[b, rows] @ k.T), -1) @ v
    return out


def run(requests=8, prompt=600, steps=16, heads=4, group=4, dim=128, block_size=64, count=8, dtype=torch.bfloat16, seed=0):
    """Returns (milliseconds for the prompts, microseconds a step, largest error of the last
    step relative to the largest output, blocks in use)."""
    torch.manual_seed(seed)
    device, scale = "cuda", dim**-0.5
    ctx = ivf.Context(0)
    lengths = torch.linspace(prompt / 2, prompt, requests).int().tolist()
    per_request = -(-(prompt + steps + 2) // block_size)
    cache = ivf.KVCache.empty(requests * per_request, heads, dim, block_size, dtype)
    pool = torch.randperm(requests * per_request, device=device).int()
    table = torch.full((requests, per_request), -1, dtype=torch.int32, device=device)
    used = torch.zeros((), dtype=torch.int64, device=device)
    cached = torch.zeros(requests, dtype=torch.int32, device=device)

    def inputs(tokens):
        make = lambda n: torch.randn(tokens, n, dim, device=device, dtype=dtype)  # noqa: E731
        return make(heads * group), make(heads), make(heads)

    # all prompts in one batch
    added = torch.tensor(lengths, dtype=torch.int32, device=device)
    tokens = sum(lengths)
    q, k, v = inputs(tokens)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    plan = ivf.ivf_kv_plan(ctx, cached, added, block_size, table, pool, tokens, want_info=True)
    ivf.ivf_kv_append(ctx, cache, k, v, plan.slots)
    ivf.ivf_kv_attend(ctx, cache, q, plan.start, plan.request, plan.position, table, scale, max(lengths))
    end.record()
    used += plan.info[2]
    cached += added
    end.synchronize()
    prompt_ms = begin.elapsed_time(end)

    one = torch.ones_like(cached)
    ahead = torch.arange(requests, device=device)  # a step takes at most a block a request
    q, k, v = inputs(requests)

    def step():
        free = pool[(used + ahead).clamp(max=pool.numel() - 1)]
        plan = ivf.ivf_kv_plan(ctx, cached, one, block_size, table, free, requests, want_info=True)
        ivf.ivf_kv_append(ctx, cache, k, v, plan.slots)
        blocks = ivf.ivf_kv_select(ctx, cache, q, plan.request, plan.position, table, count)
        out, _ = ivf.ivf_kv_attend(ctx, cache, q, plan.start, plan.request, plan.position, table, scale, 1, blocks=blocks)
        used.add_(plan.info[2])
        cached.add_(one)
        return out, blocks

    # once outside a graph, so that the workspace has its size
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, blocks = step()
    begin.record()
    for _ in range(steps):
        for t in (q, k, v):
            t.normal_()
        graph.replay()
    end.record()
    end.synchronize()
    step_us = begin.elapsed_time(end) * 1e3 / steps

    now = [n + 1 + steps for n in lengths]
    assert cached.tolist() == now
    want = reference(ctx, cache, q, table, now, blocks, scale)
    error = float((out.cpu().double() - want).abs().max() / want.abs().max())
    in_use = int(used)
    ctx.close()
    return prompt_ms, step_us, error, in_use


def main():
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("requests", 32), ("prompt", 4000), ("steps", 64), ("heads", 8), ("group", 4), ("dim", 128),
                          ("block-size", 64), ("count", 16)):
        parser.add_argument("--" + name, type=int, default=default)
    args = parser.parse_args()
    prompt_ms, step_us, error, in_use = run(args.requests, args.prompt, args.steps, args.heads, args.group, args.dim,
                                            args.block_size, args.count)
    print("prompts of %d requests: %.2f ms; %d decoding steps: %.0f us each; %d blocks in use; last step off by %.1e"
          % (args.requests, prompt_ms, args.steps, step_us, in_use, error))


if __name__ == "__main__":
    main()
