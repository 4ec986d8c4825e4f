"""Several samples of each prompt over the paged 4-bit key/value cache: forked after the prompt,
decoded with capped, windowed attention and sampled tokens, and, when half of them have ended,
the rest moved together.

    python examples/parallel_samples.py --prompts 4 --samples 8 --prompt 3000 --steps 64

The model is one attention layer with random weights between an embedding and its transpose. A
decoding step is embed, plan, append, attend, project and sample; it is captured once and replayed,
with its inputs, lengths, tables and free blocks in buffers that stay where they are. The last step
is checked against fp64 over what the cache holds, its tokens against its logits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_08751_amd as ivf  # noqa: E402


def attention(ctx, cache, q, table, n, window, sink, cap, scale):
    """fp64 attention of one token at position n - 1 over what the cache holds of its request, on the host."""
    bs, group = cache.block_size, q.shape[0] // cache.heads
    pos = torch.arange(n)
    slots = table.cpu()[pos // bs].long() * bs + pos % bs
    k, v, _ = ivf.ivf_kv_read(ctx, cache, slots.cuda())
    k, v = (x.cpu().double().repeat_interleave(group, 1) for x in (k, v))
    score = cap * torch.tanh(scale * torch.einsum("jhd,hd->hj", k, q.cpu().double()) / cap)
    score[:, (pos >= sink) & (pos < n - window)] = -torch.inf
    return torch.einsum("hj,jhd->hd", torch.softmax(score, -1), v)


def sampled(logits, u, temperature, top_k, top_p):
    """The tokens of ivf_sample in fp64, on the host."""
    x = logits.cpu().double()
    w = torch.exp((x - x.amax(1, keepdim=True)) / temperature)
    order = torch.sort(x, descending=True, stable=True)[1][:, :top_k]
    ranked = w.gather(1, order)
    before = torch.cumsum(ranked, 1) - ranked
    ranked[before >= top_p * ranked.sum(1, keepdim=True)] = 0
    total = torch.cumsum(torch.zeros_like(w).scatter_(1, order, ranked), 1)
    return (total <= u.cpu().double()[:, None] * total[:, -1:]).sum(1)


def follow(last, token, request):
    """Writes a batch's tokens to its requests' entries of `last`, which has one entry more: the padding's (request -1)."""
    last.scatter_(0, torch.where(request >= 0, request, last.shape[0] - 1).long(), token)


def run(prompts=2, samples=4, prompt=300, steps=12, heads=2, group=4, dim=64, block_size=32, vocab=5000, window=128, sink=4,
        cap=30.0, dtype=torch.bfloat16, seed=0):
    """Returns a dict: microseconds a step, the last step's largest error relative to its largest output, whether
    its tokens are those of its logits in fp64, blocks in use before and after half of the samples ended,
    blocks moved, and the tokens [samples, steps]."""
    torch.manual_seed(seed)
    ctx, bs, rows, scale = ivf.Context(0), block_size, prompts * (1 + samples), dim**-0.5
    wide = heads * group * dim
    rand = lambda *shape: torch.randn(*shape, device="cuda")  # noqa: E731
    embed = rand(vocab, wide).to(dtype)
    w_qkv, w_out = (rand(wide, (heads * (group + 2)) * dim) * wide**-0.5).to(dtype), (rand(wide, wide) * 3 * wide**-0.5).to(dtype)
    longest = prompt + 2 * steps + 4
    cols = -(-longest // bs)
    blocks = rows * cols
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((rows, cols), -1, dtype=torch.int32, device="cuda")
    cached = torch.zeros(rows, dtype=torch.int32, device="cuda")
    free = torch.randperm(blocks, device="cuda").int()  # from `used` on
    used = torch.zeros((), dtype=torch.int64, device="cuda")

    def layer(tokens, plan, longest):
        q, k, v = (embed[tokens.long()] @ w_qkv).unflatten(1, (-1, dim)).split([heads * group, heads, heads], 1)
        ivf.ivf_kv_append(ctx, cache, k, v, plan.slots)
        out, _ = ivf.ivf_kv_attend(ctx, cache, q, plan.start, plan.request, plan.position, table, scale, longest, cap=cap,
                                   first=plan.position - (window - 1), prefix=(plan.position + 1).clamp(max=sink))
        return q, out

    # the prompts, in the first rows
    lengths = [prompt - 7 * i for i in range(prompts)]
    added = i32(*lengths, *[0] * (rows - prompts))
    plan = ivf.ivf_kv_plan(ctx, cached, added, bs, table, free, sum(lengths), want_info=True)
    tokens = torch.randint(0, vocab, (sum(lengths),), device="cuda")
    layer(tokens, plan, max(lengths))
    used += plan.info[2]
    cached += added

    # their samples, in the other rows; the prompts themselves end: their blocks are the samples'
    parent = torch.arange(prompts, device="cuda").repeat_interleave(samples).int()
    child = torch.arange(prompts, rows, device="cuda").int()
    fork = ivf.ivf_kv_fork(ctx, parent, child, cached, bs, table, free[int(used):], want_info=True)
    ivf.ivf_kv_copy(ctx, cache, fork.to, fork.source)
    used += fork.info[1]
    cached[:prompts] = 0

    # a decoding step of one token for every request that goes on; the others bring none
    live = (cached > 0).int()
    last = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    last[prompts:rows] = tokens[plan.start[1:prompts + 1].long() - 1].int().repeat_interleave(samples)
    uniform = torch.zeros(rows, device="cuda")
    full = lambda v, kind: torch.full((rows,), v, dtype=kind, device="cuda")  # noqa: E731
    limits = dict(temperature=full(0.8, torch.float32), top_k=full(50, torch.int32), top_p=full(0.95, torch.float32))
    ahead, logits = torch.arange(rows, device="cuda"), torch.zeros(rows, vocab, device="cuda")

    def step():
        plan = ivf.ivf_kv_plan(ctx, cached, live, bs, table, free[(used + ahead).clamp(max=blocks - 1)], rows, want_info=True)
        at = plan.request.long().clamp(min=0)  # the batch's rows: its live requests, then padding
        q, out = layer(last[at], plan, 1)
        logits.copy_((out.flatten(1) @ w_out) @ embed.T)
        token, _ = ivf.ivf_sample(ctx, logits, uniform, **limits)
        follow(last, token, plan.request)
        used.add_(plan.info[2])
        cached.add_(live)
        return q, out, token, plan.request

    side = torch.cuda.Stream()
    keep = [x.clone() for x in (cached, table, used, last, cache.records, cache.summary, cache.weight)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once outside a graph, so that the workspace has its size; then taken back
        step()
    side.synchronize()
    for x, y in zip((cached, table, used, last, cache.records, cache.summary, cache.weight), keep):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        q, out, token, request = step()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    drawn = []

    def decode(n):
        for _ in range(n):
            uniform.uniform_()
            graph.replay()
            drawn.append(last[prompts:rows].clone())

    begin.record()
    decode(steps)
    end.record()
    end.synchronize()

    # every other sample ends; what is left is moved together
    before = int(ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks).info[0])
    cached[prompts + 1::2] = 0
    live.copy_((cached > 0).int())
    found = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks, moves=blocks)
    ivf.ivf_kv_copy(ctx, cache, found.to, found.source)
    in_use, moved, _ = found.info.tolist()
    free.copy_(found.free)
    used.zero_()
    decode(steps)
    torch.cuda.synchronize()

    requests = [r for r in request.tolist() if r >= 0]
    want = torch.stack([attention(ctx, cache, q[i], table[r], int(cached[r]), window, sink, cap, scale) for i, r in enumerate(requests)])
    n = len(requests)
    error = float((out[:n].cpu().double() - want).abs().max() / want.abs().max())
    same = bool((sampled(logits[:n], uniform[:n], limits["temperature"][:1].cpu().double(), 50, limits["top_p"][:1].cpu().double())
                 == token[:n].cpu()).all())
    ctx.close()
    return dict(step_us=begin.elapsed_time(end) * 1e3 / steps, error=error, same=same, before=before, in_use=in_use, moved=moved,
                live=n, tokens=torch.stack(drawn, 1).cpu())


def main():
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("prompts", 4), ("samples", 8), ("prompt", 3000), ("steps", 64), ("heads", 8), ("group", 4), ("dim", 128),
                          ("block-size", 64), ("vocab", 32000), ("window", 1024)):
        parser.add_argument("--" + name, type=int, default=default)
    args = parser.parse_args()
    r = run(args.prompts, args.samples, args.prompt, args.steps, args.heads, args.group, args.dim, args.block_size, args.vocab,
            args.window)
    print("%d steps of %d samples: %.0f us each; blocks in use %d, after half of them ended %d (%d moved); last step off by %.1e, "
          "tokens %s" % (args.steps, args.prompts * args.samples, r["step_us"], r["before"], r["in_use"], r["moved"], r["error"],
                         "as in fp64" if r["same"] else "not as in fp64"))


if __name__ == "__main__":
    main()
