"""The rest of a serving loop over the paged 4-bit key/value cache: attention whose scores are capped, get a
bias that grows with distance, or are masked by window, document or prefix; requests that share their
context's blocks (fork) and blocks that are found free again or moved together (reclaim), with the copies that
both ask for; and the tokens sampled from a step's logits. Each case is one pass through one of them, from
one short request to batches of long contexts, in the operators' plain form or through the package's public
entry points.

The score of query and key at positions p and j of a request is x = scale q.k, capped to cap tanh(x / cap),
less slope |p - j| of the query head. A row sees the keys j with first <= j <= p or j < prefix, where first and
prefix are given for each token: a sliding window with the context's first tokens, a document of its own behind
a shared head, a prefix that sees itself in both directions.

A fork gives a request the blocks of another and a copy of the last one, where that is partly filled. Reclaiming
lists the blocks that no request holds, after moving blocks of high numbers into free ones of low numbers.

Sampling orders a row's logits, largest first (ties: lowest index first), with weights w = exp((x - max) /
temperature): of the first top_k, the shortest run whose weights reach top_p of theirs, and of that the weights
of at least min_p; the token is the first index at which the running sum of what is left, over the
indexes in their order, passes u times its whole. Temperature 0 takes the largest logit.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SCALE_RANGE = {"bf16": (-125, 125), "f16": (-13, 13)}  # of a scale's exponent: its codes are normal numbers of the type
SINK = 4  # tokens at a context's beginning that a window keeps
TAIL = 32  # tokens at a prompt's end that see all documents


# ------------------------------------------------------------------ the cases

def listed():
    layout = dict(heads=8, group=4, dim=128, block=64)
    return [
        # One short request, one token, capped scores: latency.
        dict(name="capped_decode_1", kind="attend", type="f16", requests=1, prompts=0, added=1, context=777, heads=4,
             group=2, dim=64, block=16, cap=30.0, slopes=False, mask="", span=0),
        # Single tokens over whole long contexts with a bias by distance, the largest read of the cache.
        dict(name="biased_decode_64", kind="attend", type="bf16", requests=64, prompts=0, added=1, context=32_000,
             cap=0.0, slopes=True, mask="", span=0, **layout),
        # Single tokens that see a window of long contexts, and their first tokens.
        dict(name="window_decode_32", kind="attend", type="bf16", requests=32, prompts=0, added=1, context=50_000,
             cap=50.0, slopes=False, mask="window", span=4096, **layout),
        # Retrieved documents behind a shared head, each seeing itself and the head; the question behind them sees all.
        dict(name="documents_prompt_4k", kind="attend", type="bf16", requests=1, prompts=1, added=4000, context=611,
             cap=0.0, slopes=False, mask="documents", span=450, **layout),
        # A piece of a prompt whose first part sees itself in both directions, capped and biased.
        dict(name="prefix_prompt_2k", kind="attend", type="f16", requests=1, prompts=1, added=2048, context=8192,
             cap=30.0, slopes=True, mask="prefix", span=0, **layout),
        # Eight samples of one prompt.
        dict(name="fork_8", kind="fork", type="bf16", parents=1, children=8, context=3001, heads=4, dim=64, block=32),
        # A batch of prompts, 16 samples each.
        dict(name="fork_1024", kind="fork", type="bf16", parents=64, children=16, context=8000, heads=8, dim=128, block=64),
        # The free blocks after some requests of a small batch have ended.
        dict(name="reclaim_16", kind="reclaim", type="bf16", requests=16, context=4000, heads=2, dim=64, block=64,
             moves=0),
        # Half of a batch has ended: what is left is moved together.
        dict(name="reclaim_moved_64", kind="reclaim", type="f16", requests=64, context=16_000, heads=8, dim=128,
             block=64, moves=4096),
        # The next token of one request.
        dict(name="sample_1", kind="sample", type="f32", requests=1, vocab=32_000, mode="top_p"),
        # A step of a batch whose requests all ask for something else, with a large vocabulary.
        dict(name="sample_64_mixed", kind="sample", type="bf16", requests=64, vocab=128_000, mode="mixed"),
        # A large batch without limits on the tokens, odd rows.
        dict(name="sample_250_whole", kind="sample", type="f16", requests=250, vocab=100_003, mode="whole"),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "fork", "reclaim", "sample", "sample"])
    if kind == "sample":
        requests = _between(rng, 1, 256)
        return dict(kind=kind, type=rng.choice(["bf16", "f16", "f32"]), requests=requests,
                    vocab=_between(rng, 50, min(150_000, 25_000_000 // requests)),
                    mode=rng.choice(["mixed", "mixed", "whole", "top_k", "top_p", "greedy"]))
    block = rng.choice([16, 32, 64, 64, 128])
    heads, group = rng.choice([(8, 4), (8, 8), (4, 6), (2, 7), (1, 20), (12, 1), (5, 3)])
    case = dict(kind=kind, type=rng.choice(["bf16", "f16"]), heads=heads, dim=rng.choice([64, 96, 128, 128, 192, 256]),
                block=block)
    width = max(1.0, heads * case["dim"] / 1024.0)  # of a token, in the listed cases' measure
    if kind == "fork":
        parents = _between(rng, 1, 64)
        children = _between(rng, 1, 1024 / parents / width / max(1, block / 64))
        return dict(case, parents=parents, children=children, context=_between(rng, 1, min(8000, 500_000 / width / parents)))
    if kind == "reclaim":
        requests = _between(rng, 1, 64)
        return dict(case, requests=requests, context=_between(rng, 1, min(16_000, 500_000 / width / requests)),
                    moves=rng.choice([0, _between(rng, 1, 4096)]))
    shape = rng.choice(["decode", "decode", "prompt", "mixed"])
    if shape == "decode":
        requests = _between(rng, 1, 64)
        prompts, added = 0, 1
        context = _between(rng, 1, min(50_000, max(64, 2_000_000 / width / requests)))
    else:
        prompts = 1
        requests = 1 if shape == "prompt" else rng.randint(2, 8)
        rows = 2048 * 32 / (heads * group) / requests * min(1.0, 128 / case["dim"])
        added = _between(rng, 2, max(4, min(4096, rows)))
        context = _between(rng, 1, 8000)
    mask = rng.choice(["", "window", "documents", "prefix"])
    cap = rng.choice([0.0, 0.0, 5.0, 30.0, 50.0])
    return dict(case, group=group, requests=requests, prompts=prompts, added=added, context=context, cap=cap,
                slopes=rng.choice([False, True]), mask=mask,
                span=_between(rng, 10, 8000) if mask == "window" else _between(rng, 10, 1000) if mask == "documents" else 0)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(tokens in the cache before the call, new tokens) of each request: from the case alone."""
    if case["kind"] in ("fork", "reclaim"):
        count = case["parents"] if case["kind"] == "fork" else case["requests"]
        rng = random.Random("%d %d" % (count, case["context"]))
        return [max(1, int(case["context"] * math.exp(-1.5 * rng.random() * (i > 0)))) for i in range(count)], []
    rng = random.Random("%(requests)d %(prompts)d %(added)d %(context)d" % case)
    cached = [int(case["context"] * math.exp(-2.0 * rng.random() * (i > 0))) for i in range(case["requests"])]
    added = [max(1, int(case["added"] * (1.0 - 0.6 * rng.random() * (i > 0)))) if i < case["prompts"] else 1
             for i in range(case["requests"])]
    return cached, added


def _ceil(a, b):
    return -(-a // b)


def _ended(case):
    """Which requests of a reclaim case have ended: every other one, the longest among those that go on."""
    return [i % 2 == 1 for i in range(case["requests"])]


def _ranges(case):
    """For each request (first, prefix) of its new tokens, as two lists."""
    cached, added = _lengths(case)
    out = []
    for m, a in zip(cached, added):
        p = range(m, m + a)
        if case["mask"] == "window":
            out.append(([max(0, x - case["span"] + 1) for x in p], [min(SINK, x + 1) for x in p]))
        elif case["mask"] == "documents":
            alone = a - TAIL if a > 2 * TAIL else 0  # tokens that belong to documents
            out.append(([m + i // case["span"] * case["span"] if i < alone else 0 for i in range(a)],
                        [m if i < alone else 0 for i in range(a)]))
        elif case["mask"] == "prefix":
            out.append(([0] * a, [m + 3 * a // 4] * a))
        else:
            out.append(([0] * a, [0] * a))
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _power(e):
    """2^e in fp32."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x, kind):
    """Codes (0 ... 15) and scale exponents of x [..., dim] in groups of 32 channels."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    bits = top.view(torch.int32)
    e = (bits >> 23) - 129 + ((bits & 0x7FFFFF) > 0x600000).int()  # amax / 2^e in (3.5, 7]
    e = e.clamp(*SCALE_RANGE[kind])
    a = g.abs() * _power(-e)
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = code + 8 * (g < 0).byte()
    return code.flatten(-2), e.squeeze(-1)


def _pack(k, v, kind):
    """Records [blocks, heads, bytes] of keys and values [blocks, heads, tokens, dim]."""
    (kc, ke), (vc, ve) = _quantise(k, kind), _quantise(v, kind)
    parts = [kc[..., 0::2] | (kc[..., 1::2] << 4), vc[..., 0::2] | (vc[..., 1::2] << 4),
             (ke + 127).byte(), (ve + 127).byte().transpose(-1, -2)]
    return torch.cat([p.flatten(-2) for p in parts], -1)


def _unpack(records, block, dim):
    """fp32 keys and values [..., tokens, dim] of records [..., bytes]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=records.device)
    table = torch.cat([table, -table])
    k, v, ks, vs = records.split([block * dim // 2, block * dim // 2, block * dim // 32, block * dim // 32], -1)

    def values(b, e):
        b = b.unflatten(-1, (block, dim // 2))
        code = torch.stack([b & 15, b >> 4], -1).flatten(-2)
        return (table[code.int()].unflatten(-1, (-1, 32)) * _power(e).unsqueeze(-1)).flatten(-2)

    ke = ks.unflatten(-1, (block, dim // 32)).int() - 127
    ve = vs.unflatten(-1, (dim // 32, block)).transpose(-1, -2).int() - 127
    return values(k, ke), values(v, ve)


def _cache(s, g, blocks):
    """A cache whose blocks hold random tokens."""
    case = s["case"]
    shape = (blocks, case["heads"], case["block"], case["dim"])
    strong = 1.0 + 3.0 * (torch.rand(case["heads"], 1, case["dim"], generator=g, device=DEV) < 0.05)
    k = (torch.randn(shape, generator=g, device=DEV) * strong).to(TYPES[case["type"]])
    v = torch.randn(shape, generator=g, device=DEV).to(TYPES[case["type"]])
    s["records"] = _pack(k, v, case["type"])
    s["summary"] = torch.randint(-127, 128, (blocks, case["heads"], case["dim"]), generator=g, device=DEV).to(torch.int8)
    s["weight"] = torch.rand(blocks, case["heads"], generator=g, device=DEV)
    return strong


def _tables(lens, bs, cols, rows, ids):
    """Block tables [rows, cols] of requests of these lengths, ids taken in order."""
    need = _i32([_ceil(n, bs) for n in lens]).long()
    first = torch.cumsum(need, 0) - need
    col = torch.arange(cols, device=DEV)
    table = torch.full((rows, cols), -1, dtype=torch.int32, device=DEV)
    table[: len(lens)] = torch.where(col < need[:, None], ids[(first[:, None] + col).clamp(max=ids.numel() - 1)], -1)
    return table


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(0x5E21000 + int(seed))
    s = dict(case=case)
    if case["kind"] == "sample":
        return _prepare_sample(s, g)
    cached, added = _lengths(case)
    bs = case["block"]
    if case["kind"] == "fork":
        parents, children = case["parents"], case["parents"] * case["children"]
        need = sum(_ceil(n, bs) for n in cached)
        blocks = need + children + 8
        ids = torch.randperm(blocks, generator=g, device=DEV).int()
        s["table"] = _tables(cached, bs, _ceil(max(cached), bs) + 4, parents + children, ids)
        s["cached"] = _i32(cached + [0] * children)
        s["free"] = ids[need:]
        s["parent"] = _i32([i for i in range(parents) for _ in range(case["children"])])
        s["child"] = (parents + torch.randperm(children, generator=g, device=DEV)).int()
        _cache(s, g, blocks)
        return s
    if case["kind"] == "reclaim":
        need = sum(_ceil(n, bs) for n in cached)
        s["blocks"] = need + 40
        ids = torch.randperm(s["blocks"], generator=g, device=DEV).int()
        s["table"] = _tables(cached, bs, _ceil(max(cached), bs) + 4, len(cached), ids)
        s["cached"] = _i32([0 if ended else n for n, ended in zip(cached, _ended(case))])
        _cache(s, g, s["blocks"])
        return s
    total, tokens = [a + b for a, b in zip(cached, added)], sum(added)
    need = [_ceil(n, bs) for n in total]
    blocks = sum(need) + 8
    ids = torch.randperm(blocks, generator=g, device=DEV).int()
    s["table"] = _tables(total, bs, max(need) + 3, len(total), ids)
    s.update(cached=_i32(cached), tokens=tokens, longest=max(added), most=max(total))
    s["start"] = _i32([sum(added[:i]) for i in range(len(added) + 1)])
    s["request"] = torch.repeat_interleave(torch.arange(len(added), device=DEV), _i32(added).long(),
                                           output_size=tokens).int()
    s["position"] = (torch.arange(tokens, device=DEV) - s["start"][s["request"].long()]
                     + s["cached"][s["request"].long()]).int()
    if case["mask"]:
        ranges = _ranges(case)
        s["first"] = _i32([x for r in ranges for x in r[0]])
        s["prefix"] = _i32([x for r in ranges for x in r[1]])
    heads, group, dim = case["heads"], case["group"], case["dim"]
    if case["slopes"]:  # a geometric row, as heads of different reach have
        s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, heads * group + 1, device=DEV) / (heads * group)).float()
    strong = _cache(s, g, blocks)
    qkv = torch.randn(tokens, heads * (group + 2), dim, generator=g, device=DEV)  # of one projection
    qkv[:, : heads * group] *= 1.5 / strong.squeeze(1).repeat_interleave(group, 0)
    s["q"] = qkv.to(TYPES[case["type"]])[:, : heads * group]
    s["scale"] = 1.0 / math.sqrt(dim)
    return s


def _prepare_sample(s, g):
    case = s["case"]
    rows, vocab, mode = case["requests"], case["vocab"], case["mode"]
    wide = torch.randn(rows, vocab + (-vocab) % 64, generator=g, device=DEV) * 2.2  # the projection's width
    likely = torch.randint(0, vocab, (rows, 20), generator=g, device=DEV)
    wide.scatter_add_(1, likely, 3.0 + 5.0 * torch.rand(rows, 20, generator=g, device=DEV))
    if mode == "mixed":  # every fourth request allows some tokens only
        barred = torch.rand(wide.shape, generator=g, device=DEV) < 0.5
        barred[torch.arange(rows, device=DEV) % 4 != 1] = False
        wide.masked_fill_(barred, -math.inf)
    if mode == "whole":  # rows as a program hands them over that cut the padding off
        s["logits"] = wide[:, :vocab].to(TYPES[case["type"]]).contiguous()
    else:
        s["logits"] = wide.to(TYPES[case["type"]])[:, :vocab]
    s["uniform"] = torch.rand(rows, generator=g, device=DEV)
    pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(0, len(v), (rows,), generator=g, device=DEV)]  # noqa: E731
    if mode == "mixed":
        s.update(temperature=pick(0.0, 0.3, 0.7, 1.0, 1.0, 1.3), top_k=pick(0, 0, 1, 20, 50, 400).int(),
                 top_p=pick(1.0, 1.0, 0.95, 0.9, 0.5), min_p=pick(0.0, 0.0, 0.0, 0.05, 0.2))
    elif mode == "whole":
        s.update(temperature=pick(0.8, 1.0, 1.2))
    elif mode == "top_k":
        s.update(temperature=pick(0.7, 1.0), top_k=pick(10, 40, 64, 1000).int())
    elif mode == "top_p":
        s.update(temperature=pick(0.7, 1.0), top_p=pick(0.9, 0.95))
    else:
        s.update(temperature=pick(0.0))
    return s


# ------------------------------------------------------------------ the plain forms

def _padded(s, x):
    """x [tokens, ...] as [requests, longest, ...], and each token's place there."""
    place = (torch.arange(s["tokens"], device=DEV) - s["start"][s["request"].long()]).long()
    out = x.new_zeros(s["case"]["requests"], s["longest"], *x.shape[1:])
    out[s["request"].long(), place] = x
    return out, place


def _attend(s):
    case, heads, bs, dim = s["case"], s["case"]["heads"], s["case"]["block"], s["case"]["dim"]
    cols = _ceil(s["most"], bs)
    records = s["records"][s["table"][:, :cols].clamp(min=0).long()]  # [requests, cols, heads, bytes]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _unpack(records, bs, dim))
    q, place = _padded(s, s["q"].float())
    after, _ = _padded(s, s["position"] + 1)  # 0 in the padding
    q = q.unflatten(2, (heads, -1)).transpose(1, 2).flatten(2, 3)  # [requests, heads, longest * group, dim]
    score = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()) * s["scale"]
    score = score.unflatten(2, (s["longest"], -1))  # [requests, heads, longest, group, keys]
    if case["cap"]:
        score = score.div_(case["cap"]).tanh_().mul_(case["cap"])
    key = torch.arange(cols * bs, device=DEV)
    if case["slopes"]:
        apart = (after[..., None] - 1 - key).abs().float()[:, None, :, None]
        score = score.addcmul_(s["slopes"].view(heads, 1, -1, 1), apart, value=-1.0)
    seen = key < after[..., None]
    if case["mask"]:
        seen = (seen & (key >= _padded(s, s["first"])[0][..., None])) | (key < _padded(s, s["prefix"])[0][..., None])
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (s["longest"], -1)) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)
    pick = lambda x: x[s["request"].long(), :, place].flatten(1, 2)  # noqa: E731
    return pick(out).to(s["q"].dtype), pick(lse).contiguous()


def _copy(s, source, to):
    """Copies blocks; entries of -1 copy nothing (here: a block that is not written onto itself)."""
    idle = source.max()
    source, to = torch.where(source >= 0, source, idle).long(), torch.where(to >= 0, to, idle).long()
    for x in (s["records"], s["summary"], s["weight"]):
        x[to] = x[source]
    return s["records"], s["summary"], s["weight"]


def _fork(s):
    bs, free, table, cached = s["case"]["block"], s["free"], s["table"], s["cached"]
    parent, child = s["parent"].long(), s["child"].long()
    n = cached[parent]
    used = ((n + bs - 1) // bs).long()
    partly = n % bs != 0
    rank = torch.cumsum(partly, 0) - partly.long()
    got = partly & (rank < free.numel())
    to = torch.where(got, free[rank.clamp(max=free.numel() - 1)], -1)
    source = torch.where(got, table[parent, (used - 1).clamp(min=0)], -1)
    col = torch.arange(table.shape[1], device=DEV)
    rows = torch.where(col < used[:, None], table[parent], -1)
    rows = torch.where((col == used[:, None] - 1) & partly[:, None], to[:, None], rows)
    table, cached = table.index_copy(0, child, rows), cached.index_copy(0, child, n)
    return (table, cached, source, to) + _copy(s, source, to)


def _reclaim(s):
    bs, table, blocks, moves = s["case"]["block"], s["table"], s["blocks"], s["case"]["moves"]
    held = torch.arange(table.shape[1], device=DEV) < ((s["cached"] + bs - 1) // bs)[:, None]
    used = torch.zeros(blocks + 1, dtype=torch.int64, device=DEV)
    used[torch.where(held, table, blocks).long()] = 1
    used = used[:blocks]
    count = used.sum()
    block = torch.arange(blocks, device=DEV)
    high, low = (used == 1) & (block >= count), (used == 0) & (block < count)
    made = torch.minimum(high.sum(), torch.full_like(count, moves))

    def in_order(chosen, room):
        """The chosen blocks in ascending order, -1 behind them, and each one's rank."""
        rank = torch.cumsum(chosen, 0) - 1
        out = torch.full((room + 1,), -1, dtype=torch.int32, device=DEV)
        out[torch.where(chosen & (rank < room), rank, room)] = block.int()
        out[room] = -1
        return out[:room], rank

    source, rank = in_order(high, moves)
    to, hole = in_order(low, moves)
    moved, filled = high & (rank < made), low & (hole < made)
    goes = torch.where(moved, torch.cat([to, to.new_zeros(1)])[rank.clamp(0, moves)], block.int())
    table = torch.where(held, goes[table.clamp(min=0).long()], table)
    free, _ = in_order(((used == 0) & ~filled) | moved, blocks)
    info = torch.stack([count, made, blocks - count])
    if not moves:
        return table, free, info
    return (table, free, source, to, info) + _copy(s, source, to)


def _sample(s):
    x = s["logits"].double()
    rows, vocab = x.shape
    top = x.amax(1, keepdim=True)
    t = s["temperature"].double()[:, None]
    w = torch.exp((x - top) / torch.where(t > 0, t, 1.0))
    # greedy rows: the first of the largest, alone
    index = torch.arange(vocab, device=DEV)
    best = torch.where(x == top, index, vocab).amin(1, keepdim=True)
    w = torch.where(t > 0, w, (index == best).double())
    if "top_k" in s or "top_p" in s or "min_p" in s:
        _, order = torch.sort(x, dim=1, descending=True, stable=True)
        ranked = w.gather(1, order)
        total = torch.cumsum(ranked, 1)
        keep = torch.full((rows, 1), vocab, device=DEV)
        if "top_k" in s:
            k = s["top_k"].long()[:, None]
            keep = torch.where(k > 0, k.clamp(max=vocab), keep)
        kept = index < keep
        if "top_p" in s:
            p = s["top_p"].double()[:, None]
            enough = p * total.gather(1, keep - 1)
            kept &= (p >= 1.0) | (total - ranked < enough) | (index == 0)
        if "min_p" in s:
            kept &= (ranked >= s["min_p"].double()[:, None]) | (index == 0)
        w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, ranked, 0.0))
    total = torch.cumsum(w, 1)
    token = (total <= s["uniform"].double()[:, None] * total[:, -1:]).sum(1)
    logprob = torch.log(w.gather(1, token[:, None]) / total[:, -1:]).squeeze(1)
    return token.int(), logprob.float()


# ------------------------------------------------------------------ the framework's entry points

def _handles(s):
    """The context and the cache's handle that a program keeps."""
    import paper_2608_08751_amd as ivf

    if "context" not in s:
        s["context"] = ivf.Context(0)
        if "records" in s:
            s["cache"] = ivf.KVCache(s["records"], s["summary"], s["weight"], s["case"]["block"],
                                     TYPES[s["case"]["type"]])
    return ivf, s["context"], s.get("cache")


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if not own:
        return {"attend": _attend, "fork": _fork, "reclaim": _reclaim, "sample": _sample}[kind](s)
    ivf, ctx, cache = _handles(s)
    if kind == "attend":
        return ivf.ivf_kv_attend(ctx, cache, s["q"], s["start"], s["request"], s["position"], s["table"], s["scale"],
                                 s["longest"], cap=case["cap"], slopes=s.get("slopes"), first=s.get("first"),
                                 prefix=s.get("prefix"))
    if kind == "sample":
        return ivf.ivf_sample(ctx, s["logits"], s["uniform"], temperature=s.get("temperature"), top_k=s.get("top_k"),
                              top_p=s.get("top_p"), min_p=s.get("min_p"))
    table, cached = s["table"].clone(), s["cached"]  # the calls change them in place
    if kind == "fork":
        cached = cached.clone()
        fork = ivf.ivf_kv_fork(ctx, s["parent"], s["child"], cached, case["block"], table, s["free"])
        ivf.ivf_kv_copy(ctx, cache, fork.to, fork.source)
        return table, cached, fork.source, fork.to, s["records"], s["summary"], s["weight"]
    found = ivf.ivf_kv_reclaim(ctx, cached, case["block"], table, s["blocks"], moves=case["moves"])
    if not case["moves"]:
        return table, found.free, found.info
    ivf.ivf_kv_copy(ctx, cache, found.to, found.source)
    return table, found.free, found.source, found.to, found.info, s["records"], s["summary"], s["weight"]


# ------------------------------------------------------------------ work and exact values

def work(case):
    if case["kind"] == "sample":
        n = float(case["requests"]) * case["vocab"]
        return {"bytes": n * (4 if case["type"] == "f32" else 2) + 28.0 * case["requests"], "flops": 3.0 * n}
    cached, added = _lengths(case)
    bs, heads, dim = case["block"], case["heads"], case["dim"]
    of_block = heads * (bs * dim * 17.0 / 16 + dim + 4)
    held = [_ceil(n, bs) for n in cached]
    cols = max(held) + 4
    if case["kind"] == "fork":
        rows = case["parents"] * case["children"]
        copies = sum(n % bs != 0 for n in cached) * case["children"]
        # the tables come back whole, changed
        return {"bytes": copies * 2 * of_block + 4.0 * sum(held) + 4.0 * (case["parents"] + rows) * cols + 24.0 * rows, "flops": 0.0}
    if case["kind"] == "reclaim":
        live = sum(n for n, ended in zip(held, _ended(case)) if not ended)
        blocks = sum(held) + 40
        high = live * (blocks - live) // blocks  # blocks lie at random: about so many at or above `live`
        moved = min(high, case["moves"])
        return {"bytes": moved * (2 * of_block + 12) + 4.0 * live + 4.0 * blocks + 4.0 * len(held) * cols, "flops": 0.0}
    token = heads * dim * 17.0 / 16.0  # of the cache, keys and values
    row = 2.0 * heads * case["group"] * dim
    read = seen = 0
    for m, a, (first, prefix) in zip(cached, added, _ranges(case)):
        touched = bytearray(m + a)
        if case["mask"] in ("", "prefix"):
            touched = [1] * (m + a)
        for p, f, e in zip(range(m, m + a), first, prefix):
            lo = max(f, e)
            seen += min(e, m + a) + max(0, p + 1 - lo)
            if case["mask"] not in ("", "prefix"):
                touched[:e] = b"\1" * e
                if p >= lo:
                    touched[lo: p + 1] = b"\1" * (p + 1 - lo)
        read += sum(touched)
    return {"bytes": read * token + sum(added) * (2 * row + 4 * heads * case["group"] + 16),
            "flops": 4.0 * heads * case["group"] * dim * seen}


def _exact_sample(s):
    """Row by row from the definition: the weights sorted in 64 bits."""
    import numpy as np

    rows, vocab = s["logits"].shape
    x = s["logits"].double().cpu().numpy()
    get = lambda name, default: s[name].double().cpu().numpy() if name in s else np.full(rows, default)  # noqa: E731
    u, t, k = get("uniform", 0.0), get("temperature", 1.0), get("top_k", 0.0)
    top_p, min_p = get("top_p", 1.0), get("min_p", 0.0)
    token, logprob = np.zeros(rows, np.int32), np.zeros(rows)
    for r in range(rows):
        if t[r] <= 0:
            token[r] = int(np.argmax(x[r]))
            continue
        order = np.lexsort((np.arange(vocab), -x[r]))
        if k[r] > 0:
            order = order[: int(k[r])]
        w = np.exp((x[r][order] - x[r].max()) / t[r])
        if top_p[r] < 1:
            order = order[: max(1, int(np.searchsorted(np.cumsum(w), top_p[r] * w.sum(), side="left")) + 1)]
            w = w[: len(order)]
        n = max(1, int((w >= min_p[r]).sum()))
        order, w = order[:n], w[:n]
        by_index = np.argsort(order)
        order, w = order[by_index], w[by_index]
        running = np.cumsum(w)
        at = min(int(np.searchsorted(running, u[r] * running[-1], side="right")), n - 1)
        token[r], logprob[r] = order[at], math.log(w[at] / running[-1])
    return torch.from_numpy(token), torch.from_numpy(logprob)


def exact(case, seed):
    """Attention in 64 bits, request by request; the sampled tokens and their log-probabilities, row by row."""
    if case["kind"] in ("fork", "reclaim"):
        return None
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    bs, dim, heads, group, n = case["block"], case["dim"], case["heads"], case["group"], case["block"] * case["dim"]
    steps = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=DEV) / 2

    def values(records, part):
        """One of the two arrays of records [n, heads, bytes], fp64 [n, heads, bs, dim]."""
        b = records[..., part * n // 2: (part + 1) * n // 2].reshape(*records.shape[:-1], bs, dim // 2).long()
        e = records[..., n + part * n // 32: n + (part + 1) * n // 32].double()
        e = e.reshape(*e.shape[:-1], bs, dim // 32) if part == 0 else e.reshape(*e.shape[:-1], dim // 32, bs).mT
        out = torch.empty(*b.shape[:-1], dim, dtype=torch.float64, device=DEV)
        for odd in (0, 1):
            c = (b >> (4 * odd)) & 15
            out[..., odd::2] = steps[c & 7] * (1 - 2 * (c >> 3))
        return out * torch.pow(2.0, e - 127.0).repeat_interleave(32, -1)

    cached, added = _lengths(case)
    out = torch.zeros(s["tokens"], heads * group, dim, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["tokens"], heads * group, dtype=torch.float64, device=DEV)
    begin = 0
    for b, (m, a, (first, prefix)) in enumerate(zip(cached, added, _ranges(case))):
        total = m + a
        records = s["records"][s["table"][b, : _ceil(total, bs)].long()]
        k, v = (values(records, part).permute(1, 0, 2, 3).reshape(heads, -1, dim)[:, :total] for part in (0, 1))
        first, prefix = (torch.tensor(x, device=DEV) for x in (first, prefix))
        for i in range(0, a, 256):
            j = min(i + 256, a)
            at, key = torch.arange(m + i, m + j, device=DEV)[:, None], torch.arange(total, device=DEV)[None]
            away = torch.where(key < prefix[i:j, None], False, (key > at) | (key < first[i:j, None]))
            far = torch.where(key > at, key - at, at - key).double()
            for h in range(heads):
                for o in range(h * group, (h + 1) * group):
                    score = s["scale"] * (s["q"][begin + i: begin + j, o].double() @ k[h].mT.contiguous())
                    if case["cap"]:
                        score = case["cap"] * (1.0 - 2.0 / (1.0 + torch.exp(2.0 * score / case["cap"])))
                    if case["slopes"]:
                        score = score - s["slopes"][o].double() * far
                    score[away] = -math.inf
                    lse[begin + i: begin + j, o] = torch.logsumexp(score, -1)
                    out[begin + i: begin + j, o] = torch.exp(score - lse[begin + i: begin + j, o, None]) @ v[h]
        begin += a
    return out, lse
