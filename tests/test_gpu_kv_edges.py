"""Edges of the paged 4-bit key/value cache's operators on the GPU, against the definitions
in fp64 (tests/kv_model.py). Attention is held to what its roundings allow, as in
tests/test_gpu_kv.py (check_attend)."""
import numpy as np
import pytest

import kv_model as M
from test_gpu_kv import as_np, batch, check_attend, ctx, dev, dtype_of, ints, make, queries  # noqa: F401 (ctx: a fixture)

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f16"]


def attend_held(ctx, kind, cache, table, keys, values, start, request, position, q, bs, scale, longest):  # noqa: F811
    """Attention of a batch held to the model; query rows that are not finite are NaN where they see a key."""
    import paper_2608_08751_amd as ivf

    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), scale, longest)
    clean = as_np(q)
    spoilt = ~np.isfinite(clean).all(-1)
    clean = np.where(spoilt[..., None], 0.0, clean)
    want, want_lse = M.attend(clean, keys, values, cache.heads, request, position, table, bs, scale)
    spoilt &= want_lse > -np.inf
    want[spoilt], want_lse[spoilt] = np.nan, np.nan
    smax = abs(scale) * np.abs(clean).sum(-1).max() * np.nanmax(np.abs(keys))
    check_attend(out, lse, want, want_lse, kind, np.nanmax(np.abs(values)), smax)


def test_a_captured_call_survives_a_larger_workspace():
    # a decoding step whose key ranges are split is captured; then a call that needs more replaces the workspace.
    # Replays write their parts into memory that is nobody else's.
    import torch

    import paper_2608_08751_amd as ivf

    own = ivf.Context(0)
    heads, group, dim, bs, lens = 2, 4, 128, 64, [5000, 3000]
    cache, table, keys, values = make(own, "bf16", lens, heads, dim, bs, 95)
    start, request, position = batch(lens, [1, 1])
    args = [ints(start), ints(request), ints(position), ints(table)]
    q = queries(2, heads * group, dim, "bf16", 1, strided=False)
    assert cache.attend_bytes(own, heads * group, 2, 2, table.shape[1], 0, 1) > 0  # parts lie in the workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ivf.ivf_kv_attend(own, cache, q, *args, 0.1, 1)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = ivf.ivf_kv_attend(own, cache, q, *args, 0.1, 1)
    old = own._ws.numel()
    new = 100  # a piece of a prompt, split into more parts
    s2, r2, p2 = batch(lens[:1], [new])
    q2 = queries(new, heads * group, dim, "bf16", 2)
    assert cache.attend_bytes(own, heads * group, new, 1, table.shape[1], 0, new) > old
    want2, want_lse2 = M.attend(as_np(q2), keys, values, heads, r2, p2, table[:1], bs, 0.1)
    others = []
    for i in range(3):
        out2, lse2 = ivf.ivf_kv_attend(own, cache, q2, ints(s2), ints(r2), ints(p2), ints(table[:1]), 0.1, new)
        for stream in (torch.cuda.current_stream(), side):
            with torch.cuda.stream(stream):
                others += [torch.full((old,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(8)]
        fresh = queries(2, heads * group, dim, "bf16", 10 + i, strided=False)
        q.copy_(fresh)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all((x == 0x5A).all() for x in others)
        want, want_lse = M.attend(as_np(fresh), keys, values, heads, request, position, table, bs, 0.1)
        check_attend(out, lse, want, want_lse, "bf16", np.nanmax(np.abs(values)), 50.0)
        check_attend(out2, lse2, want2, want_lse2, "bf16", np.nanmax(np.abs(values)), 50.0)
    own.close()


# the single-token kernel; the prompt kernel, its key range whole and split
@pytest.mark.parametrize("kind,new,group,dim,bs", [("bf16", 9, 2, 64, 16), ("f16", 300, 2, 64, 16), ("bf16", 200, 1, 128, 64),
                                                   ("f16", 90, 3, 256, 32)])
def test_the_most_negative_positions_see_nothing(ctx, kind, new, group, dim, bs):  # noqa: F811
    n = new + 500
    cache, table, keys, values = make(ctx, kind, [n], 2, dim, bs, 91)
    start, request, position = batch([n], [new])
    for i, p in enumerate((-(2**31), -(2**31) + 5, -(2**31) + 70, -(2**31) + 4000, -1, -64)):
        position[(i + 1) * new // 8] = p
    q = queries(new, 2 * group, dim, kind, 92)
    attend_held(ctx, kind, cache, table, keys, values, start, request, position, q, bs, dim**-0.5, new)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [0.125, -0.125])
@pytest.mark.parametrize("new,dim", [(2, 64), (70, 64), (70, 96), (200, 128), (70, 192), (70, 256)])
def test_queries_of_infinity_whose_scores_are_all_the_lowest(ctx, kind, scale, new, dim):  # noqa: F811
    # one channel of the keys is negative in every token: an infinity there scores -infinity (or, by the scale's
    # sign, +infinity) with every key, the softmax of which is no number
    import paper_2608_08751_amd as ivf

    heads, n, bs = 2, new + 40, 16
    rng = np.random.default_rng(dim)
    kv = rng.standard_normal((n, 2, heads, dim))
    kv[:, 0, :, dim - 9] = -2.0
    kv = dev(kv.astype(np.float32), dtype_of(kind))
    blocks = -(-n // bs)
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, kv.dtype)
    ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], dev(np.arange(n, dtype=np.int64)))
    k, v = M.store(as_np(kv[:, 0]), as_np(kv[:, 1]), kind)
    assert (k[:, :, dim - 9] < 0).all()
    pad = lambda x: np.concatenate([x, np.zeros((blocks * bs - n, heads, dim))])  # noqa: E731
    keys, values = (pad(x).reshape(blocks, bs, heads, dim).transpose(0, 2, 1, 3) for x in (k, v))
    table = np.arange(blocks, dtype=np.int32)[None]
    start, request, position = batch([n], [new])
    position[1] = -1  # a row that sees nothing stays empty whatever its query holds
    q = queries(new, heads * 2, dim, kind, 93)
    q[0, 1, dim - 9], q[1, :, dim - 9] = float("inf"), float("inf")
    q[new // 2, 3, dim - 9], q[new - 1, 0, dim - 9] = float("inf"), -float("inf")
    attend_held(ctx, kind, cache, table, keys, values, start, request, position, q, bs, scale, new)


@pytest.mark.parametrize("tokens", [0, 5, 1000])
def test_plan_of_no_requests(ctx, tokens):  # noqa: F811
    import torch

    import paper_2608_08751_amd as ivf

    none = torch.empty(0, dtype=torch.int32, device="cuda")
    torch.full((4 * tokens + 64,), 77, dtype=torch.int32, device="cuda")  # what the outputs' memory may hold before
    plan = ivf.ivf_kv_plan(ctx, none, none, 16, none.view(0, 9), ints([4, 2]), tokens, want_info=True)
    assert plan.start.tolist() == [0] and plan.info.tolist() == [0, 0, 0, 0]
    for x in (plan.slots, plan.request, plan.position):
        assert x.shape == (tokens,) and (x == -1).all()


def test_plan_of_no_requests_writes_what_is_asked_for(ctx):  # noqa: F811
    import torch

    import paper_2608_08751_amd as ivf
    from paper_2608_08751_amd import _binding as B

    lib, handle = ctx.bind()
    start = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    assert lib.ivf_kv_plan(handle, None, None, 0, 16, None, 0, None, 0, 0, B._ptr(start), None, None, None,
                           None) == ivf.IVF_OK
    assert lib.ivf_kv_plan(handle, None, None, 0, 16, None, 0, None, 0, 0, None, None, None, None, None) == ivf.IVF_OK
    assert start.tolist() == [0, 77, 77]


USES = {"plan": ("cached", "added", "table", "free"), "append": ("k", "v", "slots"), "read": ("slots", "free"),
        "select": ("q", "request", "position", "table"),
        "attend": ("q", "start", "request", "position", "table", "blocks", "out", "lse")}


def arguments():
    """Tensors for a call each on a cache of 4 blocks of 16 tokens, 2 heads of 64 channels."""
    import torch

    return {"q": queries(3, 4, 64, "bf16", 1), "k": queries(3, 2, 64, "bf16", 2), "v": queries(3, 2, 64, "bf16", 3),
            "slots": dev(np.arange(3, dtype=np.int64)), "start": ints([0, 3]), "request": ints([0, 0, 0]),
            "position": ints([0, 1, 2]), "table": ints([[0, 1]]), "blocks": ints(np.zeros((3, 2, 1))),
            "cached": ints([0]), "added": ints([3]), "free": ints([1]),
            "out": torch.empty(3, 4, 64, device="cuda", dtype=torch.bfloat16), "lse": torch.empty(3, 4, device="cuda")}


def call(name, ctx, cache, a):  # noqa: F811
    import paper_2608_08751_amd as ivf

    if name == "plan":
        ivf.ivf_kv_plan(ctx, a["cached"], a["added"], 16, a["table"], a["free"], 3)
    elif name == "append":
        ivf.ivf_kv_append(ctx, cache, a["k"], a["v"], a["slots"])
    elif name == "read":
        ivf.ivf_kv_read(ctx, cache, a["slots"], a["free"])
    elif name == "select":
        ivf.ivf_kv_select(ctx, cache, a["q"], a["request"], a["position"], a["table"], 2)
    else:
        ivf.ivf_kv_attend(ctx, cache, a["q"], a["start"], a["request"], a["position"], a["table"], 0.1, 3,
                          blocks=a["blocks"], out=a["out"], out_lse=a["lse"])


def test_tensors_of_another_device_are_refused(ctx):  # noqa: F811
    # arguments on the host; all of device 0 with a context that says it is device 1's
    import paper_2608_08751_amd as ivf

    cache = ivf.KVCache.empty(4, 2, 64, 16, dtype_of("bf16"))
    other = ivf.Context(0)
    other.device = 1
    for name, used in USES.items():
        good = arguments()
        call(name, ctx, cache, good)
        with pytest.raises((TypeError, ValueError), match="device"):
            call(name, other, cache, good)
        for x in used:
            with pytest.raises((TypeError, ValueError), match="device"):
                call(name, ctx, cache, {**good, x: good[x].cpu()})
    other.close()
    with pytest.raises(ValueError, match="device"):
        ivf.KVCache(cache.records, cache.summary, cache.weight.cpu(), 16, dtype_of("bf16"))


@pytest.mark.parametrize("name,x", [("select", "q"), ("attend", "q"), ("append", "k"), ("append", "v")])
def test_rows_that_require_a_gradient_are_refused(ctx, name, x):  # noqa: F811
    import torch

    import paper_2608_08751_amd as ivf

    cache = ivf.KVCache.empty(4, 2, 64, 16, dtype_of("bf16"))
    a = arguments()
    a[x] = a[x].clone().requires_grad_()
    with pytest.raises(RuntimeError, match="gradient"):
        call(name, ctx, cache, a)
    with torch.no_grad():
        call(name, ctx, cache, a)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ["tokens", "prompt", "selected"])
def test_key_ranges_whole_and_in_parts(ctx, kind, form):  # noqa: F811
    # the same rows with a short table (or list of blocks), whole, and with one padded far beyond it, in parts
    import paper_2608_08751_amd as ivf

    heads, group, dim, bs = 2, 4, 64, 16
    lens, new = ([200], [100]) if form == "prompt" else ([900, 3, 960], [1, 1, 1])
    cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, 96)
    start, request, position = batch(lens, new)
    T, B = len(request), len(lens)
    q = queries(T, heads * group, dim, kind, 97)
    wide = np.pad(table, ((0, 0), (0, 4000 - table.shape[1])), constant_values=-1)
    short, long = None, None
    if form == "selected":
        short = np.full((T, heads, 20), -1, np.int32)
        for t, p in enumerate(position):
            kept = np.random.default_rng(t).permutation(p // bs + 1)[:18]
            short[t, :, : len(kept)] = np.sort(kept)
        long = np.pad(short, ((0, 0), (0, 0), (0, 300)), constant_values=-1)
    want, want_lse = M.attend(as_np(q), keys, values, heads, request, position, table, bs, 0.125, short)
    for t, blocks, parts in ((table, short, False), (table if form == "selected" else wide, long, True)):
        need = cache.attend_bytes(ctx, heads * group, T, B, t.shape[1], 0 if blocks is None else blocks.shape[2], max(new))
        assert (need > 0) == parts
        out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(t), 0.125, max(new),
                                     blocks=None if blocks is None else ints(blocks))
        check_attend(out, lse, want, want_lse, kind, np.nanmax(np.abs(values)), 50.0)


@pytest.mark.parametrize("new", [3, 70])  # the single-token kernel, the prompt kernel
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45])
def test_scales_of_zero(ctx, new, scale):  # noqa: F811
    # every key that a row sees weighs the same, a masked one nothing
    n, heads, bs = new + 90, 2, 16
    cache, table, keys, values = make(ctx, "bf16", [n], heads, 64, bs, 98)
    start, request, position = batch([n], [new])
    position[1] = -1
    table[0, 2] = -1
    q = queries(new, 2 * heads, 64, "bf16", 99)
    attend_held(ctx, "bf16", cache, table, keys, values, start, request, position, q, bs, scale, new)


@pytest.mark.parametrize("new", [3, 70])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scores_beyond_fp32(ctx, new, dim):  # noqa: F811
    # of magnitude 2^200: -infinity counts as masked, +infinity is no number
    import paper_2608_08751_amd as ivf

    n, bs, big = new + 20, 16, 2.0**100
    kv = np.full((n, 2, 1, dim), big)
    kv[:, 1] = np.random.default_rng(dim).standard_normal((n, 1, dim))
    kv[5, 0] = 0.0  # a key whose score is 0
    kv = dev(kv.astype(np.float32), dtype_of("bf16"))
    cache = ivf.KVCache.empty(-(-n // bs), 1, dim, bs, dtype_of("bf16"))
    ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], dev(np.arange(n, dtype=np.int64)))
    _, v = M.store(as_np(kv[:, 0]), as_np(kv[:, 1]), "bf16")
    start, request, position = batch([n], [new])
    position[1] = 4  # does not see it
    q = np.full((new, 2, dim), -big, np.float32)
    q[2, 1] = big
    out, lse = ivf.ivf_kv_attend(ctx, cache, dev(q, dtype_of("bf16")), ints(start), ints(request), ints(position),
                                 ints(np.arange(-(-n // bs))[None]), 1.0, new)
    want, want_lse = np.tile(v[5, 0], (new, 2, 1)), np.zeros((new, 2))
    want[1], want_lse[1] = 0.0, -np.inf
    want[2, 1], want_lse[2, 1] = np.nan, np.nan
    check_attend(out, lse, want, want_lse, "bf16", np.abs(v).max(), 1.0)
