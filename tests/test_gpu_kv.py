"""The paged 4-bit key/value cache on the GPU against the definitions in fp64
(tests/kv_model.py). What is stored and selected has to be equal. Attention is
held to what its roundings allow: probabilities and outputs are rounded to the
cache's type (unit u = 2^-8 for bf16, 2^-11 for f16, half of it each for
rounding to nearest), so with |v| <= vmax an output is off by at most
(u / 2) (|out| + vmax) up to fp32 terms; 1.2 u (|out| + vmax) / 2 + 1e-5 vmax is
allowed. The log-sum-exp is an fp32 sum: 2e-6 (1 + |lse|) plus the scores' own
rounding, 1e-6 of the largest |score|."""
import numpy as np
import pytest

import kv_model as M

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f16"]


@pytest.fixture(scope="module")
def ctx():
    import torch

    import paper_2608_08751_amd as ivf

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = ivf.Context(0)
    yield c
    c.close()


def dtype_of(kind):
    import torch

    return {"bf16": torch.bfloat16, "f16": torch.float16}[kind]


def as_np(t):
    return t.detach().cpu().double().numpy()


def dev(a, kind=None):
    import torch

    t = torch.as_tensor(np.ascontiguousarray(a)).cuda()
    return t if kind is None else t.to(kind)


def ints(a):
    return dev(np.asarray(a, np.int32))


def make(ctx, kind, lens, heads, dim, bs, seed, spare=3, scale_k=1.0, shuffle=True):
    """A cache that holds requests of these lengths (written by ivf_kv_append), its
    table, and keys and values as stored, fp64 [blocks, heads, bs, dim]."""
    import torch

    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(seed)
    need = [-(-n // bs) for n in lens]
    cols, blocks = max(max(need), 1) + 2, sum(need) + spare
    ids = rng.permutation(blocks) if shuffle else np.arange(blocks)
    table = np.full((len(lens), cols), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
    cache.records.fill_(255)  # unused slots read as NaN
    T = sum(lens)
    kv = rng.standard_normal((T, 2, heads, dim)) * (1 + 7 * (rng.random((1, 1, heads, dim)) < 0.05))
    kv[:, 0] *= scale_k
    kv = dev(kv.astype(np.float32), dtype_of(kind))
    slots = [int(table[b, p // bs]) * bs + p % bs for b, n in enumerate(lens) for p in range(n)]
    if T:
        ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], dev(np.array(slots, np.int64)))
    keys, values = (np.full((blocks * bs, heads, dim), np.nan) for _ in range(2))
    if T:
        k, v = as_np(kv[:, 0]), as_np(kv[:, 1])
        keys[slots], values[slots] = M.store(k, v, kind)
    split = lambda x: x.reshape(blocks, bs, heads, dim).transpose(0, 2, 1, 3)  # noqa: E731
    torch.cuda.synchronize()
    return cache, table, split(keys), split(values)


def batch(lens, new):
    """start, request, position of the last new[b] tokens of each request."""
    start = np.concatenate([[0], np.cumsum(new)])
    request = np.repeat(np.arange(len(lens)), new)
    position = np.concatenate([np.arange(n - a, n) for n, a in zip(lens, new)]) if sum(new) else np.zeros(0)
    return start.astype(np.int32), request.astype(np.int32), position.astype(np.int32)


def queries(T, Hq, dim, kind, seed, strided=True):
    rng = np.random.default_rng(seed + 1000)
    wide = dev(rng.standard_normal((max(T, 1), Hq + 3, dim)).astype(np.float32), dtype_of(kind))[:T]
    return wide[:, 2:2 + Hq] if strided else wide[:, 2:2 + Hq].contiguous()


def check_attend(out, lse, want, want_lse, kind, vmax, smax):
    u = {"bf16": 2.0**-8, "f16": 2.0**-11}[kind]
    out, lse = as_np(out), as_np(lse)
    assert (np.isnan(out) == np.isnan(want)).all() and (np.isnan(lse) == np.isnan(want_lse)).all()
    fine = ~np.isnan(want)
    err = np.abs(out - want)[fine]
    tol = (0.6 * u * (np.abs(want) + vmax) + 1e-5 * vmax)[fine]
    assert (err <= tol).all(), "off by %g (allowed %g)" % (err.max(), tol[np.argmax(err / tol)])
    inf = np.isinf(want_lse)
    assert (np.isinf(lse) == inf).all() and (lse[inf] == want_lse[inf]).all()
    ok = ~inf & ~np.isnan(want_lse)
    assert (np.abs(lse - want_lse)[ok] <= 2e-6 * (1 + np.abs(want_lse[ok])) + 1e-6 * smax).all()


def run_attend(ctx, kind, lens, new, heads, group, dim, bs, seed, count=0, scale=None, spoil=None, scale_k=1.0):
    import paper_2608_08751_amd as ivf

    cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, seed, scale_k=scale_k)
    start, request, position = batch(lens, new)
    T = len(request)
    q = queries(T, heads * group, dim, kind, seed)
    blocks = None
    if count:
        rng = np.random.default_rng(seed + 5)
        blocks = np.full((T, heads, count), -1, np.int32)
        for t in range(T):
            n = position[t] // bs + 1
            for h in range(heads):
                kept = np.sort(rng.permutation(n)[: rng.integers(0, count + 1)])
                blocks[t, h, : len(kept)] = kept
    if spoil:
        spoil(table, position, blocks)
    scale = scale or dim**-0.5
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), scale,
                                 int(max(new)), blocks=None if blocks is None else ints(blocks))
    qn = as_np(q)
    want, want_lse = M.attend(qn, keys, values, heads, request, position, table, bs, scale, blocks)
    vmax = np.nanmax(np.abs(values), initial=1.0)
    smax = abs(scale) * np.abs(qn).sum(-1).max() * np.nanmax(np.abs(keys), initial=1.0)
    check_attend(out, lse, want, want_lse, kind, vmax, smax)


# ---- tables and slots -----------------------------------------------------------

PLANS = [
    dict(B=1, cached=0, added=1, bs=64),
    dict(B=1, cached=64, added=1, bs=64),
    dict(B=1, cached=63, added=1, bs=64),
    dict(B=7, cached=100, added=40, bs=16),
    dict(B=300, cached=500, added=3, bs=128),
    dict(B=2048, cached=90, added=2, bs=32),
    dict(B=2049, cached=90, added=2, bs=32),
    dict(B=5000, cached=40, added=1, bs=16),
    dict(B=16384, cached=3, added=1, bs=16),
]


def run_plan(ctx, cached, added, bs, cols, free, tokens, seed=0):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(seed)
    B = len(cached)
    table = rng.integers(-1, 1 << 20, (B, cols)).astype(np.int32)
    got = ints(table)
    plan = ivf.ivf_kv_plan(ctx, ints(cached), ints(added), bs, got, ints(free), tokens, want_info=True)
    start, slots, request, position, info = M.plan(np.asarray(cached), np.asarray(added), bs, table, free, tokens)
    assert (got.cpu().numpy() == table).all()
    for x, y in zip(plan, (start, slots, request, position, info)):
        assert (x.cpu().numpy() == np.asarray(y)).all()


@pytest.mark.parametrize("c", PLANS, ids=lambda c: "B%d-%d+%d-bs%d" % (c["B"], c["cached"], c["added"], c["bs"]))
def test_plan(ctx, c):
    rng = np.random.default_rng(c["B"])
    cached, added = rng.integers(0, c["cached"] + 1, c["B"]), rng.integers(0, c["added"] + 1, c["B"])
    cached[0], added[0] = c["cached"], c["added"]
    cols = -(-(c["cached"] + c["added"]) // c["bs"]) + 1
    free = rng.permutation(3 * c["B"] + 50)[: 2 * c["B"] + 40]
    run_plan(ctx, cached, added, c["bs"], cols, free, int(added.sum()))


def test_plan_short_of_blocks_columns_and_room(ctx):
    cached, added = [30, 0, 17, -4, 5, 100], [50, 0, 40, 3, -2, 70]
    total = sum(max(a, 0) for a in added)
    run_plan(ctx, cached, added, 16, 4, [9, 4, 7], total)  # few free blocks, few columns
    run_plan(ctx, cached, added, 16, 12, [], total)  # none free
    run_plan(ctx, cached, added, 16, 12, list(range(30)), total + 9)  # more room than tokens
    run_plan(ctx, [0, 0], [0, 0], 16, 3, [1], 0)  # no tokens


# ---- writing and reading --------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,bs,heads", [(64, 16, 1), (96, 32, 3), (128, 64, 2), (192, 128, 1), (256, 16, 5)])
def test_append_read(ctx, kind, dim, bs, heads):
    import torch

    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(dim + bs)
    blocks = 9
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
    cache.summary.fill_(77)
    cache.weight.fill_(-3.0)
    stored_k, stored_v = (np.zeros((blocks * bs, heads, dim)) for _ in range(2))
    order = rng.permutation(blocks)
    run = [int(b) * bs + p for b in order for p in range(bs)]
    at, full = 0, set()
    for n in (1, bs - 1, bs, 2 * bs + 3, 0, 5, bs + 1):  # a call each
        slots = run[at:at + n]
        at += n
        # magnitudes from subnormal to the type's largest
        x = rng.standard_normal((n, 2, heads, dim)) * np.exp2(rng.integers(-20, 14, (n, 2, heads, 1)).astype(float))
        x[..., :32] *= 0.0 if n == 5 else 1.0
        if kind == "bf16":
            x[..., 32:64] *= 2.0**80
        wide = dev(x.astype(np.float32), dtype_of(kind))
        ivf.ivf_kv_append(ctx, cache, wide[:, 0], wide[:, 1], dev(np.array(slots, np.int64)))
        if n:
            stored_k[slots], stored_v[slots] = M.store(as_np(wide[:, 0]), as_np(wide[:, 1]), kind)
        full |= {s // bs for s in slots if s % bs == bs - 1}
    slots = run[:at]
    ids = np.arange(-1, blocks + 1)
    k, v, mean = ivf.ivf_kv_read(ctx, cache, dev(np.array(slots + [-1, blocks * bs], np.int64)), ints(ids))
    k, v, mean = as_np(k), as_np(v), as_np(mean)
    assert (k[:at] == stored_k[slots]).all() and (v[:at] == stored_v[slots]).all()
    assert np.isnan(k[at:]).all() and np.isnan(v[at:]).all()
    assert np.isnan(mean[0]).all() and np.isnan(mean[-1]).all()
    codes, weight = cache.summary.cpu().numpy(), cache.weight.cpu().numpy()
    for b in range(blocks):
        for h in range(heads):
            if b in full:
                want, w = M.summary(stored_k[b * bs:(b + 1) * bs, h])
                assert (codes[b, h] == want).all() and weight[b, h] == w
            else:
                assert (codes[b, h] == 77).all() and weight[b, h] == -3.0  # untouched
            assert (mean[1 + b, h] == (codes[b, h].astype(np.float32) * weight[b, h]).astype(np.float64)).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", KINDS)
def test_stored_values_are_the_nearest(ctx, kind):
    # every 16-bit value between the codes of one scale, ties among them
    import torch

    import paper_2608_08751_amd as ivf

    grid = np.arange(0, 7 + 1 / 64, 1 / 64)
    x = np.zeros((len(grid), 1, 64))
    x[:, 0, 0] = grid
    x[:, 0, 1] = -grid
    x[:, 0, 2] = 7.0  # sets the scale: 1
    x[:, 0, 32] = grid * 2.0**-5
    x[:, 0, 33] = 7.0 * 2.0**-5
    x[:, 0, 34:] = -grid[:, None] * 2.0**-5
    t = dev(x.astype(np.float32), dtype_of(kind))
    cache = ivf.KVCache.empty(-(-len(grid) // 16), 1, 64, 16, dtype_of(kind))
    slots = dev(np.arange(len(grid), dtype=np.int64))
    ivf.ivf_kv_append(ctx, cache, t, t.neg(), slots)
    k, v, _ = ivf.ivf_kv_read(ctx, cache, slots)
    want = M.quantise(as_np(t), kind)
    assert (as_np(k) == want).all() and (as_np(v) == -want).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", KINDS)
def test_extreme_magnitudes(ctx, kind):
    import paper_2608_08751_amd as ivf

    big = {"bf16": 3.3e38, "f16": 65504.0}[kind]
    tiny = {"bf16": 2.0**-133, "f16": 2.0**-24}[kind]
    x = np.zeros((4, 1, 64))
    x[0], x[1], x[2] = big, tiny, -big / 3
    x[3, 0, ::2] = big
    t = dev(x.astype(np.float32), dtype_of(kind))
    cache = ivf.KVCache.empty(1, 1, 64, 16, dtype_of(kind))
    slots = dev(np.arange(4, dtype=np.int64))
    ivf.ivf_kv_append(ctx, cache, t, t, slots)
    k, v, _ = ivf.ivf_kv_read(ctx, cache, slots)
    want = M.quantise(as_np(t), kind)
    assert np.isfinite(want).all() and (as_np(k) == want).all() and (as_np(v) == want).all()


@pytest.mark.parametrize("kind", KINDS)
def test_slots_outside_the_cache_are_skipped(ctx, kind):
    import torch

    import paper_2608_08751_amd as ivf

    cache = ivf.KVCache.empty(2, 2, 64, 16, dtype_of(kind))
    before = [t.clone() for t in (cache.records, cache.summary, cache.weight)]
    x = torch.ones(3, 2, 64, device="cuda", dtype=dtype_of(kind))
    ivf.ivf_kv_append(ctx, cache, x, x, dev(np.array([-1, 2 * 16, 1 << 40], np.int64)))
    assert all((a == b).all() for a, b in zip(before, (cache.records, cache.summary, cache.weight)))


# ---- selection ------------------------------------------------------------------

SELECTS = [
    # lens, new, heads, group, dim, bs, first, last, count
    ([1], [1], 1, 1, 64, 16, 1, 1, 2),
    ([16], [1], 1, 2, 64, 16, 0, 1, 1),
    ([400, 17, 33], [1, 1, 1], 2, 4, 128, 16, 1, 2, 8),
    ([700, 5], [9, 5], 3, 2, 96, 16, 1, 1, 12),
    ([1300], [70], 2, 7, 128, 32, 2, 1, 9),
    ([2100, 40, 900], [33, 1, 20], 1, 20, 256, 16, 0, 2, 30),
    ([900, 64], [1, 1], 5, 3, 192, 64, 1, 1, 4),
    ([3000], [1], 1, 4, 64, 16, 3, 4, 64),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("i", range(len(SELECTS)))
def test_select(ctx, kind, i):
    import paper_2608_08751_amd as ivf

    lens, new, heads, group, dim, bs, first, last, count = SELECTS[i]
    cache, table, keys, _ = make(ctx, kind, lens, heads, dim, bs, 40 + i)
    start, request, position = batch(lens, new)
    q = queries(len(request), heads * group, dim, kind, i)
    got = ivf.ivf_kv_select(ctx, cache, q, ints(request), ints(position), ints(table), count, first=first, last=last)
    want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), heads, request, position, table,
                    bs, first, last, count)
    assert (got.cpu().numpy() == want).all()


@pytest.mark.parametrize("tokens", [1, 40])
def test_select_ties_holes_and_rows_without_blocks(ctx, tokens):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(3)
    heads, group, dim, bs, cols, B = 2, 2, 64, 16, 70, 2
    cache = ivf.KVCache.empty(90, heads, dim, bs, dtype_of("bf16"))
    # few different summaries, so that most scores tie; some weights 0
    cache.summary.copy_(dev(rng.integers(-2, 3, (90, heads, 1)).astype(np.int8)).expand(90, heads, dim))
    cache.weight.copy_(dev((rng.integers(0, 3, (90, heads)) / 2.0).astype(np.float32)))
    table = rng.integers(0, 90, (B, cols)).astype(np.int32)
    table[0, 5:9], table[1, 0], table[1, 50], table[0, cols - 1] = -1, -7, 90, 1 << 30
    T = B * tokens
    request = np.repeat(np.arange(B), tokens)
    position = rng.integers(0, cols * bs, T)
    position[-1], position[0] = -1, cols * bs + 500  # sees nothing; beyond the table
    request[1 % T] = 5 if tokens > 1 else request[1 % T]
    q = queries(T, heads * group, dim, "bf16", 9)
    q[T // 2] = 0
    for first, last, count in ((1, 1, 3), (0, 3, 20), (30, 30, 64)):
        got = ivf.ivf_kv_select(ctx, cache, q, ints(request), ints(position), ints(table), count, first=first, last=last)
        want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), heads, request, position,
                        table, bs, first, last, count)
        assert (got.cpu().numpy() == want).all()


def test_select_queries_that_are_not_finite(ctx):
    import paper_2608_08751_amd as ivf

    cache, table, _, _ = make(ctx, "bf16", [500], 1, 64, 16, 8)
    q = queries(3, 4, 64, "bf16", 2)
    q[0, 1, 3], q[1, 0, 0], q[1, 1, 0], q[2] = float("nan"), float("inf"), -float("inf"), float("nan")
    pos = np.array([499, 400, 499])
    got = ivf.ivf_kv_select(ctx, cache, q, ints([0, 0, 0]), ints(pos), ints(table), 9)
    want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), 1, [0, 0, 0], pos, table, 16, 1,
                    1, 9)
    assert (got.cpu().numpy() == want).all()


def test_select_long_tables(ctx):
    # more columns than the tiles hold, and more than 64 KB of keys
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(5)
    for cols, T in ((2500, 6), (20000, 2), (32768, 1)):
        cache = ivf.KVCache.empty(cols + 1, 1, 64, 16, dtype_of("f16"))
        cache.summary.copy_(dev(rng.integers(-127, 128, (cols + 1, 1, 64)).astype(np.int8)))
        cache.weight.copy_(dev(rng.random((cols + 1, 1)).astype(np.float32)))
        table = rng.permutation(cols + 1)[None, :cols].astype(np.int32)
        pos = np.arange(T) + cols * 16 - T
        q = queries(T, 3, 64, "f16", cols)
        got = ivf.ivf_kv_select(ctx, cache, q, ints([0] * T), ints(pos), ints(table), 100)
        want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), 1, [0] * T, pos, table, 16,
                        1, 1, 100)
        assert (got.cpu().numpy() == want).all()


# ---- attention ------------------------------------------------------------------

ATTENDS = [
    # lens, new, heads, group, dim, bs
    ([1], [1], 1, 1, 64, 16),
    ([15, 16, 17], [1, 1, 1], 1, 2, 64, 16),
    ([31, 32, 33, 64, 65], [1, 1, 1, 1, 1], 2, 4, 128, 32),
    ([700, 1, 250], [1, 1, 1], 2, 8, 128, 64),
    ([333], [1], 1, 20, 96, 16),
    ([129, 128, 127], [1, 1, 1], 3, 5, 192, 128),
    ([1000], [1], 2, 1, 256, 16),
    ([40], [40], 2, 4, 128, 16),
    ([300, 20, 77], [45, 1, 3], 2, 3, 64, 32),
    ([200, 90], [200, 0], 1, 7, 96, 64),
    ([513], [130], 1, 4, 256, 64),
    ([260, 19], [70, 19], 1, 2, 192, 16),
    ([2500, 2400], [2, 1], 1, 4, 128, 64),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("i", range(len(ATTENDS)))
def test_attend(ctx, kind, i):
    run_attend(ctx, kind, *ATTENDS[i], seed=i)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("i,count", [(0, 1), (2, 2), (3, 7), (4, 21), (5, 2), (6, 40), (7, 3), (8, 5), (9, 2), (10, 6),
                                     (11, 9), (12, 30)])
def test_attend_selected(ctx, kind, i, count):
    run_attend(ctx, kind, *ATTENDS[i], seed=100 + i, count=count)


@pytest.mark.parametrize("count", [0, 12])
def test_rows_that_see_nothing_and_tables_with_holes(ctx, count):
    def spoil(table, position, blocks):
        table[0, 1], table[0, 4], table[1, :], table[2, 0] = -1, 1 << 30, -5, -1
        position[3], position[-1] = -1, -100
        if blocks is not None:
            blocks[0, 0, :] = -1
            blocks[1, 0, :3] = [900, 1 << 30, -3]
            blocks[2, 0, :4] = [7, 2, 2, 0]  # any order, twice

    run_attend(ctx, "bf16", [300, 40, 100, 64], [6, 4, 5, 7], 2, 3, 64, 16, seed=7, count=count, spoil=spoil)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale,scale_k", [(3.0, 8.0), (-0.7, 1.0), (1e-6, 1.0), (0.088, 1000.0)])
def test_scales_and_sharp_softmax(ctx, kind, scale, scale_k):
    run_attend(ctx, kind, [400, 33], [3, 1], 2, 4, 128, 32, seed=21, scale=scale, scale_k=scale_k)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("count", [0, 25])
def test_tokens_that_are_not_finite_reach_only_rows_that_see_them(ctx, kind, count):
    import torch

    import paper_2608_08751_amd as ivf

    heads, group, dim, bs, n, new = 2, 2, 128, 16, 390, 70
    cache, table, keys, values = make(ctx, kind, [n], heads, dim, bs, 31)
    # token 350: a NaN in the value of head 0; token 370: an infinity in the key of head 1
    for p, h, part in ((350, 0, 1), (370, 1, 0)):
        kv = torch.ones(2, 1, heads, dim, device="cuda", dtype=dtype_of(kind))
        kv[part, 0, h, 40] = float("nan") if part else -float("inf")
        slot = int(table[0, p // bs]) * bs + p % bs
        ivf.ivf_kv_append(ctx, cache, kv[0], kv[1], dev(np.array([slot], np.int64)))
        k, v = M.store(as_np(kv[0]), as_np(kv[1]), kind)
        keys[table[0, p // bs], :, p % bs], values[table[0, p // bs], :, p % bs] = k[0], v[0]
        rk, rv, _ = ivf.ivf_kv_read(ctx, cache, dev(np.array([slot], np.int64)))
        assert (np.isnan(as_np(rk)) == np.isnan(k)).all() and (np.isnan(as_np(rv)) == np.isnan(v)).all()
    start, request, position = batch([n], [new])
    q = queries(new, heads * group, dim, kind, 3)
    blocks = None
    if count:
        blocks = np.sort(np.stack([np.random.default_rng(t).permutation(25)[:count] for t in range(new * heads)]))
        blocks = blocks.reshape(new, heads, count).astype(np.int32)
        blocks[::3, :, 21:] = -1
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), 0.1, new,
                                 blocks=None if blocks is None else ints(blocks))
    want, want_lse = M.attend(as_np(q), keys, values, heads, request, position, table, bs, 0.1, blocks)
    assert np.isnan(want).any() and not np.isnan(want).all()
    check_attend(out, lse, want, want_lse, kind, np.nanmax(np.abs(values)), 100.0)


def test_split_parts_and_one_part_agree(ctx):
    # the same rows with a long and a short table: the key range is split in one call only
    import paper_2608_08751_amd as ivf

    lens = [900, 3, 2000]
    cache, table, keys, values = make(ctx, "f16", lens, 2, 64, 16, 50)
    start, request, position = batch(lens, [1, 1, 1])
    q = queries(3, 8, 64, "f16", 1)
    wide = np.full((3, 4000), -1, np.int32)
    wide[:, : table.shape[1]] = table
    want, want_lse = M.attend(as_np(q), keys, values, 2, request, position, table, 16, 0.125)
    for t in (table, wide):
        out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(t), 0.125, 1)
        check_attend(out, lse, want, want_lse, "f16", np.nanmax(np.abs(values)), 50.0)


def test_record_offsets_beyond_32_bits(ctx):
    # 33,000 blocks of 128 tokens x 4 heads x 256 channels: 4.5 GB of records
    import torch

    import paper_2608_08751_amd as ivf

    blocks, heads, dim, bs = 33000, 4, 256, 128
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of("bf16"))
    assert cache.records.numel() > 1 << 32
    rng = np.random.default_rng(1)
    ids = np.array([blocks - 1, 0, blocks - 7], np.int32)
    table = np.concatenate([ids, [-1]]).astype(np.int32)[None]
    n = 3 * bs - 5
    kv = dev(rng.standard_normal((2, n, heads, dim)).astype(np.float32), dtype_of("bf16"))
    slots = np.array([int(table[0, p // bs]) * bs + p % bs for p in range(n)], np.int64)
    ivf.ivf_kv_append(ctx, cache, kv[0], kv[1], dev(slots))
    k, v, mean = ivf.ivf_kv_read(ctx, cache, dev(slots), ints([blocks - 1]))
    wk, wv = M.store(as_np(kv[0]), as_np(kv[1]), "bf16")
    assert (as_np(k) == wk).all() and (as_np(v) == wv).all()
    code, w = M.summary(wk[:bs, 3])
    assert (as_np(mean)[0, 3] == (code.astype(np.float32) * w)).all()
    keys, values = {}, {}
    big = np.zeros((3, heads, bs, dim)), np.zeros((3, heads, bs, dim))
    for x, src in zip(big, (wk, wv)):
        for p in range(n):
            x[p // bs, :, p % bs] = src[p]
    q = queries(1, 8, dim, "bf16", 4)
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints([0, 1]), ints([0]), ints([n - 1]), ints(table), 0.0625, 1)
    want, want_lse = M.attend(as_np(q), *big, heads, [0], [n - 1], np.arange(4, dtype=np.int32)[None], bs, 0.0625)
    check_attend(out, lse, want, want_lse, "bf16", np.abs(wv).max(), 30.0)
    del cache
    torch.cuda.empty_cache()


def test_other_stream_and_graph_replay(ctx):
    # a decoding step captured once and replayed on other inputs in the same buffers
    import torch

    import paper_2608_08751_amd as ivf

    lens = [70, 33]
    cache, table, keys, values = make(ctx, "bf16", lens, 2, 128, 16, 60)
    start, request, position = batch(lens, [1, 1])
    args = [ints(start), ints(request), ints(position), ints(table)]
    q = queries(2, 8, 128, "bf16", 1, strided=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        blocks = ivf.ivf_kv_select(ctx, cache, q, *args[1:], 3)
        ivf.ivf_kv_attend(ctx, cache, q, *args, 0.1, 1, blocks=blocks)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            blocks = ivf.ivf_kv_select(ctx, cache, q, *args[1:], 3)
            out, lse = ivf.ivf_kv_attend(ctx, cache, q, *args, 0.1, 1, blocks=blocks)
    for i in range(3):
        fresh = queries(2, 8, 128, "bf16", 10 + i, strided=False)
        q.copy_(fresh)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want_b = M.select(as_np(fresh), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), 2, request, position,
                          table, 16, 1, 1, 3)
        assert (blocks.cpu().numpy() == want_b).all()
        want, want_lse = M.attend(as_np(fresh), keys, values, 2, request, position, table, 16, 0.1, want_b)
        check_attend(out, lse, want, want_lse, "bf16", np.nanmax(np.abs(values)), 30.0)


# ---- precision and the forms that larger batches take ------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,new", [(64, 1), (128, 1), (256, 1), (128, 70)])
def test_scores_of_channels_far_apart(ctx, kind, dim, new):
    # One key a row, so that the log-sum-exp is its score. In each group of 32 one channel of the
    # query is large, the others 2^-7 ... 2^-13 of it. A score may be off by a query rounding of 2^-19 of the largest
    # channel of a group for each of the group's channels, and by fp32 sums: 2^-20 of sum |q k|.
    import paper_2608_08751_amd as ivf

    B, rng = 64 if new == 1 else 1, np.random.default_rng(dim)
    cache, table, keys, _ = make(ctx, kind, [1] * B, 2, dim, 16, 70)
    start, request = np.arange(B + 1) * new, np.repeat(np.arange(B), new)
    T = B * new
    x = rng.standard_normal((T, 6, dim)) * np.exp2(-rng.integers(7, 14, (T, 6, dim)).astype(float))
    x[..., rng.integers(0, 32, dim // 32) + np.arange(0, dim, 32)] = rng.standard_normal((T, 6, dim // 32)) + 2
    q = dev(x.astype(np.float32), dtype_of(kind))
    _, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(np.zeros(T)), ints(table), 1.0, new)
    qn = as_np(q).reshape(T, 2, 3, dim)
    k = np.stack([keys[table[b, 0], :, 0] for b in request])[:, :, None]
    want = (qn * k).sum(-1)
    grouped = lambda a: np.abs(a).reshape(*a.shape[:-1], -1, 32)  # noqa: E731
    allowed = (2.0**-19 * (grouped(qn).max(-1) * grouped(k).sum(-1)).sum(-1) + 2.0**-20 * np.abs(qn * k).sum(-1)
               + 2.0**-21 * (1 + np.abs(want)))
    assert (np.abs(as_np(lse).reshape(T, 2, 3) - want) <= allowed).all()


@pytest.mark.parametrize("count", [0, 4])
@pytest.mark.parametrize("new", [2, 70])
def test_attend_queries_that_are_not_finite(ctx, count, new):
    # their rows are NaN where they see a key, empty where they see none; no other row changes
    import paper_2608_08751_amd as ivf

    cache, table, keys, values = make(ctx, "bf16", [100], 2, 64, 16, 71)
    start, request, position = batch([100], [new])
    position[1] = -1
    q = queries(new, 4, 64, "bf16", 5)
    q[0, 1, 3], q[0, 2, 40], q[1, :, 0] = float("nan"), float("inf"), float("nan")
    blocks = np.tile(np.arange(count, dtype=np.int32), (new, 2, 1)) if count else None
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), 0.125, new,
                                 blocks=None if blocks is None else ints(blocks))
    clean = as_np(q)
    bad = ~np.isfinite(clean).all(-1)
    want, want_lse = M.attend(np.where(bad[..., None], 0.0, clean), keys, values, 2, request, position, table, 16, 0.125,
                              blocks)
    bad[position < 0] = False
    want[bad], want_lse[bad] = np.nan, np.nan
    check_attend(out, lse, want, want_lse, "bf16", np.nanmax(np.abs(values)), 30.0)


# tokens with blocks of their own: four waves a unit, one wave a unit, rows beyond 8, wide channels
@pytest.mark.parametrize("kind,heads,group,dim,bs,new,count", [
    ("bf16", 8, 2, 64, 16, 100, 4), ("f16", 8, 12, 128, 32, 90, 3), ("bf16", 8, 2, 128, 16, 400, 5),
    ("f16", 8, 12, 64, 16, 390, 4), ("bf16", 8, 1, 96, 64, 400, 2), ("f16", 8, 3, 192, 16, 130, 3),
    ("bf16", 8, 9, 256, 16, 130, 3)])
def test_many_tokens_with_selected_blocks(ctx, kind, heads, group, dim, bs, new, count):
    run_attend(ctx, kind, [new + 300, 40], [new, 3], heads, group, dim, bs, seed=80, count=count)


# many requests: a unit for every wave, more units than are shared out, each beside a long table
@pytest.mark.parametrize("kind,B,heads,group,dim,longest", [
    ("bf16", 150, 2, 4, 128, 60), ("f16", 1040, 1, 1, 64, 1100), ("bf16", 520, 8, 2, 64, 1100),
    ("f16", 140, 2, 11, 96, 1300), ("bf16", 130, 3, 2, 256, 1200)])
def test_many_requests(ctx, kind, B, heads, group, dim, longest):
    lens = np.random.default_rng(B).integers(1, 40, B)
    lens[B // 2] = longest
    run_attend(ctx, kind, lens.tolist(), [1] * B, heads, group, dim, 16, seed=81)


@pytest.mark.parametrize("kind,lens,new,heads,group,dim,bs", [
    ("bf16", [5000], [100], 1, 2, 128, 64),  # few rows, long: the keys are split
    ("f16", [260, 9, 300, 1, 1, 400], [200, 1, 3, 1, 1, 90], 2, 4, 64, 16),  # small requests between prompts
    ("bf16", [150, 3, 200], [150, 3, 200], 2, 3, 192, 32),
    ("f16", [140, 2, 1, 180], [140, 2, 1, 180], 1, 5, 256, 16),
])
def test_prompts_beside_small_requests(ctx, kind, lens, new, heads, group, dim, bs):
    run_attend(ctx, kind, lens, new, heads, group, dim, bs, seed=82)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_append_read_of_many_tokens(ctx, kind, dim):
    # scattered slots, some outside the cache
    import paper_2608_08751_amd as ivf

    T, heads, bs, blocks = 2500, 2, 32, 90
    rng = np.random.default_rng(dim)
    slots = rng.permutation(blocks * bs)[:T]
    slots[::97] = -1
    x = rng.standard_normal((T, 2, heads, dim)) * np.exp2(rng.integers(-6, 7, (T, 2, heads, 1)).astype(float))
    kv = dev(x.astype(np.float32), dtype_of(kind))
    kv[7, 0, 0, 5], kv[9, 1, 1, dim - 1] = float("nan"), float("inf")
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
    ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], dev(slots.astype(np.int64)))
    k, v, _ = ivf.ivf_kv_read(ctx, cache, dev(slots.astype(np.int64)))
    wk, wv = M.store(as_np(kv[:, 0]), as_np(kv[:, 1]), kind)
    wk[slots < 0], wv[slots < 0] = np.nan, np.nan
    assert np.array_equal(as_np(k), wk, equal_nan=True) and np.array_equal(as_np(v), wv, equal_nan=True)


@pytest.mark.parametrize("dtype", KINDS)
def test_example_runs_and_agrees_with_fp64(ctx, dtype):
    # relative to the largest output: (u / 2) (1 + vmax / outmax), with vmax / outmax below 12 here
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(__file__), "..", "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    _, _, error, in_use = module.run(requests=5, prompt=200, steps=20, heads=2, group=3, dim=64, block_size=16, count=6,
                                     dtype=dtype_of(dtype))
    assert error <= 13 * {"bf16": 2.0**-9, "f16": 2.0**-12}[dtype]
    lengths = [int(100 + 25 * i) for i in range(5)]
    assert in_use == sum(-(-(n + 21) // 16) for n in lengths)


# many tokens a request: tiles of 16 tokens, some of which span requests
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,new,heads,group,dim,bs,first,last,count", [
    ([900], [400], 2, 7, 128, 32, 2, 1, 9),
    ([500, 40, 300], [200, 37, 150], 2, 2, 96, 16, 1, 1, 12),
    ([420, 33], [390, 3], 2, 1, 256, 16, 0, 2, 7),
    ([2600], [110], 7, 4, 64, 16, 1, 2, 20),
    ([1400], [160], 5, 3, 192, 16, 1, 1, 64),
])
def test_select_many_tokens(ctx, kind, lens, new, heads, group, dim, bs, first, last, count):
    import paper_2608_08751_amd as ivf

    cache, table, _, _ = make(ctx, kind, lens, heads, dim, bs, 90 + dim)
    _, request, position = batch(lens, new)
    position[5], request[7] = -1, len(lens)  # a token that sees nothing, one of no request
    q = queries(len(request), heads * group, dim, kind, 6)
    q[11], q[12, 0, 3] = 0, float("nan")
    got = ivf.ivf_kv_select(ctx, cache, q, ints(request), ints(position), ints(table), count, first=first, last=last)
    want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), heads, request, position, table,
                    bs, first, last, count)
    assert (got.cpu().numpy() == want).all()


def test_select_ties_and_holes_of_many_tokens(ctx):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(13)
    heads, group, dim, bs, cols, B, tokens = 2, 2, 64, 16, 70, 2, 200
    cache = ivf.KVCache.empty(90, heads, dim, bs, dtype_of("f16"))
    cache.summary.copy_(dev(rng.integers(-2, 3, (90, heads, 1)).astype(np.int8)).expand(90, heads, dim))
    cache.weight.copy_(dev((rng.integers(0, 3, (90, heads)) / 2.0).astype(np.float32)))
    table = rng.integers(0, 90, (B, cols)).astype(np.int32)
    table[0, 5:9], table[1, 0], table[1, 50], table[0, cols - 1] = -1, -7, 90, 1 << 30
    request = np.repeat(np.arange(B), tokens)
    position = rng.integers(0, cols * bs, B * tokens)
    position[0] = cols * bs + 500  # beyond the table
    q = queries(B * tokens, heads * group, dim, "f16", 14)
    for first, last, count in ((1, 1, 3), (0, 3, 20), (30, 30, 64)):
        got = ivf.ivf_kv_select(ctx, cache, q, ints(request), ints(position), ints(table), count, first=first, last=last)
        want = M.select(as_np(q), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), heads, request, position,
                        table, bs, first, last, count)
        assert (got.cpu().numpy() == want).all()


# every number of waves a unit, below and above the limits, tables shared out and whole, for every width
@pytest.mark.parametrize("kind,B,heads,longest", [("bf16", 40, 1, 900), ("f16", 34, 1, 2000), ("bf16", 6, 2, 1900),
                                                  ("f16", 17, 8, 3900), ("bf16", 130, 2, 4400)])
@pytest.mark.parametrize("dim,group", [(64, 4), (96, 12), (128, 8), (192, 1), (256, 3)])
def test_requests_beside_long_tables(ctx, kind, B, heads, longest, dim, group):
    lens = np.random.default_rng(B).integers(1, 70, B)
    lens[B // 3] = longest
    run_attend(ctx, kind, lens.tolist(), [1] * B, heads, group, dim, 32, seed=83)


@pytest.mark.parametrize("kind,T,heads,dim,bs", [("bf16", 300, 2, 64, 128), ("f16", 1000, 1, 96, 16),
                                                 ("bf16", 2500, 2, 128, 64), ("f16", 5000, 1, 256, 32),
                                                 ("bf16", 900, 3, 192, 16)])
def test_summaries_of_scattered_tokens(ctx, kind, T, heads, dim, bs):
    # half of every block by an earlier call, the rest, in any order, by this one; some tokens are not finite
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(T)
    blocks = T // (bs // 2)
    order = rng.permutation(blocks * bs)
    first = order[order % bs < bs // 2]  # the slots before the middle, and then the others
    second = order[order % bs >= bs // 2]
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
    cache.summary.fill_(77)
    stored = np.zeros((blocks * bs, heads, dim))
    for slots in (first, second):
        x = rng.standard_normal((len(slots), 2, heads, dim)) * np.exp2(rng.integers(-6, 7, (len(slots), 2, heads, 1)))
        kv = dev(x.astype(np.float32), dtype_of(kind))
        kv[3, 0, 0, 5], kv[11, 1, 0, dim - 1] = float("nan"), float("inf")
        assert (cache.summary == 77).all()  # nothing full yet
        ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], dev(slots.astype(np.int64)))
        stored[slots], _ = M.store(as_np(kv[:, 0]), as_np(kv[:, 1]), kind)
    codes, weight = cache.summary.cpu().numpy(), cache.weight.cpu().numpy()
    for b in range(blocks):
        for h in range(heads):
            want, w = M.summary(stored[b * bs:(b + 1) * bs, h])
            assert (codes[b, h] == want).all() and weight[b, h] == w


@pytest.mark.parametrize("new", [3, 200])  # one by one; in tiles
@pytest.mark.parametrize("junk", [float("nan"), -float("inf"), float("inf"), -2.0])
def test_select_weights_never_written(ctx, new, junk):
    # a token's own block is among the selected whatever its weight holds before its last slot is written
    import paper_2608_08751_amd as ivf

    heads, n, bs = 4, 1003, 16
    cache, table, _, _ = make(ctx, "bf16", [n], heads, 64, bs, 21)
    open_block = int(table[0, (n - 1) // bs])
    cache.weight[open_block] = junk
    cache.weight[int(table[0, 20])] = junk  # and one that is ranked
    cache.summary[open_block] = -77
    weights = cache.weight.cpu().numpy().copy()
    weights[~(np.isfinite(weights) & (weights >= 0))] = 0
    _, request, position = batch([n], [new])
    q = queries(new, 2 * heads, 64, "bf16", 4)
    got = ivf.ivf_kv_select(ctx, cache, q, ints(request), ints(position), ints(table), 7).cpu().numpy()
    want = M.select(as_np(q), cache.summary.cpu().numpy(), weights, heads, request, position, table, bs, 1, 1, 7)
    assert (got == want).all()
    assert (got.max(-1) == position[:, None] // bs).all()


@pytest.mark.parametrize("new", [2, 70])
def test_positions_up_to_the_last_of_a_table(ctx, new):
    # a table of 2^31 - 16 keys that names its first block and its last ones: the rows of the last tokens equal
    # those of a short request with the same blocks
    import torch

    import paper_2608_08751_amd as ivf

    heads, group, dim, bs, far = 1, 2, 64, 16, 6
    n = (1 + far) * bs
    cache, table, keys, values = make(ctx, "bf16", [n], heads, dim, bs, 33)
    cols = (1 << 27) - 1
    wide = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    wide[0, 0] = int(table[0, 0])
    wide[0, cols - far:] = ints(table[0, 1:1 + far])
    start, request, position = batch([n], [new])
    q = queries(new, heads * group, dim, "bf16", 5)
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position + (cols - far - 1) * bs), wide,
                                 0.125, new)
    want, want_lse = M.attend(as_np(q), keys, values, heads, request, position, table, bs, 0.125)
    vmax = np.nanmax(np.abs(values))
    smax = 0.125 * np.abs(as_np(q)).sum(-1).max() * np.nanmax(np.abs(keys))
    check_attend(out, lse, want, want_lse, "bf16", vmax, smax)


@pytest.mark.parametrize("group,new", [(4, 3), (2, 50), (16, 4)])
def test_requests_of_more_tokens_than_longest_says(ctx, group, new):
    # nothing is written past the workspace or the outputs, and requests that keep to `longest` are right
    import ctypes

    import torch

    import paper_2608_08751_amd as ivf
    from paper_2608_08751_amd import _binding as B

    heads, dim, bs, lens = 2, 64, 16, [5000, 700, 4800]
    cache, table, keys, values = make(ctx, "bf16", lens, heads, dim, bs, 61)
    start, request, position = batch(lens, [1, new, 1])
    T, Hq = len(request), heads * group
    q = queries(T, Hq, dim, "bf16", 3)
    own = ivf.Context(0)
    need = own.lib.ivf_kv_attend_bytes(cache.ref, Hq, T, 3, table.shape[1], 0, 1)
    assert need > 0  # the key ranges are shared out
    ws = torch.full((need + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
    out = torch.zeros(T + 64, Hq, dim, dtype=q.dtype, device="cuda")
    lse = torch.zeros(T + 64, Hq, device="cuda")
    args = [ints(start), ints(request), ints(position), ints(table)]
    lib, handle = own.bind()
    assert lib.ivf_set_workspace(handle, B._ptr(ws), need) == B.IVF_OK
    st = lib.ivf_kv_attend(handle, cache.ref, B._ptr(q), q.stride(0), q.stride(1), Hq, T, *map(B._ptr, args), 3,
                           table.shape[1], None, 0, ctypes.c_float(0.125), 1, B._ptr(out), B._ptr(lse))
    assert st == B.IVF_OK
    torch.cuda.synchronize()
    own.close()
    assert (ws[need:] == 0x5A).all() and not out[T:].any() and not lse[T:].any()
    want, want_lse = M.attend(as_np(q), keys, values, heads, request, position, table, bs, 0.125)
    kept = [0, T - 1]
    check_attend(out[kept], lse[kept], want[kept], want_lse[kept], "bf16", np.nanmax(np.abs(values)),
                 0.125 * np.abs(as_np(q)).sum(-1).max() * np.nanmax(np.abs(keys)))


def test_select_more_tokens_than_a_launch_holds(ctx):
    # 2^32 threads are 4,194,304 workgroups: tokens on both sides of where the second launch begins
    import torch

    import paper_2608_08751_amd as ivf

    n, bs, T = 300, 16, 4_200_000
    cache, table, _, _ = make(ctx, "bf16", [n], 1, 64, bs, 12)
    # a table of more columns than the tiles hold: a workgroup a token
    wide = np.full((1, 2100), -1, np.int32)
    wide[0, : table.shape[1]] = table[0]
    few = queries(997, 1, 64, "bf16", 8, strided=False)
    q = few.repeat(T // 997 + 1, 1, 1)[:T]
    position = ints(np.arange(T) * 7 % n)
    request = torch.zeros(T, dtype=torch.int32, device="cuda")
    got = ivf.ivf_kv_select(ctx, cache, q, request, position, ints(wide), 4)
    period = 997 * n  # tokens after which queries and positions are the same again
    want = ivf.ivf_kv_select(ctx, cache, q[:period], request[:period], position[:period], ints(wide), 4)
    assert (got == want.repeat(T // period + 1, 1, 1)[:T]).all()
    some = np.arange(0, period, 4001)
    ref = M.select(as_np(q[some]), cache.summary.cpu().numpy(), cache.weight.cpu().numpy(), 1, [0] * len(some),
                   position.cpu().numpy()[some], wide, bs, 1, 1, 4)
    assert (want.cpu().numpy()[some] == ref).all()
