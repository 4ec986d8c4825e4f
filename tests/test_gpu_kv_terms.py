"""Attention over the paged 4-bit cache with terms in its scores (cap, bias by distance, first, prefix) on the GPU,
against the definition of include/ivf.h in fp64. Tolerances: those of tests/test_gpu_kv.py for the scores without
terms (outputs 0.6 u (|out| + vmax) + 1e-5 vmax, log-sum-exps 2e-6 (1 + |lse|) + 1e-6 of the largest sum of |q k| before the cap, whose slope is at most 1), and
for the terms, with x the largest |bias| a row may see, in units of 2^-24: the slope's conversion to the base 2,
the distance (above 2^24), the fused product and sum each round once, so a score is off by 4 x 2^-24 = 2^-22 x, a
probability and its sum by that much relatively, an output by 2^-21 x vmax; the cap's tanh is off by 3 ulp of 1
and its conversion and product by half of one each: 4 2^-23 cap < 5e-7 cap a score, 1e-6 cap vmax an output."""
import math

import numpy as np
import pytest

import kv_model as M
from test_gpu_kv import as_np, batch, dev, dtype_of, ints, make, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch

    import paper_2608_08751_amd as ivf

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = ivf.Context(0)
    yield c
    c.close()


def model(q, keys, values, heads, request, position, table, bs, scale, blocks=None, cap=0.0, slopes=None, first=None,
          prefix=None):
    """fp64 (out, lse, largest |bias| of a row): the definition, row by row."""
    T, Hq, dim = q.shape
    group, cols = Hq // heads, table.shape[1]
    out, lse, far = np.zeros((T, Hq, dim)), np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for t in range(T):
        b, p = int(request[t]), int(position[t])
        if b < 0 or b >= table.shape[0] or p < 0:
            continue
        lo, end = (0 if first is None else int(first[t])), (0 if prefix is None else int(prefix[t]))
        for h in range(heads):
            k, v, at = [], [], []
            for j in range(cols) if blocks is None else [int(x) for x in blocks[t, h]]:
                if j < 0 or j >= cols or not 0 <= table[b, j] < keys.shape[0]:
                    continue
                pos = np.arange(j * bs, (j + 1) * bs)
                seen = ((pos >= lo) & (pos <= p)) | (pos < end)
                x = int(table[b, j])
                k.append(keys[x, h][seen])
                v.append(values[x, h][seen])
                at.append(pos[seen])
            if not at or not sum(map(len, at)):
                continue
            k, v, at = np.concatenate(k), np.concatenate(v), np.concatenate(at)
            nan = np.isnan(k).any() or np.isnan(v).any()
            for g in range(h * group, (h + 1) * group):
                if nan:
                    out[t, g] = lse[t, g] = np.nan
                    continue
                s = scale * (k @ q[t, g])
                if cap:
                    s = cap * np.tanh(s / cap)
                if slopes is not None:
                    bias = float(slopes[g]) * np.abs(p - at)
                    far[t, g] = np.abs(bias).max()
                    s = s - bias
                m = s.max()
                e = np.exp(s - m)
                lse[t, g] = m + math.log(e.sum())
                out[t, g] = (e / e.sum()) @ v
    return out, lse, far


def largest_score(q, keys, scale):
    return abs(scale) * np.abs(q).sum(-1).max() * np.nanmax(np.abs(keys), initial=1.0)


def check(out, lse, want, kind, vmax, smax, cap):
    want, want_lse, far = want
    u = {"bf16": 2.0**-8, "f16": 2.0**-11}[kind]
    out, lse = as_np(out), as_np(lse)
    assert (np.isnan(out) == np.isnan(want)).all() and (np.isnan(lse) == np.isnan(want_lse)).all()
    fine = ~np.isnan(want)
    tol = 0.6 * u * (np.abs(want) + vmax) + (1e-5 + 2.0**-21 * far[..., None] + 1e-6 * cap) * vmax
    err = np.abs(out - want)
    assert (err[fine] <= tol[fine]).all(), "off by %g" % np.nanmax(err / tol)
    inf = np.isinf(want_lse)
    assert (np.isinf(lse) == inf).all() and (lse[inf] == want_lse[inf]).all()
    ok = ~inf & ~np.isnan(want_lse)
    off = np.abs(lse[ok] - want_lse[ok]) / (2e-6 * (1 + np.abs(want_lse[ok])) + 1e-6 * smax + 2.0**-22 * far[ok] + 5e-7 * cap)
    assert (off <= 1).all(), "lse off by %g of what is allowed" % off.max()


def sights(mask, lens, new, request, position, rng):
    """(first, prefix) of every token."""
    T, p = len(position), position.astype(np.int64)
    total, chunk = np.asarray(lens)[request], np.asarray(new)[request]
    start = total - chunk
    none = np.zeros(T, np.int64)
    if mask == "window":
        w = np.array([1, 5, 37, 300])[rng.integers(0, 4, T)]
        return p - w + 1, np.minimum(rng.integers(0, 6, T), p + 1)
    if mask == "one window":
        return p - 99, np.minimum(4, p + 1)
    if mask == "documents":
        return start + (p - start) // 41 * 41, np.minimum(start, 33)
    if mask == "prefix":
        return none, start + 2 * chunk // 3
    if mask == "prefix only":
        return p + 1, np.minimum(total, 20)
    if mask == "mixed":  # every row something else: nothing, its own key, the whole request, values outside
        first = np.where(rng.random(T) < 0.3, p + 1 + rng.integers(0, 50, T), rng.integers(-9, p + 1))
        prefix = np.where(rng.random(T) < 0.5, rng.integers(-9, 1, T), rng.integers(0, total + 1))
        return first, prefix
    raise ValueError(mask)


def run(ctx, kind, lens, new, heads, group, dim, bs, seed, mask=None, cap=0.0, slopes=None, count=0, scale=None, spoil=None,
        sight=None):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(seed + 77)
    cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, seed)
    start, request, position = batch(lens, new)
    T, Hq = len(request), heads * group
    q = queries(T, Hq, dim, kind, seed)
    blocks = None
    if count:
        blocks = np.full((T, heads, count), -1, np.int32)
        for t in range(T):
            n = -(-lens[request[t]] // bs)
            for h in range(heads):
                kept = np.sort(rng.permutation(n)[: rng.integers(0, count + 1)])
                blocks[t, h, : len(kept)] = kept
    first = prefix = None
    if mask:
        first, prefix = sights(mask, lens, new, request, position, rng)
    if sight:
        first, prefix = sight(position.astype(np.int64))
    slope = None
    if slopes is not None:
        slope = np.resize(np.asarray(slopes, np.float32), Hq)
    if spoil:
        spoil(cache, table, position, first, prefix, keys, values)
    scale = scale or dim**-0.5
    as_i = lambda x: None if x is None else ints(x)  # noqa: E731
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), scale, int(max(new)),
                                 blocks=as_i(blocks), cap=cap, slopes=None if slope is None else dev(slope),
                                 first=as_i(first), prefix=as_i(prefix))
    qn = as_np(q)
    want = model(qn, keys, values, heads, request, position, table, bs, scale, blocks, cap, slope, first, prefix)
    vmax = np.nanmax(np.abs(values), initial=1.0)
    smax = largest_score(qn, keys, scale)
    check(out, lse, want, kind, vmax, smax, cap)
    return as_np(out), as_np(lse)


MASKS = ["window", "one window", "documents", "prefix", "prefix only", "mixed"]
LAYOUTS = [  # single tokens, few keys; a longer context; small prompts; a prompt; prompts in parts; both
    dict(lens=[1, 17, 63, 200], new=[1] * 4, heads=2, group=4, dim=64, bs=16),
    dict(lens=[2999, 1], new=[1, 1], heads=3, group=1, dim=128, bs=64),
    dict(lens=[900, 45, 0, 130], new=[3, 4, 0, 2], heads=2, group=7, dim=96, bs=32),
    dict(lens=[413], new=[390], heads=1, group=3, dim=128, bs=64),
    dict(lens=[900], new=[70], heads=2, group=2, dim=64, bs=16),
    dict(lens=[350, 777, 1, 300, 90], new=[300, 1, 1, 90, 5], heads=1, group=2, dim=192, bs=128),
    dict(lens=[260, 31], new=[100, 31], heads=1, group=5, dim=256, bs=16),
]


def name(c):
    return "%s+%s-%dx%d-d%d-bs%d" % (c["lens"], c["new"], c["heads"], c["group"], c["dim"], c["bs"])


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_masks(ctx, c, mask):
    run(ctx, "bf16" if c["dim"] % 128 else "f16", seed=len(mask), mask=mask, **c)


@pytest.mark.parametrize("terms", [dict(), dict(cap=5.0, slopes=[0.2, 0.003])], ids=["sights", "all"])
@pytest.mark.parametrize("c", [
    dict(lens=[1200], new=[1100], heads=4, group=8, dim=64, bs=16), dict(lens=[1100, 700, 650], new=[600, 1, 500], heads=8, group=4, dim=128, bs=64),
    dict(lens=[480, 90, 3, 600], new=[400, 9, 1, 300], heads=3, group=4, dim=192, bs=32)], ids=name)
def test_a_few_rows_that_see_much_more(ctx, c, terms):
    """The last rows of every request see all,
    some in the middle nothing, the others a short window and a few first keys."""
    rng = np.random.default_rng(1)

    def sight(p):
        start, request, position = batch(c["lens"], c["new"])
        last = np.asarray(c["lens"])[request] - position <= 7
        kind = rng.random(len(p)) < 0.1
        return np.where(last, 0, np.where(kind, p + 1, p - 20)), np.where(last | kind, 0, np.minimum(p + 1, 3))

    run(ctx, "bf16" if c["dim"] == 128 else "f16", seed=8, sight=sight, **terms, **c)


@pytest.mark.parametrize("kind,cap,scale", [("bf16", 0.02, None), ("f16", 1.0, None), ("bf16", 5.0, -0.2), ("f16", 30.0, 0.9),
                                            ("bf16", 2.0**-40, None), ("f16", 2.0**40, None)])
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_caps(ctx, c, kind, cap, scale):
    run(ctx, kind, seed=int(cap) % 97, cap=cap, scale=scale, **c)


@pytest.mark.parametrize("slopes", [[0.5, 0.05, 0.004], [0.0], [-0.01, 3.0]], ids=str)
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_slopes(ctx, c, slopes):
    run(ctx, "f16" if c["dim"] % 128 else "bf16", seed=len(slopes), slopes=slopes, **c)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("slope", [2.0**14, 1e6, 1e19, 3.4e38])
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_slopes_beyond_any_score(ctx, c, slope, kind):
    # A key one further away weighs exp(-2^14) = 0, so that a row is its own token's value. Its probability is rounded
    # once, over a sum that is not, and the result once: 2 u.
    import paper_2608_08751_amd as ivf

    lens, new, heads, group, dim, bs = (c[k] for k in ("lens", "new", "heads", "group", "dim", "bs"))
    cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, 5)
    start, request, position = batch(lens, new)
    T, Hq = len(request), heads * group
    out, lse = ivf.ivf_kv_attend(ctx, cache, queries(T, Hq, dim, kind, 5), ints(start), ints(request), ints(position), ints(table),
                                 dim**-0.5, int(max(new)), slopes=dev(np.full(Hq, slope, np.float32)))
    out, lse = as_np(out).reshape(T, Hq, dim), as_np(lse)
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    u = {"bf16": 2.0**-8, "f16": 2.0**-11}[kind]
    for t in range(T):
        block, at = table[request[t], position[t] // bs], position[t] % bs
        for g in range(Hq):
            v = values[block, g // group, at]
            assert (np.abs(out[t, g] - v) <= 2.01 * u * np.abs(v)).all(), (t, g)


@pytest.mark.parametrize("mask,cap", [(None, 0.0), ("mixed", 0.0), ("prefix", 0.0), ("mixed", 5.0), ("one window", 5.0)], ids=str)
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_slopes_that_are_no_number(ctx, c, mask, cap):
    """Their heads' rows are no number where they see a key; rows that see none, and the other heads, are as ever."""
    for kind, slopes in (("bf16", [math.nan, 0.05]), ("f16", [0.3, -math.nan, 0.0])):
        out, lse = run(ctx, kind, seed=len(slopes), mask=mask, cap=cap, slopes=slopes, **c)
        bad = np.isnan(np.resize(slopes, lse.shape[1]))
        assert not np.isnan(lse[:, ~bad]).any() and (np.isnan(lse[:, bad]) == ~np.isinf(lse[:, bad])).all()
        assert bad.all() or np.isfinite(out[:, ~bad]).all()


@pytest.mark.parametrize("kind,T,heads,group,dim,bs,count", [("bf16", 5, 2, 12, 128, 64, 4), ("f16", 300, 8, 2, 96, 16, 3), ("f16", 30, 2, 4, 192, 32, 6)])
def test_slopes_that_are_no_number_and_selected_blocks(ctx, kind, T, heads, group, dim, bs, count):
    lens = [max(T // 2, 1) + 150, T - max(T // 2, 1) + 333]
    run(ctx, kind, lens, [max(T // 2, 1), T - max(T // 2, 1)], heads, group, dim, bs, T, mask="mixed", slopes=[0.1, math.nan, 0.002],
        count=count)


@pytest.mark.parametrize("mask", ["window", "prefix", "mixed"])
@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_all_terms(ctx, c, mask):
    run(ctx, "bf16", seed=3, mask=mask, cap=4.0, slopes=[0.3, 0.01], **c)


@pytest.mark.parametrize("kind,T,heads,group,dim,bs,count", [
    ("bf16", 3, 2, 4, 64, 16, 5), ("f16", 40, 1, 3, 128, 32, 9), ("bf16", 5, 2, 12, 128, 64, 4), ("f16", 300, 8, 2, 96, 16, 3),
    ("bf16", 700, 3, 9, 64, 16, 2), ("f16", 30, 2, 4, 192, 32, 6), ("bf16", 9, 1, 16, 256, 64, 3)])
@pytest.mark.parametrize("mask", ["one window", "mixed"])
def test_selected_blocks(ctx, kind, T, heads, group, dim, bs, count, mask):
    lens = [max(T // 2, 1) + 150, T - max(T // 2, 1) + 333]
    run(ctx, kind, lens, [max(T // 2, 1), T - max(T // 2, 1)], heads, group, dim, bs, T, mask=mask, cap=9.0, slopes=[0.1, 0.002],
        count=count)


@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_rows_that_see_nothing(ctx, c):
    # first past every key, no prefix: zeros and -infinity
    out, lse = run(ctx, "bf16", seed=1, sight=lambda p: (p + 1, 0 * p), cap=3.0, slopes=[0.1], **c)
    assert not out.any() and (lse == -np.inf).all()
    # first at the largest int32, the prefix at the lowest
    out, lse = run(ctx, "f16", seed=2, sight=lambda p: (0 * p + 2**31 - 1, 0 * p - 2**31), **c)
    assert not out.any() and (lse == -np.inf).all()


@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_sights_at_their_ends(ctx, c):
    # the lowest first; prefixes beyond the table see what the table names (here: the requests' blocks, whose unused slots
    # hold zeros)
    def zeros(cache, table, position, first, prefix, keys, values):
        import torch

        import paper_2608_08751_amd as ivf

        block, place = np.nonzero(np.isnan(keys).any((1, 3)))
        x = torch.zeros(len(block), cache.heads, cache.dim, device="cuda", dtype=cache.dtype)
        ivf.ivf_kv_append(ctx, cache, x, x, dev(block * c["bs"] + place))
        keys[np.isnan(keys)] = 0
        values[np.isnan(values)] = 0

    run(ctx, "bf16", seed=4, sight=lambda p: (0 * p - 2**31, 0 * p), **c)
    run(ctx, "f16", seed=5, sight=lambda p: (0 * p, 0 * p + 2**31 - 1), spoil=zeros, slopes=[0.02], **c)


@pytest.mark.parametrize("c", LAYOUTS, ids=name)
def test_what_nobody_sees_may_be_anything(ctx, c):
    """Blocks between the first tokens and every window are given back: no table entry, or another's bytes."""
    def spoil(cache, table, position, first, prefix, keys, values):
        start, request, _ = batch(c["lens"], c["new"])
        for b in range(len(c["lens"])):
            own = request == b
            if not own.any():
                continue
            lo, end = int(np.maximum(first[own], 0).min()), int(prefix[own].max())
            for j in range(-(-end // c["bs"]), lo // c["bs"]):
                if j % 2:
                    table[b, j] = -1
                else:
                    cache.records[int(table[b, j])] = 255
                    keys[table[b, j]] = values[table[b, j]] = np.nan

    run(ctx, "bf16", seed=6, mask="one window", spoil=spoil, slopes=[0.01], **c)


def test_nan_keys_reach_the_rows_that_see_them_alone(ctx):
    """A token stored as NaN inside the strips of others' windows."""
    import torch

    import paper_2608_08751_amd as ivf

    for new, lens in (([1] * 4, [40, 70, 100, 130]), ([90], [130])):
        heads, group, dim, bs, kind = 2, 4, 128, 16, "bf16"
        cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, 9)
        start, request, position = batch(lens, new)
        bad = [(b, p) for b in range(len(lens)) for p in (3, 38, lens[b] - 20) if p < lens[b]]
        bad += [(1, 69)] if len(lens) > 1 else []  # that a single token sees
        slots = [int(table[b, p // bs]) * bs + p % bs for b, p in bad]
        k = torch.full((len(bad), heads, dim), float("inf"), device="cuda", dtype=dtype_of(kind))
        ivf.ivf_kv_append(ctx, cache, k, torch.zeros_like(k), dev(np.array(slots, np.int64)))
        for s in slots:
            keys[s // bs, :, s % bs] = values[s // bs, :, s % bs] = np.nan
        first, prefix = position - np.arange(len(position)) % 21, np.arange(len(position)) % 5
        q = queries(len(request), heads * group, dim, kind, 9)
        out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), 0.1, max(new),
                                     cap=20.0, first=ints(first), prefix=ints(prefix))
        want = model(as_np(q), keys, values, heads, request, position, table, bs, 0.1, None, 20.0, None, first, prefix)
        assert np.isnan(want[0]).any() and not np.isnan(want[0]).all()
        check(out, lse, want, kind, np.nanmax(np.abs(values)), largest_score(as_np(q), keys, 0.1), 20.0)


@pytest.mark.parametrize("cap", [0.0, 7.0])
@pytest.mark.parametrize("T", [1, 90])
def test_queries_that_are_not_finite(ctx, T, cap):
    import torch

    import paper_2608_08751_amd as ivf

    lens = [120]
    cache, table, keys, values = make(ctx, "f16", lens, 2, 64, 16, 3)
    start, request, position = batch(lens, [T])
    q = torch.randn(T, 4, 64, device="cuda", dtype=torch.float16)
    q[0, 0, 3], q[-1, 1, 60], q[T // 2, 3, 9] = float("nan"), float("inf"), float("-inf")
    first = position + 1 - 4 * (np.arange(T) % 2 == 0)  # every other row sees nothing
    out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), 0.1, T, cap=cap,
                                 slopes=torch.full((4,), 0.1, device="cuda"), first=ints(first))
    bad = ~torch.isfinite(q).all(-1).cpu().numpy() & (first <= position)[:, None]
    assert (np.isnan(as_np(out)).all(-1) == bad).all() and (np.isnan(as_np(lse)) == bad).all()
    empty = first > position
    assert (as_np(lse)[empty] == -np.inf).all() and not as_np(out)[empty].any()


def test_positions_beyond_the_table(ctx):
    """The bias goes by the position, also where the table ends long before it; above 2^24 the distance rounds."""
    import paper_2608_08751_amd as ivf

    for far in (5000, 2**25 + 3, 2**31 - 1):
        for T in (1, 80):
            cache, table, keys, values = make(ctx, "bf16", [160], 1, 64, 16, 5)
            table = table[:, :10].copy()
            position = np.full(T, far)
            q = queries(T, 2, 64, "bf16", T)
            slopes = np.array([2.0**-22, 2.0**-27], np.float32)
            out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints([0, T]), ints([0] * T), ints(position), ints(table), 0.125, T,
                                         slopes=dev(slopes))
            want = model(as_np(q), keys, values, 1, np.zeros(T), position, table, 16, 0.125, None, 0.0, slopes)
            check(out, lse, want, "bf16", np.nanmax(np.abs(values)), largest_score(as_np(q), keys, 0.125), 0.0)


def test_terms_of_nothing_change_little(ctx):
    """first 0, prefix 0, slopes 0 and a cap far above the scores: the call without terms, to its roundings."""
    import torch

    import paper_2608_08751_amd as ivf

    for lens, new in (([700, 33], [1, 1]), ([300], [200])):
        cache, table, _, _ = make(ctx, "f16", lens, 2, 128, 32, 11)
        start, request, position = batch(lens, new)
        q = queries(len(request), 8, 128, "f16", 11)
        call = lambda **k: ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position), ints(table), 0.09,  # noqa: E731
                                             max(new), **k)
        out, lse = call()
        zero = ints(0 * position)
        for k in (dict(first=zero), dict(prefix=zero), dict(slopes=torch.zeros(8, device="cuda")), dict(cap=1e9)):
            o, s = call(**k)
            assert float((o.float() - out.float()).abs().max()) <= 2.0**-10 * float(out.float().abs().max())
            assert float((s - lse).abs().max()) <= 1e-5
        same = call(cap=0.0)  # without any, the call itself
        assert torch.equal(same[0], out) and torch.equal(same[1], lse)


def test_captured(ctx):
    """A captured call on a stream of its own, replayed with other lengths, masks and slopes in the same buffers."""
    import torch

    import paper_2608_08751_amd as ivf

    heads, group, dim, bs, kind = 2, 4, 128, 32, "bf16"
    lens = [2900, 1500, 64]
    cache, table, keys, values = make(ctx, kind, lens, heads, dim, bs, 21)
    _, request, position = batch(lens, [1, 1, 1])
    pos, first, prefix, slopes = ints(position), ints(position), ints(position), torch.zeros(8, device="cuda")
    start, req, tab = ints([0, 1, 2, 3]), ints(request), ints(table)
    q = queries(3, 8, dim, kind, 21, strided=False)

    def step():
        return ivf.ivf_kv_attend(ctx, cache, q, start, req, pos, tab, 0.09, 1, cap=8.0, slopes=slopes, first=first, prefix=prefix)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse = step()
    rng = np.random.default_rng(1)
    for _ in range(4):
        p = np.array([rng.integers(0, n) for n in lens])
        f, e, s = p - rng.integers(0, 700, 3), np.minimum(rng.integers(0, 900, 3), lens), rng.random(8).astype(np.float32) / 50
        for t, x in ((pos, p), (first, f), (prefix, e)):
            t.copy_(torch.from_numpy(x.astype(np.int32)))
        slopes.copy_(torch.from_numpy(s))
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = model(as_np(q), keys, values, heads, request, p, table, bs, 0.09, None, 8.0, s, f, e)
        check(out, lse, want, kind, np.nanmax(np.abs(values)), largest_score(as_np(q), keys, 0.09), 8.0)
        eager = step()
        assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)


def test_arguments(ctx):
    import torch

    import paper_2608_08751_amd as ivf

    cache, table, _, _ = make(ctx, "bf16", [40], 1, 64, 16, 1)
    q = torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)
    call = lambda **k: ivf.ivf_kv_attend(ctx, cache, q, ints([0, 2]), ints([0, 0]), ints([38, 39]), ints(table), 0.1, 2, **k)  # noqa: E731
    for bad, error in ((dict(slopes=torch.zeros(3, device="cuda")), ValueError), (dict(slopes=torch.zeros(4)), TypeError),
                       (dict(slopes=torch.zeros(4, device="cuda").half()), TypeError), (dict(first=ints([0])), ValueError),
                       (dict(prefix=ints([0, 0]).long()), TypeError), (dict(cap=-1.0), ivf.IvfError),
                       (dict(cap=float("nan")), ivf.IvfError), (dict(cap=1e-13), ivf.IvfError),
                       (dict(slopes=torch.zeros(4, device="cuda", requires_grad=True)), RuntimeError)):
        with pytest.raises(error):
            call(**bad)
    with torch.no_grad():
        call(slopes=torch.zeros(4, device="cuda", requires_grad=True))
