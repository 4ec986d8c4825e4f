"""The definitions of the paged 4-bit key/value cache in numpy fp64, written from
the text of include/ivf.h: what the tests compare the kernels with."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXPONENTS = {"f16": (-13, 13), "bf16": (-125, 125)}


def quantise(x, kind):
    """Values that x [..., dim] is stored as, NaN groups apart (fp64)."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    amax = np.abs(g).max(-1, keepdims=True)
    _, e = np.frexp(amax)  # amax = m 2^e, m in [.5, 1)
    unit = e - 3.0
    unit = unit + (amax > 7.0 * np.exp2(unit))
    unit = np.exp2(np.clip(np.where(amax > 0, unit, -1000.0), *EXPONENTS[kind]))
    a = np.abs(g) / unit
    # nearest level; between two the one of even code
    d = np.abs(a[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    pick = np.where(d == best, np.arange(8) % 2 * 100 + np.arange(8), 1000).argmin(-1)
    return (np.sign(g) * LEVELS[pick] * unit).reshape(x.shape)


def store(k, v, kind):
    """(keys, values) as read back: fp64, NaN in the groups where either is not finite."""
    bad = ~(np.isfinite(k) & np.isfinite(v)).reshape(*k.shape[:-1], -1, 32).all(-1)
    bad = np.repeat(bad, 32, -1)
    clean = lambda x: quantise(np.where(bad, 0.0, x), kind)  # noqa: E731
    return np.where(bad, np.nan, clean(k)), np.where(bad, np.nan, clean(v))


def summary(keys):
    """(codes, weight) of the keys [tokens, dim] of a full block, in the definition's fp32 steps."""
    total = np.where(np.isnan(keys), 0.0, keys).sum(0).astype(np.float32)
    mean = total * np.float32(1.0 / keys.shape[0])
    amax = np.abs(mean).max()
    if not (amax >= np.float32(2.0**-100) and np.isfinite(amax)):
        return np.zeros(keys.shape[1], np.int8), np.float32(0)
    return np.rint(mean * (np.float32(127) / amax)).astype(np.int8), amax / np.float32(127)


def plan(cached, added, bs, table, free, tokens):
    """The definition of ivf_kv_plan, request by request; table is changed in place."""
    free = list(free)
    cols = table.shape[1]
    start, slots, request, position = [0], [], [], []
    used = 0
    asked = beyond = 0
    for b, (c, a) in enumerate(zip(np.maximum(cached, 0).tolist(), np.maximum(added, 0).tolist())):
        old, now = -(-c // bs), -(-(c + a) // bs)
        beyond += now > cols
        for j in range(min(old, cols), cols):
            table[b, j] = -1
        for j in range(old, min(now, cols)):
            asked += 1
            if used < len(free):
                table[b, j] = free[used]
                used += 1
        for i in range(a):
            p = c + i
            j = p // bs
            slots.append(int(table[b, j]) * bs + p % bs if j < cols and table[b, j] >= 0 else -1)
            request.append(b)
            position.append(p)
        start.append(start[-1] + a)
    info = [start[-1], asked, used, beyond]
    pad = lambda v: np.array((v + [-1] * tokens)[:tokens])  # noqa: E731
    return np.minimum(start, tokens), pad(slots), pad(request), pad(position), info


def select(q, summaries, weights, heads, request, position, table, bs, first, last, count):
    """The definition of ivf_kv_select: q fp64 [T, query heads, dim]; int32 [T, heads, count]."""
    T, Hq, dim = q.shape
    blocks, out = summaries.shape[0], np.full((T, heads, count), -1, np.int32)
    group = Hq // heads
    for t in range(T):
        b, p = int(request[t]), int(position[t])
        if b < 0 or b >= table.shape[0] or p < 0:
            continue
        n = min(p // bs + 1, table.shape[1])
        for h in range(heads):
            with np.errstate(invalid="ignore"):
                u = q[t, h * group:(h + 1) * group].sum(0).astype(np.float32)
            u[~np.isfinite(u)] = 0
            amax = np.abs(u).max()
            c = np.rint(u * (np.float32(127) / amax)).astype(np.int64) if amax >= np.float32(2.0**-100) else 0 * u
            forced, ranked = [], []
            for j in range(n):
                x = int(table[b, j])
                if x < 0 or x >= blocks:
                    continue
                if j < min(first, n) or j >= max(n - last, first):
                    forced.append(j)
                else:
                    s = np.float32(int((c * summaries[x, h].astype(np.int64)).sum())) * weights[x, h]
                    ranked.append((-s, j))
            ends = min(first, n) + n - max(n - last, min(first, n))
            kept = sorted(forced + [j for _, j in sorted(ranked)[: count - ends]])
            out[t, h, : len(kept)] = kept
    return out


def attend(q, keys, values, heads, request, position, table, bs, scale, blocks=None):
    """fp64 attention: q [T, Hq, dim], keys and values [blocks, heads, bs, dim] as read back."""
    T, Hq, dim = q.shape
    group = Hq // heads
    out, lse = np.zeros((T, Hq, dim)), np.full((T, Hq), -np.inf)
    for t in range(T):
        b, p = int(request[t]), int(position[t])
        if b < 0 or b >= table.shape[0] or p < 0:
            continue
        for h in range(heads):
            cols = range(table.shape[1]) if blocks is None else [int(j) for j in blocks[t, h]]
            k, v = [], []
            for j in cols:
                if j < 0 or j >= table.shape[1] or j * bs > p:
                    continue
                x = int(table[b, j])
                if x < 0 or x >= keys.shape[0]:
                    continue
                n = min(bs, p + 1 - j * bs)
                k.append(keys[x, h, :n])
                v.append(values[x, h, :n])
            if not k:
                continue
            k, v = np.concatenate(k), np.concatenate(v)
            # one NaN in a token's key or value makes the whole row NaN
            nan = np.isnan(k).any() or np.isnan(v).any()
            for g in range(h * group, (h + 1) * group):
                if nan:
                    out[t, g] = lse[t, g] = np.nan
                    continue
                s = scale * (k @ q[t, g])
                m = s.max()
                e = np.exp(s - m)
                lse[t, g] = m + math.log(e.sum())
                out[t, g] = (e / e.sum()) @ v
    return out, lse
