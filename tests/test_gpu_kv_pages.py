"""Forking, copying and reclaiming blocks of the paged 4-bit key/value cache on the GPU, against the text of
include/ivf.h in Python. Tables, lengths, pairs, lists and bytes have to be equal."""
import numpy as np
import pytest

import kv_model as M
from test_gpu_kv import batch, check_attend, dev, dtype_of, ints, make, as_np

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


# ---- the definitions ------------------------------------------------------------

def fork_model(parent, child, cached, bs, table, free):
    """(source, to, info); cached and table are changed in place."""
    B, cols = table.shape
    n = len(parent)
    valid = [0 <= p < B and 0 <= c < B and p != c for p, c in zip(parent, child)]
    parents = {p for p, ok in zip(parent, valid) if ok}
    source, to, asked = [-1] * n, [-1] * n, 0
    for i in range(n):
        if not valid[i] or child[i] in parents or any(valid[j] and child[j] == child[i] for j in range(i + 1, n)):
            continue
        m = int(cached[parent[i]])
        row = np.full(cols, -1, np.int32)
        held = min(-(-max(m, 0) // bs), cols)
        row[:held] = table[parent[i], :held]
        last = -(-max(m, 0) // bs) - 1
        if m > 0 and m % bs and last < cols and row[last] >= 0:
            new = int(free[asked]) if asked < len(free) else -1
            asked += 1
            if new >= 0:
                source[i], to[i] = int(row[last]), new
            row[last] = new
        table[child[i]], cached[child[i]] = row, m
    return source, to, [asked, min(asked, len(free))]


def reclaim_model(cached, bs, table, blocks, moves):
    """(free, source, to, info); table is changed in place."""
    held = [(b, j) for b in range(len(cached)) for j in range(min(-(-max(int(cached[b]), 0) // bs), table.shape[1]))
            if 0 <= table[b, j] < blocks]
    used = {int(table[b, j]) for b, j in held}
    U = len(used)
    high = sorted(x for x in used if x >= U)
    low = [x for x in range(U) if x not in used]
    goes = dict(list(zip(high, low))[:moves])
    for b, j in held:
        table[b, j] = goes.get(int(table[b, j]), int(table[b, j]))
    now = {goes.get(x, x) for x in used}
    free = [x for x in range(blocks) if x not in now]
    pad = lambda v, n: list(v) + [-1] * (n - len(v))  # noqa: E731
    return pad(free, blocks), pad(goes.keys(), moves), pad(goes.values(), moves), [U, len(goes), blocks - U]


# ---- forks ----------------------------------------------------------------------

def run_fork(ctx, parent, child, cached, bs, table, free):
    import paper_2608_08751_amd as ivf

    got_cached, got_table = ints(cached), ints(table)
    got = ivf.ivf_kv_fork(ctx, ints(parent), ints(child), got_cached, bs, got_table, ints(free), want_info=True)
    cached, table = np.array(cached, np.int32), np.array(table, np.int32)
    source, to, info = fork_model(list(parent), list(child), cached, bs, table, list(free))
    assert (got_table.cpu().numpy() == table).all() and (got_cached.cpu().numpy() == cached).all()
    assert got.source.tolist() == source and got.to.tolist() == to and got.info.tolist() == info


FORKS = [  # B, n, longest, block size, free blocks
    (2, 1, 1, 16, 5), (3, 2, 700, 64, 5), (9, 8, 3001, 32, 20), (40, 64, 900, 16, 3), (300, 250, 5000, 16, 100),
    (2048, 2048, 40, 128, 3000), (2049, 5, 100, 16, 5), (5, 2049, 100, 16, 5), (5000, 9000, 60, 16, 2000),
    (16384, 16384, 20, 16, 16384),
]


@pytest.mark.parametrize("B,n,longest,bs,n_free", FORKS)
def test_fork(ctx, B, n, longest, bs, n_free):
    rng = np.random.default_rng(B + n)
    cols = -(-longest // bs) + 2
    cached = rng.integers(0, longest + 1, B)
    cached[0] = longest
    table = rng.integers(0, 1 << 20, (B, cols)).astype(np.int32)
    half = max(1, B // 2)
    parent = rng.integers(0, half, n)
    child = half + (np.arange(n) % max(1, B - half)) if n <= 3000 else rng.permutation(np.r_[half:B, rng.integers(0, B, n)])[:n]
    run_fork(ctx, parent, child, cached, bs, table, rng.permutation(1 << 16)[:n_free])


def test_fork_lengths(ctx):
    # none, negative, a whole block, one more, beyond the table, a last block that no entry names
    cached = [0, -7, 16, 17, 100, 40, 5, 64] + [3] * 9
    table = np.arange(17 * 4).reshape(17, 4).astype(np.int32)
    table[5, 2] = -1
    run_fork(ctx, [0, 1, 2, 3, 4, 5, 6, 7], np.arange(8, 16), cached, 16, table, [900, 901, 902, 903])
    run_fork(ctx, [0, 1, 2, 3, 4, 5, 6, 7], np.arange(8, 16), cached, 16, table, [900])  # too few
    run_fork(ctx, [6, 6, 6], [8, 9, 10], cached, 16, table, [])  # none free


def test_fork_rows_that_do_not_count(ctx):
    cached = [20, 33, 7, 9, 50, 1]
    table = np.arange(24).reshape(6, 4).astype(np.int32)
    free = list(range(100, 120))
    run_fork(ctx, [0, 1, 0], [3, 3, 3], cached, 16, table, free)  # one child: the last fork counts
    run_fork(ctx, [0, 1], [1, 2], cached, 16, table, free)  # a child that is a parent
    run_fork(ctx, [0, 1], [1, 0], cached, 16, table, free)
    run_fork(ctx, [2, 0, -1, 0, 6, 1], [2, 6, 0, -5, 0, 4], cached, 16, table, free)  # itself, outside
    run_fork(ctx, [0, 3, 0], [3, -1, 4], cached, 16, table, free)  # an invalid fork makes no parent
    run_fork(ctx, [0, 7, 1], [3, 3, 4], cached, 16, table, free)  # nor the last of a child


def test_fork_of_long_rows_and_of_nothing(ctx):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(5)
    table = rng.integers(0, 1 << 30, (3, 5000)).astype(np.int32)
    run_fork(ctx, [1, 1], [0, 2], [7, 16 * 4999 + 3, 9], 16, table, [5, 6])
    run_fork(ctx, [1, 1], [0, 2], [7, 16 * 5000, 9], 16, table, [5, 6])
    got = ivf.ivf_kv_fork(ctx, ints([]), ints([]), ints([7, 8, 9]), 16, ints(table), ints([1]), want_info=True)
    assert got.source.numel() == 0 and got.info.tolist() == [0, 0]


# ---- copies ---------------------------------------------------------------------

@pytest.mark.parametrize("kind,heads,dim,bs", [("bf16", 1, 64, 16), ("f16", 3, 96, 32), ("bf16", 8, 128, 64),
                                                ("f16", 5, 192, 128), ("bf16", 2, 256, 16), ("f16", 7, 96, 16)])
def test_copy(ctx, kind, heads, dim, bs):
    import torch

    import paper_2608_08751_amd as ivf

    g = torch.Generator(device="cuda")
    g.manual_seed(dim)

    def filled(blocks):
        c = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
        c.records.random_(0, 256, generator=g)
        c.summary.random_(-128, 128, generator=g)
        c.weight.normal_(generator=g)
        return c

    a, b = filled(23), filled(40)
    pairs = {a: ([3, -1, 0, 22, 23, 7, 1 << 30], [5, 4, -1, 6, 9, 40, 10]), b: ([39, 0, -1, 5, 40, 24], [22, 3, 2, 23, 0, 1])}
    for src, (source, to) in pairs.items():
        for dst in (src, b if src is a else a):
            want = [x.clone() for x in (dst.records, dst.summary, dst.weight)]
            at = (src.records.clone(), src.summary.clone(), src.weight.clone())
            for s, t in zip(source, to):
                if 0 <= s < src.blocks and 0 <= t < dst.blocks:
                    for x, y in zip(want, at):
                        x[t] = y[s]
            ivf.ivf_kv_copy(ctx, dst, ints(to), ints(source), source_cache=None if dst is src else src)
            for x, y in zip((dst.records, dst.summary, dst.weight), want):
                assert torch.equal(x, y)
    ivf.ivf_kv_copy(ctx, a, ints([]), ints([]))


def test_copy_of_many_pairs(ctx):
    import torch

    import paper_2608_08751_amd as ivf

    c = ivf.KVCache.empty(30_000, 1, 64, 16)
    c.records.random_(0, 256)
    c.weight.normal_()
    order = torch.randperm(30_000, device="cuda").int()
    source, to = order[:15_000].contiguous(), order[15_000:].contiguous()
    records, weight = c.records.clone(), c.weight.clone()
    records[to.long()], weight[to.long()] = records[source.long()], weight[source.long()]
    ivf.ivf_kv_copy(ctx, c, to, source)
    assert torch.equal(c.records, records) and torch.equal(c.weight, weight)


# ---- the free blocks, and moves -------------------------------------------------

def run_reclaim(ctx, cached, bs, table, blocks, moves):
    import paper_2608_08751_amd as ivf

    got_table = ints(table)
    got = ivf.ivf_kv_reclaim(ctx, ints(cached), bs, got_table, blocks, moves=moves)
    table = np.array(table, np.int32)
    free, source, to, info = reclaim_model(cached, bs, table, blocks, moves)
    assert got.info.tolist() == info
    assert got.source.tolist() == source and got.to.tolist() == to
    assert (got.free.cpu().numpy() == np.array(free)).all()
    assert (got_table.cpu().numpy() == table).all()


RECLAIMS = [  # requests, columns, blocks, block size, moves: in one workgroup, and in several launches
    (1, 1, 1, 16, 0), (1, 3, 31, 64, 5), (4, 9, 64, 16, 40), (3, 10_000, 32_768, 16, 32_768), (3, 10_000, 32_767, 16, 99), (3, 10_000, 32_769, 16, 99), (16, 70, 1100, 64, 2000), (7, 300, 2101, 16, 3),
    (60, 260, 10_000, 32, 100), (1, 16_384, 20_000, 16, 9999),
    (70, 300, 15_001, 32, 0), (70, 300, 15_001, 32, 10_000), (70, 300, 200_000, 32, 17), (3, 9, 300_001, 16, 50),
    (2000, 40, 70_000, 16, 70_000), (1, 20_000, 66_000, 16, 66_000),
]


@pytest.mark.parametrize("B,cols,blocks,bs,moves", RECLAIMS)
def test_reclaim(ctx, B, cols, blocks, bs, moves):
    rng = np.random.default_rng(B + cols + blocks)
    table = rng.integers(0, blocks, (B, cols)).astype(np.int32)
    table[rng.random((B, cols)) < 0.1] = -1
    if B > 1:
        table[1] = table[0]  # shared blocks
    table[-1, 0], table[0, -1] = blocks, 1 << 30  # outside
    cached = rng.integers(-bs, bs * (cols + 2), B)
    cached[B // 2:B // 2 + B // 3] = 0
    run_reclaim(ctx, cached, bs, table, blocks, moves)


@pytest.mark.parametrize("blocks,cols", [(96, 40), (97, 40), (300_000, 150_000), (300_032, 150_016)])
def test_reclaim_all_none_and_already_together(ctx, blocks, cols):
    every = np.arange(2 * cols).reshape(2, cols).astype(np.int32)  # 0 ... 2 cols - 1
    full = [cols * 16, cols * 16]
    run_reclaim(ctx, full, 16, every, blocks, 10)  # together
    run_reclaim(ctx, full, 16, blocks - 1 - every, blocks, 3 * cols)  # at the upper end
    run_reclaim(ctx, [0, -1], 16, every, blocks, 10)  # none
    run_reclaim(ctx, full, 16, every, 2 * cols, 10)  # all


def test_reclaim_without_requests_and_without_lists(ctx):
    import torch

    import paper_2608_08751_amd as ivf

    for blocks in (5, 70, 300_000):
        got = ivf.ivf_kv_reclaim(ctx, ints([]), 16, ints(np.zeros((0, 3))), blocks, moves=4)
        assert got.free.tolist() == list(range(blocks)) and got.source.tolist() == [-1] * 4
        assert got.info.tolist() == [0, 0, blocks]
        info = torch.zeros(3, dtype=torch.int64, device="cuda")
        lib, handle = ctx.bind()
        assert lib.ivf_kv_reclaim(handle, None, 0, 16, None, 0, blocks, 0, None, None, None, info.data_ptr()) == 0
        assert info.tolist() == [0, 0, blocks]


# ---- together -------------------------------------------------------------------

@pytest.mark.parametrize("kind,dim,bs,length", [("bf16", 128, 32, 77), ("f16", 64, 16, 64), ("bf16", 96, 64, 5)])
def test_samples_of_one_prompt(ctx, kind, dim, bs, length):
    """A prompt, four samples of it that each go on alone, two of which end; the others are moved together."""
    import torch

    import paper_2608_08751_amd as ivf

    heads, group, samples, rng = 2, 3, 4, np.random.default_rng(length)
    blocks, cols = 60, -(-(length + 80) // bs) + 1
    cache = ivf.KVCache.empty(blocks, heads, dim, bs, dtype_of(kind))
    cache.records.fill_(255)
    pool = ints(rng.permutation(blocks))
    table = ints(np.full((samples + 1, cols), -1))
    cached = ints([0] * (samples + 1))
    keys = [np.zeros((0, heads, dim))] * (samples + 1)
    values = list(keys)
    free = pool

    def go_on(added):
        nonlocal cached, free
        T = sum(added)
        kv = dev(rng.standard_normal((T, 2, heads, dim)).astype(np.float32), dtype_of(kind))
        plan = ivf.ivf_kv_plan(ctx, cached, ints(added), bs, table, free, T, want_info=True)
        ivf.ivf_kv_append(ctx, cache, kv[:, 0], kv[:, 1], plan.slots)
        free = free[int(plan.info[2]):].contiguous()
        k, v = M.store(as_np(kv[:, 0]), as_np(kv[:, 1]), kind)
        at = 0
        for b, a in enumerate(added):
            keys[b], values[b] = np.concatenate([keys[b], k[at:at + a]]), np.concatenate([values[b], v[at:at + a]])
            at += a
        cached = cached + ints(added)

    def check():
        live = [b for b in range(samples + 1) if len(keys[b])]
        q = dev(rng.standard_normal((len(live), heads * group, dim)).astype(np.float32), dtype_of(kind))
        lens = [len(keys[b]) for b in live]
        start, request, position = batch(lens, [1] * len(live))
        out, lse = ivf.ivf_kv_attend(ctx, cache, q, ints(start), ints(request), ints(position),
                                     table[dev(np.array(live))].contiguous(), dim**-0.5, 1)
        whole = max(lens)
        pad = lambda x: np.stack([np.concatenate([x[b], np.zeros((whole - len(x[b]), heads, dim))]) for b in live])  # noqa: E731
        want, want_lse = M.attend(as_np(q), pad(keys).transpose(0, 2, 1, 3), pad(values).transpose(0, 2, 1, 3), heads,
                                  request, position, np.arange(len(live))[:, None], whole, dim**-0.5)
        check_attend(out, lse, want, want_lse, kind, max(np.abs(x).max() for x in values if x.size), 30.0)

    go_on([length] + [0] * samples)
    check()
    fork = ivf.ivf_kv_fork(ctx, ints([0] * samples), ints(range(1, samples + 1)), cached, bs, table, free, want_info=True)
    ivf.ivf_kv_copy(ctx, cache, fork.to, fork.source)
    free = free[int(fork.info[1]):].contiguous()
    for b in range(1, samples + 1):
        keys[b], values[b] = keys[0], values[0]
    check()
    for _ in range(3):
        go_on([0] + [int(x) for x in rng.integers(1, 20, samples)])
    check()
    for b in (0, 2, 3):  # the prompt too: its blocks are the samples'
        cached[b] = 0
        keys[b] = values[b] = np.zeros((0, heads, dim))
    before = set(free.tolist())
    found = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks)
    assert before < {x for x in found.free.tolist() if x >= 0}
    found = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks, moves=blocks)
    ivf.ivf_kv_copy(ctx, cache, found.to, found.source)
    used, made, left = found.info.tolist()
    assert made > 0 and found.free.tolist() == list(range(used, blocks)) + [-1] * used and left == blocks - used
    for x in (cache.records[used:], cache.weight[used:]):  # what is free may hold anything
        x.fill_(255 if x.dtype == torch.uint8 else float("nan"))
    check()
    free = found.free[:left]
    go_on([9] + [int(x) if b in (1, 4) else 0 for b, x in zip(range(1, samples + 1), rng.integers(1, 40, samples))])
    check()


FREE_WITHOUT_BLOCKS = [  # lists that end early, as ivf_kv_reclaim writes them, and others with entries that are no block
    [], [-1], [-1] * 40, [7], [7, 9, -1, -1], [7, 9, 11, -1, -1, -1, -1, -1], [-1, 7, -1, 9, 11], list(range(100, 130)) + [-1] * 9,
    [5, -7, 6, -(2**31)]]


@pytest.mark.parametrize("free", FREE_WITHOUT_BLOCKS, ids=lambda f: "%d-of-%d" % (sum(x >= 0 for x in f), len(f)))
@pytest.mark.parametrize("n", [1, 3, 5, 30, 3000])
def test_fork_says_how_many_blocks_it_took(ctx, n, free):
    """Entries of free_blocks that are no block are not counted; the forks that they fall to have no last block."""
    import paper_2608_08751_amd as ivf

    bs, cols = 16, 3
    cached = [20] + [0] * n
    table = np.full((n + 1, cols), -1, np.int32)
    table[0, :2] = 40, 41
    got_cached, got_table = ints(cached), ints(table)
    fork = ivf.ivf_kv_fork(ctx, ints([0] * n), ints(range(1, n + 1)), got_cached, bs, got_table, ints(free), want_info=True)
    taken = (free + [-1] * n)[:n]
    want = [x if x >= 0 else -1 for x in taken]
    assert fork.info.tolist() == [n, sum(x >= 0 for x in taken)]
    assert fork.to.tolist() == want and fork.source.tolist() == [41 if x >= 0 else -1 for x in want]
    assert (got_table[1:, 1] >= 0).sum() == int(fork.info[1]) and got_cached.tolist() == [20] * (n + 1)


@pytest.mark.parametrize("free", FREE_WITHOUT_BLOCKS, ids=lambda f: "%d-of-%d" % (sum(x >= 0 for x in f), len(f)))
@pytest.mark.parametrize("B,added", [(1, 1), (1, 100), (5, 40), (40, 1), (3000, 20)])
def test_plan_says_how_many_blocks_it_took(ctx, B, added, free):
    import paper_2608_08751_amd as ivf

    bs, cols = 16, -(-added // 16) + 1
    table = ints(np.full((B, cols), -1))
    plan = ivf.ivf_kv_plan(ctx, ints([0] * B), ints([added] * B), bs, table, ints(free), B * added, want_info=True)
    asked = B * -(-added // bs)
    taken = sum(x >= 0 for x in free[:asked])
    assert plan.info.tolist() == [B * added, asked, taken, 0]
    assert int((table >= 0).sum()) == taken
    assert int((plan.slots >= 0).sum()) == sum(min(bs, added - j * bs) for r, x in enumerate(free[:asked]) if x >= 0
                                               for j in [r % -(-added // bs)])


def test_what_reclaim_lists_runs_dry(ctx):
    """Its list as it is, padding and all, until no block is left: every call says what was missing."""
    import paper_2608_08751_amd as ivf

    bs, blocks = 16, 12
    table = np.full((9, 4), -1, np.int32)
    table[0, :3] = 2, 5, 11
    table, cached = ints(table), ints([40] + [0] * 8)
    free = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks).free
    assert free.tolist() == [0, 1, 3, 4, 6, 7, 8, 9, 10, -1, -1, -1]
    fork = ivf.ivf_kv_fork(ctx, ints([0] * 5), ints(range(1, 6)), cached, bs, table, free, want_info=True)
    assert fork.info.tolist() == [5, 5]
    free = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks).free
    plan = ivf.ivf_kv_plan(ctx, cached, ints([0] * 6 + [64, 1, 1]), bs, table, free, 66, want_info=True)
    assert plan.info.tolist() == [66, 6, 4, 0]  # four blocks were free
    assert (plan.slots < 0).tolist() == [False] * 64 + [True] * 2
    cached += ints([0] * 6 + [64, 0, 0])
    free = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks).free
    assert free.tolist() == [-1] * blocks
    fork = ivf.ivf_kv_fork(ctx, ints([0]), ints([7]), cached, bs, table, free, want_info=True)
    assert fork.info.tolist() == [1, 0] and fork.to.tolist() == [-1]


@pytest.mark.parametrize("T", [300_000, 1_000_000])
def test_plan_of_many_blocks_says_how_many_it_took(ctx, T):
    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(T)
    asked = -(-T // 16)
    free = np.where(rng.random(asked + 50) < 0.1, -1, np.arange(asked + 50))
    plan = ivf.ivf_kv_plan(ctx, ints([0]), ints([T]), 16, ints(np.full((1, asked), -1)), ints(free), T, want_info=True)
    assert plan.info.tolist() == [T, asked, int((free[:asked] >= 0).sum()), 0]


@pytest.mark.parametrize("blocks", [25_000, 60_000])
def test_captured_on_another_stream(ctx, blocks):
    """Fork, copy and reclaim as a graph, replayed on other lengths and tables in the same buffers."""
    import torch

    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(3)
    B, cols, bs, moves = 40, 500, 16, 3000
    cache = ivf.KVCache.empty(blocks, 1, 64, bs)
    table, cached, free = ints(np.zeros((B, cols))), ints(np.zeros(B)), ints(np.zeros(30))
    parent, child = ints(np.zeros(12)), ints(np.zeros(12))

    def fill():
        perm = rng.permutation(blocks)
        host = dict(table=perm[30:30 + B * cols].reshape(B, cols).astype(np.int32), cached=rng.integers(0, bs * cols, B).astype(np.int32),
                    free=perm[:30].astype(np.int32), parent=rng.integers(0, 20, 12).astype(np.int32),
                    child=rng.integers(15, 40, 12).astype(np.int32))
        for t, name in ((table, "table"), (cached, "cached"), (free, "free"), (parent, "parent"), (child, "child")):
            t.copy_(torch.from_numpy(host[name]))
        cache.records.random_(0, 256)
        return host

    def step():
        fork = ivf.ivf_kv_fork(ctx, parent, child, cached, bs, table, free, want_info=True)
        ivf.ivf_kv_copy(ctx, cache, fork.to, fork.source)
        found = ivf.ivf_kv_reclaim(ctx, cached, bs, table, blocks, moves=moves)
        ivf.ivf_kv_copy(ctx, cache, found.to, found.source)
        return fork, found

    side = torch.cuda.Stream()
    fill()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fork, found = step()
    for _ in range(4):
        h = fill()
        records = cache.records.cpu().numpy().copy()
        graph.replay()
        torch.cuda.synchronize()
        source, to, info = fork_model(h["parent"].tolist(), h["child"].tolist(), h["cached"], bs, h["table"], h["free"].tolist())
        assert fork.source.tolist() == source and fork.to.tolist() == to and fork.info.tolist() == info
        ok = [i for i in range(12) if to[i] >= 0]
        records[[to[i] for i in ok]] = records[[source[i] for i in ok]]
        lists = reclaim_model(h["cached"], bs, h["table"], blocks, moves)
        for got, want in zip((found.free, found.source, found.to, found.info), lists):
            assert got.tolist() == want
        n = lists[3][1]
        records[lists[2][:n]] = records[lists[1][:n]]
        assert (table.cpu().numpy() == h["table"]).all() and (cache.records.cpu().numpy() == records).all()


def test_arguments(ctx):
    import paper_2608_08751_amd as ivf

    table, cached = ints(np.zeros((3, 4))), ints([1, 2, 3])
    with pytest.raises(TypeError):
        ivf.ivf_kv_fork(ctx, ints([0]).long(), ints([1]), cached, 16, table, ints([1]))
    with pytest.raises(ValueError):
        ivf.ivf_kv_fork(ctx, ints([0]), ints([1, 2]), cached, 16, table, ints([1]))
    with pytest.raises(ValueError):
        ivf.ivf_kv_fork(ctx, ints([0]), ints([1]), cached[:2], 16, table, ints([1]))
    with pytest.raises(ValueError):
        ivf.ivf_kv_reclaim(ctx, cached, 16, table.t(), 10)
    with pytest.raises(ValueError):
        ivf.ivf_kv_reclaim(ctx, cached, 16, table, 0)
    with pytest.raises(TypeError):
        ivf.ivf_kv_reclaim(ctx, cached.cpu(), 16, table, 10)
    a, b = ivf.KVCache.empty(4, 1, 64, 16), ivf.KVCache.empty(4, 1, 128, 16)
    with pytest.raises(ivf.IvfError):
        ivf.ivf_kv_copy(ctx, a, ints([1]), ints([0]), source_cache=b)
    with pytest.raises(ValueError):
        ivf.ivf_kv_copy(ctx, a, ints([1]), ints([0, 2]))
