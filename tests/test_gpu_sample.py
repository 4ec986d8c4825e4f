"""Token sampling on the GPU against the definition of include/ivf.h in fp64. Tokens have to be equal: a draw or a limit
lies within 2^-43 V of a border between two tokens with a probability of about 2 V^2 2^-43, below 1e-2 for all rows
here together at V = 2^20 and 1e-6 at 10,000 (and the seeds are fixed). Log-probabilities are fp32: half a
step, 2^-24 |x|, and the weights' 2^-44 each of at least one, V 2^-44 < 1e-7: 2e-7 (1 + |x|) is allowed."""
import numpy as np
import pytest

from test_gpu_kv import dev, dtype_of

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


def model(x, u, t=1.0, k=0, p=1.0, floor=0.0):
    """(token, log-probability) of one row x (fp64)."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, 3.4028234663852886e38))
    m = x.max()
    if m == -np.inf:
        return -1, -np.inf
    if not t > 0:
        return int(np.argmax(x)), 0.0
    order = np.lexsort((np.arange(len(x)), -x))
    if 0 < k < len(x):
        order = order[:k]
    with np.errstate(invalid="ignore"):
        w = np.exp((x[order] - m) / min(t, 2.0**60))
    if p < 1:
        order = order[: int(np.searchsorted(np.cumsum(w), max(p, 0.0) * w.sum())) + 1]
        w = w[: len(order)]
    if floor > 0:
        n = max(1, int((w >= min(floor, 1.0)).sum()))
        order, w = order[:n], w[:n]
    by = np.argsort(order)
    order, w = order[by], w[by]
    c = np.cumsum(w)
    u = 0.0 if np.isnan(u) else max(u, 0.0)
    if u >= 1:
        i = int(np.nonzero(w >= 2.0**-44)[0][-1])
    else:
        i = int(np.searchsorted(c, u * c[-1], side="right"))
    return int(order[i]), float(np.log(w[i]) - np.log(c[-1]))


def tensor(x, kind):
    import torch

    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.float32 if kind == "f32" else dtype_of(kind))


def run(ctx, x, u, kind=None, **limits):
    """x: a tensor [T, V] on the GPU; limits: arrays [T] or None."""
    import paper_2608_08751_amd as ivf

    T = x.shape[0]
    types = dict(temperature=np.float32, top_k=np.int32, top_p=np.float32, min_p=np.float32)
    given = {n: np.asarray(v, types[n]) for n, v in limits.items() if v is not None}
    u = np.asarray(u, np.float32)
    token, logprob = ivf.ivf_sample(ctx, x, dev(u), **{n: dev(v) for n, v in given.items()})
    rows, token, logprob = x.double().cpu().numpy(), token.cpu().numpy(), logprob.cpu().numpy().astype(np.float64)
    default = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    for r in range(T):
        t, k, p, f = (float(given[n][r]) if n in given else default[n] for n in ("temperature", "top_k", "top_p", "min_p"))
        want, lp = model(rows[r], float(u[r]), t, int(k), p, f)
        assert token[r] == want, (r, int(token[r]), want, t, k, p, f, float(u[r]))
        assert logprob[r] == lp if np.isinf(lp) else abs(logprob[r] - lp) <= 2e-7 * (1 + abs(lp)), (r, logprob[r], lp)
    return token


def logits(rng, T, V, spread=2.5):
    x = rng.standard_normal((T, V)) * spread
    x[np.arange(T)[:, None], rng.integers(0, V, (T, min(V, 20)))] += 3 + 5 * rng.random((T, min(V, 20)))
    return x


LIMITS = ["none", "temperature", "top_k", "top_p", "min_p", "all"]
SIZES = [(3, 1), (4, 2), (5, 7), (3, 8), (6, 100), (4, 511), (3, 513), (5, 8191), (3, 8193), (8, 32_000), (3, 100_003)]


def some(rng, T, V, which):
    on = lambda n: which in (n, "all")  # noqa: E731
    pick = lambda *v: np.array(v)[rng.integers(0, len(v), T)]  # noqa: E731
    return dict(temperature=pick(0.0, 0.2, 0.7, 1.0, 1.5, 4.0) if on("temperature") else None,
                top_k=pick(0, 1, 2, 50, max(1, V // 2), V, V + 1) if on("top_k") else None,
                top_p=pick(0.0, 0.1, 0.5, 0.9, 0.999, 1.0, 1.5) if on("top_p") else None,
                min_p=pick(0.0, 0.001, 0.05, 0.5, 1.0) if on("min_p") else None)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("which", LIMITS)
@pytest.mark.parametrize("T,V", SIZES)
def test_sample(ctx, T, V, which, kind):
    rng = np.random.default_rng(V + len(which))
    for again in range(2):
        x = tensor(logits(rng, T, V), kind)
        run(ctx, x, rng.random(T), **some(rng, T, V, which))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_largest_vocabulary(ctx, kind):
    rng = np.random.default_rng(1)
    x = tensor(logits(rng, 3, 1 << 20), kind)
    for which in ("none", "top_p", "all"):
        run(ctx, x, rng.random(3), **some(rng, 3, 1 << 20, which))
    flat = tensor(rng.standard_normal((2, 1 << 20)) * 1e-3, kind)
    run(ctx, flat, [0.999, 0.5], top_p=[0.7, 0.2], top_k=[900_000, 0])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 9, 1000, 20_000])
def test_equal_logits(ctx, V, kind):
    """Ties go to the lowest index: all equal, two values, zeros of both signs."""
    rng = np.random.default_rng(V)
    T = 8
    limits = dict(top_k=[0, 1, V // 2 + 1, V, 3, 0, 0, 5], top_p=[1, 1, 1, 0.5, 0.4, 0.5, 0.25, 0.0], min_p=[0, 0, 0, 0, 1, 1, 0, 0])
    for x in (np.full((T, V), -3.25), np.where(rng.random((T, V)) < 0.5, 1.0, 1.5), np.where(rng.random((T, V)) < 0.5, -0.0, 0.0),
              np.round(rng.standard_normal((T, V)))):
        x = tensor(x, kind)
        run(ctx, x, rng.random(T), **limits)
        run(ctx, x, np.zeros(T), **limits)
        run(ctx, x, np.full(T, 1 - 2.0**-24), **limits)
        run(ctx, x, rng.random(T), temperature=[0, -1, 0, 0, 0, 0, 0, float("nan")])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite(ctx, kind):
    rng = np.random.default_rng(2)
    inf, nan = np.inf, np.nan
    T, V = 12, 3001
    x = logits(rng, T, V)
    x[0] = -inf  # no token
    x[1] = nan
    x[2, 1:] = -inf  # one
    x[3, ::2] = -inf
    x[4, 5:3000] = nan
    x[5, [7, 100, 2999]] = inf
    x[6, 3] = inf
    x[7, :] = inf
    x[8, rng.random(V) < 0.5] = nan
    x[9, :-1] = -inf
    x[10, ::3], x[10, 1::3] = nan, -inf
    x[11] = -6e4 + rng.integers(0, 64, V) * 32.0
    x = tensor(x, kind)
    for which in LIMITS:
        run(ctx, x, rng.random(T), **some(rng, T, V, which))
    run(ctx, x, rng.random(T), top_k=np.full(T, 2), top_p=np.full(T, 0.9))
    run(ctx, x, rng.random(T), top_k=np.full(T, V - 1))


@pytest.mark.parametrize("bits", [0x7FC0, 0xFFC0, 0x7F81, 0xFFBF])
def test_numbers_of_no_kind(ctx, bits):
    """Quiet and signaling ones of both signs count as -infinity."""
    import torch

    rng = np.random.default_rng(bits)
    x = tensor(logits(rng, 4, 20_000), "bf16")
    where = torch.from_numpy(rng.random((4, 20_000)) < 0.3).cuda()
    x = torch.where(where, torch.full_like(x, bits - 65536 if bits > 32767 else bits, dtype=torch.int16), x.view(torch.int16))
    x = x.view(torch.bfloat16)
    assert bool(torch.isnan(x)[where].all())
    for which in LIMITS:
        run(ctx, x, rng.random(4), **some(rng, 4, 20_000, which))


def test_arguments_beyond_their_ranges(ctx):
    rng = np.random.default_rng(4)
    inf, nan = np.inf, np.nan
    x = tensor(logits(rng, 10, 5000), "f32")
    u = [0.0, -0.0, -3.0, nan, 1 - 2.0**-24, 0.5, 1.0, 7.0, inf, 0.3]
    run(ctx, x, u)
    run(ctx, x, u, top_k=[-5, -(2**31), 2**31 - 1, 5000, 5001, 0, 4999, 1, 2, 3])
    run(ctx, x, rng.random(10), top_p=[-1, nan, inf, -inf, 2, 1, 1 - 2.0**-24, 1e-30, 0, 0.5])
    run(ctx, x, rng.random(10), min_p=[-1, nan, inf, -inf, 2, 1, 1e-30, 1e-45, 0, 0.5])
    run(ctx, x, rng.random(10), temperature=[inf, 1e30, 3e38, 1e-30, 1e-45, 1e-3, 2.0**60, 100.0, -inf, -0.0],
        top_p=[0.5, 0.5, 1, 0.9, 0.5, 0.5, 0.7, 0.7, 0.5, 0.5], top_k=[0, 70, 9, 3, 0, 5, 4000, 0, 7, 7])


def test_wide_ranges(ctx):
    """fp32 logits from the least to the largest, and rows whose spread is below their rounding."""
    rng = np.random.default_rng(5)
    T, V = 6, 4000
    x = np.empty((T, V))
    x[0] = np.sign(rng.standard_normal(V)) * np.exp(rng.uniform(-100, 88, V))
    x[1] = 3e38 * rng.uniform(-1, 1, V)
    x[2] = 1e-44 * rng.integers(-50, 50, V)
    x[3] = 1e6 + rng.integers(0, 30, V) / 16
    x[4] = -1e-6 * rng.random(V)
    x[5] = 1e30 * rng.random(V)
    x = tensor(x, "f32")
    for t in (1.0, 1e-6, 1e20, np.inf):
        for which in ("none", "top_k", "top_p", "all"):
            run(ctx, x, rng.random(T), **{**some(rng, T, V, which), "temperature": np.full(T, t)})


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_strides_and_alignment(ctx, kind):
    rng = np.random.default_rng(6)
    wide = tensor(logits(rng, 9, 10_007), kind)
    for at, n, step in ((0, 10_007, 1), (1, 9000, 1), (3, 77, 2), (5, 8192, 3), (7, 8200, 1), (2, 5, 1)):
        x = wide[::step, at:at + n]
        T = x.shape[0]
        run(ctx, x, rng.random(T), **some(rng, T, n, "all"))
    row = wide[:1].expand(5, -1)  # one row for all
    run(ctx, row, rng.random(5), top_p=np.full(5, 0.9))


@pytest.mark.parametrize("limits", [dict(), dict(top_k=40), dict(top_p=0.8), dict(top_k=300, top_p=0.9, min_p=0.01)], ids=str)
def test_draws_cover_the_distribution(ctx, limits):
    """4,096 evenly spread numbers: every token gets its share, in the order of the indexes."""
    rng = np.random.default_rng(7)
    T = 4096
    x = tensor(logits(rng, 1, 1000, 1.0), "f32").expand(T, -1)
    u = (np.arange(T) + 0.5) / T
    token = run(ctx, x, u, **{n: np.full(T, v) for n, v in limits.items()})
    assert (np.diff(token) >= 0).all()


def test_captured_on_another_stream(ctx):
    import torch

    import paper_2608_08751_amd as ivf

    rng = np.random.default_rng(8)
    T, V = 5, 40_000
    x, u = tensor(logits(rng, T, V), "bf16"), dev(np.zeros(T, np.float32))
    t, k, p = dev(np.ones(T, np.float32)), dev(np.zeros(T, np.int32)), dev(np.ones(T, np.float32))
    step = lambda: ivf.ivf_sample(ctx, x, u, temperature=t, top_k=k, top_p=p)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        token, logprob = step()
    for again in range(4):
        x.copy_(tensor(logits(rng, T, V), "bf16"))
        for a, b in ((u, rng.random(T)), (t, rng.random(T) + 0.3), (k, rng.integers(0, 90, T)), (p, rng.uniform(0.5, 1.1, T))):
            a.copy_(torch.from_numpy(np.asarray(b)))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        assert torch.equal(eager[0], token) and torch.equal(eager[1], logprob)
        run(ctx, x, u.cpu().numpy(), temperature=t.cpu().numpy(), top_k=k.cpu().numpy(), top_p=p.cpu().numpy())


def test_no_rows_and_refused_arguments(ctx):
    import torch

    import paper_2608_08751_amd as ivf

    x, u = torch.zeros(3, 10, device="cuda"), torch.zeros(3, device="cuda")
    token, logprob = ivf.ivf_sample(ctx, x[:0], u[:0])
    assert token.shape == logprob.shape == (0,)
    for args, more, error in (((x.double(), u), {}, TypeError), ((x.cpu(), u), {}, TypeError), ((x.t()[:3], u), {}, ValueError),
                              ((x[0], u), {}, ValueError), ((x, u[:2]), {}, ValueError), ((x, u.double()), {}, TypeError),
                              ((x, u), dict(top_k=u), TypeError), ((x, u), dict(temperature=u[:1]), ValueError),
                              ((x, u), dict(min_p=u.cpu()), TypeError), ((x[:, :0], u), {}, ValueError),
                              ((torch.zeros(1, 2**20 + 1, device="cuda"), u[:1]), {}, ivf.IvfError),
                              ((x.clone().requires_grad_(), u), {}, RuntimeError)):
        with pytest.raises(error):
            ivf.ivf_sample(ctx, *args, **more)


def test_a_temperature_that_requires_a_gradient_is_refused(ctx):
    """The log-probabilities go by it, and there is no backward pass; without gradients it is taken as it is."""
    import torch

    import paper_2608_08751_amd as ivf

    x, u = torch.randn(3, 10, device="cuda"), torch.rand(3, device="cuda")
    t = torch.ones(3, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError):
        ivf.ivf_sample(ctx, x, u, temperature=t)
    want = ivf.ivf_sample(ctx, x, u, temperature=t.detach())
    with torch.no_grad():
        got = ivf.ivf_sample(ctx, x, u, temperature=t)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
