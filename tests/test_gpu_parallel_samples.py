"""The example that forks prompts into samples, decodes them with sampled tokens and moves together what is left."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "parallel_samples.py")
    spec = importlib.util.spec_from_file_location("parallel_samples", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("kw", [dict(), dict(prompts=3, samples=5, prompt=150, heads=1, group=7, dim=96, block_size=16, window=40),
                                dict(prompts=1, samples=2, prompt=31, steps=3, vocab=301, window=9)], ids=["default", "odd", "small"])
def test_parallel_samples(example, kw):
    import torch

    for dtype, u in ((torch.bfloat16, 2.0**-8), (torch.float16, 2.0**-11)):
        r = example.run(dtype=dtype, **kw)
        # outputs of weighted means: their rounding and the probabilities', u / 2 each of the largest value (about
        # four times the largest output, as values here are of one normal distribution and outputs of the mean of some)
        assert r["error"] <= 4 * u + 1e-4
        assert r["same"]
        samples, prompts = kw.get("samples", 4), kw.get("prompts", 2)
        assert r["live"] == prompts * samples - prompts * samples // 2
        assert r["in_use"] < r["before"] and r["moved"] > 0
        assert r["tokens"].shape == (prompts * samples, 2 * kw.get("steps", 12))
        assert 0 <= int(r["tokens"].min()) and int(r["tokens"].max()) < kw.get("vocab", 5000)


@pytest.mark.parametrize("kw", [dict(), dict(prompts=3, samples=5, prompt=150, heads=1, group=7, dim=96, block_size=16, window=40),
                                dict(prompts=1, samples=2, prompt=31, steps=3, vocab=301, window=9)], ids=["default", "odd", "small"])
def test_every_step_goes_on_from_the_tokens_drawn(example, kw, monkeypatch):
    """What each step sampled, recorded by the captured step itself, against the tokens that the example returns: the last
    sample is live beside the batch's padding."""
    import torch

    prompts, samples, steps = kw.get("prompts", 2), kw.get("samples", 4), kw.get("steps", 12)
    rows = prompts * (1 + samples)
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    tokens, requests = (torch.full((2 * steps + 1, rows), -2, dtype=torch.int32, device="cuda") for _ in range(2))
    plan_of, sample_of, plans = example.ivf.ivf_kv_plan, example.ivf.ivf_sample, []

    def plan(*args, **more):
        plans.append(plan_of(*args, **more))
        return plans[-1]

    def sample(*args, **more):
        token, logprob = sample_of(*args, **more)
        tokens.index_copy_(0, count, token[None])
        requests.index_copy_(0, count, plans[-1].request[None])
        count.add_(1)
        return token, logprob

    monkeypatch.setattr(example.ivf, "ivf_kv_plan", plan)
    monkeypatch.setattr(example.ivf, "ivf_sample", sample)
    got = example.run(**kw)["tokens"]
    assert int(count) == 2 * steps + 1  # the step outside the graph, then every replay
    tokens, requests = tokens[1:].tolist(), requests[1:].tolist()
    for i in range(2 * steps):
        live = [r for r in requests[i] if r >= 0]
        assert live == [r for r in range(prompts, rows) if i < steps or (r - prompts) % 2 == 0]
        want = got[:, i - 1].tolist() if i else [None] * (rows - prompts)
        for r, token in zip(live, tokens[i]):
            want[r - prompts] = token
        assert got[:, i].tolist() == want, i
