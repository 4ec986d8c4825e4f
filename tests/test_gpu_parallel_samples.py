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
