"""How the example of several samples hands a step's tokens to its requests, on the CPU."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "parallel_samples.py")
    spec = importlib.util.spec_from_file_location("parallel_samples", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("prompts,samples", [(2, 4), (3, 5), (1, 2), (1, 1)])
@pytest.mark.parametrize("half", [False, True])
def test_every_live_request_gets_its_token(example, prompts, samples, half):
    """The ended requests leave as many rows of padding in the batch; the last request is live beside them."""
    rows = prompts * (1 + samples)
    live = [r for r in range(prompts, rows) if not half or (r - prompts) % 2 == 0]
    request = torch.tensor(live + [-1] * (rows - len(live)), dtype=torch.int32)
    token = 1000 + torch.arange(rows, dtype=torch.int32)
    last = torch.arange(rows + 1, dtype=torch.int32)
    example.follow(last, token, request)
    assert last[:rows].tolist() == [1000 + live.index(r) if r in live else r for r in range(rows)]
