"""Edges of the paged 4-bit key/value cache's operators on the GPU, against the definitions
in fp64 (tests/kv_model.py). Attention is held to what its roundings allow, as in
tests/test_gpu_kv.py (check_attend)."""
import numpy as np
import pytest

import kv_model as M
from test_gpu_kv import as_np, batch, check_attend, ctx, dev, dtype_of, ints, make, queries  # noqa: F401 (ctx: a fixture)

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f16"]


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
