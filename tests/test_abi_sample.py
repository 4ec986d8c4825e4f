"""The C entry point of token sampling on the CPU: what it refuses, before any device is touched (fake device addresses,
never dereferenced; a validation-only context reports IVF_EDEVICE once every check has passed)."""
from paper_2608_08751_amd import _binding as B
from test_abi_kv import GB, P, vctx  # noqa: F401 (vctx: a fixture)


def sample(ctx, logits=P(0), dt=B.IVF_BF16, stride=1024, T=10, V=1000, uniform=P(GB), temperature=P(2 * GB), top_k=P(3 * GB),
           top_p=P(4 * GB), min_p=P(5 * GB), token=P(6 * GB), logprob=P(7 * GB)):
    return ctx.lib.ivf_sample(ctx.handle, logits, dt, stride, T, V, uniform, temperature, top_k, top_p, min_p, token, logprob)


def test_sample_refusals(vctx):  # noqa: F811
    vctx.lib.ivf_set_workspace(vctx.handle, (1 << 46) + (1 << 40), 1 << 36)
    assert sample(vctx) == B.IVF_EDEVICE  # every check passed
    assert sample(vctx, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None) == B.IVF_EDEVICE
    assert sample(vctx, T=0, logits=None, uniform=None, token=None) == B.IVF_OK
    assert sample(vctx, logits=P(2)) == sample(vctx, stride=0) == sample(vctx, stride=3) == B.IVF_EDEVICE
    assert sample(vctx, dt=B.IVF_F32, logits=P(4), V=1 << 20, stride=1 << 20) == B.IVF_EDEVICE
    assert sample(vctx, dt=B.IVF_U8) == sample(vctx, dt=9) == sample(vctx, V=(1 << 20) + 1) == B.IVF_EUNSUPPORTED
    assert sample(vctx, T=1 << 22, stride=0, uniform=P(8 * GB)) == sample(vctx, T=1 << 60) == B.IVF_EUNSUPPORTED
    for bad in (dict(T=-1), dict(V=0), dict(stride=-1), dict(stride=(1 << 40) + 1), dict(logits=None), dict(uniform=None),
                dict(token=None), dict(logits=P(1)), dict(dt=B.IVF_F32, logits=P(2)), dict(uniform=P(GB + 2)),
                dict(top_k=P(3 * GB + 1)), dict(logprob=P(7 * GB + 2)), dict(token=P(0)), dict(logprob=P(GB)),
                dict(token=P(3 * GB)), dict(logprob=P(6 * GB + 4))):
        assert sample(vctx, **bad) == B.IVF_EINVAL, bad
        assert vctx.error()
    assert vctx.lib.ivf_sample(None, None, 2, 0, 0, 1, None, None, None, None, None, None, None) == B.IVF_EINVAL


def test_sample_bytes_are_what_the_call_asks_for(vctx):  # noqa: F811
    off = dict(temperature=None, top_k=None, top_p=None, min_p=None)
    for T, V in ((1, 1), (1, 32_000), (3, 1 << 20), (64, 128_000), (250, 100_003), (300, 1000), (5000, 20_000)):
        for cuts in (0, 1):
            need = vctx.lib.ivf_sample_bytes(T, V, cuts)
            vctx.lib.ivf_set_workspace(vctx.handle, None, 0)
            got = sample(vctx, T=T, V=V, stride=V, **({} if cuts else off))
            assert got == (B.IVF_ENOMEM if need else B.IVF_EDEVICE), (T, V, cuts)
            assert not need or str(need) in vctx.error()
            vctx.lib.ivf_set_workspace(vctx.handle, (1 << 46) + (1 << 40), need)
            assert sample(vctx, T=T, V=V, stride=V, **({} if cuts else off)) == B.IVF_EDEVICE
    for T, V in ((0, 100), (-1, 100), (1, 0), (1, (1 << 20) + 1), (1 << 22, 100_000), (1 << 60, 100_000)):
        assert vctx.lib.ivf_sample_bytes(T, V, 1) == 0
