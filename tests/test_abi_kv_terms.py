"""The attention call with terms in its scores, on the CPU: what it refuses, before any device is touched (fake device
addresses, never dereferenced; a validation-only context reports IVF_EDEVICE once every check has passed)."""
import ctypes
import math

import pytest

from paper_2608_08751_amd import _binding as B
from test_abi_kv import GB, P, cache, vctx  # noqa: F401 (vctx: a fixture)


def attend(ctx, terms=None, T=50, longest=50, scale=0.1, out=P(12 * GB), lse=P(13 * GB), blocks=None, count=0):
    return ctx.lib.ivf_kv_attend_terms(ctx.handle, cache(), P(6 * GB), 4096, 128, 32, T, P(7 * GB), P(8 * GB), P(9 * GB),
                                       P(10 * GB), 5, 100, blocks, count, scale, longest, terms, out, lse)


def given(cap=0.0, slopes=None, first=None, prefix=None):
    return ctypes.byref(B._KvTermsStruct(cap, slopes, first, prefix))


@pytest.fixture()
def ctx(vctx):  # noqa: F811
    vctx.lib.ivf_set_workspace(vctx.handle, (1 << 46) + (1 << 40), 1 << 36)
    return vctx


def test_terms_that_are_taken(ctx):
    assert attend(ctx) == attend(ctx, given()) == B.IVF_EDEVICE  # every check passed
    for terms in (dict(cap=30.0), dict(cap=2.0**-40), dict(cap=2.0**40), dict(slopes=P(14 * GB)), dict(first=P(14 * GB + 4)),
                  dict(prefix=P(14 * GB)), dict(cap=1.0, slopes=P(14 * GB), first=P(15 * GB), prefix=P(15 * GB))):
        assert attend(ctx, given(**terms)) == B.IVF_EDEVICE, terms
        assert attend(ctx, given(**terms), blocks=P(16 * GB), count=8) == B.IVF_EDEVICE, terms
    assert attend(ctx, given(cap=5.0), scale=0.0) == attend(ctx, given(cap=5.0), scale=-3.0) == B.IVF_EDEVICE
    assert attend(ctx, given(cap=math.nan), T=0) == B.IVF_OK


def test_terms_that_are_refused(ctx):
    for cap in (-1.0, math.nan, math.inf, -math.inf, 2.0**-41, 2.0**41, 1e-45):
        assert attend(ctx, given(cap=cap)) == B.IVF_EINVAL, cap
        assert "cap" in ctx.error()
    for scale, cap in ((1e30, 1e-12), (1e-30, 1e12), (1e-45, 1.0)):  # scale / cap beyond fp32, or not normal
        assert attend(ctx, given(cap=cap), scale=scale) == B.IVF_EINVAL, (scale, cap)
        assert "cap" in ctx.error()
    for terms in (dict(slopes=P(14 * GB + 2)), dict(first=P(14 * GB + 1)), dict(prefix=P(14 * GB + 3)), dict(slopes=P(12 * GB)),
                  dict(first=P(12 * GB + 64)), dict(prefix=P(13 * GB))):
        assert attend(ctx, given(**terms)) == B.IVF_EINVAL, terms
    assert attend(ctx, given(cap=1.0), scale=math.inf) == B.IVF_EINVAL
    assert ctx.lib.ivf_kv_attend_terms(None, None, None, 0, 0, 0, 0, None, None, None, None, 0, 0, None, 0, 0.0, 0, None, None, None) == B.IVF_EINVAL


def test_the_workspace_is_that_of_the_call_without_terms(ctx):
    ctx.lib.ivf_set_workspace(ctx.handle, None, 0)
    need = ctx.lib.ivf_kv_attend_bytes(cache(), 32, 50, 5, 100, 0, 50)
    assert attend(ctx, given(cap=1.0)) == (B.IVF_ENOMEM if need else B.IVF_EDEVICE)
