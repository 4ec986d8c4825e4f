"""The key/value cache's C entry points on the CPU: what they refuse, before any
device is touched (a validation-only context reports IVF_EDEVICE once every
check has passed)."""
import ctypes

import pytest

import paper_2608_08751_amd as ivf
from paper_2608_08751_amd import _binding as B

BASE = 0x7F0000000000  # fake device addresses, never dereferenced
GB = 1 << 30


def P(off):
    return ctypes.c_void_p(BASE + off)


@pytest.fixture()
def vctx():
    ctx = ivf.Context(-1)
    yield ctx
    ctx.close()


def cache(records=P(0), summary=P(4 * GB), weight=P(5 * GB), blocks=1000, bs=64, heads=8, dim=128, dtype=B.IVF_BF16):
    return ctypes.byref(B._KvCacheStruct(records, summary, weight, blocks, bs, heads, dim, dtype))


BAD_CACHES = [
    (dict(bs=48), B.IVF_EUNSUPPORTED), (dict(bs=0), B.IVF_EUNSUPPORTED), (dict(bs=256), B.IVF_EUNSUPPORTED),
    (dict(dim=100), B.IVF_EUNSUPPORTED), (dict(dim=32), B.IVF_EUNSUPPORTED), (dict(dtype=B.IVF_F32), B.IVF_EUNSUPPORTED),
    (dict(dtype=9), B.IVF_EUNSUPPORTED), (dict(heads=0), B.IVF_EINVAL), (dict(blocks=0), B.IVF_EINVAL),
    (dict(blocks=1 << 31), B.IVF_EINVAL), (dict(records=None), B.IVF_EINVAL), (dict(summary=None), B.IVF_EINVAL),
    (dict(weight=P(5 * GB + 4)), B.IVF_EINVAL),
]


def plan(ctx, cached=P(0), added=P(GB), n=10, bs=64, table=P(2 * GB), cols=40, free=P(3 * GB), n_free=100, T=50,
         start=P(4 * GB), slots=P(5 * GB), request=P(6 * GB), position=P(7 * GB), info=P(8 * GB)):
    return ctx.lib.ivf_kv_plan(ctx.handle, cached, added, n, bs, table, cols, free, n_free, T, start, slots, request,
                               position, info)


def test_plan_refusals(vctx):
    assert plan(vctx) == B.IVF_EDEVICE  # every check passed
    assert plan(vctx, info=None) == B.IVF_EDEVICE
    assert plan(vctx, free=None, n_free=0) == B.IVF_EDEVICE
    assert plan(vctx, T=0, slots=None, request=None, position=None) == B.IVF_EDEVICE
    assert plan(vctx, cached=P(4), free=P(3 * GB + 12)) == B.IVF_EDEVICE  # aligned to their elements
    assert plan(vctx, n=0) == B.IVF_OK
    assert plan(vctx, bs=20) == B.IVF_EUNSUPPORTED
    assert plan(vctx, n=16385) == B.IVF_EUNSUPPORTED
    assert plan(vctx, T=1 << 31) == B.IVF_EUNSUPPORTED
    for bad in (dict(n=-1), dict(T=-1), dict(n_free=-1), dict(cols=0), dict(cols=(1 << 31) // 64), dict(cached=None),
                dict(added=None), dict(table=None), dict(free=None), dict(start=None), dict(slots=None),
                dict(request=None), dict(position=None), dict(cached=P(2)), dict(slots=P(5 * GB + 4)),
                dict(table=P(0)), dict(start=P(2 * GB)), dict(slots=P(4 * GB)), dict(info=P(5 * GB))):
        assert plan(vctx, **bad) == B.IVF_EINVAL, bad
        assert vctx.error()
    assert vctx.lib.ivf_kv_plan(None, None, None, 1, 64, None, 1, None, 0, 0, None, None, None, None, None) == B.IVF_EINVAL


def append(ctx, c=None, k=P(6 * GB), kt=1536, kh=128, v=P(7 * GB), vt=1024, vh=128, slots=P(8 * GB), T=100):
    return ctx.lib.ivf_kv_append(ctx.handle, c or cache(), k, kt, kh, v, vt, vh, slots, T)


def test_append_refusals(vctx):
    assert append(vctx) == B.IVF_EDEVICE
    assert append(vctx, T=0) == B.IVF_OK
    assert append(vctx, kh=0, kt=0) == B.IVF_EDEVICE  # one row for all
    assert append(vctx, T=1 << 31) == B.IVF_EUNSUPPORTED
    for bad in (dict(T=-1), dict(k=None), dict(v=None), dict(slots=None), dict(k=P(6 * GB + 8)), dict(kt=1028),
                dict(vh=-8), dict(kh=4), dict(slots=P(8 * GB + 4)), dict(k=P(64)), dict(v=P(4 * GB)),
                dict(slots=P(5 * GB)), dict(kt=1 << 31)):
        assert append(vctx, **bad) == B.IVF_EINVAL, bad
    for bad, status in BAD_CACHES:
        assert append(vctx, cache(**bad)) == status, bad
    assert vctx.lib.ivf_kv_append(vctx.handle, None, P(0), 8, 8, P(0), 8, 8, P(0), 1) == B.IVF_EINVAL


def read(ctx, c=None, slots=P(6 * GB), T=100, k=P(7 * GB), v=P(8 * GB), blocks=P(9 * GB), n=10, mean=P(10 * GB)):
    return ctx.lib.ivf_kv_read(ctx.handle, c or cache(), slots, T, k, v, blocks, n, mean)


def test_read_refusals(vctx):
    assert read(vctx) == B.IVF_EDEVICE
    assert read(vctx, k=None) == B.IVF_EDEVICE
    assert read(vctx, n=0, blocks=None, mean=None) == B.IVF_EDEVICE
    assert read(vctx, T=0, n=0) == B.IVF_OK
    assert read(vctx, k=None, v=None, n=0) == B.IVF_OK
    for bad in (dict(T=-1), dict(n=-1), dict(slots=None), dict(blocks=None), dict(mean=None), dict(k=P(7 * GB + 2)),
                dict(v=P(7 * GB)), dict(k=P(0)), dict(mean=P(6 * GB))):
        assert read(vctx, **bad) == B.IVF_EINVAL, bad
    for bad, status in BAD_CACHES:
        assert read(vctx, cache(**bad)) == status, bad


def select(ctx, c=None, q=P(6 * GB), qt=4096, qh=128, heads=32, T=100, request=P(7 * GB), position=P(8 * GB),
           table=P(9 * GB), n=10, cols=500, first=1, last=1, count=16, out=P(10 * GB)):
    return ctx.lib.ivf_kv_select(ctx.handle, c or cache(), q, qt, qh, heads, T, request, position, table, n, cols, first,
                                 last, count, out)


def test_select_refusals(vctx):
    assert select(vctx) == B.IVF_EDEVICE
    assert select(vctx, T=0) == B.IVF_OK
    assert select(vctx, cols=32769, c=cache(bs=16)) == B.IVF_EUNSUPPORTED
    assert select(vctx, T=1 << 31) == B.IVF_EUNSUPPORTED
    for bad in (dict(heads=0), dict(heads=12), dict(first=-1), dict(last=0), dict(count=1), dict(count=4097), dict(T=-1),
                dict(n=0), dict(cols=0), dict(q=None), dict(request=None), dict(position=None), dict(table=None),
                dict(out=None), dict(qt=100), dict(q=P(6 * GB + 2)), dict(out=P(7 * GB)), dict(out=P(4 * GB)),
                dict(position=P(8 * GB + 1))):
        assert select(vctx, **bad) == B.IVF_EINVAL, bad
    for bad, status in BAD_CACHES:
        assert select(vctx, cache(**bad)) == status, bad


def attend(ctx, c=None, q=P(6 * GB), qt=4096, qh=128, heads=32, T=100, start=P(6 * GB + (1 << 29)), request=P(7 * GB),
           position=P(8 * GB), table=P(9 * GB), n=10, cols=500, blocks=None, count=0, scale=0.1, longest=5,
           out=P(10 * GB), lse=P(11 * GB)):
    return ctx.lib.ivf_kv_attend(ctx.handle, c or cache(), q, qt, qh, heads, T, start, request, position, table, n, cols,
                                 blocks, count, scale, longest, out, lse)


def test_attend_refusals(vctx):
    vctx.lib.ivf_set_workspace(vctx.handle, P(64 * GB), 64 * GB)
    assert attend(vctx) == B.IVF_EDEVICE
    assert attend(vctx, lse=None) == B.IVF_EDEVICE
    assert attend(vctx, request=None) == B.IVF_EDEVICE
    assert attend(vctx, blocks=P(12 * GB), count=8, start=None) == B.IVF_EDEVICE
    assert attend(vctx, T=0) == B.IVF_OK
    assert attend(vctx, T=1 << 31) == B.IVF_EUNSUPPORTED
    for bad in (dict(heads=0), dict(heads=12), dict(T=-1), dict(n=0), dict(cols=0), dict(count=3), dict(q=None),
                dict(start=None), dict(position=None), dict(table=None), dict(out=None), dict(longest=0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(blocks=P(12 * GB)),
                dict(blocks=P(12 * GB), count=4097), dict(blocks=P(12 * GB), count=8, request=None),
                dict(out=P(10 * GB + 8)), dict(lse=P(11 * GB + 2)), dict(out=P(6 * GB)), dict(lse=P(10 * GB)),
                dict(out=P(4 * GB))):
        assert attend(vctx, **bad) == B.IVF_EINVAL, bad
    for bad, status in BAD_CACHES:
        assert attend(vctx, cache(**bad)) == status, bad


def test_attend_workspace(vctx):
    f = vctx.lib.ivf_kv_attend_bytes
    need = f(cache(), 32, 2, 2, 500, 0, 1)
    assert need > 0  # two tokens over long tables are split
    assert f(cache(), 32, 4096, 1, 500, 0, 4096) == 0  # many rows are not
    assert f(cache(dim=100), 32, 2, 2, 500, 0, 1) == 0
    assert f(cache(), 31, 2, 2, 500, 0, 1) == 0
    assert f(None, 32, 2, 2, 500, 0, 1) == 0
    small = dict(T=2, n=2, longest=1)
    vctx.lib.ivf_set_workspace(vctx.handle, P(64 * GB), need - 1)
    assert attend(vctx, **small) == B.IVF_ENOMEM
    assert str(need) in vctx.error()
    vctx.lib.ivf_set_workspace(vctx.handle, P(64 * GB), need)
    assert attend(vctx, **small) == B.IVF_EDEVICE


def test_calls_beyond_a_launch(vctx):
    # a launch holds fewer than 2^32 threads: 2048 / dim tokens of a head take 256, a wave attends for a token
    far = [P(n << 40) for n in range(1, 6)]
    big = dict(c=cache(heads=1), T=(1 << 28) - 16)  # 2^32 - 256 threads
    assert append(vctx, k=far[0], v=far[1], slots=far[2], kt=128, vt=128, **big) == B.IVF_EDEVICE
    assert read(vctx, slots=far[0], k=far[1], v=far[2], n=0, **big) == B.IVF_EDEVICE
    assert read(vctx, slots=far[0], k=far[1], v=far[2], n=17, **big) == B.IVF_EUNSUPPORTED
    big["T"] += 1
    assert append(vctx, k=far[0], v=far[1], slots=far[2], kt=128, vt=128, **big) == B.IVF_EUNSUPPORTED
    assert read(vctx, slots=far[0], k=far[1], v=far[2], n=0, **big) == B.IVF_EUNSUPPORTED
    rows = dict(c=cache(heads=1), heads=1, q=far[0], qt=128, request=far[1], position=P((2 << 40) + (4 << 30)),
                start=far[4], blocks=far[2], count=2, out=far[3], lse=None, longest=1)
    assert attend(vctx, T=(1 << 26) - 16, **rows) == B.IVF_EDEVICE
    assert attend(vctx, T=1 << 26, **rows) == B.IVF_EUNSUPPORTED
    assert select(vctx, c=cache(heads=1), heads=1, q=far[0], qt=128, request=far[1], position=far[2], out=far[3],
                  T=1 << 28) == B.IVF_EDEVICE  # several launches
