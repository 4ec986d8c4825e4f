"""The C entry points that share, copy and reclaim the cache's blocks, on the CPU: what they refuse, before any
device is touched (fake device addresses, never dereferenced; a validation-only context reports IVF_EDEVICE
once every check has passed)."""
import pytest

from paper_2608_08751_amd import _binding as B
from test_abi_kv import BAD_CACHES, GB, P, cache, vctx  # noqa: F401 (vctx: a fixture)


def fork(ctx, parent=P(0), child=P(GB), n=10, cached=P(2 * GB), rows=20, bs=64, table=P(3 * GB), cols=40, free=P(4 * GB),
         n_free=100, source=P(5 * GB), to=P(6 * GB), info=P(7 * GB)):
    return ctx.lib.ivf_kv_fork(ctx.handle, parent, child, n, cached, rows, bs, table, cols, free, n_free, source, to, info)


def test_fork_refusals(vctx):  # noqa: F811
    assert fork(vctx) == B.IVF_EDEVICE  # every check passed
    assert fork(vctx, info=None) == fork(vctx, free=None, n_free=0) == B.IVF_EDEVICE
    assert fork(vctx, n=0, parent=None, child=None, source=None, to=None) == B.IVF_EDEVICE
    assert fork(vctx, n=0, info=None, table=None) == B.IVF_OK
    assert fork(vctx, n=16384, rows=16384) == B.IVF_EDEVICE
    for bad in (dict(bs=20), dict(n=16385), dict(rows=16385)):
        assert fork(vctx, **bad) == B.IVF_EUNSUPPORTED, bad
    for bad in (dict(n=-1), dict(n_free=-1), dict(rows=0), dict(cols=0), dict(cols=(1 << 31) // 64), dict(parent=None),
                dict(child=None), dict(cached=None), dict(table=None), dict(free=None), dict(source=None), dict(to=None),
                dict(parent=P(2)), dict(info=P(7 * GB + 4)), dict(table=P(0)), dict(cached=P(GB)), dict(source=P(4 * GB)),
                dict(to=P(5 * GB)), dict(info=P(3 * GB)), dict(cached=P(3 * GB))):
        assert fork(vctx, **bad) == B.IVF_EINVAL, bad
        assert vctx.error()
    assert vctx.lib.ivf_kv_fork(None, None, None, 0, None, 0, 64, None, 0, None, 0, None, None, None) == B.IVF_EINVAL


def copy(ctx, dst=None, src=None, to=P(6 * GB), source=P(7 * GB), n=10):
    return ctx.lib.ivf_kv_copy(ctx.handle, dst or cache(), src or cache(), to, source, n)


def test_copy_refusals(vctx):  # noqa: F811
    far = dict(records=P(10 * GB), summary=P(14 * GB), weight=P(15 * GB))
    assert copy(vctx) == B.IVF_EDEVICE
    assert copy(vctx, n=0, to=None, source=None) == B.IVF_OK
    assert copy(vctx, src=cache(blocks=5, **far)) == copy(vctx, dst=cache(**far)) == B.IVF_EDEVICE
    assert copy(vctx, src=cache(blocks=500)) == B.IVF_EDEVICE  # the same arrays, seen shorter
    assert copy(vctx, n=1 << 31) == B.IVF_EUNSUPPORTED
    for other in (dict(bs=32), dict(heads=4), dict(dim=64), dict(dtype=B.IVF_F16)):
        assert copy(vctx, src=cache(**far, **other)) == B.IVF_EINVAL, other
    for bad in (dict(n=-1), dict(to=None), dict(source=None), dict(to=P(6 * GB + 2)), dict(source=P(64)), dict(to=P(4 * GB)),
                dict(src=cache(records=P(4096))), dict(src=cache(records=P(10 * GB))),
                dict(src=cache(**{**far, "weight": P(4 * GB)}))):
        assert copy(vctx, **bad) == B.IVF_EINVAL, bad
        assert vctx.error()
    for bad, status in BAD_CACHES:
        assert copy(vctx, cache(**bad)) == status and copy(vctx, src=cache(**bad)) == status, bad
    assert vctx.lib.ivf_kv_copy(vctx.handle, None, None, None, None, 1) == B.IVF_EINVAL


def reclaim(ctx, cached=P(0), rows=20, bs=64, table=P(GB), cols=40, blocks=1000, moves=10, free=P(2 * GB), source=P(3 * GB),
            to=P(4 * GB), info=P(5 * GB)):
    return ctx.lib.ivf_kv_reclaim(ctx.handle, cached, rows, bs, table, cols, blocks, moves, free, source, to, info)


def test_reclaim_refusals(vctx):  # noqa: F811
    assert reclaim(vctx) == B.IVF_EDEVICE
    assert reclaim(vctx, rows=0, cached=None, table=None, cols=0) == B.IVF_EDEVICE
    assert reclaim(vctx, moves=0, source=None, to=None) == reclaim(vctx, free=None) == reclaim(vctx, info=None) == B.IVF_EDEVICE
    assert reclaim(vctx, moves=0, free=None, info=None) == B.IVF_OK  # nothing is asked for
    assert reclaim(vctx, bs=8) == B.IVF_EUNSUPPORTED
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=(1 << 31) // 64), dict(blocks=0), dict(blocks=1 << 31), dict(moves=-1),
                dict(moves=1 << 31), dict(cached=None), dict(table=None), dict(source=None), dict(to=None), dict(table=P(2)),
                dict(free=P(2 * GB + 1)), dict(info=P(5 * GB + 4)), dict(table=P(0)), dict(free=P(0)), dict(source=P(2 * GB)),
                dict(to=P(3 * GB)), dict(info=P(GB)), dict(free=P(GB))):
        assert reclaim(vctx, **bad) == B.IVF_EINVAL, bad
        assert vctx.error()
    assert vctx.lib.ivf_kv_reclaim(None, None, 0, 64, None, 0, 1, 0, None, None, None, None) == B.IVF_EINVAL


@pytest.mark.parametrize("rows,cols,blocks,moves", [(20, 40, 1000, 10), (64, 300, 1000, 0), (64, 300, 1000, 5), (2, 3, 1 << 19, 0),
                                                    (1 << 20, 2000, (1 << 31) - 1, 9), (0, 0, 1 << 20, 3)])
def test_reclaim_bytes_are_what_the_call_asks_for(vctx, rows, cols, blocks, moves):  # noqa: F811
    need = vctx.lib.ivf_kv_reclaim_bytes(rows, 64, cols, blocks, moves)
    vctx.lib.ivf_set_workspace(vctx.handle, None, 0)
    far = dict(table=P(1 << 34), free=P(1 << 35), source=P(1 << 36), to=P(1 << 37), info=P(1 << 38))
    assert reclaim(vctx, rows=rows, cols=cols, blocks=blocks, moves=moves, **far) == (B.IVF_ENOMEM if need else B.IVF_EDEVICE)
    assert not need or str(need) in vctx.error()


def test_reclaim_bytes_of_refused_sizes(vctx):  # noqa: F811
    for sizes in ((-1, 64, 40, 1 << 20, 0), (1, 20, 40, 1 << 20, 0), (1, 64, 0, 1 << 20, 0), (1, 64, 40, 0, 0),
                  (1, 64, 40, 1 << 31, 0), (1, 64, 40, 1 << 20, -1), (1, 64, 1 << 30, 1 << 20, 0), (1 << 31, 64, 40, 1 << 20, 0)):
        assert vctx.lib.ivf_kv_reclaim_bytes(*sizes) == 0, sizes
