"""Sizes at which the key/value cache's C entry points refuse, on the CPU (fake device
addresses, never dereferenced)."""
import subprocess
import sys

import pytest

from paper_2608_08751_amd import _binding as B
from test_abi_kv import attend, cache, vctx  # noqa: F401 (vctx: a fixture)


# (query heads, T, B, columns, count, longest) that the attention call refuses
REFUSED = [(32, 1 << 40, 1 << 40, 500, 0, 1), (32, 2, 2, (1 << 31) - 1, 0, 1), (1 << 20, 2, 2, 500, 0, 1),
           (32, 2, 2, 500, 5000, 1), (32, 2, 2, 500, -1, 1), (32, 2, 1 << 31, 500, 0, 1), (32, 2, 0, 500, 0, 1),
           (32, 2, 2, 0, 0, 1), (32, 2, 2, 500, 0, 0), (32, -1, 2, 500, 0, 1)]


@pytest.mark.parametrize("sizes", REFUSED)
def test_attend_bytes_of_refused_sizes(vctx, sizes):  # noqa: F811
    assert vctx.lib.ivf_kv_attend_bytes(cache(), *sizes) == 0


def test_attend_bytes_of_a_product_of_2_to_the_64():
    # 2^52 tokens of 4,096 heads, in a process of its own: a division by zero would end it
    code = ("import ctypes\nfrom paper_2608_08751_amd import _binding as B\n"
            "c = B._KvCacheStruct(1 << 20, 1 << 40, 1 << 41, 1000, 64, 4096, 128, B.IVF_BF16)\n"
            "print(B.load_library().ivf_kv_attend_bytes(ctypes.byref(c), 4096, 1 << 52, 1, 500, 8, 1))")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["0"], (r.returncode, r.stderr[-300:])


def test_attend_bytes_are_what_the_call_asks_for(vctx):  # noqa: F811
    for T, n, cols, longest in ((2, 2, 500, 1), (64, 64, 600, 1), (100, 1, 500, 100), (9, 2, 500, 8), (5000, 1, 500, 5000)):
        need = vctx.lib.ivf_kv_attend_bytes(cache(), 32, T, n, cols, 0, longest)
        vctx.lib.ivf_set_workspace(vctx.handle, None, 0)
        got = attend(vctx, T=T, n=n, cols=cols, longest=longest)
        assert got == (B.IVF_ENOMEM if need else B.IVF_EDEVICE)
        assert not need or str(need) in vctx.error()


def test_attend_scales_beyond_fp32_to_the_base_2(vctx):  # noqa: F811
    # scale log2(e) is an fp32 factor: infinite, it would make a score of 0 no number
    vctx.lib.ivf_set_workspace(vctx.handle, (1 << 46) + (1 << 40), 1 << 36)
    for scale in (2.3e38, -2.3e38, 0.0, 1e-45):
        assert attend(vctx, scale=scale) == B.IVF_EDEVICE  # every check passed
    for scale in (2.4e38, -3.4e38, float("inf")):
        assert attend(vctx, scale=scale) == B.IVF_EINVAL
        assert "scale" in vctx.error()
