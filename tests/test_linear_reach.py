"""The sizes of test_gpu_linear_reach.py run the forms they are for (no GPU needed)."""

import ctypes
import os

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

BF16, E4M3 = 1, 3


def query(name, *args):
    f = getattr(P.lib(), name)
    f.argtypes = [ctypes.c_int64] + [ctypes.c_int] * (len(args) - 1)
    return f(*args)


def test_few_tokens():
    import test_gpu_linear_reach as cases
    seen = set()
    for M, N, K in cases.FEW:
        for dtype, size in ((BF16, 2), (E4M3, 1)):
            waves, form = query("terra_internal_linear_few_waves", M, N, K, dtype), query("terra_internal_linear_form", M, N, K, dtype, 1)
            seen.add((form, waves))
            mt, rt = form % 10, 1 + form // 10
            at_once = 4 if mt + rt <= 3 else 2 if mt + rt <= 5 else 1       # pieces of 128 bytes whose loads go out together
            if size * K // 128 >= 2 * waves * at_once:
                seen.add("turns of %d" % at_once)
            if waves * mt * rt * 16 * 20 * 4 == 160 * 1024:
                seen.add("all of LDS")
    assert {(1, 4), (1, 8), (1, 16), (2, 16), (4, 16), (12, 16), (12, 8), (14, 16), (14, 8)} <= seen
    assert {"turns of 4", "turns of 2", "turns of 1", "all of LDS"} <= seen


def test_weight_gradients():
    import test_gpu_linear_reach as cases
    for M, N, K in cases.WALKS:
        f = query("terra_internal_linear_wgrad_form", M, N, K, 1)
        assert f // 100 == 8 and -(-N // 256) * -(-K // 256) * (f % 100) > 256 and (N % 256 or K % 256)


def test_tiles():
    import test_gpu_linear_reach as cases
    seen = set()
    for M, N, K in cases.TILES:
        for dtype in (BF16, E4M3):
            f = query("terra_internal_linear_form", M, N, K, dtype, 1)
            seen.add((f // 1000 % 10, f // 100 % 10, min(2, f % 100), f // 10000))
    # (padded, form, in slices, whole rounds and a rest)
    assert {(0, 8, 1, 1), (0, 2, 1, 0), (0, 2, 2, 0), (0, 0, 1, 0), (0, 0, 2, 0), (1, 2, 1, 0), (1, 8, 1, 0)} <= seen
