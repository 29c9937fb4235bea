"""What the operators' workspace queries promise over a range of rows (no GPU needed)."""

import ctypes
import os

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

ROWS = sorted({1, 2, 3, 5, 63, 64, 65, 255, 257, 512, 513, 767, 769, 1023, 1024, 1025, 1279, 1281, 2048, 4999, 5119, 5121, 20000,
               138240, 10 ** 7})
COLS = [1, 64, 511, 512, 513, 768, 1001, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 20000]


@pytest.mark.parametrize("cols", COLS)
def test_norm_of_more_rows_serves_fewer(cols):
    need = [P.terra_rmsnorm_bwd_workspace_bytes(r, cols) for r in ROWS]
    assert need == sorted(need) and need[0] > 0


def test_norm_call_takes_what_any_larger_query_gives():
    """The workspace check alone: a workspace at an odd address is refused as such only once it is large enough."""
    from paper_2608_15211_amd import operators as ops
    A = 1 << 20
    for cols in COLS:
        for r in ROWS:
            n = P.terra_rmsnorm_bwd_workspace_bytes(r, cols)
            d = ops.terra_rmsnorm_desc(r, cols, 0.0, cols, cols, cols, cols, 0)
            call = lambda b: ops.lib().terra_rmsnorm_bwd(d, 1, A, A, A, None, None, None, A, A + 4, b, None)  # noqa: E731
            assert call(ctypes.c_size_t(n)) == 1 and b"aligned" in P.lib().terra_last_error()
            assert call(ctypes.c_size_t(3)) == 3


def test_linear_is_for_its_own_sizes():
    """Products of few tiles take contraction slices, and more tokens none: the header's warning."""
    f = P.terra_linear_fwd_workspace_bytes
    assert f(1024, 768, 4096, "bf16") > f(138240, 768, 4096, "bf16") == 0
