"""Sizes that do not fit the C ABI's 32 bits are refused and not cut to their low bits (no
GPU needed: tensors without memory, and the library's own checks)."""

import os

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

BIG = 2 ** 32


def meta(*dims, dtype=torch.bfloat16):
    return torch.empty(*dims, dtype=dtype, device="meta")


@pytest.fixture
def ops(monkeypatch):
    """The binding with its device checks and the stream taken out; a call that the library would launch fails the test."""
    from paper_2608_15211_amd import operators as o

    def call(fn, device, *args):
        status = fn(*args, None)
        assert status, "the library took the call"
        P._check(status)

    monkeypatch.setattr(o, "_input", lambda t, name: t.get_device())
    monkeypatch.setattr(o, "_call", call)
    return o


def test_workspace_queries():
    assert P.terra_rmsnorm_bwd_workspace_bytes(8, 768) > 0 and P.terra_linear_bwd_workspace_bytes(100, 64, 64, "bf16") > 0
    assert P.terra_linear_fwd_workspace_bytes(100, 64, 4096, "bf16") > 0
    for cols in (BIG + 768, BIG, 2 ** 31, 2 ** 24 + 1):
        assert P.terra_rmsnorm_bwd_workspace_bytes(8, cols) == 0
    for n in (BIG + 64, 2 ** 31):
        for query in (P.terra_linear_fwd_workspace_bytes, P.terra_linear_bwd_workspace_bytes):
            assert query(100, n, 4096, "bf16") == 0 and query(100, 64, n, "bf16") == 0


def test_norm(ops):
    x = meta(2, BIG + 8)
    for call in (lambda: P.terra_rmsnorm_fwd(x), lambda: P.terra_rmsnorm_bwd(x, x, meta(2, dtype=torch.float32))):
        with pytest.raises(P.TerraError, match="2\\^24"):
            call()


def test_linear(ops):
    ws = meta(1, dtype=torch.uint8)
    with pytest.raises(P.TerraError, match="2\\^26"):
        P.terra_linear_fwd(meta(100, 8), meta(BIG + 8, 8), workspace=ws)
    with pytest.raises(P.TerraError, match="2\\^26"):
        P.terra_linear_fwd(meta(100, BIG + 8), meta(8, BIG + 8), workspace=ws)
    with pytest.raises(P.TerraError, match="2\\^26"):
        P.terra_linear_bwd(meta(100, 8), meta(100, BIG + 8), meta(8, BIG + 8), workspace=ws)


def test_rope(ops):
    plan = P.terra_plan_rope(64)
    with pytest.raises(P.TerraError, match="256 heads"):
        P.terra_rope_fwd(plan, meta(1, BIG + 4, 64), grid=(1, 1))
    with pytest.raises(P.TerraError, match="256 heads"):
        P.terra_rope_bwd(plan, meta(1, 2, 64), meta(1, BIG + 4, 64), grid=(1, 1))
    # the two counts' sum leaves 32 bits
    with pytest.raises(P.TerraError, match="256 heads"):
        P.terra_rope_fwd(plan, meta(1, 2 ** 31 - 1, 64), meta(1, 2 ** 31 - 1, 64), grid=(1, 1))
    for grid in ((BIG + 4, 4), (4, BIG + 4), (-BIG + 2, 2)):
        with pytest.raises(P.TerraError, match="grid_h"):
            P.terra_rope_fwd(plan, meta(16, 2, 64), grid=grid)
    for kw in (dict(head_dim=BIG + 64, rot_dim=64), dict(head_dim=64, rot_dim=BIG + 64), dict(head_dim=64, axes=BIG + 1)):
        with pytest.raises(P.TerraError):
            P.terra_plan_rope(**kw)
