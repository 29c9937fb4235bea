"""Outputs over inputs: the calls that the header allows in place, and refusals of those that
would read what they have written (no GPU needed: every call is refused or has no rows).

The allowed ones are told from the refused by the last check, the workspace's or the
launch's: nothing is launched, since no device is there."""

import os

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

INVALID = 1
BF16, F32 = 1, 0
A, B, C, D, E = ((i + 1) << 24 for i in range(5))       # addresses that are never used


@pytest.fixture(autouse=True)
def _no_gpu():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where nothing can be launched")


def ops():
    from paper_2608_15211_amd import operators
    return operators


def refused(fn, *args):
    """Whether the call is refused for its addresses or strides."""
    s = fn(*args)
    message = P.lib().terra_last_error()
    assert s != 0
    if s == INVALID:
        assert b"in place" in message or b"same memory" in message, message
    return s == INVALID


def norm_fwd(x=A, res=B, z=C, y=D, q=None, **d):
    kw = dict(rows=3, cols=8, eps=1e-5, x_ld=8, res_ld=8, z_ld=8, y_ld=8, q_ld=8)
    kw.update(d)
    return refused(ops().lib().terra_rmsnorm_fwd, ops().terra_rmsnorm_desc(**kw), BF16, x, res, None, z, y, q, q and E, None, None)


def test_norm_forward():
    assert not norm_fwd()
    assert not norm_fwd(y=A) and not norm_fwd(z=A) and not norm_fwd(z=B) and not norm_fwd(y=A, z=B) and not norm_fwd(y=B, z=A)
    assert norm_fwd(y=C) and norm_fwd(y=A, z=A) and norm_fwd(z=B, y=B)
    assert norm_fwd(y=A, x_ld=16) and norm_fwd(z=A, z_ld=9) and norm_fwd(z=B, res_ld=9) and norm_fwd(y=B, y_ld=16)
    assert norm_fwd(q=A) and norm_fwd(q=B) and norm_fwd(q=C) and norm_fwd(q=D)
    assert not norm_fwd(res=A) and not norm_fwd(res=A, z=A) and norm_fwd(res=A, res_ld=16, z=A)


def norm_bwd(dy=A, z=B, dz=C, dx=D, **d):
    kw = dict(rows=3, cols=8, eps=0.0, x_ld=8, res_ld=8, z_ld=8, y_ld=8, q_ld=0)
    kw.update(d)
    return refused(ops().lib().terra_rmsnorm_bwd, ops().terra_rmsnorm_desc(**kw), BF16, dy, z, E, None, dz, dx, None, None, 0, None)


def test_norm_backward():
    assert not norm_bwd() and not norm_bwd(dx=A) and not norm_bwd(dx=B) and not norm_bwd(dx=C) and not norm_bwd(dz=A, dx=A)
    assert norm_bwd(dx=A, x_ld=16) and norm_bwd(dx=B, z_ld=16) and norm_bwd(dx=C, res_ld=16)


def lin_fwd(x=A, w=B, res=None, y=C, pre=None, **d):
    kw = dict(M=3, N=16, K=16, x_ld=16, w_ld=16, y_ld=16, res_ld=16, pre_ld=16, act=0, out_dtype=BF16)
    kw.update(d)
    return refused(ops().lib().terra_linear_fwd, ops().terra_linear_desc(**kw), BF16, x, None, w, None, None, res, y, pre, None, 0, None)


def test_linear_forward():
    assert not lin_fwd() and not lin_fwd(res=C) and not lin_fwd(res=D, pre=E) and not lin_fwd(res=D, pre=D) and not lin_fwd(res=A)
    assert lin_fwd(y=A) and lin_fwd(y=B) and lin_fwd(pre=A) and lin_fwd(pre=B) and lin_fwd(pre=C)
    assert lin_fwd(res=C, res_ld=32) and lin_fwd(res=D, pre=D, pre_ld=32)


def lin_bwd(dy=A, x=B, w=C, pre=None, dx=D, dw=E, db=None, act=0, **d):
    kw = dict(M=3, N=16, K=16, x_ld=16, w_ld=16, y_ld=16, pre_ld=16, dx_ld=16, dw_ld=16, act=act)
    kw.update(d)
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    return refused(ops().lib().terra_linear_bwd, ops().terra_linear_desc(**kw), BF16, dy, x, w, pre, dx, dw, BF16, db,
                   (ws.data_ptr() + 15) // 16 * 16, 1 << 15, None)


def test_linear_backward():
    assert not lin_bwd() and not lin_bwd(dx=B, dw=None) and not lin_bwd(dx=None, dw=C) and not lin_bwd(x=A)
    assert lin_bwd(dx=A) and lin_bwd(dx=B) and lin_bwd(dx=C) and lin_bwd(dw=A) and lin_bwd(dw=B) and lin_bwd(dx=D, dw=D)
    assert lin_bwd(dw=C) and lin_bwd(dx=None, dw=A)
    F = 9 << 24
    assert lin_bwd(pre=F, act=2, dx=F) and lin_bwd(pre=F, act=2, dw=F) and not lin_bwd(pre=F, act=0, dx=F)


def rope(q, k, fn="terra_rope_fwd"):
    o = ops()
    T = lambda i, out: o.terra_rope_tensor(i, out, 2, 128, 64, 128, 64)  # noqa: E731
    return refused(getattr(o.lib(), fn), P.terra_plan_rope(64), BF16, 4, None, 2, 2, T(*q), k and T(*k), None)


@pytest.mark.parametrize("fn", ["terra_rope_fwd", "terra_rope_bwd"])
def test_rope(fn):
    assert not rope((A, B), None, fn) and not rope((A, A), (B, B), fn) and not rope((A, B), (A, C), fn)
    assert rope((A, C), (B, C), fn) and rope((A, B), (B, C), fn) and rope((A, C), (B, A), fn) and rope((A, B), (B, A), fn)
