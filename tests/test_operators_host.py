"""Host-side checks of the norm, the linear layer and the rotary positions (no
GPU needed): what the C ABI and the binding refuse before any device work, the
workspaces, and the rotary plan against a plain computation."""

import ctypes
import math
import os

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16, F16, E4M3 = 0, 1, 2, 3
A = 1 << 20                 # an address that is never used: every call below is refused, or has no rows


def ops():
    from paper_2608_15211_amd import operators
    return operators


def status(fn, *args):
    s = fn(*args)
    assert (P.lib().terra_last_error() == b"") == (s == OK)
    return s


# --------------------------------------------------------------------- norm
def norm_fwd(dtype=BF16, x=A, res=None, gain=None, z=None, y=A, q=None, qs=None, rstd=None, **d):
    kw = dict(rows=3, cols=8, eps=1e-5, x_ld=8, res_ld=8, z_ld=8, y_ld=8, q_ld=8)
    kw.update(d)
    return status(ops().lib().terra_rmsnorm_fwd, ops().terra_rmsnorm_desc(**kw), dtype, x, res, gain, z, y, q, qs, rstd, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=0), OK), (dict(rows=0, x=None, y=None), OK), (dict(rows=-1), INVALID), (dict(cols=0), INVALID),
    (dict(cols=(1 << 24) + 1, x_ld=1 << 30, y_ld=1 << 30), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(dtype=E4M3), INVALID), (dict(dtype=7), INVALID),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(q=A), INVALID), (dict(qs=A), INVALID), (dict(x_ld=7), INVALID),
    (dict(y_ld=7), INVALID), (dict(res=A, res_ld=0), INVALID), (dict(z=A, z_ld=-8), INVALID), (dict(q=A, qs=A, q_ld=1), INVALID),
    (dict(x_ld=1 << 40), UNSUPPORTED), (dict(x=A + 1), INVALID), (dict(y=A + 2, dtype=F32), INVALID), (dict(gain=A + 2), INVALID),
    (dict(rstd=A + 1), INVALID), (dict(q=A, qs=A + 2), INVALID)])
def test_norm_forward_refuses(kw, want):
    assert norm_fwd(**kw) == want


def norm_bwd(dtype=BF16, dy=A, z=A, rstd=A, gain=None, dz=None, dx=A, dgain=None, ws=None, n=0, **d):
    kw = dict(rows=3, cols=8, eps=0.0, x_ld=8, res_ld=8, z_ld=8, y_ld=8, q_ld=0)
    kw.update(d)
    return status(ops().lib().terra_rmsnorm_bwd, ops().terra_rmsnorm_desc(**kw), dtype, dy, z, rstd, gain, dz, dx, dgain, ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=0), OK), (dict(dx=None), INVALID), (dict(dy=None), INVALID), (dict(z=None), INVALID), (dict(rstd=None), INVALID),
    (dict(dgain=A), WORKSPACE), (dict(dgain=A, ws=A, n=31), WORKSPACE), (dict(dgain=A, ws=A + 4, n=1 << 20), INVALID),
    (dict(dgain=A + 2, ws=A, n=1 << 20), INVALID), (dict(y_ld=1), INVALID), (dict(dz=A, res_ld=1), INVALID), (dict(x_ld=1), INVALID),
    (dict(dtype=5), INVALID)])
def test_norm_backward_refuses(kw, want):
    assert norm_bwd(**kw) == want


def test_norm_workspace():
    assert P.terra_rmsnorm_bwd_workspace_bytes(-1, 8) == 0 and P.terra_rmsnorm_bwd_workspace_bytes(8, 0) == 0
    assert P.terra_rmsnorm_bwd_workspace_bytes(0, 8) == 0
    for rows in (1, 5, 1000, 10 ** 6, 2 ** 40):
        n = P.terra_rmsnorm_bwd_workspace_bytes(rows, 768)
        assert n % (768 * 4) == 0 and 0 < n <= 2048 * 768 * 4


# ------------------------------------------------------------------- linear
def lin_fwd(dtype=BF16, x=A, xs=None, w=A, wsc=None, bias=None, res=None, y=A, pre=None, ws=None, n=0, **d):
    kw = dict(M=3, N=8, K=16, x_ld=16, w_ld=16, y_ld=8, res_ld=8, pre_ld=8, act=0, out_dtype=BF16)
    kw.update(d)
    return status(ops().lib().terra_linear_fwd, ops().terra_linear_desc(**kw), dtype, x, xs, w, wsc, bias, res, y, pre, ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(M=0), OK), (dict(M=0, x=None), OK), (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID),
    (dict(M=1 << 31), UNSUPPORTED), (dict(N=(1 << 26) + 1), UNSUPPORTED), (dict(K=(1 << 26) + 1), UNSUPPORTED), (dict(M=1 << 30, N=1 << 20, y_ld=1 << 20), UNSUPPORTED),
    (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(dtype=F32), UNSUPPORTED), (dict(dtype=9), INVALID),
    (dict(out_dtype=F32), INVALID), (dict(out_dtype=F16), INVALID), (dict(dtype=E4M3), INVALID),
    (dict(dtype=E4M3, xs=A), INVALID), (dict(dtype=E4M3, xs=A, wsc=A, out_dtype=E4M3), INVALID), (dict(xs=A), INVALID), (dict(wsc=A), INVALID),
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(x_ld=15), INVALID), (dict(w_ld=0), INVALID),
    (dict(y_ld=7), INVALID), (dict(res=A, res_ld=7), INVALID), (dict(pre=A, pre_ld=7), INVALID), (dict(x=A + 1), INVALID),
    (dict(y=A + 1), INVALID), (dict(bias=A + 2), INVALID), (dict(M=100, N=64, K=4096, x_ld=4096, w_ld=4096, y_ld=64), WORKSPACE)])
def test_linear_forward_refuses(kw, want):
    assert lin_fwd(**kw) == want


def lin_bwd(dtype=BF16, dy=A, x=A, w=A, pre=None, dx=A, dw=A, dwt=F32, db=A, ws=A, n=1 << 20, **d):
    kw = dict(M=3, N=8, K=16, x_ld=16, w_ld=16, y_ld=8, pre_ld=8, dx_ld=16, dw_ld=16, act=0)
    kw.update(d)
    return status(ops().lib().terra_linear_bwd, ops().terra_linear_desc(**kw), dtype, dy, x, w, pre, dx, dw, dwt, db, ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=F32), UNSUPPORTED), (dict(dtype=E4M3), UNSUPPORTED), (dict(dtype=4), INVALID), (dict(dx=None, dw=None, db=None), INVALID),
    (dict(dwt=F16), INVALID), (dict(dwt=E4M3), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID),
    (dict(act=2), INVALID), (dict(act=2, pre=A, pre_ld=3), INVALID), (dict(dx_ld=15), INVALID), (dict(dw_ld=15), INVALID),
    (dict(y_ld=7), INVALID), (dict(ws=None), WORKSPACE), (dict(n=16), WORKSPACE), (dict(ws=A + 8), INVALID), (dict(dw=A + 2), INVALID),
    (dict(M=-1), INVALID)])
def test_linear_backward_refuses(kw, want):
    assert lin_bwd(**kw) == want


def test_linear_workspaces():
    f, b = P.terra_linear_fwd_workspace_bytes, P.terra_linear_bwd_workspace_bytes
    assert f(0, 8, 8, "bf16") == f(1, 4096, 4096, "bf16") == f(-1, 8, 8, "bf16") == f(8, 8, 8, "f32") == 0
    assert b(8, 8, 8, "e4m3") == 0 and b(8, 0, 8, "bf16") == 0
    assert f(138240, 2304, 768, "bf16") == 0
    assert b(1000, 2000, 512, "f16") >= 1000 * 2000 * 2 + 512 * 2000 * 2
    for M in (0, 1, 63, 1000, 138240):
        assert 0 < b(M, 768, 768, "bf16") < 3 * (M + 768) * 768 * 2 + 64 * 768 * 768 * 4 + 512 * 768 * 4 + (1 << 20)


def test_linear_cases_reach_every_form():
    """The GPU tests' sizes run each of the library's forms (256 compute units)."""
    import test_gpu_linear as cases
    L = P.lib()
    L.terra_internal_linear_form.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    L.terra_internal_linear_wgrad_form.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    few, forms, wgrad = set(), set(), set()
    for M, N, K in cases.SIZES + [(256 * 43 + 19, 1536, 64)]:
        for dtype in (BF16, E4M3):
            f = L.terra_internal_linear_form(M, N, K, dtype, 1)
            (few if M <= 64 else forms).add(f if M <= 64 else (f // 10000, f // 1000 % 10, f // 100 % 10, min(2, f % 100)))
    for M, N, K in cases.BWD:
        f = L.terra_internal_linear_wgrad_form(M, N, K, 1)
        wgrad.add((f // 100, min(2, f % 100)))
    assert few == {1, 2, 4, 11, 12, 14}
    # (whole rounds and a rest, padded, form, in slices)
    assert {f[1:] for f in forms} >= {(0, 8, 1), (0, 2, 1), (0, 2, 2), (0, 0, 1), (0, 0, 2), (1, 8, 1), (1, 2, 1)}
    assert any(f[0] for f in forms)
    assert wgrad >= {(2, 1), (2, 2), (8, 2)}
    # rows at odd places
    assert L.terra_internal_linear_form(333, 130, 70, BF16, 0) // 100 == 0


# --------------------------------------------------------------------- rope
def rope_desc(**kw):
    d = dict(head_dim=64, rot_dim=64, axes=1, layout=1, scaling=0, base=1e4, factor=1.0, orig_len=0.0, beta_fast=32.0, beta_slow=1.0,
             attn_scale=0.0)
    d.update(kw)
    return ops().terra_rope_desc(**d)


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(axes=0), INVALID), (dict(axes=3), INVALID), (dict(rot_dim=0), INVALID), (dict(rot_dim=66), INVALID),
    (dict(rot_dim=33), INVALID), (dict(rot_dim=62, axes=2), INVALID), (dict(head_dim=258), UNSUPPORTED), (dict(head_dim=1, rot_dim=2), INVALID),
    (dict(layout=2), INVALID), (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(base=0.5), INVALID), (dict(base=math.nan), INVALID),
    (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=1, factor=math.inf), INVALID), (dict(scaling=2, rot_dim=2), INVALID),
    (dict(scaling=2, rot_dim=4, axes=2, factor=2.0), INVALID), (dict(scaling=3, factor=2.0), INVALID),
    (dict(scaling=3, factor=2.0, orig_len=64.0, beta_slow=32.0), INVALID), (dict(scaling=3, factor=2.0, orig_len=64.0), OK),
    (dict(attn_scale=-1.0), INVALID), (dict(attn_scale=math.nan), INVALID)])
def test_rope_plan_refuses(kw, want):
    assert status(ops().lib().terra_plan_rope, rope_desc(**kw), ops().terra_rope_plan()) == want


def rope(tokens=4, dtype=BF16, pos=None, h=2, w=2, q=None, k=None, plan=None, fn="terra_rope_fwd"):
    T = lambda **kw: ops().terra_rope_tensor(**{**dict(in_=A, out=A + 4096, heads=2, in_token=128, in_head=64, out_token=128, out_head=64), **kw})  # noqa: E731
    if plan is None:
        plan = P.terra_plan_rope(64)
    return status(getattr(ops().lib(), fn), plan, dtype, tokens, pos, h, w, None if q is False else T(**(q or {})),
                  None if k is None else T(**k), None)


@pytest.mark.parametrize("fn", ["terra_rope_fwd", "terra_rope_bwd"])
@pytest.mark.parametrize("kw,want", [
    (dict(tokens=0), OK), (dict(tokens=0, k={}), OK), (dict(tokens=-1), INVALID), (dict(tokens=1 << 31), UNSUPPORTED), (dict(dtype=E4M3), INVALID),
    (dict(q=False), INVALID), (dict(h=0), INVALID), (dict(h=1 << 16, w=1 << 15), INVALID), (dict(pos=A + 2), INVALID),
    (dict(q=dict(heads=0)), INVALID), (dict(q=dict(in_=None)), INVALID), (dict(k=dict(out=None)), INVALID), (dict(q=dict(in_=A + 1)), INVALID),
    (dict(q=dict(out=A + 2), dtype=F32), INVALID), (dict(q=dict(in_token=-1)), INVALID), (dict(q=dict(in_head=1 << 31)), INVALID),
    (dict(q=dict(out_token=100)), INVALID), (dict(k=dict(out_head=63)), INVALID), (dict(q=dict(out_token=0)), INVALID),
    (dict(q=dict(out=A, in_token=256)), INVALID), (dict(q=dict(heads=200, out_token=1 << 14), k=dict(heads=57, out_token=1 << 14)), UNSUPPORTED)])
def test_rope_refuses(kw, want, fn):
    assert rope(fn=fn, **kw) == want


def test_rope_refuses_a_made_up_plan():
    p = ops().terra_rope_plan(rope_desc(), 16, 1.0)
    assert rope(plan=p, tokens=0) == INVALID
    assert rope(plan=ops().terra_rope_plan(), tokens=0) == INVALID


@pytest.mark.parametrize("kw", [
    dict(head_dim=64), dict(head_dim=128, rot_dim=96, axes=2, base=100.0), dict(head_dim=64, scaling="linear", factor=4.0),
    dict(head_dim=64, scaling="ntk", factor=8.0, base=1e6), dict(head_dim=256, scaling="yarn", factor=16.0, orig_len=4096),
    dict(head_dim=64, scaling="yarn", factor=2.0, orig_len=8192, attn_scale=1.25), dict(head_dim=2), dict(head_dim=64, base=1.0)])
def test_rope_plan_values(kw):
    from operator_refs import rope_freqs
    plan = P.terra_plan_rope(**kw)
    part = kw.get("rot_dim", kw["head_dim"]) // kw.get("axes", 1)
    f = rope_freqs(part, kw.get("base", 1e4), **{n: kw[n] for n in ("scaling", "factor", "orig_len") if n in kw})
    assert plan.pairs == part // 2
    for i, v in enumerate(f):
        # float64 pow and products on either side: a few 2^-52, and half a 2^-64 turn
        assert abs(plan.turns[i] / 2.0 ** 64 - v / (2 * math.pi)) <= 1e-13 * v + 2.0 ** -63
    assert not any(plan.turns[part // 2:])
    want = kw.get("attn_scale") or (0.1 * math.log(kw["factor"]) + 1 if kw.get("scaling") == "yarn" else 1.0)
    assert abs(plan.scale - want) < 1e-6


# ------------------------------------------------------------- the binding
def test_binding_refuses_host_tensors_and_names():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(16, 8, dtype=torch.bfloat16)
    for call in (lambda: P.terra_rmsnorm_fwd(x), lambda: P.terra_linear_fwd(x, w), lambda: P.terra_linear_bwd(x, x, w),
                 lambda: P.terra_rmsnorm_bwd(x, x, torch.zeros(4)), lambda: P.terra_rope_fwd(P.terra_plan_rope(8), x[:, None], grid=(2, 2))):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="layout"):
        P.terra_plan_rope(64, layout="thirds")
    with pytest.raises(ValueError, match="scaling"):
        P.terra_plan_rope(64, scaling="more")
    with pytest.raises(P.TerraError):
        P.terra_plan_rope(64, rot_dim=65)


def test_calls_go_to_the_tensors_device(monkeypatch):
    """On another device than the current one: there, on its stream; back afterwards."""
    o, at = ops(), [0]

    class Device:
        def __init__(self, i):
            self.i = i

        def __enter__(self):
            self.was, at[0] = at[0], self.i

        def __exit__(self, *a):
            at[0] = self.was

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(o, "_current_device", lambda: at[0])
    monkeypatch.setattr(o, "_raw_stream", lambda i: 100 + i)
    seen = []
    call = lambda *a: seen.append((at[0], a)) or 0  # noqa: E731
    o._call(call, 0, "x")
    o._call(call, 3, "y")
    assert seen == [(0, ("x", 100)), (3, ("y", 103))] and at[0] == 0


def test_row_strides():
    """Which views are matrices."""
    o, t = ops(), torch.zeros(4, 6, 10)
    assert o._stride(t, "t") == 10
    assert o._stride(t[:, :, 2:7], "t") == 10
    assert o._stride(t[:, 3], "t") == 60
    assert o._stride(t[1:2, :, :3], "t") == 10
    assert o._stride(torch.zeros(10), "t") == 10
    assert o._stride(torch.zeros(30)[::3][:1], "t") == 1
    assert o._stride(torch.zeros(0, 5), "t") == 5
    for bad in (t[:, :4, :], t.transpose(1, 2), t[:, :, ::2], torch.zeros(1, 8).expand(3, 8), torch.zeros(20).as_strided((4, 8), (4, 1))):
        with pytest.raises(ValueError):
            o._stride(bad, "t")


def test_importing_the_package_leaves_torch_out():
    import subprocess
    import sys
    code = "import sys, paper_2608_15211_amd as P; assert 'torch' not in sys.modules; P.terra_plan_rope; assert 'torch' in sys.modules"
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    with pytest.raises(AttributeError):
        P.terra_no_such_call
