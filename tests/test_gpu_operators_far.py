"""The operators on tensors of more than 2^31 elements: zeros but for the last
rows, which are held to float64 (bounds: operator_refs.py)."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
ROWS, COLS, LAST = 950007, 2304, 300      # 2.19e9 elements


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    assert ROWS * COLS > 2 ** 31
    yield
    torch.cuda.empty_cache()


def normal(*dims, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*dims, generator=g, device="cuda")).to(dtype)


def far(*dims, dtype=BF16, seed=0):
    """Zeros; the last LAST rows normal."""
    x = torch.zeros(*dims, dtype=dtype, device="cuda")
    x[-LAST:] = normal(LAST, *dims[1:], seed=seed).to(dtype)
    return x


def test_norm():
    x, gain, rstd = far(ROWS, COLS, seed=1), 1 + 0.1 * normal(COLS, seed=2), torch.empty(ROWS, device="cuda")
    y, _ = P.terra_rmsnorm_fwd(x, gain, rstd=rstd)
    _, ref, r = R.rms_fwd(x[-LAST:], None, gain, 1e-5)
    c = R.rms_terms(COLS) * R.U
    R.within("y", y[-LAST:], ref, (R.half(BF16) + 2 * c) * ref.abs())
    R.within("rstd", rstd[-LAST:], r, 2 * c * r)
    assert not bool(y[:-LAST].any())
    dx, dg = P.terra_rmsnorm_bwd(y, x, rstd, gain, dz=x)
    rx, rg, mx, mg = R.rms_bwd(y[-LAST:], x[-LAST:], rstd[-LAST:], gain, x[-LAST:])
    R.within("dx", dx[-LAST:], rx, R.half(BF16) * rx.abs() + 68 * R.U * mx + torch.finfo(BF16).tiny)
    # sums with zeros are exact: LAST of them are not, and what is at z-hat and dy z-hat
    R.within("dgain", dg, rg, (LAST + 4) * R.U * mg)


@pytest.mark.parametrize("dtype,first,K", [(BF16, 0, COLS), (F16, 1, COLS - 8), (E4M3, 0, COLS), (BF16, 0, COLS - 1)])
def test_linear_forward(dtype, first, K):
    """Rows at 16-byte places, at others, in 8 bits, and of odd length."""
    x = far(ROWS, COLS, dtype=dtype, seed=1)[:, first:first + K]
    w, bias = normal(COLS, K, seed=2, scale=K ** -0.5).to(dtype), normal(COLS, seed=3)
    sx = sw = None
    if dtype == E4M3:
        sx, sw = torch.ones(ROWS, device="cuda"), torch.ones(COLS, device="cuda")
        sx[-LAST:] = 1 + torch.arange(LAST, device="cuda") / 512
    y = P.terra_linear_fwd(x, w, bias, act="silu", x_scale=sx, w_scale=sw)
    t, ref, off = R.lin_fwd(x[-LAST:], w, bias, "silu", None, None if sx is None else sx[-LAST:], sw)
    R.within("y", y[-LAST:], ref, R.lin_fwd_bound(t, ref, off, y.dtype, "silu", None))
    # before them the activation of the bias alone
    assert bool((y[:-LAST] == y[:1]).all())


@pytest.mark.parametrize("N,K", [(COLS, 64), (64, COLS)])
def test_linear_backward(N, K):
    x, w, dy, pre = far(ROWS, K, seed=1), normal(N, K, dtype=BF16, seed=2), far(ROWS, N, seed=3), far(ROWS, N, seed=4)
    dx, dw, db = P.terra_linear_bwd(dy, x, w, pre, act="gelu")
    ref, mag, dyc = R.lin_bwd(dy[-LAST:], x[-LAST:], w, pre[-LAST:], "gelu")
    h = R.half(BF16)
    R.within("dx", dx[-LAST:], ref[0], h * ref[0].abs() + (h + (N + 4) * R.U) * 1.01 * mag[0] + torch.finfo(BF16).tiny)
    assert not bool(dx[:-LAST].any())
    R.within("dw", dw, ref[1], (h + (LAST + 4) * R.U) * 1.01 * mag[1] + torch.finfo(F32).tiny)
    R.within("db", db, ref[2], (LAST + 4) * R.U * mag[2] + 1e-6 * dyc)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope(layout):
    heads, hd = COLS // 32, 32
    q = far(ROWS, heads, hd, seed=1)
    plan = P.terra_plan_rope(hd, layout=layout)
    out, _ = P.terra_rope_fwd(plan, q, grid=(1, ROWS))
    pos = torch.arange(ROWS - LAST, ROWS, device="cuda")[:, None]
    y, off = R.rope(q[-LAST:], pos, R.rope_freqs(hd, 10000.0), 1, hd, layout, 1.0)
    R.within("q", out[-LAST:], y, R.half(BF16) * y.abs() + (1 + R.half(BF16)) * off)
    assert not bool(out[:-LAST].any())
