"""Matrices whose rows lie megabytes apart: a tile's or a slice's rows span more than 2^31 bytes,
past what a buffer descriptor's offsets reach.  Against float64 (bounds: operator_refs.py)."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402
from test_gpu_linear import check, normal  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.empty_cache()


def apart(t, ld, first=0):
    """A copy of t whose rows are ld elements apart, NaN between them."""
    big = torch.full((t.shape[0], ld), float("nan"), dtype=t.dtype, device="cuda")
    v = big[:, first:first + t.shape[1]]
    v.copy_(t)
    return v


@pytest.mark.parametrize("first", [0, 3])
def test_linear_forward(first):
    M, N, K, ld = 300, 130, 104, (1 << 22) + 8
    assert 256 * ld * 2 > 2 ** 31
    x, w, res = normal(M, K, dtype=BF16, seed=1), normal(N, K, dtype=BF16, seed=2, scale=K ** -0.5), normal(M, N, dtype=BF16, seed=3)
    y = apart(torch.zeros_like(res), ld, first)
    P.terra_linear_fwd(apart(x, ld, first), w, act="silu", res=apart(res, ld), out=y)
    check(y, None, x, w, None, "silu", res)
    del y
    y = P.terra_linear_fwd(x, apart(w, (1 << 24) + 8, first), act="silu", res=res)
    check(y, None, x, w, None, "silu", res)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("M,ld", [(3000, (1 << 19) + 8), (300, (1 << 22) + 8)])
def test_linear_backward(M, ld, act):
    """Slices of tokens that span more than 2^31 bytes, and tiles that do."""
    N, K = 136, 72
    assert min(M, 256) * ld * 2 > 2 ** 31 or M * ld * 2 > 2 ** 31
    x, w, dy, pre = normal(M, K, dtype=BF16, seed=1), normal(N, K, dtype=BF16, seed=2), normal(M, N, dtype=BF16, seed=3), normal(M, N, dtype=BF16, seed=4)
    dx = apart(torch.zeros_like(x), ld)
    out = (dx, torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda"))
    P.terra_linear_bwd(apart(dy, ld), apart(x, ld), w, apart(pre, ld), act=act, out=out)
    ref, mag, dyc = R.lin_bwd(dy, x, w, pre, act)
    h = R.half(BF16) if act != "none" else 0
    R.within("dx", out[0], ref[0], R.half(BF16) * ref[0].abs() + (h + (N + 4) * R.U) * 1.01 * mag[0] + torch.finfo(BF16).tiny)
    R.within("dw", out[1], ref[1], (h + (M + 4) * R.U) * 1.01 * mag[1])
    R.within("db", out[2], ref[2], (M + 4) * R.U * mag[2] + 1e-6 * dyc)


@pytest.mark.parametrize("cols", [104, 1001])
def test_norm(cols):
    rows, ld = 1100, (1 << 21) + 3
    x, res, gain = normal(rows, cols, dtype=BF16, seed=1), normal(rows, cols, dtype=BF16, seed=2), 1 + 0.1 * normal(cols, seed=3)
    y, z = P.terra_rmsnorm_fwd(x, gain, res=res)
    a, b = apart(x, ld), apart(res, ld, 5)
    P.terra_rmsnorm_fwd(a, gain, res=b, out=a, z=b)
    assert torch.equal(a, y) and torch.equal(b, z)
    rstd = (z.double().square().mean(-1) + 1e-5).rsqrt().float()
    dx, dg = P.terra_rmsnorm_bwd(x, z, rstd, gain, dz=res)
    got, g = P.terra_rmsnorm_bwd(a.copy_(x), b, rstd, gain, dz=res, out=(a, torch.empty_like(dg)))
    assert torch.equal(got, dx) and torch.equal(g, dg)


def test_rope():
    """Heads 2^31 - 8 elements apart, and tokens 2^23."""
    T, hd = 200, 64
    plan = P.terra_plan_rope(hd, rot_dim=40)
    q = normal(T, 2, hd, dtype=BF16, seed=1)
    want, _ = P.terra_rope_fwd(plan, q, grid=(1, T))
    ld, far = 1 << 23, 2 ** 31 - 8
    big = torch.zeros(far + T * hd, dtype=BF16, device="cuda")
    v = big.as_strided((T, 2, hd), (hd, far, 1))
    v.copy_(q)
    got, _ = P.terra_rope_fwd(plan, v, grid=(1, T), out=(v, None))
    assert torch.equal(got, want)
    v = big.as_strided((T, 2, hd), (ld, hd, 1))
    v.copy_(q)
    got, _ = P.terra_rope_fwd(plan, v, grid=(1, T))
    assert torch.equal(got, want)
