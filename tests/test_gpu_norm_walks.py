"""The root-mean-square norm where a wave or a workgroup walks several rows, none
of them zero: what is carried from row to row (the next row's loads, the gain's gradient),
in every form.  Against float64 (bounds: operator_refs.py)."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
# (rows, cols) of the forward and of the backward, and of the forward alone
BOTH = [(16000, 65), (10000, 64), (9001, 512), (10007, 768), (9001, 1001), (4001, 2048), (4001, 2001), (2700, 4096), (2700, 4091),
        (1700, 4100), (1300, 8191), (1300, 8192), (1100, 8200), (1301, 12003)]
FORWARD = [(1100, 16384), (1100, 16391)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def normal(*dims, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*dims, generator=g, device="cuda")).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", BOTH + FORWARD)
def test_forward(rows, cols, dtype):
    x, res = normal(rows, cols, dtype=dtype, seed=1), normal(rows, cols, dtype=dtype, seed=2, scale=2)
    gain, rstd = 1 + 0.1 * normal(cols, seed=3), torch.empty(rows, device="cuda")
    q, s = torch.empty(rows, cols, dtype=E4M3, device="cuda"), torch.empty(rows, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    P.terra_rmsnorm_fwd(x, gain, res=res, out=y, z=z, rstd=rstd, q=q, q_scale=s)
    zz, yy, rr = R.rms_fwd(x, res, gain, 1e-5)
    c = R.rms_terms(cols) * R.U
    R.within("z", z, zz, (R.half(dtype) + 2 * R.U) * zz.abs() + torch.finfo(dtype).tiny)
    R.within("y", y, yy, (R.half(dtype) + c) * yy.abs() + torch.finfo(dtype).tiny)
    R.within("rstd", rstd, rr, c * rr)
    top = yy.abs().amax(-1) / 448
    R.within("scale", s, top, 2 * c * top)
    v = yy / s.double()[:, None]
    R.within("q", q.float(), v, (1 + 8 * c) * (v.abs() * 2.0 ** -4).clamp_min(2.0 ** -10))
    # in place, y over x and z over res; and y over x alone
    a, b = x.clone(), res.clone()
    P.terra_rmsnorm_fwd(a, gain, res=b, out=a, z=b)
    assert torch.equal(a, y) and torch.equal(b, z)
    a = x.clone()
    P.terra_rmsnorm_fwd(a, gain, res=res, out=a, z=b)
    assert torch.equal(a, y) and torch.equal(b, z)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", BOTH)
def test_backward(rows, cols, dtype):
    dy, z = normal(rows, cols, dtype=dtype, seed=1), normal(rows, cols, dtype=dtype, seed=2, scale=2)
    dz, gain = normal(rows, cols, dtype=dtype, seed=4), 1 + 0.1 * normal(cols, seed=3)
    rstd = R.rms_fwd(z, None, None, 1e-5)[2].float()
    blocks = P.terra_rmsnorm_bwd_workspace_bytes(rows, cols) // (4 * cols)
    for g, r in ((gain, dz), (None, None)):
        dx, dg = torch.empty_like(dy), torch.empty(cols, device="cuda")
        P.terra_rmsnorm_bwd(dy, z, rstd, g, dz=r, out=(dx, dg))
        rx, rg, mx, mg = R.rms_bwd(dy, z, rstd, g, r)
        # a row's mean: up to 32 sums in a thread (cols / 1024 in long rows), 26 more and 4 products
        R.within("dx", dx, rx, R.half(dtype) * rx.abs() + (max(32, cols / 1024) + 36) * R.U * mx + torch.finfo(dtype).tiny)
        # a column's sum: z-hat, the rows that a slot walks (at most rows / blocks), four waves,
        # blocks / 128 partial sums in each of four chains, these and 32 threads
        R.within("dgain", dg, rg, (rows / blocks + blocks / 128 + 45) * R.U * mg)
        for i in range(3):                         # in place of dy and of dz; each gradient by itself
            t = [dy.clone(), dz.clone()]
            out = ((t[0], None), (t[1], None), (None, torch.empty_like(dg)))[i]
            if i == 1 and r is None:
                continue
            P.terra_rmsnorm_bwd(t[0], z, rstd, g, dz=None if r is None else t[1], out=out)
            assert torch.equal(out[0], dx) if i < 2 else torch.equal(out[1], dg)
