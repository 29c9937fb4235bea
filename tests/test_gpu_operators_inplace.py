"""The in-place calls that the header allows, against the same calls with outputs of their own:
bit for bit, in the forms that hold rows in different ways and walk several."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def normal(*dims, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*dims, generator=g, device="cuda").to(BF16)


@pytest.mark.parametrize("rows,cols", [(9001, 512), (10007, 768), (4001, 2001), (1700, 4100), (1100, 16384), (600, 20003)])
def test_norm(rows, cols):
    x, res, gain = normal(rows, cols, seed=1), normal(rows, cols, seed=2), 1 + 0.1 * normal(cols, seed=3).float()
    y, z = P.terra_rmsnorm_fwd(x, gain, res=res)
    for over in ("y", "z", "both"):              # y over res, z over x
        a, b = x.clone(), res.clone()
        yy, zz = P.terra_rmsnorm_fwd(a, gain, res=b, out=b if over != "z" else None, z=a if over != "y" else None)
        assert torch.equal(yy, y) and torch.equal(zz, z)
        assert (over == "z" or yy is b) and (over == "y" or zz is a)
    rstd = (z.double().square().mean(-1) + 1e-5).rsqrt().float()
    dx, dg = P.terra_rmsnorm_bwd(x, z, rstd, gain, dz=res)
    zz, again = z.clone(), torch.empty_like(dg)
    P.terra_rmsnorm_bwd(x, zz, rstd, gain, dz=res, out=(zz, again))
    assert torch.equal(zz, dx) and torch.equal(again, dg)


@pytest.mark.parametrize("M,N,K", [(7, 300, 520), (130, 1000, 2048), (300, 2305, 96), (1017, 771, 1003), (256 * 43 + 19, 1536, 64)])
def test_linear(M, N, K):
    x, w, res, bias = normal(M, K, seed=1), normal(N, K, seed=2), normal(M, N, seed=3), normal(N, seed=4).float()
    pre = torch.empty_like(res)
    y = P.terra_linear_fwd(x, w, bias, act="silu", res=res, pre=pre)
    r = res.clone()
    assert torch.equal(P.terra_linear_fwd(x, w, bias, act="silu", res=r, pre=r), y) and torch.equal(r, pre)
    r, p = res.clone(), torch.empty_like(res)
    P.terra_linear_fwd(x, w, bias, act="silu", res=r, pre=p, out=r)
    assert torch.equal(r, y) and torch.equal(p, pre)
