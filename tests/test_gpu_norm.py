"""The root-mean-square norm on the GPU against float64 (bounds: operator_refs.py)."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def normal(*dims, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*dims, generator=g, device="cuda")).to(dtype)


def check_fwd(x, gain, res, got, eps=1e-5):
    z, y, rstd = R.rms_fwd(x, res, gain, eps)
    c = R.rms_terms(x.shape[-1]) * R.U
    dt = x.dtype
    out, zz = got["out"], got["z"]
    if zz is not None:
        R.within("z", zz, z, (R.half(dt) + 2 * R.U) * z.abs() + torch.finfo(dt).tiny)
    if out is not None:
        R.within("y", out, y, (R.half(dt) + c) * y.abs() + torch.finfo(dt).tiny)
    if got.get("rstd") is not None:
        R.within("rstd", got["rstd"], rstd.reshape(-1), c * rstd.reshape(-1))
    if got.get("q") is not None:
        s = got["q_scale"].double().reshape(rstd.shape)
        ref = (y.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
        R.within("scale", s, ref, 2 * c * ref)
        v = y / s[..., None]
        # half a step of e4m3, and of its smallest numbers
        R.within("q", got["q"].float(), v, (1 + 8 * c) * (v.abs() * 2.0 ** -4).clamp_min(2.0 ** -10))


def run_fwd(x, gain, res, q8=False, y=True):
    rows = x.numel() // x.shape[-1]
    got = {"rstd": torch.empty(rows, device="cuda")}
    kw = {}
    if q8:
        kw = {"q": torch.empty(x.shape, dtype=E4M3, device="cuda"), "q_scale": torch.empty(rows, device="cuda")}
        if y:
            kw["out"] = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    out, z = P.terra_rmsnorm_fwd(x, gain, res=res, rstd=got["rstd"], **kw)
    return {**got, **kw, "out": out, "z": z}


# every way a row is held: one wave, 256 and 1024 threads, and longer; odd lengths
ROWS_COLS = [(1, 1), (1, 7), (3, 8), (1, 4096), (5, 513), (1025, 64), (1030, 509), (1100, 768), (1500, 1001),
             (1031, 2048), (260, 4100), (300, 8191), (7, 8200), (3, 16391), (2, 32768), (3, 40003)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", ROWS_COLS)
def test_forward(rows, cols, dtype):
    x, res = normal(rows, cols, dtype=dtype, seed=1), normal(rows, cols, dtype=dtype, seed=2, scale=2)
    gain = 1 + 0.1 * normal(cols, seed=3)
    check_fwd(x, gain, res, run_fwd(x, gain, res))
    check_fwd(x, None, None, run_fwd(x, None, None))
    check_fwd(x, gain, res, run_fwd(x, gain, res, q8=True, y=rows % 2 == 1))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", ROWS_COLS)
def test_backward(rows, cols, dtype):
    dy, z = normal(rows, cols, dtype=dtype, seed=1), normal(rows, cols, dtype=dtype, seed=2, scale=2)
    dz, gain = normal(rows, cols, dtype=dtype, seed=4), 1 + 0.1 * normal(cols, seed=3)
    rstd = R.rms_fwd(z, None, None, 1e-5)[2].float()
    for g, r in ((gain, dz), (None, None), (gain, None)):
        dg = torch.empty(cols, device="cuda")
        dx = torch.empty_like(dy)
        P.terra_rmsnorm_bwd(dy, z, rstd, g, dz=r, out=(dx, dg))
        rx, rg, mx, mg = R.rms_bwd(dy, z, rstd, g, r)
        # a row's mean: up to 32 sums in a thread (cols / 1024 in long rows), 26 more and 4 products
        c = (max(32, cols / 1024) + 36) * R.U
        R.within("dx", dx, rx, R.half(dtype) * rx.abs() + c * mx + torch.finfo(dtype).tiny)
        # a column's sum: the rows of a wave, four waves, 16 + 32 partial sums
        R.within("dgain", dg, rg, (rows / 64 + 64) * R.U * mg)
        only, none = P.terra_rmsnorm_bwd(dy, z, rstd, g, dz=r, out=(torch.empty_like(dy), None))
        assert none is None and torch.equal(only, dx)
        again = torch.empty(cols, device="cuda")
        P.terra_rmsnorm_bwd(dy, z, rstd, g, dz=r, out=(None, again))
        assert torch.equal(again, dg)


def test_backward_against_differences():
    x, dy = normal(3, 40, seed=1), normal(3, 40, seed=2)
    gain = 1 + 0.1 * normal(40, seed=3)
    z, y, rstd = R.rms_fwd(x, None, gain, 1e-5)
    dx, dg = P.terra_rmsnorm_bwd(dy, x, rstd.float(), gain)
    loss = lambda a, g: float((R.rms_fwd(a, None, g, 1e-5)[1] * dy.double()).sum())  # noqa: E731
    h = 1e-4
    for i in (0, 17, 39):
        e = torch.zeros(3, 40, dtype=torch.float64, device="cuda")
        e[1, i] = h
        d = (loss(x.double() + e, gain.double()) - loss(x.double() - e, gain.double())) / (2 * h)
        assert abs(d - float(dx[1, i])) < 1e-5        # third derivatives times h^2, float32's rounding
        d = (loss(x.double(), gain.double() + e[1]) - loss(x.double(), gain.double() - e[1])) / (2 * h)
        assert abs(d - float(dg[i])) < 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_offsets(dtype):
    """Parts of wider tensors, at odd places; what lies around the outputs stays."""
    rows, cols = 37, 203
    big = lambda s: normal(rows, cols + 61, dtype=dtype, seed=s)  # noqa: E731
    x, res = big(1)[:, 3:3 + cols], big(2)[:, 5:5 + cols]
    outs = [torch.full((rows, cols + 9), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    z, y = outs[0][:, 1:1 + cols], outs[1][:, 2:2 + cols]
    P.terra_rmsnorm_fwd(x, None, res=res, out=y, z=z)
    check_fwd(x, None, res, {"out": y, "z": z})
    for o, lo in zip(outs, (1, 2)):
        assert bool((o[:, :lo] == 7).all()) and bool((o[:, lo + cols:] == 7).all())
    q = torch.zeros((rows, cols + 3), dtype=torch.uint8, device="cuda").view(E4M3)[:, 1:1 + cols]
    s = torch.empty(rows, device="cuda")
    P.terra_rmsnorm_fwd(x, None, q=q, q_scale=s)
    check_fwd(x, None, None, {"out": None, "z": None, "q": q, "q_scale": s})


@pytest.mark.parametrize("rows,cols", [(1030, 509), (5, 4096), (2, 40003)])
def test_in_place(rows, cols):
    x, res = normal(rows, cols, dtype=BF16, seed=1), normal(rows, cols, dtype=BF16, seed=2)
    ref_y, ref_z = P.terra_rmsnorm_fwd(x, None, res=res)
    a, b = x.clone(), res.clone()
    P.terra_rmsnorm_fwd(a, None, res=b, out=a, z=b)
    assert torch.equal(a, ref_y) and torch.equal(b, ref_z)
    rstd = R.rms_fwd(ref_z, None, None, 1e-5)[2].float()
    dx, _ = P.terra_rmsnorm_bwd(x, ref_z, rstd, None, dz=res)
    for i in range(2):
        t = [x.clone(), res.clone()]
        P.terra_rmsnorm_bwd(t[0], ref_z, rstd, None, dz=t[1], out=(t[i], None))
        assert torch.equal(t[i], dx)


def test_more_rows_than_one_round():
    x = normal(9001, 65, dtype=BF16, seed=1)
    check_fwd(x, None, None, run_fwd(x, None, None, q8=True))


@pytest.mark.parametrize("cols", [64, 3001, 40003])
def test_zeros_infinities_nan(cols):
    x = normal(6, cols, seed=1)
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    x[3] = 1e-30
    x[4] = 1e30           # its square is beyond float32: 1/rms is 0
    q, s = torch.empty((6, cols), dtype=E4M3, device="cuda"), torch.empty(6, device="cuda")
    y = torch.empty_like(x)
    P.terra_rmsnorm_fwd(x, None, out=y, q=q, q_scale=s)
    assert bool((y[0] == 0).all()) and float(s[0]) == 2.0 ** -126 and bool((q[0].float() == 0).all())
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(s[1])) and bool(torch.isnan(q[1].float()).all())
    assert bool(torch.isnan(y[2, 5])) and float(y[2, 0]) == 0 and bool(torch.isnan(s[2]))
    tiny = R.rms_fwd(x[3:4], None, None, 1e-5)[1][0]
    # as every y: its own rounding (2^-24 of 3.2e-28 is 1.9e-35 already) and 1/rms's
    R.within("tiny", y[3], tiny, (1 + R.rms_terms(cols)) * R.U * tiny)
    assert bool((y[4] == 0).all()) and bool((q[4].float() == 0).all())
    check_fwd(x[5:], None, None, {"out": y[5:], "z": None, "q": q[5:], "q_scale": s[5:]})


def test_no_rows():
    x = torch.empty((0, 32), dtype=BF16, device="cuda")
    y, z = P.terra_rmsnorm_fwd(x, None, res=x)
    assert y.shape == x.shape and z.shape == x.shape
    dx, dg = P.terra_rmsnorm_bwd(x, x, torch.empty(0, device="cuda"), torch.ones(32, device="cuda"))
    assert dx.shape == x.shape and bool((dg == 0).all())
