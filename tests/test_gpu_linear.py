"""The linear layer on the GPU against float64 (bounds: operator_refs.py)."""

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


def quantised(x):
    s = (x.abs().amax(-1, keepdim=True) / 448).clamp_min(2.0 ** -126)
    return (x / s).to(E4M3), s.squeeze(-1)


def operands(M, N, K, dtype):
    x, w = normal(M, K, seed=1), normal(N, K, seed=2, scale=K ** -0.5)
    if dtype != E4M3:
        return x.to(dtype), w.to(dtype), None, None
    (x, sx), (w, sw) = quantised(x), quantised(w)
    return x, w, sx, sw


def check(y, pre, x, w, bias, act, res, sx=None, sw=None):
    t, ref, off = R.lin_fwd(x, w, bias, act, res, sx, sw)
    off = off.reshape(ref.shape)
    R.within("y", y, ref, R.lin_fwd_bound(t, ref, off, y.dtype, act, res))
    if pre is not None:
        R.within("pre", pre, t, R.half(y.dtype) * t.abs() + 2 * off + torch.finfo(y.dtype).tiny)


# (M, N, K): few tokens in each of its tilings, odd everywhere; one tile and
# several of both tile sizes; contraction slices; lengths that the direct loads
# do not take
SIZES = [(1, 1, 1), (1, 16, 64), (1, 77, 130), (1, 4096, 768), (3, 33, 1000), (16, 100, 256), (17, 48, 72), (33, 130, 515),
         (48, 300, 64), (64, 65, 1024), (65, 64, 64), (100, 129, 40), (128, 128, 512), (130, 1000, 2048), (200, 257, 1111),
         (513, 8, 4096), (300, 2305, 96), (1017, 771, 1003), (2500, 2000, 264), (4000, 4200, 128),
         (5, 16400, 72), (20, 16390, 64), (40, 16500, 136), (2000, 2000, 2003), (6000, 2100, 1003),
         (5000, 4100, 1024)]


@pytest.mark.parametrize("dtype", [BF16, F16, E4M3])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_forward(M, N, K, dtype):
    x, w, sx, sw = operands(M, N, K, dtype)
    to = F16 if dtype == F16 or (dtype == E4M3 and M % 2) else BF16
    bias, res = normal(N, seed=3), normal(M, N, dtype=to, seed=4)
    kw = {"x_scale": sx, "w_scale": sw, "out_dtype": to}
    for act, b, r, keep in (("none", None, None, False), ("gelu", bias, None, True), ("silu", bias, res, True),
                            ("relu", None, res, False)):
        pre = torch.empty(M, N, dtype=to, device="cuda") if keep else None
        y = P.terra_linear_fwd(x, w, b, act=act, res=r, pre=pre, **kw)
        assert y.dtype == to
        check(y, pre, x, w, b, act, r, sx, sw)


def test_whole_rounds_and_the_rest():
    """More row tiles than whole rounds of one tile a compute unit."""
    M, N, K = 256 * 43 + 19, 1536, 64
    x, w, _, _ = operands(M, N, K, BF16)
    bias, res, pre = normal(N, seed=3), normal(M, N, dtype=BF16, seed=4), torch.empty(M, N, dtype=BF16, device="cuda")
    y = P.terra_linear_fwd(x, w, bias, act="gelu", res=res, pre=pre)
    check(y, pre, x, w, bias, "gelu", res)
    x, w, sx, sw = operands(M, N, K, E4M3)
    check(P.terra_linear_fwd(x, w, bias, res=res, x_scale=sx, w_scale=sw), None, x, w, bias, "none", res, sx, sw)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("M", [1, 20, 64, 300])
def test_strides_and_offsets(M, dtype):
    """Parts of wider tensors; what lies around y and pre stays, y in place of res too."""
    N, K = 150, 200
    x, w, sx, sw = operands(M, N + 6, K + 50, dtype)
    bias = normal(N, seed=3)
    for lo in (0, 1, 16):
        xs, ws = x[:, lo:lo + K], w[3:3 + N, lo:lo + K]
        wsc = None if sw is None else sw[3:3 + N].clone()
        wide = [torch.full((M, N + 11), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
        y, pre = wide[0][:, 5:5 + N], wide[1][:, 8:8 + N]
        res = normal(M, N, dtype=BF16, seed=5)
        y.copy_(res)
        P.terra_linear_fwd(xs, ws, bias, act="silu", res=y, x_scale=sx, w_scale=wsc, out=y, pre=pre)
        check(y, pre, xs, ws, bias, "silu", res, sx, wsc)
        for o, a in zip(wide, (5, 8)):
            assert bool((o[:, :a] == 7).all()) and bool((o[:, a + N:] == 7).all())


def test_nothing_behind_a_row_counts():
    """NaN and infinities next to every row, in x and in w."""
    for M in (1, 40, 70, 200):
        for K in (100, 104):
            X, W = normal(M, K + 24, dtype=BF16, seed=1), normal(90, K + 24, dtype=BF16, seed=2)
            X[:, :8], W[:, :8], X[:, 8 + K:], W[:, 8 + K:] = float("nan"), float("inf"), float("inf"), float("nan")
            x, w = X[:, 8:8 + K], W[:, 8:8 + K]
            check(P.terra_linear_fwd(x, w), None, x, w, None, "none", None)
            dy = normal(M, 90, dtype=BF16, seed=3)
            dx, dw, db = P.terra_linear_bwd(dy, x, w)
            assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all()) and bool(torch.isfinite(db).all())


def test_infinities_and_nan_in_place():
    x, w = normal(5, 64, dtype=BF16, seed=1), normal(40, 64, dtype=BF16, seed=2)
    x[1, 3] = float("nan")
    x[2, 7] = float("inf")
    y = P.terra_linear_fwd(x, w, act="relu")
    assert bool(torch.isnan(y[1]).all())
    assert torch.equal(torch.isinf(y[2]), w[:, 7] > 0) and bool((y[2][w[:, 7] < 0] == 0).all())
    check(y[3:], None, x[3:], w, None, "relu", None)


BWD = [(1, 1, 1), (1, 64, 40), (5, 33, 70), (64, 128, 256), (100, 129, 40), (130, 1000, 72), (1017, 771, 403),
       (3000, 200, 512), (5000, 520, 96), (20000, 64, 64), (9001, 40, 1544)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("M,N,K", BWD)
def test_backward(M, N, K, dtype):
    x, w, _, _ = operands(M, N, K, dtype)
    dy, pre = normal(M, N, dtype=dtype, seed=3), normal(M, N, dtype=dtype, seed=4, scale=2)
    for act, dwt in (("none", F32), ("gelu", dtype), ("silu", F32), ("relu", dtype)):
        out = (torch.empty(M, K, dtype=dtype, device="cuda"), torch.empty(N, K, dtype=dwt, device="cuda"),
               torch.empty(N, device="cuda"))
        P.terra_linear_bwd(dy, x, w, pre, act=act, out=out)
        ref, mag, dyc = R.lin_bwd(dy, x, w, pre, act)
        # dt's rounding to the operands' type (none without an activation), the sums, the output's own
        h = R.half(dtype) if act != "none" else 0
        R.within("dx", out[0], ref[0], R.half(dtype) * ref[0].abs() + (h + (N + 4) * R.U) * 1.01 * mag[0] + torch.finfo(dtype).tiny)
        own = R.half(dwt) if dwt != F32 else 0
        R.within("dw", out[1], ref[1], own * ref[1].abs() + (h + (M + 4) * R.U) * 1.01 * mag[1] + torch.finfo(dwt).tiny)
        R.within("db", out[2], ref[2], (M + 4) * R.U * mag[2] + 1e-6 * dyc)
        # each gradient by itself has the same bits
        for i in range(3):
            one = [None] * 3
            one[i] = torch.empty_like(out[i])
            P.terra_linear_bwd(dy, x, w, pre, act=act, out=one)
            assert torch.equal(one[i], out[i])


def test_backward_against_differences():
    M, N, K = 6, 24, 40
    x, w, _, _ = operands(M, N, K, F16)
    dy, bias = normal(M, N, dtype=F16, seed=3), normal(N, seed=4)
    pre = torch.empty(M, N, dtype=F16, device="cuda")
    P.terra_linear_fwd(x, w, bias, act="gelu", pre=pre)
    dx, dw, db = P.terra_linear_bwd(dy, x, w, pre, act="gelu")
    loss = lambda a, b, c: float((R.lin_fwd(a, b, c, "gelu", None)[1] * dy.double()).sum())  # noqa: E731
    X, W, B, h = x.double(), w.double(), bias.double(), 1e-4
    for t, got, at in ((X, dx, (2, 5)), (W, dw, (7, 11)), (B, db, (3,))):
        e = torch.zeros_like(t)
        e[at] = h
        args = [(X, W, B), (X, W, B)]
        plus = [v + e if v is t else v for v in args[0]]
        minus = [v - e if v is t else v for v in args[1]]
        d = (loss(*plus) - loss(*minus)) / (2 * h)
        # roundings of pre, dt and the output to half steps of 2^-11, over sums of a few units
        assert abs(d - float(got[at])) < 2e-2 * max(1.0, abs(d))


def test_backward_strides_and_offsets():
    M, N, K = 333, 130, 70
    X, W = normal(M, K + 20, dtype=BF16, seed=1), normal(N + 2, K + 20, dtype=BF16, seed=2)
    DY, PRE = normal(M, N + 20, dtype=BF16, seed=3), normal(M, N + 20, dtype=BF16, seed=4)
    for lo in (0, 3, 8):
        x, w, dy, pre = X[:, lo:lo + K], W[1:1 + N, lo:lo + K], DY[:, lo:lo + N], PRE[:, lo + 1:lo + 1 + N]
        plain = [t.contiguous() for t in (dy, x, w, pre)]
        for act in ("none", "gelu"):
            ref = P.terra_linear_bwd(*plain, act=act)
            wide = torch.full((M, K + 5), 7.0, dtype=BF16, device="cuda")
            dww = torch.full((N, K + 5), 7.0, device="cuda")
            out = (wide[:, 2:2 + K], dww[:, 2:2 + K], torch.empty(N, device="cuda"))
            P.terra_linear_bwd(dy, x, w, pre, act=act, out=out)
            (rx, rw, rb), mag, _ = R.lin_bwd(dy, x, w, pre, act)
            h = R.half(BF16) if act != "none" else 0
            R.within("dx", out[0], rx, R.half(BF16) * rx.abs() + (h + (N + 4) * R.U) * 1.01 * mag[0])
            R.within("dw", out[1], rw, (h + (M + 4) * R.U) * 1.01 * mag[1])
            R.within("db", out[2], ref[2], 0)
            assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + K:] == 7).all())
            assert bool((dww[:, :2] == 7).all()) and bool((dww[:, 2 + K:] == 7).all())


def test_no_tokens():
    w = normal(48, 64, dtype=BF16)
    y = P.terra_linear_fwd(torch.empty((0, 64), dtype=BF16, device="cuda"), w)
    assert y.shape == (0, 48)
    e = torch.empty((0, 48), dtype=BF16, device="cuda")
    for dwt in (F32, BF16):
        out = (torch.empty((0, 64), dtype=BF16, device="cuda"), torch.full((48, 64), 3.0, dtype=dwt, device="cuda"),
               torch.full((48,), 3.0, device="cuda"))
        P.terra_linear_bwd(e, torch.empty((0, 64), dtype=BF16, device="cuda"), w, out=out)
        assert bool((out[1] == 0).all()) and bool((out[2] == 0).all())


def test_same_bits_every_time():
    x, w, _, _ = operands(700, 520, 2048, BF16)
    dy = normal(700, 520, dtype=BF16, seed=3)
    first = (P.terra_linear_fwd(x, w), *P.terra_linear_bwd(dy, x, w))
    for _ in range(3):
        for a, b in zip(first, (P.terra_linear_fwd(x, w), *P.terra_linear_bwd(dy, x, w))):
            assert torch.equal(a, b)
