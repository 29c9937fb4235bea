"""The 8-bit output of the root-mean-square norm: its scale is that of the row's y,
and q the nearest e4m3 value to the float32 quotient y / q_scale, for every way a row is held."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

pytestmark = pytest.mark.gpu
F32, E4M3 = torch.float32, torch.float8_e4m3fn
# (rows, cols): one wave, 256, 512 and 1024 threads a row, and rows that are read again; whole chunks and not
SIZES = [(1030, 64), (1030, 509), (40, 1001), (40, 4096), (30, 8191), (20, 16384), (6, 16391), (5, 40003)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def quantise(x, gain, eps=1e-5):
    """(y, q, q_scale) of float32 rows, on the host."""
    rows, cols = x.shape
    y, q = torch.empty_like(x), torch.empty(rows, cols, dtype=E4M3, device="cuda")
    s = torch.empty(rows, device="cuda")
    P.terra_rmsnorm_fwd(x, gain, eps=eps, out=y, q=q, q_scale=s)
    return y.cpu(), q.cpu(), s.cpu()


def same_bits(y, q, s):
    """float32 divisions on the host are correctly rounded, and so is the step to e4m3: the bits are known."""
    assert torch.equal(s, (y.abs().amax(-1) / 448).clamp_min(2.0 ** -126))
    want = (y / s[:, None]).to(E4M3).view(torch.uint8)
    assert int((q.view(torch.uint8) != want).sum()) == 0


@pytest.mark.parametrize("rows,cols", SIZES)
def test_bits(rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= 10.0 ** torch.randint(-6, 7, (rows, 1), generator=g, device="cuda").float()
    gain = 1 + 0.1 * torch.randn(cols, generator=g, device="cuda")
    same_bits(*quantise(x, gain))
    same_bits(*quantise(x, None))


@pytest.mark.parametrize("rows,cols", SIZES)
def test_gain_beyond_the_range(rows, cols):
    """x gain leaves float32's range, above and below, where y does not."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = 1 + torch.rand(rows, cols, generator=g, device="cuda")
    # squares beyond float32: 1/rms is 0, and so is y
    y, q, s = quantise(1e30 * x, torch.full((cols,), 1e10, device="cuda"))
    assert not bool(y.any()) and not bool(q.float().any()) and bool((s == 2.0 ** -126).all())
    y, q, s = quantise(1e15 * x, torch.full((cols,), 1e25, device="cuda"))
    assert bool((y > 1e24).all()) and bool(torch.isfinite(y).all())
    same_bits(y, q, s)
    y, q, s = quantise(1e-18 * x, torch.full((cols,), 1e-25, device="cuda"), eps=0.0)
    assert bool((y > 1e-26).all()) and bool((y < 1e-24).all())
    same_bits(y, q, s)


@pytest.mark.parametrize("rows,cols", SIZES)
def test_infinite_scale(rows, cols):
    """An infinity among finite y: the scale is infinite, the finite ones stand at 0."""
    x, gain = torch.ones(rows, cols, device="cuda"), torch.ones(cols, device="cuda")
    x[:, 7], gain[7] = 4.0, 3e38
    y, q, s = quantise(x, gain)
    assert bool(torch.isinf(y[:, 7]).all()) and bool(torch.isinf(s).all())
    assert bool(torch.isnan(q[:, 7].float()).all())
    rest = torch.arange(cols) != 7
    assert bool(torch.isfinite(y[:, rest]).all()) and not bool(q[:, rest].float().any())
