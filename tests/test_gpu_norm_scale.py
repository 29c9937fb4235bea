"""The 8-bit output of the root-mean-square norm: q is the nearest e4m3 value to the
float32 quotient y / q_scale, bit for bit."""

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

pytestmark = pytest.mark.gpu
F32, E4M3 = torch.float32, torch.float8_e4m3fn
# (rows, cols): one wave, 256, 512 and 1024 threads a row; whole chunks and not
SIZES = [(1030, 64), (1030, 509), (40, 1001), (40, 4096), (30, 8191), (20, 16384)]


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

