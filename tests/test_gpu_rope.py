"""Rotary positions on the GPU against float64 (bounds: operator_refs.py)."""

import math

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def normal(*dims, dtype=F32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*dims, generator=g, device="cuda").to(dtype)


def grid_pos(T, H, W, axes):
    t = torch.arange(T, device="cuda") % (H * W)
    return torch.stack((t // W, t % W), -1) if axes == 2 else t[:, None]


def check(name, got, x, pos, plan_kw, sign=1):
    hd = x.shape[-1]
    rot, axes, layout = plan_kw.get("rot_dim") or hd, plan_kw.get("axes", 1), plan_kw.get("layout", "half")
    freq_kw = {k: plan_kw[k] for k in ("scaling", "factor", "orig_len") if k in plan_kw}
    scale = plan_kw.get("attn_scale") or (0.1 * math.log(plan_kw["factor"]) + 1 if plan_kw.get("scaling") == "yarn" else 1.0)
    freqs = R.rope_freqs(rot // axes, plan_kw.get("base", 10000.0), **freq_kw)
    flat = x.reshape(-1, *x.shape[-2:])
    y, off = R.rope(flat, pos, freqs, axes, rot, layout, scale, sign)
    # below the smallest normal number a half step is that of the smallest normal one:
    # 2^-25 in float16, which the values next to zero reach
    step = R.half(x.dtype) * y.abs().clamp_min(torch.finfo(x.dtype).tiny)
    R.within(name, got.reshape(flat.shape), y, step + (1 + R.half(x.dtype)) * off)
    assert torch.equal(got.reshape(flat.shape)[:, :, rot:], flat[:, :, rot:])


CASES = [
    # tokens, grid, q heads, k heads, head dim, plan
    (1, (1, 1), 1, 1, 2, {}),
    (1, (1, 4000), 8, 2, 64, {"layout": "interleaved"}),
    (960, (24, 40), 24, 24, 32, {"axes": 2}),
    (960, (24, 40), 24, 24, 32, {"axes": 2, "layout": "interleaved"}),
    (777, (7, 37), 3, 5, 24, {"axes": 2, "rot_dim": 20}),
    (777, (7, 37), 3, 5, 24, {"axes": 2, "rot_dim": 20, "layout": "interleaved"}),
    (531, (1, 531), 5, 1, 128, {"rot_dim": 64, "layout": "interleaved"}),
    (531, (1, 531), 5, 1, 128, {"rot_dim": 64}),
    (531, (1, 531), 4, 4, 96, {"rot_dim": 22}),
    (100, (1, 50), 2, 2, 33, {"rot_dim": 6, "layout": "interleaved"}),
    (100, (1, 50), 2, 2, 35, {"rot_dim": 24}),
    (64, (1, 64), 128, 128, 256, {}),
    (5000, (1, 5000), 1, 1, 256, {"layout": "interleaved", "base": 100.0}),
    (300, (1, 300), 6, 2, 64, {"scaling": "linear", "factor": 4.0}),
    (300, (1, 300), 6, 2, 64, {"scaling": "ntk", "factor": 8.0, "layout": "interleaved"}),
    (300, (1, 300), 6, 2, 64, {"scaling": "yarn", "factor": 8.0, "orig_len": 64}),
    (300, (10, 30), 6, 2, 64, {"scaling": "yarn", "factor": 2.0, "orig_len": 8192, "axes": 2, "attn_scale": 1.5}),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,grid,qh,kh,hd,kw", CASES)
def test_against_float64(T, grid, qh, kh, hd, kw, dtype):
    plan = P.terra_plan_rope(hd, **kw)
    q, k = normal(T, qh, hd, dtype=dtype, seed=1), normal(T, kh, hd, dtype=dtype, seed=2)
    pos = grid_pos(T, *grid, kw.get("axes", 1))
    a, b = P.terra_rope_fwd(plan, q, k, grid=grid)
    check("q", a, q, pos, kw)
    check("k", b, k, pos, kw)
    # the same positions given
    a2, b2 = P.terra_rope_fwd(plan, q, k, pos=pos.int().contiguous())
    assert torch.equal(a, a2) and torch.equal(b, b2)
    a, b = P.terra_rope_bwd(plan, q, k, grid=grid)
    check("dq", a, q, pos, kw, -1)
    check("dk", b, k, pos, kw, -1)
    only, none = P.terra_rope_bwd(plan, q, grid=grid)
    assert none is None and torch.equal(only, a)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(layout):
    T = 640
    g = torch.Generator(device="cuda").manual_seed(5)
    pos = torch.randint(-2 ** 31, 2 ** 31, (T, 1), generator=g, device="cuda").int()
    pos[:4, 0] = torch.tensor([0, 2 ** 31 - 1, -2 ** 31, -1], device="cuda").int()
    q = normal(T, 2, 64, seed=1)
    # float64 angles of 2^31 positions are off by 2^31 2^-52 = 5e-7: the reference takes the whole
    # turns off in integers, its frequencies from the plan's 2^-64 turns
    plan = P.terra_plan_rope(64, layout=layout, base=1e6)
    got, _ = P.terra_rope_fwd(plan, q, pos=pos)
    y = torch.empty_like(q, dtype=torch.float64)
    ints = [int(p) for p in pos[:, 0].cpu()]
    for i in range(32):
        assert abs(plan.turns[i] / 2.0 ** 64 * 2 * math.pi / 1e6 ** (-2 * i / 64) - 1) < 1e-12
        frac = torch.tensor([(p * plan.turns[i]) % 2 ** 64 / 2.0 ** 64 for p in ints], dtype=torch.float64, device="cuda")
        c, s = torch.cos(2 * math.pi * frac)[:, None], torch.sin(2 * math.pi * frac)[:, None]
        lo, hi = (i, i + 32) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = q[:, :, lo].double(), q[:, :, hi].double()
        y[:, :, lo], y[:, :, hi] = a * c - b * s, a * s + b * c
    R.within("q", got, y, 6e-7 * (1 + q.abs().max().double()))


def test_parts_of_a_projection_in_place_and_apart():
    """q and k as parts of one tensor, tokens of two images; outputs as NHWC, and in place."""
    B, H, W, heads, hd = 2, 9, 14, 6, 32
    qkv = normal(B, H, W, 3 * heads * hd, dtype=BF16, seed=1)
    q, k = (qkv[..., i * heads * hd:(i + 1) * heads * hd].unflatten(-1, (heads, hd)) for i in (0, 1))
    plan = P.terra_plan_rope(hd, axes=2)
    a, b = P.terra_rope_fwd(plan, q, k, grid=(H, W))
    pos = grid_pos(B * H * W, H, W, 2)
    check("q", a, q.contiguous(), pos, {"axes": 2})
    check("k", b, k.contiguous(), pos, {"axes": 2})
    before = qkv.clone()
    P.terra_rope_fwd(plan, q, k, grid=(H, W), out=(q, k))
    assert torch.equal(q, a) and torch.equal(k, b)
    assert torch.equal(qkv[..., 2 * heads * hd:], before[..., 2 * heads * hd:])


def test_head_major_and_odd_places():
    T, heads, hd = 70, 5, 40
    store = normal(heads, T, hd + 3, dtype=BF16, seed=1)
    q = store[:, :, 1:1 + hd].transpose(0, 1)
    out = torch.full((heads, T, hd + 5), 7.0, dtype=BF16, device="cuda")
    o = out[:, :, 2:2 + hd].transpose(0, 1)
    plan = P.terra_plan_rope(hd, rot_dim=24)
    P.terra_rope_fwd(plan, q, grid=(1, T), out=(o, None))
    check("q", o, q.contiguous(), grid_pos(T, 1, T, 1), {"rot_dim": 24})
    assert bool((out[:, :, :2] == 7).all()) and bool((out[:, :, 2 + hd:] == 7).all())


def test_turning_back():
    q = normal(500, 4, 64, seed=1)
    plan = P.terra_plan_rope(64)
    there, _ = P.terra_rope_fwd(plan, q, grid=(1, 500))
    back, _ = P.terra_rope_bwd(plan, there, grid=(1, 500))
    assert float((back - q).abs().max()) < 8e-7 * (2 * float(q.abs().max()))     # each way 2.5e-7 + 3 u of two channels


def test_no_tokens():
    q = torch.empty((0, 4, 32), dtype=BF16, device="cuda")
    a, b = P.terra_rope_fwd(P.terra_plan_rope(32), q, q, grid=(1, 1))
    assert a.shape == q.shape and b.shape == q.shape
