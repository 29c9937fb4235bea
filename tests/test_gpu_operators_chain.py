"""The norm, the linear layer, the rotary positions and the window attention as a
block of a model uses them, forward and backward, against float64; captured
into a graph and replayed; on another stream.

The block: x1 = x + r;  h = rms(x1);  q, k, v = h W_qkv^T (one projection);
q, k turned by their row and column;  o = window attention;
x2 = x1 + o W_o^T + b;  y = x2 + SiLU(rms(x2) W_1^T + b_1) W_2^T + b_2.
Bars as the Swin block's (test_gpu_block.py): the chain has about as many 16-bit
roundings of values of the same size, so every result is held to relative L2
1e-2 and to a max error of 1e-2 of its largest magnitude.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2608_15211_amd")

import operator_refs as R  # noqa: E402
from oracle import Geometry, attn_bwd, attn_fwd, route, unroute  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.lib()


def near(name, got, ref):
    got, ref = got.double(), ref.double().reshape(got.shape)
    err, big = float((got - ref).abs().max()), float(ref.abs().max())
    rel = float((got - ref).norm() / ref.norm())
    print("  %-6s max %.2e of the largest, rel L2 %.2e" % (name, err / big, rel), flush=True)
    assert err <= 1e-2 * big and rel <= 1e-2, name


GEOM = dict(B=2, H=20, W=29, C=96, heads=3, head_dim=32, wh=8, ww=8, sh=4, sw=4, mask_flags=1)


def params(dtype, seed=0):
    C, F = GEOM["C"], 200
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *d: torch.randn(*d, generator=g, device="cuda")  # noqa: E731
    w = {"qkv": (3 * C, C), "o": (C, C), "w1": (F, C), "w2": (C, F)}
    p = {n: (rn(*s) / s[1] ** 0.5).to(dtype) for n, s in w.items()}
    p.update(g1=1 + 0.1 * rn(C), g2=1 + 0.1 * rn(C), bo=0.02 * rn(C), b1=0.02 * rn(F), b2=0.02 * rn(C))
    shape = (GEOM["B"], GEOM["H"], GEOM["W"], C)
    p.update(x=rn(*shape).to(dtype), r=rn(*shape).to(dtype), dy=rn(*shape).to(dtype))
    p["table"] = 0.02 * rn(2 * GEOM["wh"] - 1, 2 * GEOM["ww"] - 1, GEOM["heads"])
    return p


class Block:
    """The block in the library's calls, with buffers of its own."""

    def __init__(self, p):
        B, H, W, C, heads, hd = (GEOM[n] for n in ("B", "H", "W", "C", "heads", "head_dim"))
        F, T, dt = p["w1"].shape[0], B * H * W, p["x"].dtype
        e = lambda *s, t=dt: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.p, self.plan, self.grid = p, P.terra_plan_rope(hd, axes=2), (H, W)
        n = (B, H, W)
        self.b = {"x1": e(*n, C), "h1": e(*n, C), "s1": e(T, t=f32), "qkv": e(*n, 3 * C), "q": e(*n, heads, hd), "k": e(*n, heads, hd),
                  "v": e(*n, C), "o": e(*n, C), "lse": e(B, heads, H * W, t=f32), "x2": e(*n, C), "h2": e(*n, C),
                  "s2": e(T, t=f32), "pre": e(*n, F), "a": e(*n, F), "y": e(*n, C)}
        self.g = {"a": e(*n, F), "w2": e(C, F, t=f32), "b2": e(C, t=f32), "h2": e(*n, C), "w1": e(F, C, t=f32), "b1": e(F, t=f32),
                  "x2": e(*n, C), "g2": e(C, t=f32), "o": e(*n, C), "wo": e(C, C, t=f32), "bo": e(C, t=f32),
                  "q": e(*n, C), "k": e(*n, C), "v": e(*n, C), "table": e(*p["table"].shape, t=f32), "qkv": e(*n, 3 * C),
                  "h1": e(*n, C), "wqkv": e(3 * C, C, t=f32), "x": e(*n, C), "g1": e(C, t=f32)}
        code = {BF16: "bf16", F16: "f16"}[dt]
        need = max([P.terra_linear_bwd_workspace_bytes(T, *w, code) for w in ((3 * C, C), (C, C), (F, C), (C, F))] +
                   [P.terra_linear_fwd_workspace_bytes(T, *w, code) for w in ((3 * C, C), (C, C), (F, C), (C, F))] +
                   [P.terra_rmsnorm_bwd_workspace_bytes(T, C), P.terra_winattn_bwd_workspace_bytes(GEOM, code)])
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def forward(self):
        p, b, C, heads = self.p, self.b, GEOM["C"], GEOM["heads"]
        P.terra_rmsnorm_fwd(p["x"], p["g1"], res=p["r"], eps=EPS, out=b["h1"], z=b["x1"], rstd=b["s1"])
        P.terra_linear_fwd(b["h1"], p["qkv"], out=b["qkv"], workspace=self.ws)
        q, k, v = (b["qkv"][..., i * C:(i + 1) * C] for i in range(3))
        P.terra_rope_fwd(self.plan, q.unflatten(-1, (heads, -1)), k.unflatten(-1, (heads, -1)), grid=self.grid, out=(b["q"], b["k"]))
        b["v"].copy_(v)
        P.terra_winattn_fwd_nhwc(b["q"].flatten(-2), b["k"].flatten(-2), b["v"], p["table"], GEOM, out=b["o"], lse=b["lse"])
        P.terra_linear_fwd(b["o"], p["o"], p["bo"], res=b["x1"], out=b["x2"], workspace=self.ws)
        P.terra_rmsnorm_fwd(b["x2"], p["g2"], eps=EPS, out=b["h2"], rstd=b["s2"])
        P.terra_linear_fwd(b["h2"], p["w1"], p["b1"], act="silu", out=b["a"], pre=b["pre"], workspace=self.ws)
        P.terra_linear_fwd(b["a"], p["w2"], p["b2"], res=b["x2"], out=b["y"], workspace=self.ws)
        return b["y"]

    def backward(self):
        p, b, g, C, heads, ws = self.p, self.b, self.g, GEOM["C"], GEOM["heads"], self.ws
        P.terra_linear_bwd(p["dy"], b["a"], p["w2"], out=(g["a"], g["w2"], g["b2"]), workspace=ws)
        P.terra_linear_bwd(g["a"], b["h2"], p["w1"], b["pre"], act="silu", out=(g["h2"], g["w1"], g["b1"]), workspace=ws)
        P.terra_rmsnorm_bwd(g["h2"], b["x2"], b["s2"], p["g2"], dz=p["dy"], out=(g["x2"], g["g2"]), workspace=ws)
        P.terra_linear_bwd(g["x2"], b["o"], p["o"], out=(g["o"], g["wo"], g["bo"]), workspace=ws)
        P.terra_winattn_bwd_nhwc(b["q"].flatten(-2), b["k"].flatten(-2), b["v"], b["o"], g["o"], b["lse"], p["table"], GEOM,
                                 out=(g["q"], g["k"], g["v"], g["table"]), workspace=ws)
        dq, dk, dv = (g["qkv"][..., i * C:(i + 1) * C] for i in range(3))
        split = lambda t: t.unflatten(-1, (heads, -1))  # noqa: E731
        P.terra_rope_bwd(self.plan, split(g["q"]), split(g["k"]), grid=self.grid, out=(split(dq), split(dk)))
        dv.copy_(g["v"])
        P.terra_linear_bwd(g["qkv"], b["h1"], p["qkv"], out=(g["h1"], g["wqkv"], None), workspace=ws)
        P.terra_rmsnorm_bwd(g["h1"], b["x1"], b["s1"], p["g1"], dz=g["x2"], out=(g["x"], g["g1"]), workspace=ws)
        return g

    def step(self):
        self.forward()
        self.backward()


def reference(p):
    """The same in float64, attention by the oracle."""
    g = Geometry(**GEOM)
    B, H, W, C, heads, hd = (GEOM[n] for n in ("B", "H", "W", "C", "heads", "head_dim"))
    T = B * H * W
    d = {n: v.double() for n, v in p.items()}
    leaves = {n: d[n].clone().requires_grad_() for n in ("x", "qkv", "o", "w1", "w2", "g1", "g2", "bo", "b1", "b2", "table")}
    t = torch.arange(T, device="cuda") % (H * W)
    pos = torch.stack((t // W, t % W), -1).double()
    freqs = torch.tensor(R.rope_freqs(hd // 2, 10000.0), dtype=torch.float64, device="cuda")

    def turn(z):
        z = z.reshape(T, heads, 2, 2, hd // 4)
        ang = (pos[:, :, None] * freqs)[:, None]
        a, b = z.unbind(3)
        return torch.stack((a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()), 3).reshape(B, H, W, C)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, table):
            a = [route(z.detach().cpu().numpy(), g) for z in (q, k, v)]
            ctx.a, ctx.table = a, table.detach().cpu().numpy()
            return torch.from_numpy(unroute(attn_fwd(*a, ctx.table, g)[0], g)).cuda()

        @staticmethod
        def backward(ctx, do):
            dq, dk, dv, dt = attn_bwd(*ctx.a, route(do.cpu().numpy(), g), ctx.table, g)
            return (*(torch.from_numpy(np.ascontiguousarray(unroute(z, g))).cuda() for z in (dq, dk, dv)), torch.from_numpy(dt).cuda())

    def rms(z, gain):
        return z / (z.square().mean(-1, keepdim=True) + EPS).sqrt() * gain

    L = leaves
    x1 = L["x"] + d["r"]
    q, k, v = (rms(x1, L["g1"]) @ L["qkv"].t()).split(C, -1)
    x2 = x1 + Attention.apply(turn(q), turn(k), v, L["table"]) @ L["o"].t() + L["bo"]
    u = rms(x2, L["g2"]) @ L["w1"].t() + L["b1"]
    y = x2 + (u * torch.sigmoid(u)) @ L["w2"].t() + L["b2"]
    y.backward(d["dy"])
    return y.detach(), {n: v.grad for n, v in leaves.items()}


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_block_of_operators(dtype):
    p = params(dtype)
    blk = Block(p)
    y = blk.forward()
    g = blk.backward()
    ry, rg = reference(p)
    near("y", y, ry)
    for mine, theirs in {"x": "x", "wqkv": "qkv", "wo": "o", "w1": "w1", "w2": "w2", "g1": "g1", "g2": "g2", "bo": "bo",
                         "b1": "b1", "b2": "b2", "table": "table"}.items():
        near(mine, g[mine], rg[theirs])


def test_captured_and_replayed():
    """The whole step in one graph; every replay, with eager work between, gives eager's bits for its inputs."""
    p, other = params(BF16), params(BF16, seed=9)
    eager = Block({n: v.clone() for n, v in p.items()})
    blk = Block(p)
    blk.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.step()
    for turn in range(4):
        for n in ("x", "r", "dy", "w1", "g1"):
            p[n].copy_((other if turn % 2 == 0 else params(BF16))[n])
            eager.p[n].copy_(p[n])
        for t in list(blk.b.values()) + list(blk.g.values()):
            t.zero_()
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for name in blk.b:
            assert torch.equal(blk.b[name], eager.b[name]), name
        for name in blk.g:
            assert torch.equal(blk.g[name], eager.g[name]), name


def test_another_stream():
    from paper_2608_15211_amd import operators as ops
    p = params(BF16)
    for s in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            assert ops._raw_stream(0) == torch.cuda.current_stream().cuda_stream and ops._current_device() == torch.cuda.current_device()
    first, blk = Block(p), Block({n: v.clone() for n, v in p.items()})
    first.step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        blk.step()
    s.synchronize()
    for name in blk.b:
        assert torch.equal(blk.b[name], first.b[name]), name
    for name in blk.g:
        assert torch.equal(blk.g[name], first.g[name]), name


def test_two_at_once():
    """Two steps on two streams, eager and as two graphs, each with its own workspace."""
    p = [params(BF16), params(BF16, seed=9)]
    want = [Block({n: v.clone() for n, v in q.items()}) for q in p]
    for w in want:
        w.step()
    blks = [Block(q) for q in p]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        for blk, w in zip(blks, want):
            for mine, theirs in ((blk.b, w.b), (blk.g, w.g)):
                for name in mine:
                    assert torch.equal(mine[name], theirs[name]), name
                    mine[name].zero_()
        torch.cuda.synchronize()

    for _ in range(2):
        for blk, s in zip(blks, streams):
            with torch.cuda.stream(s):
                blk.step()
        same()
    graphs = [torch.cuda.CUDAGraph() for _ in blks]
    for blk, graph in zip(blks, graphs):
        with torch.cuda.graph(graph):
            blk.step()
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        same()


# few tokens, both tile sizes in one and in several slices, whole rounds and a rest, padded copies, any alignment
@pytest.mark.parametrize("M,N,K,dtype", [(7, 300, 520, F16), (130, 1000, 2048, BF16), (300, 2304, 96, F16), (1017, 771, 1003, BF16),
                                         (2000, 2000, 2003, F16), (11000, 1536, 64, BF16), (20000, 64, 64, F16)])
def test_linear_captured(M, N, K, dtype):
    """Graphs whose outputs and workspaces were allocated while they were captured."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, dy = (torch.empty(*d, dtype=dtype, device="cuda") for d in ((M, K), (N, K), (M, N)))
    bias = torch.randn(N, generator=g, device="cuda")

    def step():
        pre = torch.empty(M, N, dtype=dtype, device="cuda")
        y = P.terra_linear_fwd(x, w, bias, act="silu", pre=pre)
        return (y, pre, *P.terra_linear_bwd(dy, x, w, pre, act="silu"))

    def fill():
        for t in (x, w, dy):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    fill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        fill()
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
            a.zero_()


@pytest.mark.parametrize("rows", [1, 16, 40, 333])
def test_norm_into_8_bit_product(rows):
    """The norm's 8-bit output and scales are what the product takes."""
    C, N = 512, 200
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(rows, C, generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.randn(N, C, generator=g, device="cuda") / C ** 0.5
    ws = (w.abs().amax(1) / 448)
    wq = (w / ws[:, None]).to(E4M3)
    q, s = torch.empty(rows, C, dtype=E4M3, device="cuda"), torch.empty(rows, device="cuda")
    y, z = P.terra_rmsnorm_fwd(x, None, res=r, q=q, q_scale=s)
    assert y is None
    out = P.terra_linear_fwd(q, wq, act="gelu", res=None, x_scale=s, w_scale=ws)
    t, ref, off = R.lin_fwd(q.float(), wq.float(), None, "gelu", None, s, ws)
    R.within("product", out, ref, R.lin_fwd_bound(t, ref, off, BF16, "gelu", None))
    # against the norm and the product without 8 bits: each element of either is off by at most
    # 2^-4 of itself (and of the smallest scale's step), so that each product is off by 2.1 2^-4
    zz, yy, _ = R.rms_fwd(x, r, None, EPS)
    plain = yy @ w.double().t()
    room = 2.1 * 2.0 ** -4 * (yy.abs() @ w.double().abs().t()) + 2.0 ** -10 * (s.double()[:, None] * w.double().abs().sum(1) + yy.abs().sum(1, keepdim=True) * ws.double())
    R.within("8 bits", R.lin_fwd(q.float(), wq.float(), None, "none", None, s, ws)[0], plain, room)
