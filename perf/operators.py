"""The Transformer operators around the window attention, as they are measured:
the root-mean-square norm with the residual's addition and an 8-bit output, the
linear layer with its epilogue, and rotary positions.

`run` computes a case in plain torch operations, or, where `own` is true, with
the library's calls.  Inputs follow the repository's synthetic recipes
(standard normal activations, weights N(0,1)/sqrt(fan_in), gains 1 + 0.1 N(0,1),
biases 0.02 N(0,1)), drawn on the device.

    norm_fwd    z = x + res; y = gain z / sqrt(mean(z^2) + eps): z, y and 1/rms, or z
                and y in e4m3 with one scale a row
    norm_bwd    dx (also the residual's gradient) and the gain's gradient
    lin_fwd     y = act(x w^T + bias) + res, x and w in 16 bits, or in e4m3 with a scale
                for each row of x and of w
    lin_bwd     the gradients of x, w and bias from dy and the stored pre-activation
    rope_fwd    the pairs of q and k turned by their positions' angles
    rope_bwd    the gradients turned back
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-5
E4M3_MAX, SCALE_MIN = 448.0, 2.0 ** -126


# -------------------------------------------------------------------- cases
def _norm(name, op, dtype, rows, cols, q8=False, res=True):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "cols": cols, "q8": q8, "res": res}


def _lin(name, op, dtype, M, N, K, act="none", bias=True, res=False, pre=False, dw="f32"):
    c = {"name": name, "op": op, "dtype": dtype, "M": M, "N": N, "K": K, "act": act, "bias": bias}
    c.update({"dw": dw} if op == "lin_bwd" else {"res": res, "pre": pre})
    return c


def _rope(name, op, dtype, B, H, W, q_heads, k_heads, hd, rot, axes, layout, base=10000.0, scaling="none", factor=1.0,
          orig=0, far=0, packed=False):
    """far: the positions are given, up to this one; 0: the grid's own.  packed: q and k are parts of one tensor."""
    return {"name": name, "op": op, "dtype": dtype, "B": B, "H": H, "W": W, "q_heads": q_heads, "k_heads": k_heads,
            "hd": hd, "rot": rot, "axes": axes, "layout": layout, "base": base, "scaling": scaling, "factor": factor,
            "orig": orig, "far": far, "packed": packed}


def listed():
    return [
        # one token of a model of width 4096 on its way into an 8-bit product: latency
        _norm("norm_fwd_1x4096_q8", "norm_fwd", "f16", 1, 4096, q8=True),
        # a training step's norm on one latitude slab, 128 x 1080 tokens of width 768
        _norm("norm_fwd_138240x768", "norm_fwd", "bf16", 138240, 768),
        # neither a whole number of vectors a row nor of rows a workgroup
        _norm("norm_fwd_15301x1001_q8", "norm_fwd", "bf16", 15301, 1001, q8=True),
        # the slab's backward, with the gradient that comes down the residual stream
        _norm("norm_bwd_138240x768", "norm_bwd", "bf16", 138240, 768),
        # the first MLP layer for one token
        _lin("lin_fwd_1x4096x1024", "lin_fwd", "bf16", 1, 4096, 1024, act="gelu"),
        # an output projection with its residual for a few tokens, 8-bit weights
        _lin("lin_fwd_16x4096x4096_e4m3", "lin_fwd", "e4m3", 16, 4096, 4096, res=True),
        # the QKV projection of the slab
        _lin("lin_fwd_138240x2304x768", "lin_fwd", "bf16", 138240, 2304, 768),
        # the first MLP layer of a quarter slab at width 1536, 8-bit operands
        _lin("lin_fwd_34560x6144x1536_e4m3", "lin_fwd", "e4m3", 34560, 6144, 1536, act="gelu"),
        # odd in every direction, activation and residual
        _lin("lin_fwd_1017x771x1003_f16", "lin_fwd", "f16", 1017, 771, 1003, act="silu", res=True, pre=True),
        # the first MLP layer's backward, a quarter slab at width 1024
        _lin("lin_bwd_34560x4096x1024", "lin_bwd", "bf16", 34560, 4096, 1024, act="gelu", dw="bf16"),
        # one long sequence, far positions, part of the head, grouped heads, float32
        _rope("rope_bwd_f32_4097_yarn", "rope_bwd", "f32", 1, 1, 4097, 8, 2, 128, 64, 1, "interleaved", 1e6, "yarn", 8.0,
              8192, far=1000000),
        # the slab's grid, rows turn one half of the head and columns the other; q and k as the QKV product leaves them
        _rope("rope_fwd_138240_24x32", "rope_fwd", "bf16", 1, 128, 1080, 24, 24, 32, 32, 2, "half", packed=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly a multiple of 64, now and then any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.3 or n < 96 else (n + 32) // 64 * 64


def draw(rng):
    """One more case: any operator, direction, type and size that the listed ones stand for."""
    most = {"bytes": max(work(c)["bytes"] for c in listed()), "flops": max(work(c)["flops"] for c in listed())}
    while True:
        kind = rng.choice(("norm", "lin", "lin", "rope"))
        if kind == "norm":
            op = rng.choice(("norm_fwd", "norm_fwd", "norm_bwd"))
            case = _norm(None, op, rng.choice(("bf16", "bf16", "f16", "f32")), _log(rng, 1, 138240), _width(rng, 64, 8192),
                         op == "norm_fwd" and rng.random() < 0.4, rng.random() < 0.8)
        elif kind == "lin":
            op = rng.choice(("lin_fwd", "lin_fwd", "lin_bwd"))
            act = rng.choice(("none", "relu", "gelu", "silu"))
            dtype = rng.choice(("bf16", "bf16", "f16") if op == "lin_bwd" else ("bf16", "bf16", "f16", "e4m3"))
            M = _log(rng, 1, 64) if rng.random() < 0.3 else _log(rng, 64, 138240)
            case = _lin(None, op, dtype, M, _width(rng, 64, 8192), _width(rng, 64, 8192), act, rng.random() < 0.8,
                        rng.random() < 0.5, act != "none" and rng.random() < 0.5, "f32" if act == "none" else dtype)
        else:
            axes, hd = rng.choice((1, 2)), rng.choice((32, 64, 128))
            rot = hd if rng.random() < 0.6 else rng.randrange(2 * axes, hd + 1, 2 * axes)
            H, W = (1, _log(rng, 1, 138240)) if axes == 1 else (_log(rng, 1, 256), _log(rng, 1, 1080))
            q_heads = rng.choice((4, 8, 12, 24, 32))
            scaling = rng.choice(("none", "none", "linear", "ntk", "yarn")) if rot > 2 * axes else "none"
            case = _rope(None, rng.choice(("rope_fwd", "rope_bwd")), rng.choice(("bf16", "bf16", "f16", "f32")),
                         rng.choice((1, 1, 2)), H, W, q_heads, rng.choice((q_heads, q_heads, q_heads // 4, 1)), hd, rot,
                         axes, rng.choice(("interleaved", "half")), rng.choice((100.0, 10000.0, 1e6)), scaling,
                         1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)), 8192 if scaling == "yarn" else 0,
                         _log(rng, 1000, 1 << 24) if rng.random() < 0.4 else 0, rng.random() < 0.5)
        del case["name"]
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def work(case):
    """Each input read once, each output written once; the products' multiplications and additions."""
    s = SIZES[case["dtype"]]
    if case["op"].startswith("norm"):
        n, rows, cols = case["rows"] * case["cols"], case["rows"], case["cols"]
        if case["op"] == "norm_fwd":
            moved = n * s * (3 if case["res"] else 1) + (n + 4 * rows if case["q8"] else n * s + 4 * rows) + 4 * cols
            return {"bytes": moved, "flops": 6 * n}
        return {"bytes": n * s * (4 if case["res"] else 3) + 4 * rows + 8 * cols, "flops": 10 * n}
    if case["op"].startswith("lin"):
        M, N, K = case["M"], case["N"], case["K"]
        if case["op"] == "lin_fwd":
            moved = (M + N) * K * s + M * N * 2 * (1 + case["res"] + case["pre"]) + 4 * N * case["bias"]
            return {"bytes": moved + (4 * (M + N) if s == 1 else 0), "flops": 2 * M * N * K}
        moved = M * N * s * (2 if case["act"] != "none" else 1) + 2 * M * K * s + N * K * (s + SIZES[case["dw"]])
        return {"bytes": moved + 4 * N * case["bias"], "flops": 4 * M * N * K}
    T = case["B"] * case["H"] * case["W"]
    n = T * (case["q_heads"] + case["k_heads"]) * case["hd"]
    return {"bytes": 2 * n * s + (4 * T * case["axes"] if case["far"] else 0), "flops": 3 * n}


# ------------------------------------------------------------------- inputs
def _quantised(x):
    scale = (x.abs().amax(dim=-1, keepdim=True) / E4M3_MAX).clamp_min(SCALE_MIN)
    return (x / scale).to(torch.float8_e4m3fn), scale.squeeze(-1)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*dims):
        return torch.randn(*dims, generator=gen, device="cuda")

    s = {}
    if case["op"].startswith("norm"):
        shape = (case["rows"], case["cols"])
        s["gain"] = 1 + 0.1 * normal(case["cols"])
        if case["op"] == "norm_fwd":
            s["x"] = normal(*shape).to(dt)
            s["res"] = (2 * normal(*shape)).to(dt) if case["res"] else None
        else:
            # what the forward left: z as it is stored, and its 1/rms
            s["z"], s["dy"] = (2 * normal(*shape)).to(dt), normal(*shape).to(dt)
            s["rstd"] = (s["z"].float().square().mean(dim=-1) + EPS).rsqrt()
            s["dz"] = normal(*shape).to(dt) if case["res"] else None
    elif case["op"].startswith("lin"):
        M, N, K = case["M"], case["N"], case["K"]
        x, w = normal(M, K), normal(N, K) / math.sqrt(K)
        out = torch.bfloat16 if case["dtype"] == "e4m3" else dt
        s["x_scale"] = s["w_scale"] = None
        if case["dtype"] == "e4m3":
            (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _quantised(x), _quantised(w)
        else:
            s["x"], s["w"] = x.to(dt), w.to(dt)
        if case["op"] == "lin_fwd":
            s["bias"] = 0.02 * normal(N) if case["bias"] else None
            s["res"] = normal(M, N).to(out) if case["res"] else None
        else:
            s["dy"] = normal(M, N).to(dt)
            s["pre"] = normal(M, N).to(dt) if case["act"] != "none" else None
    else:
        T, hd = case["B"] * case["H"] * case["W"], case["hd"]
        heads = (case["q_heads"], case["k_heads"])
        if case["packed"]:
            # two parts of a projection's output, whose rows also hold the values
            s["q"], s["k"], _ = normal(T, heads[0] + 2 * heads[1], hd).to(dt).split((*heads, heads[1]), dim=1)
        else:
            s["q"], s["k"] = normal(T, heads[0], hd).to(dt), normal(T, heads[1], hd).to(dt)
        s["pos"] = None
        if case["far"]:
            s["pos"] = torch.randint(0, case["far"], (T, case["axes"]), generator=gen, device="cuda", dtype=torch.int32)
    return s


def prepare(case, seed):
    """The inputs, and where the library runs the buffers and the plan that a program keeps."""
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2608_15211_amd as terra

        def empty(*dims, dtype=DTYPES[case["dtype"]]):
            return torch.empty(*dims, dtype=dtype, device="cuda")

        if case["op"] == "norm_fwd":
            rows, cols, q8 = case["rows"], case["cols"], case["q8"]
            s["out"] = {"z": empty(rows, cols) if case["res"] else None, "out": None if q8 else empty(rows, cols),
                        "rstd": None if q8 else empty(rows, dtype=torch.float32),
                        "q": empty(rows, cols, dtype=torch.float8_e4m3fn) if q8 else None,
                        "q_scale": empty(rows, dtype=torch.float32) if q8 else None}
        elif case["op"] == "norm_bwd":
            s["out"] = (empty(case["rows"], case["cols"]), empty(case["cols"], dtype=torch.float32))
            s["ws"] = empty(terra.terra_rmsnorm_bwd_workspace_bytes(case["rows"], case["cols"]), dtype=torch.uint8)
        elif case["op"].startswith("lin"):
            M, N, K = case["M"], case["N"], case["K"]
            need = terra.terra_linear_fwd_workspace_bytes if case["op"] == "lin_fwd" else terra.terra_linear_bwd_workspace_bytes
            s["ws"] = empty(need(M, N, K, case["dtype"]), dtype=torch.uint8)
            if case["op"] == "lin_fwd":
                to = torch.bfloat16 if case["dtype"] == "e4m3" else DTYPES[case["dtype"]]
                s["out"] = {"out": empty(M, N, dtype=to), "pre": empty(M, N, dtype=to) if case["pre"] else None}
            else:
                s["out"] = (empty(M, K), empty(N, K, dtype=DTYPES[case["dw"]]),
                            empty(N, dtype=torch.float32) if case["bias"] else None)
        else:
            s["plan"] = terra.terra_plan_rope(case["hd"], rot_dim=case["rot"], axes=case["axes"], layout=case["layout"],
                                              base=case["base"], scaling=case["scaling"], factor=case["factor"],
                                              orig_len=case["orig"])
            s["out"] = (empty(*s["q"].shape), empty(*s["k"].shape))
    return s


# ------------------------------------------------------------- plain forms
def _act(t, act):
    if act == "gelu":
        return 0.5 * t * (1 + torch.erf(t * math.sqrt(0.5)))
    return t if act == "none" else t * (t > 0) if act == "relu" else t / (1 + torch.exp(-t))


def _act_grad(t, act):
    if act == "relu":
        return (t > 0).to(t.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(t * math.sqrt(0.5))) + t * torch.exp(-0.5 * t * t) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-t))
    return s * (1 + t * (1 - s))


def _norm_fwd(case, s):
    dt = DTYPES[case["dtype"]]
    z = s["x"].float()
    if case["res"]:
        z = z + s["res"].float()
    rstd = 1 / torch.sqrt((z * z).mean(dim=-1) + EPS)
    y = z * rstd.unsqueeze(-1) * s["gain"]
    kept = {"z": z.to(dt)} if case["res"] else {}
    if not case["q8"]:
        return {"y": y.to(dt), "rstd": rstd, **kept}
    q, scale = _quantised(y)
    return {"q": q, "scale": scale, **kept}


def _norm_bwd(case, s):
    z, dy, rstd = s["z"].float(), s["dy"].float(), s["rstd"].unsqueeze(-1)
    g, zh = dy * s["gain"], z * rstd
    dx = rstd * (g - zh * (g * zh).mean(dim=-1, keepdim=True))
    if case["res"]:
        dx = dx + s["dz"].float()
    return {"dx": dx.to(DTYPES[case["dtype"]]), "dgain": (dy * zh).sum(dim=0)}


def _lin_fwd(case, s):
    to = torch.bfloat16 if case["dtype"] == "e4m3" else DTYPES[case["dtype"]]
    t = s["x"].float() @ s["w"].float().t()
    if case["dtype"] == "e4m3":
        t = t * s["x_scale"].unsqueeze(-1) * s["w_scale"]
    if case["bias"]:
        t = t + s["bias"]
    y = _act(t, case["act"])
    if case["res"]:
        y = y + s["res"].float()
    return {"y": y.to(to), **({"pre": t.to(to)} if case["pre"] else {})}


def _lin_bwd(case, s):
    dt = s["dy"].float()
    if case["act"] != "none":
        dt = dt * _act_grad(s["pre"].float(), case["act"])
    dx, dw = dt @ s["w"].float(), dt.t() @ s["x"].float()
    db = {"db": dt.sum(dim=0)} if case["bias"] else {}
    return {"dx": dx.to(DTYPES[case["dtype"]]), "dw": dw.to(DTYPES[case["dw"]]), **db}


def _positions(case, s):
    if s["pos"] is not None:
        return s["pos"].double()
    t = torch.arange(case["B"] * case["H"] * case["W"], device="cuda")
    if case["axes"] == 1:
        return (t % (case["H"] * case["W"])).double().unsqueeze(-1)
    return torch.stack((t // case["W"] % case["H"], t % case["W"]), dim=-1).double()


def _frequencies(case):
    """Angle a position, of each pair of one axis, and the factor on cosine and sine."""
    part, f = case["rot"] // case["axes"], case["factor"]
    i = torch.arange(part // 2, dtype=torch.float64, device="cuda")
    base = case["base"] * f ** (part / (part - 2)) if case["scaling"] == "ntk" else case["base"]
    freq = torch.exp(-2 * i / part * math.log(base))
    if case["scaling"] == "linear":
        freq = freq / f
    if case["scaling"] == "yarn":
        keep = ((case["orig"] * freq / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        freq = freq * (keep + (1 - keep) / f)
    return freq, 0.1 * math.log(f) + 1 if case["scaling"] == "yarn" else 1.0


def _rope_run(case, s):
    """Forward, or with the angles' signs turned round backward: all heads of q and k at once."""
    freq, scale = _frequencies(case)
    angle = _positions(case, s).unsqueeze(-1) * freq                     # token, axis, pair
    sign = 1.0 if case["op"] == "rope_fwd" else -1.0
    cos = (scale * torch.cos(angle)).float().unsqueeze(1)
    sin = (sign * scale * torch.sin(angle)).float().unsqueeze(1)
    x = torch.cat((s["q"], s["k"]), dim=1).float()
    T, heads, axes, rot = x.shape[0], x.shape[1], case["axes"], case["rot"]
    r = x[:, :, :rot].reshape(T, heads, axes, *((rot // axes // 2, 2) if case["layout"] == "interleaved" else (2, rot // axes // 2)))
    a, b = r.unbind(-1 if case["layout"] == "interleaved" else -2)
    turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1 if case["layout"] == "interleaved" else -2)
    y = torch.cat((turned.reshape(T, heads, rot), x[:, :, rot:]), dim=-1).to(DTYPES[case["dtype"]])
    q, k = y.split((case["q_heads"], case["k_heads"]), dim=1)
    return {"q": q, "k": k}


def run(s):
    case = s["case"]
    if not own:
        return {"norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd, "lin_fwd": _lin_fwd, "lin_bwd": _lin_bwd,
                "rope_fwd": _rope_run, "rope_bwd": _rope_run}[case["op"]](case, s)
    import paper_2608_15211_amd as terra

    op, out = case["op"], s["out"]
    if op == "norm_fwd":
        terra.terra_rmsnorm_fwd(s["x"], s["gain"], res=s["res"], eps=EPS, **out)
        kept = {"z": out["z"]} if case["res"] else {}
        return {"q": out["q"], "scale": out["q_scale"], **kept} if case["q8"] else {"y": out["out"], "rstd": out["rstd"], **kept}
    if op == "norm_bwd":
        terra.terra_rmsnorm_bwd(s["dy"], s["z"], s["rstd"], s["gain"], dz=s["dz"], out=out, workspace=s["ws"])
        return {"dx": out[0], "dgain": out[1]}
    if op == "lin_fwd":
        terra.terra_linear_fwd(s["x"], s["w"], s["bias"], act=case["act"], res=s["res"], x_scale=s["x_scale"],
                               w_scale=s["w_scale"], workspace=s["ws"], **out)
        return {"y": out["out"], **({"pre": out["pre"]} if case["pre"] else {})}
    if op == "lin_bwd":
        terra.terra_linear_bwd(s["dy"], s["x"], s["w"], s["pre"], act=case["act"], out=out, workspace=s["ws"])
        return {"dx": out[0], "dw": out[1], **({"db": out[2]} if case["bias"] else {})}
    call = terra.terra_rope_fwd if op == "rope_fwd" else terra.terra_rope_bwd
    grid = None if case["far"] else (case["H"], case["W"])
    call(s["plan"], s["q"], s["k"], pos=s["pos"], grid=grid, out=out)
    return {"q": out[0], "k": out[1]}


# ------------------------------------------------------------ in 64 bits
def _nearest_e4m3(v):
    """The e4m3 value next to each of v: 3 bits after the leading one, exponents from -6, ties to the even one."""
    exponent = torch.frexp(v.abs()).exponent - 1
    step = torch.ldexp(torch.ones_like(v), exponent.clamp_min(-6) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = {n: t.double() if isinstance(t, torch.Tensor) else t for n, t in _inputs(case, seed).items()}
    op = case["op"]
    if op == "norm_fwd":
        z = s["x"] + s["res"] if case["res"] else s["x"]
        mean = torch.linalg.vector_norm(z, dim=1).pow(2) / case["cols"]
        y = s["gain"] * z / (mean + EPS).sqrt()[:, None]
        kept = {"z": z} if case["res"] else {}
        if not case["q8"]:
            return {"y": y, "rstd": (mean + EPS) ** -0.5, **kept}
        scale = torch.maximum(y.max(dim=1).values, -y.min(dim=1).values) / E4M3_MAX
        return {"q": _nearest_e4m3(y / scale[:, None]), "scale": scale, **kept}
    if op == "norm_bwd":
        # y_i = gain_i z_i r: dy_i/dz_j = gain_i r (delta_ij - z_i z_j r^2 / cols)
        r, a = s["rstd"][:, None], s["dy"] * s["gain"]
        dx = r * a - s["z"] * r ** 3 * torch.linalg.vecdot(a, s["z"], dim=1)[:, None] / case["cols"]
        dgain = torch.mv((s["dy"] * s["z"]).t(), s["rstd"])
        return {"dx": dx + s["dz"] if case["res"] else dx, "dgain": dgain}
    if op == "lin_fwd":
        if case["dtype"] == "e4m3":
            s["x"], s["w"] = s["x"] * s["x_scale"][:, None], s["w"] * s["w_scale"][:, None]
        t = torch.matmul(s["w"], s["x"].t()).t()
        t = t + s["bias"] if case["bias"] else t
        y = {"none": lambda v: v, "relu": lambda v: v.clamp_min(0), "silu": lambda v: v * torch.sigmoid(v),
             "gelu": lambda v: v * torch.special.ndtr(v)}[case["act"]](t)
        return {"y": y + s["res"] if case["res"] else y, **({"pre": t} if case["pre"] else {})}
    if op == "lin_bwd":
        d, p = s["dy"], s["pre"]
        if case["act"] == "relu":
            d = torch.where(p > 0, d, 0.0)
        elif case["act"] == "gelu":
            d = d * (torch.special.ndtr(p) + p * torch.exp(-p * p / 2) * (2 * math.pi) ** -0.5)
        elif case["act"] == "silu":
            d = d * torch.sigmoid(p) * (1 + p * torch.sigmoid(-p))
        dw = torch.matmul(s["x"].t(), d).t()
        return {"dx": torch.matmul(s["w"].t(), d.t()).t(), "dw": dw, **({"db": torch.mv(d.t(), torch.ones_like(d[:, 0]))} if case["bias"] else {})}
    # each pair as a complex number, multiplied by scale exp(i angle), backward by its conjugate
    axes, rot, T = case["axes"], case["rot"], case["B"] * case["H"] * case["W"]
    part = rot // axes
    pos = s["pos"]
    if pos is None:
        u, v = torch.meshgrid(torch.arange(case["H"], device="cuda"), torch.arange(case["W"], device="cuda"), indexing="ij")
        one = (u * case["W"] + v)[..., None] if axes == 1 else torch.stack((u, v), dim=-1)
        pos = one.reshape(1, -1, axes).expand(case["B"], -1, -1).reshape(T, axes).double()
    f, scale = [], 1.0
    for i in range(part // 2):
        base, div = case["base"], 1.0
        if case["scaling"] == "linear":
            div = case["factor"]
        if case["scaling"] == "ntk":
            base *= case["factor"] ** (part / (part - 2))
        g = base ** (-2 * i / part)
        if case["scaling"] == "yarn":
            # kept where a pair turns 32 times or more over the original length, divided below one turn
            ramp = min(1.0, max(0.0, (case["orig"] * g / (2 * math.pi) - 1) / 31))
            div = 1 / (ramp + (1 - ramp) / case["factor"])
            scale = 0.1 * math.log(case["factor"]) + 1
        f.append(g / div)
    turn = pos[:, :, None] * torch.tensor(f, dtype=torch.float64, device="cuda") * (1 if op == "rope_fwd" else -1)
    turn = torch.polar(torch.full_like(turn, scale), turn)[:, None]
    outs = {}
    for n in ("q", "k"):
        y = s[n].clone()
        for a in range(axes):
            lo = a * part
            at = (slice(lo, lo + part, 2), slice(lo + 1, lo + part, 2))
            if case["layout"] == "half":
                at = (slice(lo, lo + part // 2), slice(lo + part // 2, lo + part))
            c = torch.complex(s[n][:, :, at[0]], s[n][:, :, at[1]]) * turn[:, :, a]
            y[:, :, at[0]], y[:, :, at[1]] = c.real, c.imag
        outs[n] = y
    return outs
