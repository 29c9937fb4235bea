"""Plain float64 forms of the norm, the linear layer and the rotary positions,
with the error bounds the kernels are held to (u = 2^-24, float32's half step;
half(t) = a type's half step)."""

import math

import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def within(name, got, ref, bound):
    """Every element of got within bound (a tensor or number, absolute) of ref; NaN where ref has NaN."""
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), "%s: NaN in other places" % name
    over = ((got - ref).abs() - bound)[~nan & (got != ref)]
    assert not over.numel() or float(over.max()) <= 0, "%s: %d of %d elements outside the bound, by up to %.3g" % (
        name, int((over > 0).sum()), ref.numel(), float(over.max()))


# --------------------------------------------------------------------- norm
def rms_fwd(x, res, gain, eps):
    z = x.double() + (0 if res is None else res.double())
    rstd = 1 / (z.square().mean(-1) + eps).sqrt()
    y = z * rstd[..., None] * (1 if gain is None else gain.double())
    return z, y, rstd


def rms_terms(cols):
    """Roundings of a float32 rstd, in u: up to 32 squares in a row (cols / 1024 in
    the longest rows) and 26 sums of lanes and waves, halved by the root, and 4 of its own;
    two more of a product."""
    return (max(32, cols / 1024) + 26) / 2 + 6


def rms_bwd(dy, z, rstd, gain, dz):
    """dx, dgain and the sums of magnitudes that their roundings go with."""
    d, z, r = dy.double(), z.double(), rstd.double()[..., None]
    g = d * (1 if gain is None else gain.double())
    zh = z * r
    m = (g * zh).mean(-1, keepdim=True)
    dx = r * (g - zh * m) + (0 if dz is None else dz.double())
    mag = r * (g.abs() + zh.abs() * (g * zh).abs().mean(-1, keepdim=True)) + (0 if dz is None else dz.double().abs())
    flat = (d * zh).reshape(-1, z.shape[-1])
    return dx, flat.sum(0), mag, flat.abs().sum(0)


# ------------------------------------------------------------------- linear
def act(t, name):
    if name == "relu":
        return t.clamp_min(0)
    if name == "gelu":
        return 0.5 * t * (1 + torch.erf(t / math.sqrt(2)))
    return t * torch.sigmoid(t) if name == "silu" else t


def act_grad(t, name):
    if name == "relu":
        return (t > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(t / math.sqrt(2))) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(t)
    return s * (1 + t * (1 - s)) if name == "silu" else torch.ones_like(t)


def lin_fwd(x, w, bias, name, res, x_scale=None, w_scale=None):
    """t, y and the bound on t before it is rounded: K sums of a row's products.

    Of 8-bit operands the matrix instruction adds each eight neighbours as integers
    that are aligned to the largest of the eight products and cut 13 bits below its leading
    one (seen on the instruction itself: beside +256 and -256 a third product s of the eight
    counts down to s = 2^-5 and is cut toward zero there, beside products of other
    eights it counts in full).  The other seven lose less than 2^-13 of the largest each,
    and that is at most the product of the two largest magnitudes of the eight."""
    x, w = x.double(), w.double()
    if x_scale is not None:
        x, w = x * x_scale.double()[..., None], w * w_scale.double()[:, None]
    t, mag = x @ w.t(), x.abs() @ w.abs().t()
    cut = 0
    if x_scale is not None:
        gx, gw = (torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 8)).unflatten(-1, (-1, 8)).amax(-1) for v in (x, w))
        cut = 7 * 2.0 ** -13 * (gx @ gw.t())
    if bias is not None:
        t, mag = t + bias.double(), mag + bias.double().abs()
    y = act(t, name) + (0 if res is None else res.double())
    return t, y, (x.shape[-1] + 4) * U * mag + cut


def lin_fwd_bound(t, y, off, dtype, name, res):
    """Of y: its rounding, t's error (no activation is steeper than 1.13), the
    activation's own (4e-7; exponential and reciprocal of silu to 4 u of t) and the residual's sum."""
    own = 0 if name in ("none", "relu") else 4e-7 + 8 * U * t.abs()
    more = U * (y.abs() + (0 if res is None else res.double().abs()))
    return half(dtype) * y.abs() + (1 + half(dtype)) * (1.13 * off + own + more) + torch.finfo(dtype).tiny


def lin_bwd(dy, x, w, pre, name):
    """(dx, dw, db) and their sums of magnitudes."""
    N, K = w.shape
    dy, x, w = dy.double().reshape(-1, N), x.double().reshape(-1, K), w.double()
    dt = dy * (act_grad(pre.double().reshape(-1, N), name) if name != "none" else 1)
    a = dt.abs() + (1e-6 * dy.abs() if name in ("gelu", "silu") else 0)
    return (dt @ w, dt.t() @ x, dt.sum(0)), (a @ w.abs(), a.t() @ x.abs(), a.sum(0)), dy.abs().sum(0)


# --------------------------------------------------------------------- rope
def rope_freqs(part, base, scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0):
    out = []
    for i in range(part // 2):
        b = base * factor ** (part / (part - 2)) if scaling == "ntk" else base
        f = b ** (-2 * i / part)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            g = (orig_len * f / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow)
            g = min(1.0, max(0.0, g))
            f = f * (g + (1 - g) / factor)
        out.append(f)
    return out


def rope(x, pos, freqs, axes, rot, layout, scale, sign=1):
    """x (tokens, heads, hd), pos (tokens, axes): turned x and its bound before rounding:
    cosine and sine to 2.5e-7 (the angle's 2^-25 and a polynomial's 3e-8, each with its
    float32 steps), two products and a sum."""
    y, off = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    part = rot // axes
    for a in range(axes):
        for i, f in enumerate(freqs):
            lo, hi = (a * part + 2 * i, a * part + 2 * i + 1) if layout == "interleaved" else \
                (a * part + i, a * part + i + part // 2)
            ang = sign * pos[:, a].double()[:, None] * f
            c, s = scale * torch.cos(ang), scale * torch.sin(ang)
            p, q = x[:, :, lo].double(), x[:, :, hi].double()
            y[:, :, lo], y[:, :, hi] = p * c - q * s, p * s + q * c
            off[:, :, lo] = off[:, :, hi] = scale * (2.5e-7 + 3 * U) * (p.abs() + q.abs())
    return y, off
