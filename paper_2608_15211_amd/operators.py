"""The operators around the attention: root-mean-square norm, linear layer and
rotary positions (C ABI in include/terra_swin.h, same names).

As in the rest of the binding, torch tensors are device memory and every step
runs in the library's kernels on the current stream of the tensors' device.
Tensors may be views: a matrix is any tensor whose last dimension is contiguous
and whose leading ones step through memory at one stride, rows not overlapping.
Outputs and workspaces are allocated where they are not given.
"""

import ctypes

import torch

from . import TERRA_BF16, TERRA_F16, TERRA_F32, _check
from . import lib as _load

TERRA_E4M3 = 3
TERRA_ROPE_MAX_PAIRS = 128

_CODES = {torch.float32: TERRA_F32, torch.bfloat16: TERRA_BF16, torch.float16: TERRA_F16, torch.float8_e4m3fn: TERRA_E4M3,
          "f32": TERRA_F32, "bf16": TERRA_BF16, "f16": TERRA_F16, "e4m3": TERRA_E4M3}
_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_LAYOUTS = {"interleaved": 0, "half": 1}
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class terra_rmsnorm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("eps", ctypes.c_float)] + \
        [(n, ctypes.c_int64) for n in ("x_ld", "res_ld", "z_ld", "y_ld", "q_ld")]


class terra_linear_desc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int32), ("K", ctypes.c_int32)] + \
        [(n, ctypes.c_int64) for n in ("x_ld", "w_ld", "y_ld", "res_ld", "pre_ld", "dx_ld", "dw_ld")] + \
        [("act", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


class terra_rope_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("head_dim", "rot_dim", "axes", "layout", "scaling")] + \
        [(n, ctypes.c_double) for n in ("base", "factor", "orig_len", "beta_fast", "beta_slow", "attn_scale")]


class terra_rope_plan(ctypes.Structure):
    _fields_ = [("desc", terra_rope_desc), ("pairs", ctypes.c_int32), ("scale", ctypes.c_float),
                ("turns", ctypes.c_uint64 * TERRA_ROPE_MAX_PAIRS)]


class terra_rope_tensor(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("heads", ctypes.c_int32)] + \
        [(n, ctypes.c_int64) for n in ("in_token", "in_head", "out_token", "out_head")]


_lib = None


def lib():
    """The loaded library, these entry points' argument types declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = _load()
    p, vp, i32, i64, sz = ctypes.POINTER, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    types = {"terra_rmsnorm_fwd": [p(terra_rmsnorm_desc), i32] + [vp] * 9,
             "terra_rmsnorm_bwd": [p(terra_rmsnorm_desc), i32] + [vp] * 8 + [sz, vp],
             "terra_linear_fwd": [p(terra_linear_desc), i32] + [vp] * 9 + [sz, vp],
             "terra_linear_bwd": [p(terra_linear_desc), i32] + [vp] * 6 + [i32, vp, vp, sz, vp],
             "terra_plan_rope": [p(terra_rope_desc), p(terra_rope_plan)]}
    for name in ("terra_rope_fwd", "terra_rope_bwd"):
        types[name] = [p(terra_rope_plan), i32, i64, vp, i32, i32, p(terra_rope_tensor), p(terra_rope_tensor), vp]
    for name, args in types.items():
        getattr(L, name).argtypes = args
        getattr(L, name).restype = i32
    for name, args in {"terra_rmsnorm_bwd_workspace_bytes": [i64, i32],
                       "terra_linear_fwd_workspace_bytes": [i64, i32, i32, i32],
                       "terra_linear_bwd_workspace_bytes": [i64, i32, i32, i32]}.items():
        getattr(L, name).argtypes = args
        getattr(L, name).restype = sz
    _lib = L
    return L


# ---------------------------------------------------------------- arguments
def _code(dtype):
    try:
        return _CODES[dtype]
    except KeyError:
        raise TypeError("unsupported dtype %r" % (dtype,)) from None


def _choice(value, choices, name):
    try:
        return choices[value]
    except KeyError:
        raise ValueError("%s must be one of %s, not %r" % (name, ", ".join(choices), value)) from None


def _i32(n):
    """A size for one of the library's 32-bit integers, which ctypes would cut to its low bits:
    what does not fit becomes the largest, and that is refused."""
    return n if -0x80000000 <= n < 0x80000000 else 0x7fffffff


def _on(t, name, device, dtype):
    if t.get_device() != device:
        raise ValueError("%s is on %s, expected cuda:%d" % (name, t.device, device))
    if t.dtype is not dtype:
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))


def _step(sizes, strides, name):
    """The one stride at which the places of some leading dimensions follow each other (None: at most one place)."""
    step = span = None
    for n, s in zip(reversed(sizes), reversed(strides)):
        if n == 1:
            continue
        if step is None:
            step = span = s
        if s != span:
            raise ValueError("%s: its rows do not follow each other at one stride" % name)
        span = s * n
    return step


def _stride(t, name):
    """Row stride of a matrix."""
    if t.is_contiguous():
        return t.shape[-1] if t.dim() else 1
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError("%s must be contiguous along its last dimension" % name)
    step = _step(t.shape[:-1], t.stride()[:-1], name)
    if step is None:
        return t.shape[-1]
    if step < t.shape[-1]:
        raise ValueError("%s: its rows overlap" % name)
    return step


def _matrix(t, name, device, dtype, rows, cols):
    """(address, row stride) of a rows x cols matrix; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.get_device() != device:
        _on(t, name, device, dtype)
    shape = t.shape
    if not shape or shape[-1] != cols or t.numel() != rows * cols:
        raise ValueError("%s has shape %s, expected %d rows of %d" % (name, tuple(shape), rows, cols))
    return t.data_ptr(), cols if t.is_contiguous() else _stride(t, name)


def _vector(t, name, device, n, dtype=torch.float32):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device:
        _on(t, name, device, dtype)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be contiguous with %d elements" % (name, n))
    return t.data_ptr()


def _workspace(ws, need, device):
    """(tensor, address, bytes); need(): bytes to allocate where none is given (the library checks a given one's size)."""
    if ws is None:
        n = need()
        if n == 0:
            return None, None, 0
        ws = torch.empty(n, dtype=torch.uint8, device="cuda:%d" % device)
    elif ws.dtype is not torch.uint8 or ws.get_device() != device:
        _on(ws, "workspace", device, torch.uint8)
    if not ws.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return ws, ws.data_ptr(), ws.numel()


def _input(t, name):
    """The number of its device."""
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dim() == 0:
        raise ValueError("%s must have a dimension" % name)
    return t.get_device()


# The current device and a device's current stream as plain numbers: what
# torch.cuda.current_device() and current_stream().cuda_stream return, without the objects
# they make on the way (2 us of a call's host time).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)


def _call(fn, device, *args):
    """The library's call on the device's current stream."""
    if device == _current_device():
        status = fn(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _raw_stream(device))
    if status:
        _check(status)


# ---------------------------------------------------- root-mean-square norm
def terra_rmsnorm_fwd(x, gain=None, res=None, eps=1e-5, out=None, z=None, rstd=None, q=None, q_scale=None):
    """z = x + res, y = gain z / sqrt(mean(z^2) + eps) over the last dimension.

    x (..., C) in float32, bfloat16 or float16; res like x; gain float32 (C).
    Returns (y, z): y is `out`, allocated unless q is given (with q alone no y
    is written: None); z is written if it or res is given, allocated if res
    is.  rstd: float32, one a row, receives 1 / sqrt(...) for the backward.
    q (float8_e4m3fn, like x) and q_scale (float32, one a row) receive y in
    8 bits: q * q_scale stands for y."""
    dev, dt, C = _input(x, "x"), x.dtype, x.shape[-1]
    rows = x.numel() // C if C else 0
    if (q is None) != (q_scale is None):
        raise ValueError("q and q_scale come together")
    if z is None and res is not None:
        z = torch.empty(x.shape, dtype=dt, device=x.device)
    if out is None and q is None:
        out = torch.empty(x.shape, dtype=dt, device=x.device)
    (xp, xl), (rp, rl) = _matrix(x, "x", dev, dt, rows, C), _matrix(res, "res", dev, dt, rows, C)
    (zp, zl), (yp, yl) = _matrix(z, "z", dev, dt, rows, C), _matrix(out, "out", dev, dt, rows, C)
    qp, ql = _matrix(q, "q", dev, torch.float8_e4m3fn, rows, C)
    _call(lib().terra_rmsnorm_fwd, dev, terra_rmsnorm_desc(rows, _i32(C), eps, xl, rl, zl, yl, ql), _code(dt), xp, rp,
          _vector(gain, "gain", dev, C), zp, yp, qp, _vector(q_scale, "q_scale", dev, rows), _vector(rstd, "rstd", dev, rows))
    return out, z


def terra_rmsnorm_bwd_workspace_bytes(rows, cols):
    """Workspace of terra_rmsnorm_bwd for up to `rows` rows."""
    return int(lib().terra_rmsnorm_bwd_workspace_bytes(rows, _i32(cols)))


def terra_rmsnorm_bwd(dy, z, rstd, gain=None, dz=None, out=None, workspace=None):
    """Gradients (dx, dgain) from dy, the forward's z and rstd, and dz, what
    reaches z by the residual stream; dx is the gradient of x and of res.
    `out` may hold preallocated (dx, dgain), None for one that is not wanted;
    without it dgain is computed if gain is given."""
    dev, dt, C = _input(dy, "dy"), dy.dtype, dy.shape[-1]
    rows = dy.numel() // C if C else 0
    if out is None:
        out = (torch.empty(dy.shape, dtype=dt, device=dy.device),
               None if gain is None else torch.empty(C, dtype=torch.float32, device=dy.device))
    dx, dgain = out
    ws, wp, wn = _workspace(workspace, lambda: 0 if dgain is None else lib().terra_rmsnorm_bwd_workspace_bytes(rows, _i32(C)), dev)
    (yp, yl), (zp, zl) = _matrix(dy, "dy", dev, dt, rows, C), _matrix(z, "z", dev, dt, rows, C)
    (rp, rl), (xp, xl) = _matrix(dz, "dz", dev, dt, rows, C), _matrix(dx, "dx", dev, dt, rows, C)
    _call(lib().terra_rmsnorm_bwd, dev, terra_rmsnorm_desc(rows, _i32(C), 0.0, xl, rl, zl, yl, 0), _code(dt), yp, zp,
          _vector(rstd, "rstd", dev, rows), _vector(gain, "gain", dev, C), rp, xp, _vector(dgain, "dgain", dev, C), wp, wn)
    return dx, dgain


# ------------------------------------------------------------- linear layer
def terra_linear_fwd_workspace_bytes(M, N, K, dtype):
    """Workspace of terra_linear_fwd for these sizes; fewer tokens may need more."""
    return int(lib().terra_linear_fwd_workspace_bytes(M, _i32(N), _i32(K), _code(dtype)))


def terra_linear_bwd_workspace_bytes(M, N, K, dtype):
    """Workspace of terra_linear_bwd for these sizes; fewer tokens may need more."""
    return int(lib().terra_linear_bwd_workspace_bytes(M, _i32(N), _i32(K), _code(dtype)))


def terra_linear_fwd(x, w, bias=None, act="none", res=None, x_scale=None, w_scale=None, out=None, pre=None,
                     workspace=None, out_dtype=None):
    """y = act(x w^T + bias) + res for x (..., K) and w (N, K), act one of
    none, relu, gelu, silu.  bfloat16 or float16 tensors, or float8_e4m3fn x
    and w with x_scale (float32, one a row of x) and w_scale (N), y then of
    out_dtype (default bfloat16).  pre (like y) receives what act is applied to, for the backward."""
    dev, dt = _input(x, "x"), x.dtype
    if w.dim() != 2:
        raise ValueError("w must have two dimensions")
    (N, K), code = w.shape, _code(dt)
    M = x.numel() // K if K else 0
    to = dt if code != TERRA_E4M3 else out_dtype or torch.bfloat16
    if out_dtype not in (None, to):
        raise ValueError("out_dtype is %s for %s tensors" % (to, dt))
    if out is None:
        out = torch.empty((*x.shape[:-1], N), dtype=to, device=x.device)
    (xp, xl), (wp, wl) = _matrix(x, "x", dev, dt, M, K), _matrix(w, "w", dev, dt, N, K)
    (yp, yl), (rp, rl) = _matrix(out, "out", dev, to, M, N), _matrix(res, "res", dev, to, M, N)
    pp, pl = _matrix(pre, "pre", dev, to, M, N)
    ws, sp, sn = _workspace(workspace, lambda: lib().terra_linear_fwd_workspace_bytes(M, _i32(N), _i32(K), code), dev)
    _call(lib().terra_linear_fwd, dev, terra_linear_desc(M, _i32(N), _i32(K), xl, wl, yl, rl, pl, 0, 0, _choice(act, _ACTS, "act"), _code(to)),
          code, xp, _vector(x_scale, "x_scale", dev, M), wp, _vector(w_scale, "w_scale", dev, N),
          _vector(bias, "bias", dev, N), rp, yp, pp, sp, sn)
    return out


def terra_linear_bwd(dy, x, w, pre=None, act="none", out=None, workspace=None):
    """Gradients (dx, dw, dbias) of the linear layer from dy (..., N); that of
    res is dy.  pre: as the forward left it, unless act is none.  `out` may
    hold preallocated (dx, dw, dbias), None for one that is not wanted; dw is
    float32 (which is allocated) or like w, dbias float32."""
    dev, dt = _input(dy, "dy"), dy.dtype
    if w.dim() != 2:
        raise ValueError("w must have two dimensions")
    (N, K), code = w.shape, _code(dt)
    M = dy.numel() // N if N else 0
    if out is None:
        out = (torch.empty((*dy.shape[:-1], K), dtype=dt, device=dy.device), torch.empty((N, K), dtype=torch.float32, device=dy.device),
               torch.empty(N, dtype=torch.float32, device=dy.device))
    dx, dw, db = out
    (yp, yl), (xp, xl) = _matrix(dy, "dy", dev, dt, M, N), _matrix(x, "x", dev, dt, M, K)
    (wp, wl), (pp, pl) = _matrix(w, "w", dev, dt, N, K), _matrix(pre, "pre", dev, dt, M, N)
    (ip, il), (gp, gl) = _matrix(dx, "dx", dev, dt, M, K), _matrix(dw, "dw", dev, dt if dw is None or dw.dtype == dt else torch.float32, N, K)
    ws, sp, sn = _workspace(workspace, lambda: lib().terra_linear_bwd_workspace_bytes(M, _i32(N), _i32(K), code), dev)
    _call(lib().terra_linear_bwd, dev, terra_linear_desc(M, _i32(N), _i32(K), xl, wl, yl, 0, pl, il, gl, _choice(act, _ACTS, "act"), code), code,
          yp, xp, wp, pp, ip, gp, TERRA_F32 if dw is None else _code(dw.dtype), _vector(db, "dbias", dev, N), sp, sn)
    return out


# --------------------------------------------------------- rotary positions
def terra_plan_rope(head_dim, rot_dim=None, axes=1, layout="half", base=10000.0, scaling="none", factor=1.0, orig_len=0,
                    beta_fast=32.0, beta_slow=1.0, attn_scale=0.0):
    """The plan of rotary positions that terra_rope_fwd and _bwd take: the
    first rot_dim (default: all) channels of a head turn, in `axes` (1 or 2)
    equal parts, pairs interleaved or in halves; frequencies base^(-2i/part),
    scaled for long contexts (none, linear, ntk, yarn) by `factor`."""
    d = terra_rope_desc(_i32(head_dim), _i32(head_dim if rot_dim is None else rot_dim), _i32(axes), _choice(layout, _LAYOUTS, "layout"),
                        _choice(scaling, _SCALINGS, "scaling"), base, factor, orig_len, beta_fast, beta_slow, attn_scale)
    plan = terra_rope_plan()
    _check(lib().terra_plan_rope(d, plan))
    return plan


def _heads(x, out, name, tokens, hd, device, dtype):
    shape = x.shape
    for t in (x, out):
        if t.dtype is not dtype or t.get_device() != device:
            _on(t, name if t is x else name + "'s output", device, dtype)
        if t.shape != shape or len(shape) < 2 or shape[-1] != hd or t.numel() != tokens * shape[-2] * hd:
            raise ValueError("%s has shape %s, expected (%d tokens, heads, %d)" % (name if t is x else name + "'s output", tuple(t.shape), tokens, hd))
    heads = shape[-2]
    steps = []
    for t in (x, out):
        if t.is_contiguous():
            steps += (heads * hd, hd)
        else:
            if t.stride(-1) != 1:
                raise ValueError("%s must be contiguous along its last dimension" % (name if t is x else name + "'s output"))
            steps += (_step(t.shape[:-2], t.stride()[:-2], name) or 0, t.stride(-2))
    return terra_rope_tensor(x.data_ptr(), out.data_ptr(), _i32(heads), *steps)


def _rope(fn, plan, q, k, pos, grid, out):
    dev, dt, hd = _input(q, "q"), q.dtype, plan.desc.head_dim
    if q.dim() < 2 or q.shape[-1] != hd or q.shape[-2] == 0:
        raise ValueError("q has shape %s, expected (tokens, heads, %d)" % (tuple(q.shape), hd))
    tokens = q.numel() // (q.shape[-2] * hd)
    if out is None:
        out = (torch.empty(q.shape, dtype=dt, device=q.device), None if k is None else torch.empty(k.shape, dtype=dt, device=q.device))
    tq = _heads(q, out[0], "q", tokens, hd, dev, dt)
    tk = None if k is None else _heads(k, out[1], "k", tokens, hd, dev, dt)
    if pos is not None:
        _on(pos, "pos", dev, torch.int32)
        if pos.numel() != tokens * plan.desc.axes or not pos.is_contiguous():
            raise ValueError("pos must be contiguous with %d x %d elements" % (tokens, plan.desc.axes))
    elif grid is None:
        raise ValueError("pos or grid must be given")
    h, w = (0, 0) if grid is None else (_i32(grid[0]), _i32(grid[1]))
    _call(fn, dev, plan, _code(dt), tokens, None if pos is None else pos.data_ptr(), h, w, tq, tk)
    return out


def terra_rope_fwd(plan, q, k=None, pos=None, grid=None, out=None):
    """q (..., heads, head_dim) and k, which may have other heads, turned by
    their tokens' positions: pos, int32 (tokens, axes), or the place on a
    `grid` (H, W) whose tokens follow each other (NHWC; sequences of one axis:
    (1, length)).  Returns (q, k), new or `out`, which may be (q, k)."""
    return _rope(lib().terra_rope_fwd, plan, q, k, pos, grid, out)


def terra_rope_bwd(plan, dq, dk=None, pos=None, grid=None, out=None):
    """Gradients of the turned q and k to those of q and k, as terra_rope_fwd."""
    return _rope(lib().terra_rope_bwd, plan, dq, dk, pos, grid, out)
