"""Operators between and behind the linear layers (``include/rrm.h``): argument marshalling only.

Tensors are CUDA tensors whose last axis is adjacent; the axes before it may be strided as far as they collapse to the
two (``gated_ff``: one) that the C calls take, and nothing is copied to make them so.  Results that the caller does not hand
in, and the workspace, are allocated by torch.  With ``stream`` a call runs as if that stream were the current one, its allocations
included; the caller orders it behind what its inputs wait for, and what uses its results behind it.

The calls are not differentiable by autograd: their gradients are the ``*_backward`` functions.  A tensor that requires a gradient is refused where autograd
records (under ``torch.no_grad()``, and inside an ``autograd.Function``, it is not), as the results would silently carry none.

What the checks of a call look at (shapes, strides, types) decides its descriptor and workspace too, so both are kept by it: a call with the
shapes of an earlier one takes them from a table and goes on to the pointers.  (One frame of a live video, host time of a call:
12 us with every check and structure made anew, 8 to 9 so.)
"""
from __future__ import annotations

import ctypes

import torch

from .binding import BF16, CONV, _check, _stream_ptr, lib

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
MARK_FRAMES = 64  # RRM_SCAN_MARK_FRAMES


class NormDesc(ctypes.Structure):
    """``rrm_norm_desc``"""
    _fields_ = ([(k, ctypes.c_int) for k in ("n", "positions", "c", "groups", "x_elem", "y_elem", "act")] + [("eps", ctypes.c_float)]
                + [(k, ctypes.c_int64) for k in ("x_sample", "x_position", "y_sample", "y_position", "dx_sample", "dx_position")])


class ScanDesc(ctypes.Structure):
    """``rrm_scan_desc``"""
    _fields_ = ([(k, ctypes.c_int) for k in ("n", "t", "c", "elem")]
                + [(k, ctypes.c_int64) for k in ("x_video", "x_frame", "f_video", "f_frame", "y_video", "y_frame",
                                                 "dx_video", "dx_frame", "df_video", "df_frame")])


class FFDesc(ctypes.Structure):
    """``rrm_ff_desc``"""
    _fields_ = ([(k, ctypes.c_int) for k in ("m", "k", "f", "act")]
                + [(k, ctypes.c_int64) for k in ("x_row", "wg_row", "wu_row", "h_row", "gu_row", "dx_row", "dwg_row", "dwu_row")]
                + [("unaligned", ctypes.c_int)])


# (descriptor, reference to it, bytes of workspace, device) by what the checks looked at.  Emptied when it has grown past what a program's
# shapes come to.
_plans: dict = {}


def _keep(key, desc, size_of: str, backward: int, *tensors):
    devices = {t.device.index for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError(f"tensors on several devices: {sorted(devices)}")
    if len(_plans) > 4096:
        _plans.clear()
    ref = ctypes.byref(desc)
    _plans[key] = plan = (desc, ref, getattr(lib(), size_of)(ref, backward), devices.pop())
    return plan


def _look(t):
    """What the checks look at (of a tensor made for the call nothing: its like always passes)."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.device, t.requires_grad and torch.is_grad_enabled())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _elem(t) -> int:
    if t.dtype is torch.float32:
        return 0
    if t.dtype is torch.bfloat16:
        return 1
    raise ValueError(f"expected float32 or bfloat16, got {t.dtype}")


def _expect(t, what: str, shape, dtype=None) -> None:
    if t is None:
        return
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a CUDA tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what}: requires a gradient, which the result would not carry: call under torch.no_grad() and take the "
                         "gradient from the *_backward function")


def _dense(t, what: str, shape, dtype) -> None:
    _expect(t, what, shape, dtype)
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")


def _adjacent(t, what: str) -> None:
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the last axis must be adjacent")


def _outer_inner(t, what: str):
    """Strides of the first axis and of the axes between it and the last, which have to collapse to one."""
    _adjacent(t, what)
    shape, strides = t.shape, t.stride()
    if t.dim() == 2:
        return strides[0], shape[1]
    inner = strides[-2]
    rows = shape[-2]
    for size, stride in zip(shape[-3:0:-1], strides[-3:0:-1]):
        if size != 1 and rows != 1 and stride != inner * rows:
            raise ValueError(f"{what}: the axes between the first and the last must collapse to one")
        if rows == 1:
            inner = stride
        rows *= size
    return strides[0], inner


def _frames(t, what: str):
    _adjacent(t, what)
    return t.stride(0), t.stride(1)


def _row(t, what: str) -> int:
    if t.dim() != 2:
        raise ValueError(f"{what}: expected two axes")
    _adjacent(t, what)
    return t.stride(0)


def _act(name) -> int:
    try:
        return ACTS[name]
    except (KeyError, TypeError):
        raise ValueError(f"act: expected one of {sorted(ACTS)}, got {name!r}") from None


def _workspace(nbytes: int, device):
    """A tensor (torch's blocks begin at whole 512 bytes), or None for none."""
    if not nbytes:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _elsewhere(stream, call, *args):
    """``call(*args)`` with ``stream`` (an object or a handle) current.  So its results and workspace come from memory of that stream's: a block of another stream's
    may still be in use by what that one was given earlier, which ``stream`` does not wait for.  The results are recorded on the stream
    that was current before, where the caller goes on: they must not be handed out again before that one is through with them."""
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    before = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        got = call(*args)
    for t in got if isinstance(got, tuple) else (got,):
        if all(t is not a for a in args):
            t.record_stream(before)
    return got


# -- group norm with an activation -------------------------------------------------------------------------------------

def group_norm_act(x, groups: int, gamma=None, beta=None, act: str = "none", eps: float = 1e-5, out=None, out_dtype=None, stats=None,
                   stream=None):
    """``rrm_group_norm_act``: ``x`` [n, .., c] float32 or bfloat16, channels last (2 axes: one position a sample); ``gamma``
    and ``beta`` float32 [c].  ``out`` or a new tensor of ``out_dtype`` (default: x's type) receives the result;
    ``stats``, float32 [n, groups, 2], what the backward pass needs."""
    if stream is not None:
        return _elsewhere(stream, group_norm_act, x, groups, gamma, beta, act, eps, out, out_dtype, stats)
    made = out is None
    if made:
        out = torch.empty_like(x, dtype=out_dtype)
    key = ("norm", groups, act, eps, out_dtype, _look(x), made or _look(out), _look(gamma), _look(beta), _look(stats))
    plan = _plans.get(key)
    if plan is None:
        if x.dim() < 2:
            raise ValueError("x: expected [n, .., c]")
        n, c = x.shape[0], x.shape[-1]
        _expect(x, "x", x.shape)
        _expect(out, "out", x.shape, out_dtype)
        _dense(gamma, "gamma", (c,), torch.float32)
        _dense(beta, "beta", (c,), torch.float32)
        _dense(stats, "stats", (n, groups, 2), torch.float32)
        positions = x.numel() // (n * c) if n and c else 0
        plan = _keep(key, NormDesc(n, positions, c, int(groups), _elem(x), _elem(out), _act(act), float(eps), *_outer_inner(x, "x"),
                                   *_outer_inner(out, "out"), 0, 0), "rrm_group_norm_workspace", 0, x, out, gamma, beta, stats)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_group_norm_act(plan[1], x.data_ptr(), _ptr(gamma), _ptr(beta), out.data_ptr(), _ptr(stats), _ptr(ws), plan[2],
                                    _stream_ptr(None, plan[3])))
    return out


def group_norm_act_of(layer, groups: int, gamma=None, beta=None, act: str = "none", eps: float = 1e-5, out=None, stats=None, stream=None):
    """group_norm_act of a bfloat16 convolution's stored projection (``rrm_snapshot``), read where it lies: after ``layer.step`` on the same
    stream, the next layer's input, bfloat16 [n, h_out, w_out, c_out]."""
    if stream is not None:
        return _elsewhere(stream, group_norm_act_of, layer, groups, gamma, beta, act, eps, out, stats)
    if layer.dtype != BF16 or layer.shape.kind != CONV:
        raise ValueError("layer: expected a bfloat16 convolution")
    n, h, w, c = layer.y_shape
    made = out is None
    if made:
        out = torch.empty((n, h, w, c), dtype=torch.bfloat16, device="cuda")
    key = ("norm of", groups, act, eps, n, h, w, c, made or _look(out), _look(gamma), _look(beta), _look(stats))
    plan = _plans.get(key)
    if plan is None:
        _expect(out, "out", (n, h, w, c), torch.bfloat16)
        _dense(gamma, "gamma", (c,), torch.float32)
        _dense(beta, "beta", (c,), torch.float32)
        _dense(stats, "stats", (n, groups, 2), torch.float32)
        plan = _keep(key, NormDesc(n, h * w, c, int(groups), 0, 1, _act(act), float(eps), h * w * c, c, *_outer_inner(out, "out"), 0, 0),
                     "rrm_group_norm_workspace", 0, out, gamma, beta, stats)
    ws = _workspace(plan[2], out.device)
    _check(lib().rrm_group_norm_act(plan[1], layer.snapshot_ptrs()[1], _ptr(gamma), _ptr(beta), out.data_ptr(), _ptr(stats), _ptr(ws), plan[2],
                                    _stream_ptr(None, plan[3])))
    return out


def group_norm_act_backward(dy, x, stats, gamma=None, beta=None, act: str = "none", dx=None, dgamma=None, dbeta=None, stream=None):
    """``rrm_group_norm_act_backward``: (dx, dgamma, dbeta) from ``dy`` (of the result's type and x's shape) and the ``stats`` that
    the forward pass left for the same ``x``, ``gamma``, ``beta`` and ``act``."""
    if stream is not None:
        return _elsewhere(stream, group_norm_act_backward, dy, x, stats, gamma, beta, act, dx, dgamma, dbeta)
    c = x.shape[-1]
    made = [t is None for t in (dx, dgamma, dbeta)]
    if dx is None:
        dx = torch.empty_like(x)
    if dgamma is None:
        dgamma = x.new_empty((c,), dtype=torch.float32) if gamma is None else torch.empty_like(gamma)
    if dbeta is None:
        dbeta = torch.empty_like(dgamma)
    key = ("norm back", act, _look(dy), _look(x), _look(stats), _look(gamma), _look(beta),
           made[0] or _look(dx), made[1] or _look(dgamma), made[2] or _look(dbeta))
    plan = _plans.get(key)
    if plan is None:
        if x.dim() < 2:
            raise ValueError("x: expected [n, .., c]")
        if stats.dim() != 3:
            raise ValueError("stats: expected [n, groups, 2]")
        n, groups = x.shape[0], stats.shape[1]
        _expect(x, "x", x.shape)
        _expect(dy, "dy", x.shape)
        _expect(dx, "dx", x.shape, x.dtype)
        _dense(stats, "stats", (n, groups, 2), torch.float32)
        for t, what in ((gamma, "gamma"), (beta, "beta"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            _dense(t, what, (c,), torch.float32)
        positions = x.numel() // (n * c) if n and c else 0
        plan = _keep(key, NormDesc(n, positions, c, groups, _elem(x), _elem(dy), _act(act), 1.0, *_outer_inner(x, "x"),
                                   *_outer_inner(dy, "dy"), *_outer_inner(dx, "dx")), "rrm_group_norm_workspace", 1, x, dy, stats, gamma, beta, dx, dgamma,
                     dbeta)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_group_norm_act_backward(plan[1], x.data_ptr(), stats.data_ptr(), _ptr(gamma), _ptr(beta), dy.data_ptr(), dx.data_ptr(),
                                             dgamma.data_ptr(), dbeta.data_ptr(), _ptr(ws), plan[2], _stream_ptr(None, plan[3])))
    return dx, dgamma, dbeta


# -- gated linear recurrence -------------------------------------------------------------------------------------------

def gated_scan_marks(x, stream=None):
    """A tensor for the states that a forward pass of training keeps: float32 [n, ceil(t / 64), c] for x [n, t, c].  ``stream``: the one that
    the passes run on, where it is not the current one."""
    if stream is not None:
        return _elsewhere(stream, gated_scan_marks, x)
    n, t, c = x.shape
    return x.new_empty((n, -(-t // MARK_FRAMES), c), dtype=torch.float32)


def gated_scan(x, f, h0=None, lengths=None, out=None, h_last=None, marks=None, stream=None):
    """``rrm_gated_scan``: (y, h_last) of the recurrence over ``x`` and the gates' logits ``f``, [n, t, c] float32 or bfloat16, from
    the state ``h0`` (float32 [n, c]; None: zeros).  ``lengths`` int32 [n]: frames of each video.  ``marks``: see gated_scan_marks;
    the backward pass needs them.  For one frame (t = 1) ``h_last`` may be ``h0``."""
    if stream is not None:
        return _elsewhere(stream, gated_scan, x, f, h0, lengths, out, h_last, marks)
    if x.dim() != 3:
        raise ValueError("x: expected [n, t, c]")
    n, t, c = shape = x.shape
    made = (out is None, h_last is None)
    if out is None:
        out = torch.empty_like(x)
    if h_last is None:
        h_last = x.new_empty((n, c), dtype=torch.float32)
    key = ("scan", _look(x), _look(f), _look(h0), _look(lengths), made[0] or _look(out), made[1] or _look(h_last), _look(marks))
    plan = _plans.get(key)
    if plan is None:
        _expect(x, "x", shape)
        _expect(f, "f", shape, x.dtype)
        _expect(out, "out", shape, x.dtype)
        _dense(h0, "h0", (n, c), torch.float32)
        _dense(h_last, "h_last", (n, c), torch.float32)
        _dense(lengths, "lengths", (n,), torch.int32)
        _dense(marks, "marks", (n, -(-t // MARK_FRAMES), c), torch.float32)
        plan = _keep(key, ScanDesc(n, t, c, _elem(x), *_frames(x, "x"), *_frames(f, "f"), *_frames(out, "out"), 0, 0, 0, 0),
                     "rrm_gated_scan_workspace", 0, x, f, h0, lengths, out, h_last, marks)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_gated_scan(plan[1], x.data_ptr(), f.data_ptr(), _ptr(h0), _ptr(lengths), out.data_ptr(), h_last.data_ptr(), _ptr(marks),
                                _ptr(ws), plan[2], _stream_ptr(None, plan[3])))
    return out, h_last


def gated_scan_backward(dy, x, f, marks, lengths=None, dh_last=None, dx=None, df=None, dh0=None, stream=None):
    """``rrm_gated_scan_backward``: (dx, df, dh0) from ``dy``, the forward pass's inputs and ``marks``, and the gradient
    ``dh_last`` (float32 [n, c]; None: zeros) of the last state."""
    if stream is not None:
        return _elsewhere(stream, gated_scan_backward, dy, x, f, marks, lengths, dh_last, dx, df, dh0)
    if x.dim() != 3:
        raise ValueError("x: expected [n, t, c]")
    n, t, c = shape = x.shape
    made = [g is None for g in (dx, df, dh0)]
    if dx is None:
        dx = torch.empty_like(x)
    if df is None:
        df = torch.empty_like(f)
    if dh0 is None:
        dh0 = x.new_empty((n, c), dtype=torch.float32)
    key = ("scan back", _look(dy), _look(x), _look(f), _look(marks), _look(lengths), _look(dh_last),
           made[0] or _look(dx), made[1] or _look(df), made[2] or _look(dh0))
    plan = _plans.get(key)
    if plan is None:
        for v, what in ((x, "x"), (f, "f"), (dy, "dy"), (dx, "dx"), (df, "df")):
            _expect(v, what, shape, x.dtype)
        _dense(marks, "marks", (n, -(-t // MARK_FRAMES), c), torch.float32)
        _dense(lengths, "lengths", (n,), torch.int32)
        _dense(dh_last, "dh_last", (n, c), torch.float32)
        _dense(dh0, "dh0", (n, c), torch.float32)
        plan = _keep(key, ScanDesc(n, t, c, _elem(x), *_frames(x, "x"), *_frames(f, "f"), *_frames(dy, "dy"), *_frames(dx, "dx"),
                                   *_frames(df, "df")), "rrm_gated_scan_workspace", 1, x, f, dy, marks, lengths, dh_last, dx, df, dh0)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_gated_scan_backward(plan[1], x.data_ptr(), f.data_ptr(), marks.data_ptr(), _ptr(lengths), dy.data_ptr(), _ptr(dh_last),
                                         dx.data_ptr(), df.data_ptr(), dh0.data_ptr(), _ptr(ws), plan[2], _stream_ptr(None, plan[3])))
    return dx, df, dh0


# -- gated feed-forward block ------------------------------------------------------------------------------------------

def gated_ff(x, wg, wu, act: str = "silu", out=None, save=None, stream=None):
    """``rrm_gated_ff``: act(x wg^T) * (x wu^T), bfloat16: ``x`` [m, k], ``wg`` and ``wu`` [f, k], the result [m, f].
    ``save``: two tensors [m, f] that receive the two projections for the backward pass."""
    if stream is not None:
        return _elsewhere(stream, gated_ff, x, wg, wu, act, out, save)
    made = out is None
    if made:
        out = x.new_empty((x.shape[0], wg.shape[0]))
    g, u = (None, None) if save is None else save
    px, pg, pu = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    loose = (px | pg | pu) & 15 != 0
    key = ("ff", act, loose, _look(x), _look(wg), _look(wu), made or _look(out), _look(g), _look(u))
    plan = _plans.get(key)
    if plan is None:
        bf = torch.bfloat16
        rows = [_row(t, what) for t, what in ((x, "x"), (wg, "wg"), (wu, "wu"), (out, "out"))]
        (m, k), f = x.shape, wg.shape[0]
        _expect(x, "x", (m, k), bf)
        _expect(wg, "wg", (f, k), bf)
        _expect(wu, "wu", (f, k), bf)
        _expect(out, "out", (m, f), bf)
        saved = 0
        if save is not None:
            _expect(g, "save[0]", (m, f), bf)
            _expect(u, "save[1]", (m, f), bf)
            saved = _row(g, "save[0]")
            if _row(u, "save[1]") != saved:
                raise ValueError("save: both tensors need the same strides")
        plan = _keep(key, FFDesc(m, k, f, _act(act), *rows, saved, 0, 0, 0, int(loose)), "rrm_gated_ff_workspace", 0, x, wg, wu, out, g, u)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_gated_ff(plan[1], px, pg, pu, out.data_ptr(), _ptr(g), _ptr(u), _ptr(ws), plan[2], _stream_ptr(None, plan[3])))
    return out


def gated_ff_backward(dh, x, wg, wu, g, u, act: str = "silu", dx=None, dwg=None, dwu=None, stream=None):
    """``rrm_gated_ff_backward``: (dx, dwg, dwu) from ``dh`` and the projections ``g`` and ``u`` that the forward pass saved."""
    if stream is not None:
        return _elsewhere(stream, gated_ff_backward, dh, x, wg, wu, g, u, act, dx, dwg, dwu)
    made = [t is None for t in (dx, dwg, dwu)]
    if dx is None:
        dx = torch.empty_like(x)
    if dwg is None:
        dwg = torch.empty_like(wg)
    if dwu is None:
        dwu = torch.empty_like(wu)
    px, pg, pu = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    loose = (px | pg | pu) & 15 != 0
    key = ("ff back", act, loose, _look(dh), _look(x), _look(wg), _look(wu), _look(g), _look(u),
           made[0] or _look(dx), made[1] or _look(dwg), made[2] or _look(dwu))
    plan = _plans.get(key)
    if plan is None:
        bf = torch.bfloat16
        rows = [_row(t, what) for t, what in ((x, "x"), (wg, "wg"), (wu, "wu"), (dh, "dh"), (g, "g"), (dx, "dx"), (dwg, "dwg"), (dwu, "dwu"))]
        if _row(u, "u") != rows[4]:
            raise ValueError("g, u: both tensors need the same strides")
        (m, k), f = x.shape, wg.shape[0]
        for t, what, shape in ((x, "x", (m, k)), (wg, "wg", (f, k)), (wu, "wu", (f, k)), (g, "g", (m, f)), (u, "u", (m, f)), (dh, "dh", (m, f)),
                               (dx, "dx", (m, k)), (dwg, "dwg", (f, k)), (dwu, "dwu", (f, k))):
            _expect(t, what, shape, bf)
        plan = _keep(key, FFDesc(m, k, f, _act(act), *rows, int(loose)), "rrm_gated_ff_workspace", 1, x, wg, wu, dh, g, u, dx, dwg, dwu)
    ws = _workspace(plan[2], x.device)
    _check(lib().rrm_gated_ff_backward(plan[1], px, pg, pu, g.data_ptr(), u.data_ptr(), dh.data_ptr(), dx.data_ptr(), dwg.data_ptr(), dwu.data_ptr(),
                                       _ptr(ws), plan[2], _stream_ptr(None, plan[3])))
    return dx, dwg, dwu
