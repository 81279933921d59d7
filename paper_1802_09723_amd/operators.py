"""Operators between and behind the linear layers (``include/rrm.h``): argument marshalling only.

Tensors are CUDA tensors whose last axis is adjacent; the axes before it may be strided as far as they collapse to the
two (``gated_ff``: one) that the C calls take, and nothing is copied to make them so.  Results that the caller does not hand
in, and the workspace, are allocated by torch on the current stream; with ``stream`` they are recorded on it as well.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from .binding import _check, _stream_ptr, lib

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


# Descriptors by their values, each with the bytes of workspace its call takes: a live frame's call fills in no structure.
# Emptied when it has grown past what a program's shapes come to.
_descs: dict = {}


def _desc(cls, size_of: str, backward: int, *values):
    key = (size_of, backward, values)
    got = _descs.get(key)
    if got is None:
        if len(_descs) > 4096:
            _descs.clear()
        d = cls(*values)
        got = _descs[key] = (d, ctypes.byref(d), getattr(lib(), size_of)(ctypes.byref(d), backward))
    return got


def _elem(t) -> int:
    import torch
    if t.dtype is torch.float32:
        return 0
    if t.dtype is torch.bfloat16:
        return 1
    raise ValueError(f"expected float32 or bfloat16, got {t.dtype}")


def _expect(t, what: str, shape, dtype=None):
    """The device pointer of a tensor of this shape (None: not given)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a CUDA tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _dense(t, what: str, shape, dtype):
    p = _expect(t, what, shape, dtype)
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    return p


def _outer_inner(t, what: str):
    """Strides of the first axis and of the axes between it and the last, which have to collapse to one."""
    shape, strides = t.shape, t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the last axis must be adjacent")
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


def _row(t, what: str) -> int:
    if t.dim() != 2:
        raise ValueError(f"{what}: expected two axes")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"{what}: the last axis must be adjacent")
    return t.stride(0)


def _act(name) -> int:
    try:
        return ACTS[name]
    except (KeyError, TypeError):
        raise ValueError(f"act: expected one of {sorted(ACTS)}, got {name!r}") from None


def _workspace(nbytes: int, device):
    """(tensor, pointer); torch's blocks begin at whole 512 bytes"""
    if not nbytes:
        return None, None
    import torch
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _used_on(stream, *tensors) -> None:
    """A tensor made here on the current stream and used on another must not be handed out again before that one is through."""
    if stream is None:
        return
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


# -- group norm with an activation -------------------------------------------------------------------------------------

def group_norm_act(x, groups: int, gamma=None, beta=None, act: str = "none", eps: float = 1e-5, out=None, out_dtype=None, stats=None,
                   stream=None):
    """``rrm_group_norm_act``: ``x`` [n, .., c] float32 or bfloat16, channels last (2 axes: one position a sample); ``gamma``
    and ``beta`` float32 [c].  ``out`` or a new tensor of ``out_dtype`` (default: x's type) receives the result;
    ``stats``, float32 [n, groups, 2], what the backward pass needs."""
    import torch
    if x.dim() < 2:
        raise ValueError("x: expected [n, .., c]")
    made = out is None
    if made:
        out = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=x.device)
    n, c = x.shape[0], x.shape[-1]
    px, po = _expect(x, "x", x.shape), _expect(out, "out", x.shape, out_dtype)
    xs, ys = _outer_inner(x, "x"), _outer_inner(out, "out")
    positions = x.numel() // (n * c) if n and c else 0
    d, ref, need = _desc(NormDesc, "rrm_group_norm_workspace", 0, n, positions, c, int(groups), _elem(x), _elem(out), _act(act), float(eps),
                         xs[0], xs[1], ys[0], ys[1], 0, 0)
    pg, pb = _dense(gamma, "gamma", (c,), torch.float32), _dense(beta, "beta", (c,), torch.float32)
    ps = _dense(stats, "stats", (n, groups, 2), torch.float32)
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_group_norm_act(ref, px, pg, pb, po, ps, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, out if made else None)
    return out


def group_norm_act_backward(dy, x, stats, gamma=None, beta=None, act: str = "none", dx=None, dgamma=None, dbeta=None, stream=None):
    """``rrm_group_norm_act_backward``: (dx, dgamma, dbeta) from ``dy`` (of the result's type and x's shape) and the ``stats`` that
    the forward pass left for the same ``x``, ``gamma``, ``beta`` and ``act``."""
    import torch
    if x.dim() < 2:
        raise ValueError("x: expected [n, .., c]")
    n, c = x.shape[0], x.shape[-1]
    if stats.dim() != 3:
        raise ValueError("stats: expected [n, groups, 2]")
    groups = stats.shape[1]
    made = [t is None for t in (dx, dgamma, dbeta)]
    if dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dgamma is None:
        dgamma = torch.empty(c, dtype=torch.float32, device=x.device)
    if dbeta is None:
        dbeta = torch.empty(c, dtype=torch.float32, device=x.device)
    px, pdy, pdx = _expect(x, "x", x.shape), _expect(dy, "dy", x.shape), _expect(dx, "dx", x.shape, x.dtype)
    xs, ys, gs = _outer_inner(x, "x"), _outer_inner(dy, "dy"), _outer_inner(dx, "dx")
    positions = x.numel() // (n * c) if n and c else 0
    d, ref, need = _desc(NormDesc, "rrm_group_norm_workspace", 1, n, positions, c, groups, _elem(x), _elem(dy), _act(act), 1.0,
                         xs[0], xs[1], ys[0], ys[1], gs[0], gs[1])
    ps = _dense(stats, "stats", (n, groups, 2), torch.float32)
    pg, pb = _dense(gamma, "gamma", (c,), torch.float32), _dense(beta, "beta", (c,), torch.float32)
    qg, qb = _dense(dgamma, "dgamma", (c,), torch.float32), _dense(dbeta, "dbeta", (c,), torch.float32)
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_group_norm_act_backward(ref, px, ps, pg, pb, pdy, pdx, qg, qb, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, *(t for t, was in zip((dx, dgamma, dbeta), made) if was))
    return dx, dgamma, dbeta


# -- gated linear recurrence -------------------------------------------------------------------------------------------

def gated_scan_marks(x):
    """A tensor for the states that a forward pass of training keeps: float32 [n, ceil(t / 64), c] for x [n, t, c]."""
    import torch
    n, t, c = x.shape
    return torch.empty((n, -(-t // MARK_FRAMES), c), dtype=torch.float32, device=x.device)


def _scan_shape(x):
    if x.dim() != 3:
        raise ValueError("x: expected [n, t, c]")
    return x.shape


def _frames(t, what: str):
    s = t.stride()
    if s[2] != 1 and t.shape[2] > 1:
        raise ValueError(f"{what}: the last axis must be adjacent")
    return s[0], s[1]


def gated_scan(x, f, h0=None, lengths=None, out=None, h_last=None, marks=None, stream=None):
    """``rrm_gated_scan``: (y, h_last) of the recurrence over ``x`` and the gates' logits ``f``, [n, t, c] float32 or bfloat16, from
    the state ``h0`` (float32 [n, c]; None: zeros).  ``lengths`` int32 [n]: frames of each video.  ``marks``: see gated_scan_marks;
    the backward pass needs them.  For one frame (t = 1) ``h_last`` may be ``h0``."""
    import torch
    n, t, c = _scan_shape(x)
    made = (out is None, h_last is None)
    if out is None:
        out = torch.empty((n, t, c), dtype=x.dtype, device=x.device)
    if h_last is None:
        h_last = torch.empty((n, c), dtype=torch.float32, device=x.device)
    shape = (n, t, c)
    px, pf, po = _expect(x, "x", shape), _expect(f, "f", shape, x.dtype), _expect(out, "out", shape, x.dtype)
    d, ref, need = _desc(ScanDesc, "rrm_gated_scan_workspace", 0, n, t, c, _elem(x), *_frames(x, "x"), *_frames(f, "f"),
                         *_frames(out, "out"), 0, 0, 0, 0)
    p0, pl = _dense(h0, "h0", (n, c), torch.float32), _dense(h_last, "h_last", (n, c), torch.float32)
    pn = _dense(lengths, "lengths", (n,), torch.int32)
    pm = _dense(marks, "marks", (n, -(-t // MARK_FRAMES), c), torch.float32)
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_gated_scan(ref, px, pf, p0, pn, po, pl, pm, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, out if made[0] else None, h_last if made[1] else None)
    return out, h_last


def gated_scan_backward(dy, x, f, marks, lengths=None, dh_last=None, dx=None, df=None, dh0=None, stream=None):
    """``rrm_gated_scan_backward``: (dx, df, dh0) from ``dy``, the forward pass's inputs and ``marks``, and the gradient
    ``dh_last`` (float32 [n, c]; None: zeros) of the last state."""
    import torch
    n, t, c = _scan_shape(x)
    shape = (n, t, c)
    made = [g is None for g in (dx, df, dh0)]
    if dx is None:
        dx = torch.empty(shape, dtype=x.dtype, device=x.device)
    if df is None:
        df = torch.empty(shape, dtype=x.dtype, device=x.device)
    if dh0 is None:
        dh0 = torch.empty((n, c), dtype=torch.float32, device=x.device)
    px, pf, pdy = _expect(x, "x", shape), _expect(f, "f", shape, x.dtype), _expect(dy, "dy", shape, x.dtype)
    pdx, pdf = _expect(dx, "dx", shape, x.dtype), _expect(df, "df", shape, x.dtype)
    d, ref, need = _desc(ScanDesc, "rrm_gated_scan_workspace", 1, n, t, c, _elem(x), *_frames(x, "x"), *_frames(f, "f"),
                         *_frames(dy, "dy"), *_frames(dx, "dx"), *_frames(df, "df"))
    pm = _dense(marks, "marks", (n, -(-t // MARK_FRAMES), c), torch.float32)
    pn = _dense(lengths, "lengths", (n,), torch.int32)
    pl, p0 = _dense(dh_last, "dh_last", (n, c), torch.float32), _dense(dh0, "dh0", (n, c), torch.float32)
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_gated_scan_backward(ref, px, pf, pm, pn, pdy, pl, pdx, pdf, p0, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, *(g for g, was in zip((dx, df, dh0), made) if was))
    return dx, df, dh0


# -- gated feed-forward block ------------------------------------------------------------------------------------------

def gated_ff(x, wg, wu, act: str = "silu", out=None, save=None, stream=None):
    """``rrm_gated_ff``: act(x wg^T) * (x wu^T), bfloat16: ``x`` [m, k], ``wg`` and ``wu`` [f, k], the result [m, f].
    ``save``: two tensors [m, f] that receive the two projections for the backward pass."""
    import torch
    m, k = x.shape
    f = wg.shape[0]
    made = out is None
    if made:
        out = torch.empty((m, f), dtype=torch.bfloat16, device=x.device)
    bf = torch.bfloat16
    px, pg, pu = _expect(x, "x", (m, k), bf), _expect(wg, "wg", (f, k), bf), _expect(wu, "wu", (f, k), bf)
    po = _expect(out, "out", (m, f), bf)
    sg = su = None
    row = 0
    if save is not None:
        sg, su = _expect(save[0], "save[0]", (m, f), bf), _expect(save[1], "save[1]", (m, f), bf)
        row = _row(save[0], "save[0]")
        if _row(save[1], "save[1]") != row:
            raise ValueError("save: both tensors need the same strides")
    d, ref, need = _desc(FFDesc, "rrm_gated_ff_workspace", 0, m, k, f, _act(act), _row(x, "x"), _row(wg, "wg"), _row(wu, "wu"),
                         _row(out, "out"), row, 0, 0, 0, int((px | pg | pu) & 15 != 0))
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_gated_ff(ref, px, pg, pu, po, sg, su, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, out if made else None)
    return out


def gated_ff_backward(dh, x, wg, wu, g, u, act: str = "silu", dx=None, dwg=None, dwu=None, stream=None):
    """``rrm_gated_ff_backward``: (dx, dwg, dwu) from ``dh`` and the projections ``g`` and ``u`` that the forward pass saved."""
    import torch
    m, k = x.shape
    f = wg.shape[0]
    bf = torch.bfloat16
    made = [t is None for t in (dx, dwg, dwu)]
    if dx is None:
        dx = torch.empty((m, k), dtype=bf, device=x.device)
    if dwg is None:
        dwg = torch.empty((f, k), dtype=bf, device=x.device)
    if dwu is None:
        dwu = torch.empty((f, k), dtype=bf, device=x.device)
    px, pg, pu = _expect(x, "x", (m, k), bf), _expect(wg, "wg", (f, k), bf), _expect(wu, "wu", (f, k), bf)
    sg, su, pdh = _expect(g, "g", (m, f), bf), _expect(u, "u", (m, f), bf), _expect(dh, "dh", (m, f), bf)
    qx, qg, qu = _expect(dx, "dx", (m, k), bf), _expect(dwg, "dwg", (f, k), bf), _expect(dwu, "dwu", (f, k), bf)
    row = _row(g, "g")
    if _row(u, "u") != row:
        raise ValueError("g, u: both tensors need the same strides")
    d, ref, need = _desc(FFDesc, "rrm_gated_ff_workspace", 1, m, k, f, _act(act), _row(x, "x"), _row(wg, "wg"), _row(wu, "wu"),
                         _row(dh, "dh"), row, _row(dx, "dx"), _row(dwg, "dwg"), _row(dwu, "dwu"),
                         int((px | pg | pu) & 15 != 0))
    ws, pw = _workspace(need, x.device)
    _check(lib().rrm_gated_ff_backward(ref, px, pg, pu, sg, su, pdh, qx, qg, qu, pw, need, _stream_ptr(stream)))
    _used_on(stream, ws, *(t for t, was in zip((dx, dwg, dwu), made) if was))
    return dx, dwg, dwu
