"""Operators between and behind the linear layers against plain implementations in 64 bits, at sizes, strides, masks and
types where they can go wrong; their gradients against the formulas (autograd in 64 bits) and against differences; their refusals.

Tolerances, with u = 2^-24 (float32) and v = 2^-8 (bfloat16: neighbours in [1, 2) are 2^-7 apart, a rounding is off by half of that):
  a result rounded to bfloat16 is off by v of itself, and by what it was off before;
  before that, sums of m terms held as trees of partial sums are off by some log2(m) + 8 rounding errors u of the sum of the
  magnitudes (SUM below: 32 u, enough for every m here); a gate or an activation by a few u of its magnitude, and the erf form by
  1.5e-7 (the published bound of its polynomial), which GATE = 16 u ~ 1e-6 holds.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_1802_09723_amd as rrm
from paper_1802_09723_amd import operators as ops
from paper_1802_09723_amd.binding import RRMError

gpu = pytest.mark.gpu

U = 2.0 ** -24
V = 2.0 ** -8
SUM = 32 * U
GATE = 16 * U
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def act64(act, z):
    if act == "relu":
        return torch.relu(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def check(got, want, slack, what):
    """|got - want| <= slack (a number or a tensor), plus the rounding of got's type; same shape, finite where want is."""
    got_d = got.detach().cpu().double()
    assert got_d.shape == want.shape, f"{what}: shape {tuple(got_d.shape)} != {tuple(want.shape)}"
    half = V if got.dtype == torch.bfloat16 else U
    lim = slack + half * (want.abs() + slack) + 1e-38
    err = (got_d - want).abs()
    bad = ~(err <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {err[bad].max() if bad.any() else 0} where {(lim + 0 * err)[bad].max()} is allowed"


# -- group norm ----------------------------------------------------------------------------------------------------------

def norm64(x, groups, gamma, beta, act, eps=1e-5):
    n, c = x.shape[0], x.shape[-1]
    v = x.reshape(n, -1, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    z = ((v - mean) * r).reshape(x.shape)
    z = z * gamma + beta
    return act64(act, z), mean.reshape(n, groups), r.reshape(n, groups)


def norm_slack(x64, groups, gamma, beta, stats_r):
    """What z may be off by before its rounding: the statistics' errors, magnified by r where a mean dwarfs the deviation."""
    big = float(x64.abs().max()) * float(stats_r.max()) * (float(gamma.abs().max()))
    return SUM * (big + float(beta.abs().max()) + 1) + GATE


NORM = [
    # n, positions' shape, c, groups
    (1, (1, 1), 1, 1),
    (1, (1, 1), 8, 8),      # groups of one value: variance 0
    (3, (1, 1), 64, 4),
    (1, (7, 7), 512, 32),
    (2, (5, 9), 105, 7),    # nothing divides
    (2, (13, 13), 12, 4),
    (4, (6, 5), 24, 24),    # a group a channel
    (2, (3, 3), 17, 1),     # one group
    (2, (30, 31), 40, 5),
    (1, (56, 56), 64, 32),
    (3, (4, 4), 4096, 4),
    (1, (2, 3), 5000, 1000),
    (1, (150, 151), 36, 6), # a long sample
    (1, (300, 200), 16, 2), # beyond what one workgroup holds
    (1, (1, 70000), 3, 1),
    (70, (3, 2), 30, 3),
]


@gpu
@pytest.mark.parametrize("types", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", NORM)
def test_norm_forward_and_backward(shape, types):
    n, hw, c, groups = shape
    act = ("none", "relu", "silu", "gelu")[(n + c + groups) % 4]
    tx, ty = DT[types[0]], DT[types[1]]
    g = gen(n * 1000 + c)
    x = (torch.randn(n, *hw, c, generator=g) * 1.5 + torch.randn(c, generator=g)).to(tx)
    gamma, beta = 1 + 0.2 * torch.randn(c, generator=g), 0.3 * torch.randn(c, generator=g)
    dy = torch.randn(n, *hw, c, generator=g).to(ty)
    x64 = x.double().requires_grad_()
    ga64, be64 = gamma.double().requires_grad_(), beta.double().requires_grad_()
    y64, mean64, r64 = norm64(x64, groups, ga64, be64, act)
    stats = torch.empty(n, groups, 2, device="cuda")
    xd, gd, bd = x.cuda(), gamma.cuda(), beta.cuda()
    y = rrm.group_norm_act(xd, groups, gd, bd, act, out_dtype=ty, stats=stats)
    slack = norm_slack(x64.detach(), groups, gamma, beta, r64.detach())
    check(y, y64.detach(), slack, "y")
    check(stats[..., 0], mean64.detach(), SUM * float(x.abs().max()), "mean")
    check(stats[..., 1], r64.detach(), SUM * float(r64.detach().max()) * (1 + float(x64.detach().abs().max() * r64.detach().max())), "r")

    if act == "relu":
        # where z is next to 0 its sign, and with it the slope, may fall either way: no gradient comes in there
        z = norm64(x.double(), groups, gamma.double(), beta.double(), "none")[0]
        dy = torch.where(z.abs() <= 4 * slack, torch.zeros(()), dy.float()).to(ty)
    want = torch.autograd.grad(y64, (x64, ga64, be64), dy.double())
    dx, dgamma, dbeta = rrm.group_norm_act_backward(dy.cuda(), xd, stats, gd, bd, act)
    # dz is off by the slope's error, and xh by the slack: both in sums of magnitudes
    m = (n * hw[0] * hw[1])
    mag = float(dy.abs().max()) * 1.2
    xh = float(((x64.detach().abs().max() + 3) * r64.detach().max()).clamp(min=1))
    check(dbeta, want[2], mag * (4 * slack + SUM) * math.sqrt(m) * 4, "dbeta")
    check(dgamma, want[1], mag * (4 * slack + SUM) * xh * math.sqrt(m) * 4, "dgamma")
    rr = float(r64.detach().max())
    check(dx, want[0], rr * mag * float(gamma.abs().max()) * (8 * slack + SUM) * xh * xh, "dx")


@gpu
@pytest.mark.parametrize("shape", [(2, (9, 7), 64, 8), (1, (40, 50), 32, 4), (2, (300, 120), 32, 4)])
def test_norm_of_values_far_from_zero(shape):
    """A mean a thousand deviations away: a variance from sums of squares would lose all its digits."""
    n, hw, c, groups = shape
    x = 1000 + torch.randn(n, *hw, c, generator=gen(5))
    y64, mean64, r64 = norm64(x.double(), groups, torch.ones(c).double(), torch.zeros(c).double(), "none")
    y = rrm.group_norm_act(x.cuda(), groups)
    check(y, y64, norm_slack(x.double(), groups, torch.ones(c), torch.zeros(c), r64), "y")


@gpu
def test_norm_is_by_group_and_sample():
    """Not-a-numbers and infinities of one sample's group stay in it; a constant group gives beta."""
    x = torch.randn(3, 4, 5, 32, generator=gen(1))
    x[1, 2, 2, 9] = math.nan
    x[2, 0, 0, 31] = math.inf
    x[0, :, :, 0:8] = 2.5
    y = rrm.group_norm_act(x.cuda(), 4, None, torch.full((32,), 0.25, device="cuda")).cpu()
    clean = torch.ones(3, 4, dtype=torch.bool)
    clean[1, 1] = clean[2, 3] = False
    ok = torch.isfinite(y).view(3, 20, 4, 8).permute(0, 2, 1, 3).reshape(3, 4, -1).all(-1)
    assert torch.equal(ok, clean)
    assert torch.equal(y[0, :, :, 0:8], torch.full((4, 5, 8), 0.25))


@gpu
@pytest.mark.parametrize("ty", ["f32", "bf16"])
@pytest.mark.parametrize("lo", [0, 1, 2, 8])
def test_norm_strides(ty, lo):
    """Channels out of wider maps, at every alignment, in and out; a sample axis that lies inside the positions'."""
    wide = torch.randn(2, 6, 7, 48, generator=gen(lo)).to(DT[ty]).cuda()
    x = wide[..., lo:lo + 24]
    back = torch.full((2, 6, 7, 40), 7.0, device="cuda", dtype=DT[ty])
    out = back[..., 3:27]
    g, b = torch.rand(24, device="cuda") + 0.5, torch.randn(24, device="cuda")
    stats = torch.empty(2, 6, 2, device="cuda")
    rrm.group_norm_act(x, 6, g, b, "silu", out=out, stats=stats)
    want = rrm.group_norm_act(x.contiguous(), 6, g, b, "silu")
    assert torch.equal(out, want)
    assert (back[..., :3] == 7).all() and (back[..., 27:] == 7).all()
    dy = torch.randn(2, 6, 7, 32, generator=gen(9)).to(DT[ty]).cuda()
    whole = torch.full((2, 6, 7, 33), 7.0, device="cuda", dtype=DT[ty])
    dx = whole[..., 2:26]
    got = rrm.group_norm_act_backward(dy[..., 1:25], x, stats, g, b, "silu", dx=dx)
    ref = rrm.group_norm_act_backward(dy[..., 1:25].contiguous(), x.contiguous(), stats, g, b, "silu")
    for a, e in zip(got, ref):
        assert torch.equal(a, e)
    assert (whole[..., :2] == 7).all() and (whole[..., 26:] == 7).all()
    t = torch.randn(42, 2, 24, generator=gen(3)).to(DT[ty]).cuda().transpose(0, 1)
    assert torch.equal(rrm.group_norm_act(t, 6, g, b), rrm.group_norm_act(t.contiguous(), 6, g, b))


@gpu
def test_norm_of_nothing():
    g = torch.randn(8, device="cuda")
    for shape in ((0, 3, 3, 8), (2, 0, 3, 8)):
        x = torch.empty(shape, device="cuda")
        stats = torch.empty(shape[0], 2, 2, device="cuda")
        assert rrm.group_norm_act(x, 2, g, g, "silu", stats=stats).shape == shape
        dx, dgamma, dbeta = rrm.group_norm_act_backward(x, x, stats, g, g, "silu")
        assert dx.shape == shape and not dgamma.any() and not dbeta.any()


# -- gated scan ----------------------------------------------------------------------------------------------------------

def scan64(x, f, h0, lengths):
    """frame by frame; values behind a video's end are never touched"""
    n, t, c = x.shape
    ys, hs = [], []
    for i in range(n):
        h, end, rows = h0[i], int(lengths[i]), []
        for k in range(end):
            a = torch.sigmoid(f[i, k])
            h = a * h + torch.sigmoid(-f[i, k]) * x[i, k]
            rows.append(h)
        rows += [torch.zeros(c, dtype=torch.float64)] * (t - end)
        ys.append(torch.stack(rows) if rows else torch.zeros(0, c, dtype=torch.float64))
        hs.append(h)
    return torch.stack(ys), torch.stack(hs)


def scan_inputs(n, t, c, dtype, ragged, seed=0):
    g = gen(seed + n * 7 + t * 3 + c)
    x = torch.randn(n, t, c, generator=g).to(DT[dtype])
    f = (torch.randn(n, t, c, generator=g) + 4 * torch.rand(c, generator=g)).to(DT[dtype])
    h0 = torch.randn(n, c, generator=g)
    lengths = torch.full((n,), t, dtype=torch.int32)
    if ragged:
        lengths = torch.randint(0, t + 1, (n,), generator=g, dtype=torch.int32)
        lengths[0] = 0
        for i in range(n):
            x[i, int(lengths[i]):] = math.nan
            f[i, int(lengths[i]):] = math.inf
    return x, f, h0, lengths


SCAN = [
    # n, t, c
    (1, 1, 1), (1, 1, 4096), (3, 1, 70), (2, 2, 8), (1, 63, 16), (2, 64, 33), (2, 65, 64), (3, 200, 129), (1, 513, 72),
    (2, 1000, 24), (5, 130, 520), (1, 2500, 40), (70, 9, 8),
]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", SCAN)
def test_scan_forward_and_backward(shape, ragged, dtype):
    n, t, c = shape
    x, f, h0, lengths = scan_inputs(n, t, c, dtype, ragged)
    g = gen(77)
    dy, dh = torch.randn(n, t, c, generator=g).to(DT[dtype]), torch.randn(n, c, generator=g)
    leaves = [v.double().requires_grad_() for v in (x, f, h0)]
    y64, last64 = scan64(*leaves, lengths)
    dy64 = dy.double()
    if ragged:
        for i in range(n):
            dy[i, int(lengths[i]):] = math.nan
            dy64[i, int(lengths[i]):] = 0
    total = (y64 * dy64).sum() + (last64 * dh.double()).sum()  # (videos of no frames: last64 is h0)
    want = [w if w is not None else torch.zeros_like(v) for w, v in zip(torch.autograd.grad(total, leaves, allow_unused=True), leaves)]
    xd, fd, hd = x.cuda(), f.cuda(), h0.cuda()
    ld = lengths.cuda() if ragged else None
    marks = rrm.gated_scan_marks(xd)
    y, last = rrm.gated_scan(xd, fd, hd, lengths=ld, marks=marks)
    plain, plain_last = rrm.gated_scan(xd, fd, hd, lengths=ld)
    assert torch.equal(y, plain) and torch.equal(last, plain_last)
    # a step's error is some units of the largest |h|, and later gates shrink it; memories of up to some e^8 frames add them up
    top = max(1.0, float(torch.nan_to_num(x.float(), 0).abs().max()), float(h0.abs().max()))
    slack = top * (SUM + 2 * U * math.sqrt(t) + GATE) * 2
    check(y, y64.detach(), slack, "y")
    check(last, last64.detach(), slack, "h_last")
    got = rrm.gated_scan_backward(dy.cuda(), xd, fd, marks, lengths=ld, dh_last=dh.cuda())
    # g sums some e^8 frames' dy at the most, each as well held
    gmax = float(max((w.detach().abs().max() for w in (want[2],)), default=0)) + 4 * math.sqrt(t) + 8
    # the largest |g| bounds what a gradient is off by: dx = (1 - a) g, df = g (h - x) a (1 - a)
    gs = slack / top * gmax
    check(got[0], want[0], gs, "dx")
    check(got[1], want[1], gs * 2 * top, "df")
    check(got[2], want[2], gs, "dh0")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_of_many_frames(dtype):
    """A long video with slow gates against a loop in 64 bits on the device."""
    n, t, c = 2, 20011, 24
    x, f, h0, _ = scan_inputs(n, t, c, dtype, False)
    lengths = torch.tensor([t, 15000], dtype=torch.int32)
    xd, fd, hd = x.cuda(), f.cuda(), h0.cuda()
    marks = rrm.gated_scan_marks(xd)
    y, last = rrm.gated_scan(xd, fd, hd, lengths=lengths.cuda(), marks=marks)
    a, b = torch.sigmoid(fd.double()), torch.sigmoid(-fd.double()) * xd.double()
    a[1, 15000:], b[1, 15000:] = 1, 0
    hs = torch.empty(n, t + 1, c, dtype=torch.float64, device="cuda")
    hs[:, 0] = hd.double()
    for k in range(t):
        torch.addcmul(b[:, k], a[:, k], hs[:, k], out=hs[:, k + 1])
    want = hs[:, 1:].clone()
    want[1, 15000:] = 0
    slack = 5 * (SUM + 2 * U * 64 + GATE) * 2
    check(y, want.cpu(), slack, "y")
    check(last, hs[:, t].cpu(), slack, "h_last")
    check(marks, hs[:, 0:t:64].cpu(), slack, "marks")
    dy = torch.randn(n, t, c, generator=gen(3)).to(DT[dtype]).cuda()
    got = rrm.gated_scan_backward(dy, xd, fd, marks, lengths=lengths.cuda())
    dy64 = dy.double()
    dy64[1, 15000:] = 0
    grads = torch.empty_like(want)
    carry = torch.zeros(n, c, dtype=torch.float64, device="cuda")
    for k in range(t - 1, -1, -1):
        torch.add(carry, dy64[:, k], out=grads[:, k])
        carry = grads[:, k] * a[:, k]
    dx = grads * torch.sigmoid(-fd.double())
    df = grads * (hs[:, :-1] - xd.double()) * a * torch.sigmoid(-fd.double())
    dx[1, 15000:], df[1, 15000:] = 0, 0
    gs = slack * float(grads.abs().max()) / 5
    check(got[0], dx.cpu(), gs, "dx")
    check(got[1], df.cpu(), gs * 10, "df")
    check(got[2], carry.cpu(), gs, "dh0")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(4, 5000, 130), (3, 4224, 9), (1, 9001, 5)])
def test_scan_of_one_video_by_many_workgroups(shape, dtype):
    """The state is handed on between workgroups: the same bits in every call, and those of pieces of the video but for roundings; videos end at
    the borders of what a workgroup takes, in it, at once."""
    n, t, c = shape
    x, f, h0, _ = scan_inputs(n, t, c, dtype, False)
    ends = [t, 128 * 32, 0, 64 * 33][:n]
    lengths = torch.tensor(ends, dtype=torch.int32).cuda()
    xd, fd, hd = x.cuda(), f.cuda(), h0.cuda()
    dy, dh = torch.randn(n, t, c, generator=gen(5)).to(DT[dtype]).cuda(), torch.randn(n, c, generator=gen(6)).cuda()
    first = None
    for _ in range(4):
        marks = rrm.gated_scan_marks(xd)
        y, last = rrm.gated_scan(xd, fd, hd, lengths=lengths, marks=marks)
        got = (y, last, marks, *rrm.gated_scan_backward(dy, xd, fd, marks, lengths=lengths, dh_last=dh))
        if first is None:
            first = [v.clone() for v in got]
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    slack = 5 * (SUM + 2 * U * 64 + GATE) * 2
    for i, end in enumerate(ends):
        h = hd[i:i + 1]
        assert not first[0][i, end:].any() and not first[3][i, end:].any() and not first[4][i, end:].any()
        for k in range(0, end, 500):
            e = min(end, k + 500)
            piece, h = rrm.gated_scan(xd[i:i + 1, k:e], fd[i:i + 1, k:e], h)
            check(first[0][i:i + 1, k:e], piece.double().cpu(), slack + (2 ** -8 * 5 if dtype == "bf16" else 0), "y")
        check(first[1][i:i + 1], h.double().cpu(), slack, "h_last")
        g = dh[i:i + 1]
        for k in reversed(range(0, end, 320)):  # (whole marks)
            e = min(end, k + 320)
            part = [v[i:i + 1, k:e].contiguous() for v in (dy, xd, fd)]
            dx, df, g = rrm.gated_scan_backward(*part, first[2][i:i + 1, k // 64:(e - 1) // 64 + 1].contiguous(), dh_last=g)
            gs = slack * 20 + (2 ** -8 * 20 if dtype == "bf16" else 0)
            check(first[3][i:i + 1, k:e], dx.double().cpu(), gs, "dx")
            check(first[4][i:i + 1, k:e], df.double().cpu(), gs * 10, "df")
        check(first[5][i:i + 1], g.double().cpu(), slack * 20, "dh0")


@gpu
def test_scan_gates_at_their_ends():
    """Gates of 0 and 1 from infinite and far logits: the state is x_t, or h_{t-1}, without an error; gradients stay finite."""
    x = torch.randn(1, 6, 8, generator=gen(1))
    f = torch.tensor([math.inf, -math.inf, 200.0, -200.0, math.inf, -math.inf]).view(1, 6, 1).expand(1, 6, 8).contiguous()
    h0 = torch.randn(1, 8, generator=gen(2))
    marks = rrm.gated_scan_marks(x.cuda())
    y, last = rrm.gated_scan(x.cuda(), f.cuda(), h0.cuda(), marks=marks)
    want = torch.stack([h0[0], x[0, 1], x[0, 1], x[0, 3], x[0, 3], x[0, 5]])[None]
    assert torch.equal(y.cpu(), want) and torch.equal(last.cpu(), x[:, 5])
    for t in rrm.gated_scan_backward(torch.ones(1, 6, 8, device="cuda"), x.cuda(), f.cuda(), marks):
        assert torch.isfinite(t).all()
    f[0, 2, 3] = math.nan
    y = rrm.gated_scan(x.cuda(), f.cuda(), h0.cuda())[0].cpu()
    bad = torch.isnan(y)
    assert bad[0, 2:3, 3].all() and not bad[0, :, :3].any() and not bad[0, :, 4:].any() and not bad[0, :2].any()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_of_live_videos_frame_by_frame(dtype):
    """One frame at a time, the state in place, gives what one call over all frames gives."""
    x, f, h0, _ = scan_inputs(5, 40, 100, dtype, False)
    xd, fd = x.cuda(), f.cuda()
    want, last = rrm.gated_scan(xd, fd, h0.cuda())
    h = h0.cuda()
    for k in range(40):
        y, h2 = rrm.gated_scan(xd[:, k:k + 1], fd[:, k:k + 1], h, h_last=h)
        assert h2 is h
        check(y[:, 0], want[:, k].cpu().double(), (SUM + GATE) * 10 + (V * 5 if dtype == "bf16" else 0), f"frame {k}")
    check(h, last.cpu().double(), (SUM + GATE) * 10, "state")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lo", [0, 1, 4, 8])
def test_scan_strides(dtype, lo):
    """x and f out of one joint projection, frames before videos, gradients into a joint one."""
    n, t, c = 3, 70, 40
    joint = torch.randn(t, n, 2 * c + 16, generator=gen(lo)).to(DT[dtype]).cuda().transpose(0, 1)
    x, f = joint[..., lo:lo + c], joint[..., lo + c:lo + 2 * c]
    marks = rrm.gated_scan_marks(x)
    out = torch.full((n, t, c + 9), 7.0, device="cuda", dtype=DT[dtype])
    y, last = rrm.gated_scan(x, f, marks=marks, out=out[..., lo:lo + c])
    want, wlast = rrm.gated_scan(x.contiguous(), f.contiguous(), torch.zeros(n, c, device="cuda"))
    assert torch.equal(y, want) and torch.equal(last, wlast)
    assert (out[..., :lo] == 7).all() and (out[..., lo + c:] == 7).all()
    dy = torch.randn(n, t, c, generator=gen(8)).to(DT[dtype]).cuda()
    grads = torch.full((t, n, 2 * c + 16), 7.0, device="cuda", dtype=DT[dtype]).transpose(0, 1)
    rrm.gated_scan_backward(dy, x, f, marks, dx=grads[..., lo:lo + c], df=grads[..., lo + c:lo + 2 * c])
    ref = rrm.gated_scan_backward(dy, x.contiguous(), f.contiguous(), marks)
    assert torch.equal(grads[..., lo:lo + c], ref[0]) and torch.equal(grads[..., lo + c:lo + 2 * c], ref[1])
    assert (grads[..., :lo] == 7).all() and (grads[..., lo + 2 * c:] == 7).all()
    # one x for all videos: the gradient is each video's own
    one = torch.randn(1, t, c, generator=gen(6)).to(DT[dtype]).cuda().expand(n, t, c)
    assert torch.equal(rrm.gated_scan(one, f)[0], rrm.gated_scan(one.contiguous(), f)[0])


@gpu
def test_scan_of_nothing():
    h0, dh = torch.randn(3, 8, device="cuda"), torch.randn(3, 8, device="cuda")
    x = torch.empty(3, 0, 8, device="cuda")
    y, last = rrm.gated_scan(x, x, h0)
    assert y.shape == (3, 0, 8) and torch.equal(last, h0)
    dx, df, dh0 = rrm.gated_scan_backward(x, x, x, rrm.gated_scan_marks(x), dh_last=dh)
    assert torch.equal(dh0, dh)
    x = torch.empty(0, 5, 8, device="cuda")
    y, last = rrm.gated_scan(x, x)
    assert y.shape == (0, 5, 8) and last.shape == (0, 8)
    # lengths outside of [0, t] are held to it
    x, f, h0, _ = scan_inputs(2, 10, 8, "f32", False)
    a = rrm.gated_scan(x.cuda(), f.cuda(), h0.cuda(), lengths=torch.tensor([-5, 99], dtype=torch.int32, device="cuda"))
    b = rrm.gated_scan(x.cuda(), f.cuda(), h0.cuda(), lengths=torch.tensor([0, 10], dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[1][0].cpu(), h0[0])


# -- gated feed-forward block -----------------------------------------------------------------------------------------------

FF = [
    # m, k, f
    (1, 1, 1), (1, 64, 64), (1, 4096, 256), (2, 1001, 333), (5, 72, 40), (16, 512, 512), (17, 256, 130), (33, 1000, 96),
    (64, 384, 1024), (100, 65, 67), (128, 128, 128), (129, 136, 264), (200, 1030, 300), (300, 512, 257), (513, 64, 700), (1030, 320, 520),
    (3000, 72, 104), (2100, 1001, 60), (40, 2500, 1100),  # few tiles over long sums
]


def ff_inputs(m, k, f, seed=0):
    g = gen(seed + m + 3 * k + 7 * f)
    x = torch.randn(m, k, generator=g).bfloat16()
    wg, wu = (torch.randn(f, k, generator=g) * k ** -0.5).bfloat16(), (torch.randn(f, k, generator=g) * k ** -0.5).bfloat16()
    return x, wg, wu, torch.randn(m, f, generator=g).bfloat16()


def ff_check(got, x, wg, wu, dh, act):
    """h, G, U against 64 bits; the gradients against the formulas at the G and U that were saved, with dG and dU rounded"""
    h, g, u, dx, dwg, dwu = got
    x64, wg64, wu64 = x.double(), wg.double(), wu.double()
    g64, u64 = x64 @ wg64.t(), x64 @ wu64.t()
    # a product's sums: 32 u of the sum of the magnitudes
    sg, su = SUM * (x64.abs() @ wg64.abs().t()), SUM * (x64.abs() @ wu64.abs().t())
    check(g, g64, sg, "g")
    check(u, u64, su, "u")
    a64 = act64(act, g64)
    check(h, a64 * u64, (1.2 * sg + GATE * (1 + g64.abs())) * (u64.abs() + su) + a64.abs() * su, "h")
    gs = g.cpu().double().requires_grad_()
    us = u.cpu().double()
    p = act64(act, gs)
    slope = torch.autograd.grad(p.sum(), gs)[0]
    p = p.detach()
    d64 = dh.double()
    dg, du = d64 * us * slope, d64 * p
    # rounded to bfloat16 before the products: V of each term, at random signs; 8 standard deviations of such a sum
    eg, eu = dg.abs() * (V + GATE) + GATE * (d64 * us).abs(), du.abs() * (V + GATE) + GATE * d64.abs()

    def off(e, w):
        return SUM * (e / V).matmul(w.abs()) + 8 * torch.sqrt((e * e).matmul(w * w)) + GATE * e.matmul(w.abs())

    check(dx, dg @ wg64 + du @ wu64, off(eg, wg64) + off(eu, wu64), "dx")
    check(dwg, dg.t() @ x64, off(eg.t(), x64), "dwg")
    check(dwu, du.t() @ x64, off(eu.t(), x64), "dwu")


@gpu
@pytest.mark.parametrize("shape", FF)
def test_ff_forward_and_backward(shape):
    m, k, f = shape
    act = ("silu", "gelu", "none", "relu")[(m + k + f) % 4]
    x, wg, wu, dh = ff_inputs(m, k, f)
    xd, gd, ud = x.cuda(), wg.cuda(), wu.cuda()
    g, u = torch.empty(m, f, device="cuda", dtype=torch.bfloat16), torch.empty(m, f, device="cuda", dtype=torch.bfloat16)
    h = rrm.gated_ff(xd, gd, ud, act, save=(g, u))
    assert torch.equal(h, rrm.gated_ff(xd, gd, ud, act))
    dx, dwg, dwu = rrm.gated_ff_backward(dh.cuda(), xd, gd, ud, g, u, act)
    ff_check((h, g, u, dx, dwg, dwu), x, wg, wu, dh, act)
    again = rrm.gated_ff_backward(dh.cuda(), xd, gd, ud, g, u, act)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dwg, dwu)))


@gpu
@pytest.mark.parametrize("m", [1, 3, 40, 150, 700])
@pytest.mark.parametrize("lo", [0, 1, 8])
def test_ff_strides(m, lo):
    """Both weights and both gradients as halves of joint tensors, rows out of wider ones at every alignment."""
    k, f = 104, 72
    joint = (torch.randn(2 * f, k + 16, generator=gen(lo)) * 0.1).bfloat16().cuda()
    wg, wu = joint[:f, lo:lo + k], joint[f:, lo:lo + k]
    x = torch.randn(m, k + 24, generator=gen(m)).bfloat16().cuda()[:, lo:lo + k]
    dh = torch.randn(m, f + 8, generator=gen(m + 1)).bfloat16().cuda()[:, lo % 8:lo % 8 + f]
    out = torch.full((m, f + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    both = torch.empty(m, 2 * f + 8, device="cuda", dtype=torch.bfloat16)
    g, u = both[:, lo % 8:lo % 8 + f], both[:, lo % 8 + f:lo % 8 + 2 * f]
    h = rrm.gated_ff(x, wg, wu, "silu", out=out[:, lo:lo + f], save=(g, u))
    dense = [t.contiguous() for t in (x, wg, wu)]
    assert torch.equal(h, rrm.gated_ff(*dense, "silu"))
    assert (out[:, :lo] == 7).all() and (out[:, lo + f:] == 7).all()
    dw = torch.full((2 * f, k + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    dxw = torch.full((m, k + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    rrm.gated_ff_backward(dh, x, wg, wu, g, u, "silu", dx=dxw[:, lo:lo + k], dwg=dw[:f, lo:lo + k], dwu=dw[f:, lo:lo + k])
    ref = rrm.gated_ff_backward(dh.contiguous(), *dense, g.contiguous(), u.contiguous(), "silu")
    assert torch.equal(dxw[:, lo:lo + k], ref[0]) and torch.equal(dw[:f, lo:lo + k], ref[1]) and torch.equal(dw[f:, lo:lo + k], ref[2])
    assert (dxw[:, :lo] == 7).all() and (dxw[:, lo + k:] == 7).all() and (dw[:, :lo] == 7).all() and (dw[:, lo + k:] == 7).all()


@gpu
@pytest.mark.parametrize("m", [1, 30, 200])
def test_ff_rows_stay_apart(m):
    """A row, a hidden feature or an input feature that is not a number spoils its own results alone."""
    x, wg, wu, dh = ff_inputs(m + 3, 200, 150)
    x[1, 7] = math.nan
    wg[5, 3] = math.inf
    g, u = torch.empty(m + 3, 150, device="cuda", dtype=torch.bfloat16), torch.empty(m + 3, 150, device="cuda", dtype=torch.bfloat16)
    h = rrm.gated_ff(x.cuda(), wg.cuda(), wu.cuda(), "none", save=(g, u)).cpu()
    good = torch.ones_like(h, dtype=torch.bool)
    good[1], good[:, 5] = False, False
    assert torch.isfinite(h[good]).all() and not torch.isfinite(h[1]).any()
    x[1, 7], wg[5, 3] = 1, 1
    h = rrm.gated_ff(x.cuda(), wg.cuda(), wu.cuda(), "none", save=(g, u))
    dh[2, 9] = math.nan
    dx, dwg, dwu = rrm.gated_ff_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), g, u, "none")
    rows = torch.isfinite(dx.cpu()).all(1)
    assert not rows[2] and rows[torch.arange(m + 3) != 2].all()
    for d in (dwg, dwu):
        rows = torch.isfinite(d.cpu()).all(1)
        assert not rows[9] and rows[torch.arange(150) != 9].all()


@gpu
def test_ff_of_nothing():
    x, wg, wu, dh = (t.cuda() for t in ff_inputs(0, 32, 16))
    h = rrm.gated_ff(x, wg, wu)
    assert h.shape == (0, 16)
    dx, dwg, dwu = rrm.gated_ff_backward(dh, x, wg, wu, h, h)
    assert dx.shape == (0, 32) and not dwg.any() and not dwu.any()


# -- gradients against differences --------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("which", ["norm", "scan"])
def test_gradients_against_differences(which):
    """The derivative along random directions: the kernels' gradients times the direction, against the difference quotient of the
    definitions in 64 bits."""
    g = gen(11)
    step = 1e-5
    if which == "norm":
        args = [torch.randn(2, 5, 3, 12, generator=g), 1 + 0.1 * torch.randn(12, generator=g), torch.randn(12, generator=g)]
        dy = torch.randn(2, 5, 3, 12, generator=g)
        stats = torch.empty(2, 3, 2, device="cuda")
        dev = [a.cuda() for a in args]
        rrm.group_norm_act(dev[0], 3, dev[1], dev[2], "gelu", stats=stats)
        grads = rrm.group_norm_act_backward(dy.cuda(), dev[0], stats, dev[1], dev[2], "gelu")

        def loss(v):
            return float((norm64(v[0], 3, v[1], v[2], "gelu")[0] * dy.double()).sum())
    else:
        args = [torch.randn(2, 70, 6, generator=g), torch.randn(2, 70, 6, generator=g), torch.randn(2, 6, generator=g)]
        dy, dh = torch.randn(2, 70, 6, generator=g), torch.randn(2, 6, generator=g)
        dev = [a.cuda() for a in args]
        marks = rrm.gated_scan_marks(dev[0])
        rrm.gated_scan(*dev, marks=marks)
        grads = rrm.gated_scan_backward(dy.cuda(), dev[0], dev[1], marks, dh_last=dh.cuda())

        def loss(v):
            y, last = scan64(v[0], v[1], v[2], [70, 70])
            return float((y * dy.double()).sum() + (last * dh.double()).sum())
    for k in range(3):
        d = torch.randn(args[k].shape, generator=g).double()
        lo, hi = [a.double() for a in args], [a.double() for a in args]
        lo[k] = lo[k] - step * d
        hi[k] = hi[k] + step * d
        quotient = (loss(hi) - loss(lo)) / (2 * step)
        got = float((grads[k].cpu().double() * d).sum())
        # a quotient of 64-bit losses: step^2 of the third derivatives (some tens) and 1e-16 / step of the losses (some tens)
        norm = float(grads[k].cpu().double().norm() * d.norm())
        assert abs(got - quotient) <= 1e-6 * norm + 1e-7, (which, k, got, quotient)


# -- streams, graphs, the layers' own outputs ----------------------------------------------------------------------------------

@gpu
def test_operators_on_a_stream_of_their_own_and_in_a_graph():
    """Another stream than the current one, by object and by handle; a captured chain replayed over changing inputs."""
    n, t, c = 4, 200, 64
    x, f, h0, _ = scan_inputs(n, t, c, "bf16", False)
    xd, fd, hd = x.cuda(), f.cuda(), h0.cuda()
    w = [v.cuda() for v in ff_inputs(n * t, c, 96)[1:3]]
    gamma, beta = torch.rand(c, device="cuda") + 0.5, torch.randn(c, device="cuda")

    def chain(stream=None):
        a = rrm.group_norm_act(xd, 8, gamma, beta, "silu", stream=stream)
        y, last = rrm.gated_scan(a, fd, hd, stream=stream)
        return rrm.gated_ff(y.view(n * t, c), *w, "gelu", stream=stream), last

    want = [v.clone() for v in chain()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (side, side.cuda_stream):
        got = chain(s)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = chain()
    for k in range(4):
        xd.copy_(torch.randn(n, t, c, generator=gen(k)))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        want = chain()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_scans_that_hand_on_their_state_on_two_streams_and_in_a_graph():
    """Long videos, whose blocks wait for one another: two calls at once on streams of their own, and a captured pass, both ways, replayed over
    changing inputs with the same calls between the replays; strided inputs, not-a-numbers behind the ends."""
    n, t, c = 3, 3000, 72
    x, f, h0, _ = scan_inputs(n, t, 2 * c, "bf16", False)
    ends = [t, 1000, 0]
    for i, end in enumerate(ends):
        x[i, end:], f[i, end:] = math.nan, math.inf
    lengths = torch.tensor(ends, dtype=torch.int32).cuda()
    xd, fd, hd = x.cuda()[:, :, c:], f.cuda()[:, :, :c], h0.cuda()[:, :c].contiguous()
    dy = torch.randn(n, t, c, generator=gen(8)).bfloat16().cuda()

    def both(stream=None):
        marks = rrm.gated_scan_marks(xd)
        y, last = rrm.gated_scan(xd, fd, hd, lengths=lengths, marks=marks, stream=stream)
        return (y, last, marks, *rrm.gated_scan_backward(dy, xd, fd, marks, lengths=lengths, stream=stream))

    want = [v.clone() for v in both()]
    assert all(torch.isfinite(v).all() for v in want)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [both(s) for _ in range(5) for s in sides]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for k in range(4):
        xd.copy_(torch.randn(n, t, c, generator=gen(k)))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_the_example_runs_them_together():
    """The live path against plain torch in 64 bits on the same parameters and frames; training brings the loss down."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "video_head.py")
    spec = importlib.util.spec_from_file_location("video_head", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses, logits, labels = ex.main()
    assert losses[-1] < 0.5 * losses[0] and torch.isfinite(logits).all()
    net = ex.Net(seed=3)
    frames = ex.synthetic_clip(net, 6, seed=4)
    got = [net.serve(fr).cpu().double() for fr in frames]

    def b(v):  # the roundings between the steps
        return v.float().bfloat16().double()

    def conv(x, w, stride):
        return torch.nn.functional.conv2d(x.permute(0, 3, 1, 2), b(w).permute(0, 3, 1, 2), stride=stride, padding=1).permute(0, 2, 3, 1)

    h = torch.zeros(net.n, 64, dtype=torch.float64)
    for fr, lg in zip(frames, got):
        a = b(norm64(conv(fr.cpu().double(), net.w1, 1), 8, torch.ones(32).double(), torch.zeros(32).double(), "silu")[0])
        a = b(norm64(conv(a, net.w2, 2), 8, torch.ones(64).double(), torch.zeros(64).double(), "silu")[0])
        feat = b(a.mean((1, 2)))
        gate = torch.sigmoid(b(feat @ net.gate.cpu().double().t()))
        h = gate * h + (1 - gate) * feat
        y = b(h)
        z = b(act64("silu", y @ net.wg.cpu().double().t()) * (y @ net.wu.cpu().double().t()))
        want = z @ net.out.cpu().double().t()
        # six roundings to bfloat16 stand between a frame and its logits, each off by 2^-8 of what it rounds at the most; a value
        # that another precision's sum rounds the other way moves by twice that, and the sums behind average it
        assert float((lg - want).abs().max()) <= 12 * V * float(want.abs().max()), float((lg - want).abs().max() / want.abs().max())


@gpu
def test_norm_of_a_layers_stored_projection():
    """Read in place after a delta step; the same as of a copy; other layers are refused."""
    import rrm_synth as S
    w = S.f32_to_bf16_bits(np.random.default_rng(0).normal(size=(40, 3, 3, 16)).astype(np.float32) * 0.1)
    layer = rrm.Layer(S.conv_shape(9, 11, 16, 40, 3, 1, 1, n=2), rrm.BF16, w)
    x = torch.randn(2, 9, 11, 16, generator=gen(1)).bfloat16().cuda()
    for k in range(2):
        x[:, k:k + 3, 2:5] += 1
        layer.step(x)
        stats = torch.empty(2, 5, 2, device="cuda")
        got = rrm.group_norm_act_of(layer, 5, act="relu", stats=stats)
        want = rrm.group_norm_act(layer.y_snapshot(), 5, act="relu", out_dtype=torch.bfloat16)
        assert torch.equal(got, want) and torch.isfinite(stats).all()
    layer.destroy()
    other = rrm.Layer(S.fc_shape(16, 8), rrm.BF16, S.f32_to_bf16_bits(np.ones((8, 16), np.float32)))
    with pytest.raises(ValueError, match="convolution"):
        rrm.group_norm_act_of(other, 2)
    other.destroy()


@gpu
def test_offsets_beyond_32_bits():
    """Two videos, samples or rows more than 2^32 elements apart: the same results as of their copies."""
    far = (1 << 32) + 24
    big = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
    small = torch.randn(2, 40, 24, generator=gen(2)).bfloat16().cuda()
    x = big.as_strided((2, 40, 24), (far, 24, 1))
    x.copy_(small)
    f = torch.randn(2, 40, 24, generator=gen(3)).bfloat16().cuda()
    out = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda").as_strided((2, 40, 24), (far, 24, 1))
    y, last = rrm.gated_scan(x, f, out=out)
    want, wlast = rrm.gated_scan(small, f)
    assert torch.equal(y, want) and torch.equal(last, wlast)
    marks = rrm.gated_scan_marks(small)
    rrm.gated_scan(x, f, marks=marks)
    got = rrm.gated_scan_backward(x, x, f, marks, dx=out)
    for a, e in zip(got, rrm.gated_scan_backward(small, small, f, marks)):
        assert torch.equal(a, e)
    stats = torch.empty(2, 3, 2, device="cuda")
    y = rrm.group_norm_act(x, 3, act="gelu", out=out, stats=stats)
    assert torch.equal(y, rrm.group_norm_act(small, 3, act="gelu"))
    for a, e in zip(rrm.group_norm_act_backward(x, x, stats, act="gelu", dx=out), rrm.group_norm_act_backward(small, small, stats, act="gelu")):
        assert torch.equal(a, e)
    for m in (2, 20):  # rows a gigabyte and more apart
        step = far // (m - 1) // 8 * 8
        rows = big.as_strided((m, 24), (step, 1))
        rows.copy_(torch.randn(m, 24, generator=gen(m)).bfloat16())
        x2, to = rows.contiguous(), torch.empty_strided((m, 24), (step, 1), dtype=torch.bfloat16, device="cuda")
        wg, wu = torch.randn(24, 24, generator=gen(5)).bfloat16().cuda(), torch.randn(24, 24, generator=gen(6)).bfloat16().cuda()
        g, u = torch.empty(m, 24, device="cuda", dtype=torch.bfloat16), torch.empty(m, 24, device="cuda", dtype=torch.bfloat16)
        assert torch.equal(rrm.gated_ff(rows, wg, wu, out=to, save=(g, u)), rrm.gated_ff(x2, wg, wu))
        for a, e in zip(rrm.gated_ff_backward(rows, rows, wg, wu, g, u, dx=to), rrm.gated_ff_backward(x2, x2, wg, wu, g, u)):
            assert torch.equal(a, e)


# -- refusals ------------------------------------------------------------------------------------------------------------------

def _norm_desc(**kw):
    v = dict(n=2, positions=9, c=8, groups=2, x_elem=0, y_elem=0, act=0, eps=1e-5, x_sample=72, x_position=8, y_sample=72, y_position=8,
             dx_sample=72, dx_position=8)
    v.update(kw)
    return ops.NormDesc(*v.values())


def _scan_desc(**kw):
    v = dict(n=2, t=9, c=8, elem=0, x_video=72, x_frame=8, f_video=72, f_frame=8, y_video=72, y_frame=8, dx_video=72, dx_frame=8,
             df_video=72, df_frame=8)
    v.update(kw)
    return ops.ScanDesc(*v.values())


def _ff_desc(**kw):
    v = dict(m=4, k=8, f=16, act=2, x_row=8, wg_row=8, wu_row=8, h_row=16, gu_row=16, dx_row=8, dwg_row=8, dwu_row=8)
    v.update(kw)
    return ops.FFDesc(*v.values())


def test_descriptors_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rrm.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    kinds = {"int": ctypes.c_int, "float": ctypes.c_float, "int64_t": ctypes.c_int64}
    for name, cls in (("rrm_norm_desc", ops.NormDesc), ("rrm_scan_desc", ops.ScanDesc), ("rrm_ff_desc", ops.FFDesc)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*%s;" % name, text, flags=re.S).group(1)
        fields = [(f.strip(), kinds[kind]) for kind, names in re.findall(r"\b(int64_t|int|float)\s+([a-z_0-9, \n]+);", body) for f in names.split(",")]
        assert fields == list(cls._fields_), name
    assert int(re.search(r"RRM_SCAN_MARK_FRAMES (\d+)", text).group(1)) == ops.MARK_FRAMES


def test_refusals_come_back_as_status_codes():
    """No call below reaches the device: pointers are made up."""
    L = rrm.lib()
    P = 1 << 20  # an aligned address that nothing follows
    big = 1 << 30

    def norm(d=None, x=P, y=P, gamma=None, stats=None, **kw):
        d = d or _norm_desc(**kw)
        return L.rrm_group_norm_act(ctypes.byref(d), x, gamma, None, y, stats, P, big, None)

    assert L.rrm_group_norm_act(None, P, None, None, P, None, P, big, None) == -1
    assert norm(x=None) == -1 and norm(y=None) == -1
    assert norm(groups=3) == -2 and norm(groups=0) == -2 and norm(n=-1) == -2 and norm(c=0) == -2
    assert norm(x_elem=2) == -3 and norm(y_elem=-1) == -3
    assert norm(act=4) == -8 and norm(act=-1) == -8 and norm(eps=0.0) == -8 and norm(eps=math.nan) == -8 and norm(eps=math.inf) == -8
    assert norm(x=P + 2) == -9 and norm(gamma=P + 1) == -9 and norm(stats=P + 2) == -9 and norm(y=P + 1, y_elem=1) == -9
    assert norm(y_position=7) == -2 and norm(y_sample=60) == -2 and norm(y_position=0) == -2 and norm(y_sample=-72) == -2
    assert norm(x_sample=1 << 62) == -2 and norm(x_position=-(1 << 63)) == -2
    assert norm(n=1 << 30, c=8) == -2
    assert norm(n=0) == 0 and norm(positions=0) == 0

    def norm_back(ws=P, have=big, x=P, stats=P, dy=P, dx=P, **kw):
        d = _norm_desc(**kw)
        return L.rrm_group_norm_act_backward(ctypes.byref(d), x, stats, None, None, dy, dx, P, P, ws, have, None)

    need = L.rrm_group_norm_workspace(ctypes.byref(_norm_desc()), 1)
    assert need > 0
    assert norm_back(stats=None) == -1 and norm_back(dy=None) == -1 and norm_back(ws=None) == -1
    assert norm_back(ws=P + 16) == -9 and norm_back(have=need - 1) == -10 and norm_back(dx_position=4) == -2
    assert norm_back(have=need - 1) == -10 and b"workspace" in L.rrm_last_error() and L.rrm_status_string(-10) == b"workspace too small"

    def scan(x=P, f=P, h0=None, y=P, last=None, lengths=None, **kw):
        d = _scan_desc(**kw)
        return L.rrm_gated_scan(ctypes.byref(d), x, f, h0, lengths, y, last, None, P, big, None)

    assert L.rrm_gated_scan(None, P, P, None, None, P, None, None, P, big, None) == -1
    assert scan(x=None) == -1 and scan(f=None) == -1 and scan(y=None) == -1
    assert scan(t=-1) == -2 and scan(n=-1) == -2 and scan(c=-1) == -2 and scan(n=1 << 28, c=1 << 4) == -2 and scan(n=1, t=0x7fffffff, c=1) == -2
    assert scan(elem=2) == -3 and scan(y_frame=7) == -2 and scan(y_video=8) == -2
    assert scan(f=P + 2) == -9 and scan(lengths=P + 2) == -9
    assert scan(h0=P, last=P) == -6
    assert scan(n=0) == 0 and scan(c=0) == 0

    def scan_back(marks=P, dx=P, df=P, **kw):
        d = _scan_desc(**kw)
        return L.rrm_gated_scan_backward(ctypes.byref(d), P, P, marks, None, P, None, dx, df, None, P, big, None)

    assert scan_back(marks=None) == -1 and scan_back(dx=None) == -1 and scan_back(df=None) == -1
    assert scan_back(dx_frame=7) == -2 and scan_back(df_video=9) == -2 and scan_back(dx=P + 1) == -9
    assert [L.rrm_scan_marks(t) for t in (-1, 0, 1, 64, 65)] == [0, 0, 1, 1, 2]

    def ff(x=P, wg=P, h=P, g=None, u=None, **kw):
        d = _ff_desc(**kw)
        return L.rrm_gated_ff(ctypes.byref(d), x, wg, P, h, g, u, P, big, None)

    assert L.rrm_gated_ff(None, P, P, P, P, None, None, P, big, None) == -1
    assert ff(x=None) == -1 and ff(wg=None) == -1 and ff(h=None) == -1 and ff(g=P) == -1 and ff(u=P) == -1
    assert ff(m=-1) == -2 and ff(k=0) == -2 and ff(f=0) == -2 and ff(k=1 << 25) == -2 and ff(h_row=15) == -2
    assert ff(act=7) == -8 and ff(x=P + 1) == -9 and ff(g=P, u=P, gu_row=3) == -2
    assert ff(m=0) == 0

    def ff_back(x=P, g=P, dx=P, dwg=P, dwu=P, have=big, **kw):
        d = _ff_desc(**kw)
        return L.rrm_gated_ff_backward(ctypes.byref(d), x, P, P, g, P, P, dx, dwg, dwu, P, have, None)

    assert ff_back(x=None) == -1 and ff_back(g=None) == -1 and ff_back(dwg=None) == -1 and ff_back(dwu=None) == -1
    assert ff_back(dx_row=7) == -2 and ff_back(dwg_row=4) == -2 and ff_back(have=1) == -10
    assert ff_back(dx=None, dwg=None, dwu=None) == 0


def test_the_binding_refuses_what_the_calls_cannot_take():
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="CUDA"):
        rrm.group_norm_act(x, 2)
    with pytest.raises(ValueError, match="CUDA"):
        rrm.gated_scan(x, x)
    with pytest.raises(ValueError, match="CUDA"):
        rrm.gated_ff(torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="expected \\[n, t, c\\]"):
        rrm.gated_scan(x[0], x[0])


@gpu
def test_the_binding_refuses_wrong_tensors():
    x = torch.zeros(2, 3, 3, 8, device="cuda")
    for bad in (lambda: rrm.group_norm_act(x, 2, act="tanh"), lambda: rrm.group_norm_act(x.half(), 2),
                lambda: rrm.group_norm_act(x, 2, gamma=torch.zeros(7, device="cuda")),
                lambda: rrm.group_norm_act(x, 2, gamma=torch.zeros(8, device="cuda", dtype=torch.bfloat16)),
                lambda: rrm.group_norm_act(x.transpose(2, 3), 2),
                lambda: rrm.group_norm_act(x[:, :, :2], 2),
                lambda: rrm.group_norm_act(x, 2, stats=torch.zeros(2, 4, 2, device="cuda")),
                lambda: rrm.gated_scan(x[0], x[0, :, :, :4]), lambda: rrm.gated_scan(x[0], x[0].bfloat16()),
                lambda: rrm.gated_scan(x[0], x[0], lengths=torch.zeros(3, device="cuda", dtype=torch.int64)),
                lambda: rrm.gated_ff(x[0, 0], x[0, 0], x[0, 0])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RRMError):
        rrm.group_norm_act(x, 3)
    with pytest.raises(RRMError):
        rrm.group_norm_act(x, 2, eps=0.0)
