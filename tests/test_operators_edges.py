"""The operators between and behind the linear layers where their surroundings are odd: other streams, sizes at the ends of the accepted range,
tensors that do not belong, and the kernels' variants that small shapes do not reach.  Tolerances are those of test_operators where nothing else is said."""
import contextlib
import ctypes
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_1802_09723_amd as rrm
from paper_1802_09723_amd import operators as ops
from test_operators import DT, GATE, SUM, U, V, _norm_desc, act64, gen, norm64

gpu = pytest.mark.gpu


# -- streams -------------------------------------------------------------------------------------------------------------------

BF = torch.bfloat16
# a call of each operator on small tensors, and their shapes and type
CALLS = {
    "norm": (lambda t, **kw: rrm.group_norm_act(t[0], 2, **kw), torch.float32, [(2, 3, 8)]),
    "norm_back": (lambda t, **kw: rrm.group_norm_act_backward(*t, **kw), torch.float32, [(2, 3, 8), (2, 3, 8), (2, 2, 2)]),
    "scan": (lambda t, **kw: rrm.gated_scan(*t, **kw), torch.float32, [(2, 70, 8), (2, 70, 8)]),
    "long_scan": (lambda t, **kw: rrm.gated_scan(*t, **kw), torch.float32, [(1, 900, 8), (1, 900, 8)]),
    "scan_back": (lambda t, **kw: rrm.gated_scan_backward(*t, **kw), torch.float32, [(2, 70, 8), (2, 70, 8), (2, 70, 8), (2, 2, 8)]),
    "ff": (lambda t, **kw: rrm.gated_ff(*t, **kw), BF, [(20, 9), (16, 9), (16, 9)]),
    "ff_back": (lambda t, **kw: rrm.gated_ff_backward(*t, **kw), BF, [(20, 16), (20, 8), (16, 8), (16, 8), (20, 16), (20, 16)]),
    "marks": (lambda t, **kw: rrm.gated_scan_marks(t[0], **kw), torch.float32, [(2, 70, 8)]),
}


def several(got):
    return got if isinstance(got, tuple) else (got,)


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream_is_that_streams(name, monkeypatch):
    """Results and workspace come from the pool of the stream that they are used on (a block of the current stream's may still be in use there), and
    results are recorded on the one that was current.  Without a device: the library, the streams and what counts allocations are stand-ins."""
    class Stream:
        cuda_stream = 0x100
        device = torch.device("cuda", 0)

    here, side = Stream(), Stream()
    now, taken, recorded = [here], [], []
    call, dtype, shapes = CALLS[name]
    inputs = [torch.zeros(shape, dtype=dtype) for shape in shapes]

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def counted(make):
        def wrapped(*a, **kw):
            kw.pop("device", None)
            t = make(*a, **kw)
            taken.append((now[-1], t))
            return t
        return wrapped

    class Library:
        def __getattr__(self, name):
            return (lambda *a: 256) if name.endswith("_workspace") else (lambda *a: 0)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append((s, t)))
    monkeypatch.setattr(ops, "lib", Library)
    monkeypatch.setattr(ops, "_expect", lambda *a: None)
    monkeypatch.setattr(ops, "_plans", {})
    monkeypatch.setattr(torch, "empty", counted(torch.empty))
    monkeypatch.setattr(torch, "empty_like", counted(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "new_empty", counted(torch.Tensor.new_empty))
    got = several(call(inputs, stream=side))
    assert taken and all(s is side for s, _ in taken)
    for t in got:
        assert any(r is t and s is here for s, r in recorded)


@gpu
@pytest.mark.parametrize("name", [n for n in CALLS if n != "marks"])
def test_a_call_on_another_stream_beside_one_that_uses_freed_memory(name):
    """A block that was freed while the current stream still writes it is not handed to a call on another stream."""
    call, dtype, shapes = CALLS[name]
    inputs = [torch.randn(shape, generator=gen(i)).to(dtype).cuda() for i, shape in enumerate(shapes)]
    want = [t.clone() for t in several(call(inputs))]
    side = torch.cuda.Stream()
    slow = torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        slow.add_(1.0)
    # blocks of the sizes that a call may ask for, written behind the slow work and freed before it is done
    blocks = [torch.empty(256 << k, device="cuda", dtype=torch.uint8) for k in range(12) for _ in range(8)]
    for b in blocks:
        b.fill_(77)
    del blocks, b
    got = several(call(inputs, stream=side))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_a_captured_call_on_another_stream():
    """A stream that joins a capture, and its results back on the first one: replays give what eager calls do."""
    x, f = (torch.randn(2, 700, 24, generator=gen(i)).cuda() for i in range(2))
    side = torch.cuda.Stream()

    def both():
        here = torch.cuda.current_stream()
        a = rrm.group_norm_act(x, 4, act="silu")
        side.wait_stream(here)
        y, last = rrm.gated_scan(a, f, stream=side)
        here.wait_stream(side)
        return rrm.group_norm_act(y, 4), last

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for k in range(4):
        x.copy_(torch.randn(2, 700, 24, generator=gen(k + 5)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


# -- sizes at the ends of the range ----------------------------------------------------------------------------------------------

def norm_parts64(x, groups, eps=1e-5):
    """(xh, mean, r) of a map [n, positions, c] in 64 bits, where it lies"""
    n, p, c = x.shape
    v = x.double().view(n, p, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt(((v - mean) ** 2).mean((1, 3), keepdim=True) + eps)
    return ((v - mean) * r).view(n, p, c), mean, r


def close(got, want, slack, what):
    err = (got.double() - want).abs() - slack
    assert err.max() <= 0, f"{what}: {int((err > 0).sum())} off, by {float(err.max()):.3g} more than allowed"


@gpu
@pytest.mark.parametrize("n,c,groups", [(2, 1 << 24, 1), (1, 9000000, 1000), (1, 10000001, 1), (1, (1 << 23) + 3, 1)])
def test_norm_of_very_many_channels(n, c, groups):
    """Groups of which every one has a mean and a deviation of its own, so that another one's would show: a channel's group counts in
    integers where 32-bit floats no longer tell neighbouring channels apart."""
    cg = c // groups
    g = torch.Generator(device="cuda").manual_seed(c)
    own = torch.arange(n * groups, device="cuda").view(n, 1, groups, 1)
    x = torch.empty(n, 1, c, device="cuda").normal_(generator=g)
    x = (x.view(n, 1, groups, cg) * (1 + own % 3) + (own % 5)).view(n, 1, c)
    xh, mean, r = norm_parts64(x, groups)
    stats = torch.empty(n, groups, 2, device="cuda")
    y = rrm.group_norm_act(x, groups, stats=stats)
    # a thread sums its share of the group, some cg / 512 terms, one behind the other: their roundings at random signs, eight deviations
    s = (8 * math.sqrt(cg / 512) + 32) * U
    top = float(x.abs().max()) * float(r.max())
    slack = s * (top + 1) + GATE
    close(stats[..., 0], mean.view(n, groups), s * float(x.abs().max()), "mean")
    close(stats[..., 1], r.view(n, groups), s * (1 + top) * r.view(n, groups), "r")
    close(y, xh, slack, "y")
    # with a mean and a part along xh, so that every term of the gradient counts
    dy = (0.5 + 0.7 * xh + torch.empty(n, 1, c, device="cuda").normal_(generator=g)).float()
    dx, dgamma, dbeta = rrm.group_norm_act_backward(dy, x, stats)
    v, h = dy.double().view(n, 1, groups, cg), xh.view(n, 1, groups, cg)
    p, q = v.mean((1, 3), keepdim=True), (v * h).mean((1, 3), keepdim=True)
    want = (r * (v - p - h * q)).view(n, 1, c)
    rr = r.expand(n, 1, groups, cg).reshape(n, 1, c)
    close(dx, want, rr * 4 * (s + slack) * (dy.double().abs() + 1 + 2 * xh.abs() * (1 + xh.abs())), "dx")
    close(dbeta, dy.double().sum((0, 1)), 4 * U * dy.double().abs().sum((0, 1)), "dbeta")
    close(dgamma, (dy.double() * xh).sum((0, 1)), ((slack + 4 * U * (1 + xh.abs())) * dy.double().abs()).sum((0, 1)), "dgamma")


# n, positions, c, groups at the ends of what a descriptor may say
FAR_NORM = [
    (1, 1, 0x7ffff000, 1), (1, 1, (1 << 30) + 8, 1), (1, 100, 1 << 30, 2), (1, 3, 1 << 30, 1 << 26), (1, 0x7ffff000, 1, 1), (1, 0x7ffff000, 64, 1),
    (0x7ffff000, 1, 1, 1), (0x7ffff000, 40000, 1, 1), (3, 0x7fffe000, 8, 8), (2, 0x7fffe000, 24, 4), (1, 1, 0x7ffff000, 0x7ffff000),
]


def test_norm_plans_of_the_largest_sizes():
    """The host's choice of a layout ends, and the bytes it asks for hold what the kernels keep there.  In a process of its own: it used not to end."""
    code = """
import ctypes, sys
sys.path.insert(0, sys.argv[1])
import paper_1802_09723_amd as rrm
from paper_1802_09723_amd.operators import NormDesc
for n, p, c, g in eval(sys.argv[2]):
    for x in (0, 1):
        for back in (0, 1):
            d = NormDesc(n, p, c, g, x, 0, 0, 1e-5, 0, c, 0, c, 0, c)
            print(rrm.lib().rrm_group_norm_workspace(ctypes.byref(d), back))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code, root, repr(FAR_NORM)], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr
    sizes = iter(int(v) for v in done.stdout.split())
    for n, p, c, groups in FAR_NORM:
        for x in (0, 1):
            # a value a channel and sample where samples are held, two a channel of a slice beside the groups' where not: at most about
            # 1024 slices and one for each sample and set of channels
            forward, backward = next(sizes), next(sizes)
            least, most = 8 * n * c, 8 * n * c + 8 * 1024 * 2048 * 8
            assert forward == 0 or least <= forward <= 3 * most, (n, p, c, groups, x, forward)
            assert least <= backward <= 4 * most, (n, p, c, groups, x, backward)


def test_norm_refuses_sizes_beyond_the_range():
    L = rrm.lib()
    P = 1 << 20
    for kw in (dict(n=1, positions=1, c=0x7ffff001, groups=1), dict(n=1, positions=0x7ffff001, c=1, groups=1), dict(n=0x7fffffff, positions=1, c=1, groups=1)):
        d = _norm_desc(**kw)
        assert L.rrm_group_norm_act(ctypes.byref(d), P, None, None, P, None, P, 1 << 40, None) == -2
        assert L.rrm_group_norm_act_backward(ctypes.byref(d), P, P, None, None, P, P, P, P, P, 1 << 40, None) == -2


@gpu
@pytest.mark.parametrize("positions", [0x7ffff000, (1 << 30) + 77])
def test_norm_of_very_many_positions(positions):
    """One channel, as many positions as a call takes: the last slices end where the map does, both ways."""
    x = torch.empty(1, positions, 1, device="cuda", dtype=BF).normal_(3.0, 2.0, generator=torch.Generator(device="cuda").manual_seed(5))
    parts = [slice(k, min(k + (1 << 27), positions)) for k in range(0, positions, 1 << 27)]
    flat = x.view(-1)
    mean = sum(float(flat[p].double().sum()) for p in parts) / positions
    r = (sum(float(((flat[p].double() - mean) ** 2).sum()) for p in parts) / positions + 1e-5) ** -0.5
    stats = torch.empty(1, 1, 2, device="cuda")
    y = rrm.group_norm_act(x, 1, stats=stats).view(-1)
    # a thread sums some 8192 positions of a slice one behind the other
    s = (8 * math.sqrt(positions / 1024 / 256) + 32) * U
    top = float(x.abs().max())
    assert abs(float(stats[0, 0, 0]) - mean) <= s * top and abs(float(stats[0, 0, 1]) - r) <= s * r * (1 + top * r)
    slack = s * (top * r + 1)
    for p in parts:
        want = (flat[p].double() - mean) * r
        close(y[p], want, slack + V * (want.abs() + slack), "y")
    # dy = 0.5 y + 1: <dy> = 1 and <dy xh> = 0.5 but for roundings, so dx is r times what these leave
    dy = y.mul_(0.5).add_(1).view(1, positions, 1)
    dx, dgamma, dbeta = rrm.group_norm_act_backward(dy, x, stats)
    d = dy.view(-1)
    p1 = sum(float(d[p].double().sum()) for p in parts)
    q1 = sum(float((d[p].double() * ((flat[p].double() - mean) * r)).sum()) for p in parts)
    most = 1 + 0.5 * top * r
    assert abs(float(dbeta) - p1) <= s * most * positions and abs(float(dgamma) - q1) <= (s * (1 + top * r) + slack) * most * positions
    for p in parts:
        xh = (flat[p].double() - mean) * r
        want = r * (d[p].double() - p1 / positions - xh * q1 / positions)
        off = r * 4 * (s + slack) * (1 + xh.abs()) ** 2 * most
        close(dx.view(-1)[p], want, off + V * (want.abs() + off), "dx")


@gpu
@pytest.mark.parametrize("t", [1, 17])
def test_scan_of_very_many_videos(t):
    """More videos than one launch has workgroups for (2^32 threads along an axis)."""
    n = (1 << 26) + 5 if t == 1 else (1 << 24) + 5
    g = torch.Generator(device="cuda").manual_seed(t)
    x, f = (torch.empty(n, t, 1, device="cuda", dtype=BF).normal_(generator=g) for _ in range(2))
    h0 = torch.empty(n, 1, device="cuda").normal_(generator=g)
    marks = rrm.gated_scan_marks(x)
    y, last = rrm.gated_scan(x, f, h0, marks=marks)
    slack = 8 * (SUM + GATE) * 2  # (values below 8)
    h = h0[:, 0].double()
    for k in range(t):
        a = torch.sigmoid(f[:, k, 0].double())
        h = a * h + (1 - a) * x[:, k, 0].double()
        close(y[:, k, 0], h, slack + V * (h.abs() + slack), "y")
    close(last[:, 0], h, slack, "h_last")
    dx, df, dh0 = rrm.gated_scan_backward(y, x, f, marks)
    before = [h0[:, 0].double()]  # the states again, for the gradients
    for k in range(t - 1):
        a = torch.sigmoid(f[:, k, 0].double())
        before.append(a * before[-1] + (1 - a) * x[:, k, 0].double())
    carry = torch.zeros_like(h)
    gs = slack * t
    for k in reversed(range(t)):
        a, v, grad = torch.sigmoid(f[:, k, 0].double()), x[:, k, 0].double(), y[:, k, 0].double() + carry
        want = (1 - a) * grad
        close(dx[:, k, 0], want, gs + V * (want.abs() + gs), "dx")
        want = grad * (before[k] - v) * a * (1 - a)
        close(df[:, k, 0], want, 16 * gs + V * (want.abs() + 16 * gs), "df")
        carry = a * grad
    close(dh0[:, 0], carry, gs, "dh0")


@gpu
@pytest.mark.parametrize("n,c,groups", [((1 << 24) + 9, 2, 1), (2, (1 << 27) + 64, ((1 << 27) + 64) // 16)])
def test_norm_of_very_many_samples_or_groups(n, c, groups):
    """More samples, or channels of a sample, than one launch has workgroups for."""
    cg = c // groups
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.empty(n, 1, c, device="cuda", dtype=BF).normal_(1.0, generator=g)
    dy = torch.empty(n, 1, c, device="cuda", dtype=BF).normal_(0.5, generator=g)
    stats = torch.empty(n, groups, 2, device="cuda")
    # (two values next to one another have a large r: an eps that holds it to 30)
    eps = 1e-3
    y = rrm.group_norm_act(x, groups, eps=eps, stats=stats)
    dx, dgamma, dbeta = rrm.group_norm_act_backward(dy, x, stats)
    s1, s2, m2 = (torch.zeros(c, device="cuda", dtype=torch.float64) for _ in range(3))
    flat = [t.view(n, groups, cg) for t in (x, dy, y, dx)]
    step = max(1, (1 << 25) // (n * cg)) if n < 100 else groups
    for k in range(0, groups, step):
        v, d, gy, gdx = (t[:, k:k + step].double() for t in flat)
        mean = v.mean(2, keepdim=True)
        r = 1 / torch.sqrt(((v - mean) ** 2).mean(2, keepdim=True) + eps)
        xh = (v - mean) * r
        slack = SUM * (8 * r + 1) + GATE
        close(gy, xh, slack + V * (xh.abs() + slack), "y")
        want = r * (d - d.mean(2, keepdim=True) - xh * (d * xh).mean(2, keepdim=True))
        off = r * 4 * (SUM + slack) * (1 + xh.abs()) ** 2 * (1 + d.abs().amax(2, keepdim=True))
        close(gdx, want, off + V * (want.abs() + off), "dx")
        at = slice(k * cg, (k + v.shape[1]) * cg)
        s1[at], s2[at] = d.sum(0).view(-1), (d * xh).sum(0).view(-1)
        m2[at] = (d.abs() * (SUM * (1 + xh.abs()) + slack)).sum(0).view(-1)
    close(dbeta, s1, m2, "dbeta")
    # 32 threads sum the samples of a channel one behind the other
    close(dgamma, s2, m2 * (1 + math.sqrt(n / 32)), "dgamma")


# -- values ------------------------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("ty", [torch.float32, BF])
@pytest.mark.parametrize("shape", [(1, 8, 8, 32, 4), (2, 16, 16, 64, 8), (3, 64, 64, 16, 2), (1, 256, 256, 32, 2)])
def test_norm_of_constant_groups_is_beta(shape, ty):
    """Groups of one value each, whose sums (of powers of two of them) are exact: z is beta, to the bit, for a small eps too.  Its own shift and scale
    folded into one multiply-add would leave the rounding of mean / sqrt(eps)."""
    n, h, w, c, groups = shape
    beta = torch.tensor([0.1, 0.5, 0.25, -0.7], device="cuda").repeat(c // 4)
    gamma = torch.linspace(0.5, 2.0, c, device="cuda")
    for value in (1.0, 100.0, 1000.0, -3.0):
        for eps in (1e-5, 1e-12, 1e-30):
            x = torch.full((n, h, w, c), value, device="cuda", dtype=ty)
            y = rrm.group_norm_act(x, groups, gamma, beta, eps=eps, out_dtype=torch.float32)
            assert torch.equal(y, beta.expand_as(y)), (value, eps, float((y - beta).abs().max()))


# -- tensors that do not belong ------------------------------------------------------------------------------------------------------

class Device(torch.Tensor):
    """A tensor that says it is on a device"""
    at = torch.device("cuda", 0)
    is_cuda = True

    @property
    def device(self):
        return self.at


class OtherDevice(Device):
    at = torch.device("cuda", 1)


@pytest.fixture
def without_a_device(monkeypatch):
    """Calls end at a library that does nothing; tensors are CPU ones that say otherwise."""
    class Library:
        def __getattr__(self, name):
            return (lambda *a: 0)

    class Stream:
        cuda_stream = 0x100
        device = torch.device("cuda", 0)

    monkeypatch.setattr(ops, "lib", Library)
    monkeypatch.setattr(ops, "_plans", {})
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)


def inputs_of(name, kind=Device):
    call, dtype, shapes = CALLS[name]
    return call, [torch.zeros(shape, dtype=dtype).as_subclass(kind) for shape in shapes]


@pytest.mark.parametrize("name", [n for n in CALLS if n != "marks"])
def test_gradients_are_not_lost_in_silence(name, without_a_device):
    """Every input that requires a gradient is refused where autograd records, also when the same call has been made without."""
    call, inputs = inputs_of(name)
    call(inputs)
    for t in inputs:
        t.requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            call(inputs)
        with torch.no_grad():
            call(inputs)
        with pytest.raises(ValueError, match="no_grad"):
            call(inputs)
        t.requires_grad_(False)
    call(inputs)


def test_gradients_of_the_parameters_are_not_lost_in_silence(without_a_device):
    call, (x,) = inputs_of("norm")
    gamma, beta = (torch.zeros(8, requires_grad=True).as_subclass(Device) for _ in range(2))
    for kw in (dict(gamma=gamma), dict(beta=beta)):
        with pytest.raises(ValueError, match="requires a gradient"):
            rrm.group_norm_act(x, 2, **kw)
        with torch.no_grad():
            rrm.group_norm_act(x, 2, **kw)


@pytest.mark.parametrize("name", [n for n in CALLS if n != "marks"])
def test_tensors_of_several_devices_are_refused(name, without_a_device):
    call, inputs = inputs_of(name)
    call(inputs)
    for k in range(1, len(inputs)):
        mixed = [t.as_subclass(OtherDevice) if i == k else t for i, t in enumerate(inputs)]
        with pytest.raises(ValueError, match="several devices"):
            call(mixed)


@pytest.mark.parametrize("name", [n for n in CALLS if n != "marks"])
def test_tensors_of_another_device_than_the_current_one_are_refused(name, without_a_device, monkeypatch):
    """The launch would go to the current device: also when the same call was right before."""
    call, inputs = inputs_of(name)
    current = [0]
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x100, raising=False)
    call(inputs)
    current[0] = 1
    with pytest.raises(ValueError, match="current device is 1"):
        call(inputs)
    current[0] = 0
    call(inputs)


# -- the package -----------------------------------------------------------------------------------------------------------------------

def test_the_package_is_imported_without_torch():
    """Building the library, and layers' shapes and names, need none of it; the operators bring it when they are asked for."""
    code = """
import sys
sys.path.insert(0, sys.argv[1])
import paper_1802_09723_amd as rrm
import paper_1802_09723_amd.build
assert "torch" not in sys.modules
assert {"gated_ff", "gated_scan_marks", "group_norm_act_of"} <= set(dir(rrm))
try:
    rrm.nothing
except AttributeError:
    pass
from paper_1802_09723_amd import gated_scan, operators
assert rrm.gated_scan is gated_scan is operators.gated_scan and "torch" in sys.modules
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code, root], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr


# -- the feed-forward block's tiles ------------------------------------------------------------------------------------------------------

def ff_layout(m, k, f, asked):
    d = ops.FFDesc(m, k, f, 2, k, k, k, f, f, k, k, k, 0)
    layout = (ctypes.c_int * 5)()
    assert rrm.lib().rrm_aux_ff_layout(ctypes.byref(d), asked, layout) == 0
    return list(layout)


# Shapes of every kind of tile, over more than four steps of 64 of the summed axis and by parts of it or not, ragged everywhere; rows of k that are copied
# and padded (odd k), and rows that are read where they lie
FF_FORWARD = {
    (0, False): [(4807, 305, 853), (2773, 304, 1529)], (0, True): [(4327, 4919, 67), (4123, 4072, 69)],
    (1, False): [(193, 321, 4075), (261, 320, 3491)], (1, True): [(17, 1995, 1479), (17, 1280, 2647)],
    (2, False): [(4709, 349, 385), (1095, 312, 1803)], (2, True): [(2109, 4757, 17), (4299, 2328, 23)],
    (3, False): [(19, 321, 17), (19, 312, 17)], (3, True): [(17, 1081, 19), (19, 1048, 19)],
}
FF_DX = {
    (0, False): [(3451, 2559, 301), (3535, 2576, 329)], (0, True): [(2243, 137, 3841), (4463, 168, 2463)],
    (1, False): [(451, 4225, 311), (4747, 400, 305)], (1, True): [(4197, 17, 465), (2085, 24, 979)],
    (2, False): [(4733, 839, 303), (965, 4288, 301)], (2, True): [(2049, 17, 2021), (4315, 24, 1001)],
    (3, False): [(19, 17, 305), (23, 24, 305)], (3, True): [(17, 17, 469), (17, 24, 525)],
}
FF_DW = {
    (0, False): [(311, 2179, 1801), (325, 2184, 1803)], (0, True): [(3523, 131, 4769), (4985, 136, 2971)],
    (1, False): [(313, 129, 4505), (313, 144, 4749)], (1, True): [(4197, 17, 465), (2085, 24, 979)],
    (2, False): [(319, 439, 4181), (309, 408, 4743)], (2, True): [(4863, 17, 1057), (2413, 24, 2211)],
    (3, False): [(315, 17, 19), (343, 24, 17)], (3, True): [(969, 19, 17), (997, 24, 19)],
}
# one launch for dX and both dW: (tile, dX by parts, dW by parts)
FF_BOTH = {
    (0, False, False): (905, 4413, 469), (0, False, True): (3373, 1241, 139), (0, True, False): (129, 1305, 2557), (0, True, True): (4969, 139, 1091),
    (1, False, False): (17, 3995, 401), (1, False, True): (4087, 161, 119), (1, True, False): (17, 1349, 1003), (1, True, True): (1059, 17, 1075),
    (2, False, False): (391, 4763, 197), (2, False, True): (4605, 607, 69), (2, True, False): (71, 1243, 2063), (2, True, True): (1127, 17, 2201),
    (3, False, False): (17, 19, 17), (3, False, True): (1001, 17, 17), (3, True, False): (19, 17, 449), (3, True, True): (987, 17, 243),
}
# a launch each: (tile of dX, of dW)
FF_APART = {
    (0, 1): (4299, 3749, 65), (0, 2): (4289, 3597, 147), (0, 3): (3307, 4667, 129), (1, 0): (215, 1851, 3891), (1, 1): (289, 2685, 3677),
    (1, 2): (621, 1453, 2671), (1, 3): (2863, 1405, 1437), (2, 0): (271, 4327, 3031), (2, 1): (1541, 4863, 273), (2, 2): (579, 2649, 3039),
    (2, 3): (4879, 1589, 547), (3, 0): (265, 1467, 4367), (3, 2): (315, 3155, 2437),
}


def ff_case(m, k, f):
    g = torch.Generator(device="cuda").manual_seed(m + 3 * k + 7 * f)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda").normal_(0.0, scale, generator=g).bfloat16()

    return normal(m, k), normal(f, k, scale=k ** -0.5), normal(f, k, scale=k ** -0.5), normal(m, f)


def rounded(slack, want):
    """slack, and the rounding to bfloat16"""
    return slack + V * (want.abs() + slack)


def ff_forward_close(x, wg, wu, act, h, g, u):
    """as test_operators' ff_check, on the device"""
    x64, wg64, wu64 = x.double(), wg.double(), wu.double()
    g64, u64 = x64 @ wg64.t(), x64 @ wu64.t()
    sg, su = SUM * (x64.abs() @ wg64.abs().t()), SUM * (x64.abs() @ wu64.abs().t())
    close(g, g64, rounded(sg, g64), "g")
    close(u, u64, rounded(su, u64), "u")
    a64 = act64(act, g64)
    close(h, a64 * u64, rounded((1.2 * sg + GATE * (1 + g64.abs())) * (u64.abs() + su) + a64.abs() * su, a64 * u64), "h")


def ff_backward_close(x, wg, wu, dh, g, u, act, dx=None, dw=None):
    g64 = g.double().requires_grad_()
    p = act64(act, g64)
    slope = torch.autograd.grad(p.sum(), g64)[0]
    p, u64, d64 = p.detach(), u.double(), dh.double()
    dg, du = d64 * u64 * slope, d64 * p
    # dG and dU are rounded before the products: V of each term, at random signs; eight deviations of such a sum
    eg, eu = dg.abs() * (V + GATE) + GATE * (d64 * u64).abs(), du.abs() * (V + GATE) + GATE * d64.abs()

    def off(e, w):
        return SUM * (e / V).matmul(w.abs()) + 8 * torch.sqrt((e * e).matmul(w * w)) + GATE * e.matmul(w.abs())

    x64, wg64, wu64 = x.double(), wg.double(), wu.double()
    if dx is not None:
        want = dg @ wg64 + du @ wu64
        close(dx, want, rounded(off(eg, wg64) + off(eu, wu64), want), "dx")
    if dw is not None:
        for got, d, e, what in ((dw[0], dg, eg, "dwg"), (dw[1], du, eu, "dwu")):
            want = d.t() @ x64
            close(got, want, rounded(off(e.t(), x64), want), what)


def ff_saved(x, wg, wu):
    """projections for a backward pass by itself"""
    return (x.float() @ wg.float().t()).bfloat16(), (x.float() @ wu.float().t()).bfloat16()


def ff_gradients(x, wg, wu, g, u, dh, act, dx, dwg, dwu):
    """The C call: the gradients that are not given are not asked for."""
    (m, k), f = x.shape, wg.shape[0]
    d = ops.FFDesc(m, k, f, ops.ACTS[act], k, k, k, f, f, k, k, k, 0)
    need = rrm.lib().rrm_gated_ff_workspace(ctypes.byref(d), 1)
    ws = torch.empty(need, device="cuda", dtype=torch.uint8)
    at = [t if t is None else t.data_ptr() for t in (x, wg, wu, g, u, dh, dx, dwg, dwu)]
    assert rrm.lib().rrm_gated_ff_backward(ctypes.byref(d), *at, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0


def act_of(m, k, f):
    return ("silu", "gelu")[(m + k + f) // 2 % 2]


@gpu
@pytest.mark.parametrize("tile,split,shape", [(*q, s) for q, v in FF_FORWARD.items() for s in v])
def test_ff_forward_of_every_tile(tile, split, shape):
    layout = ff_layout(*shape, 0)
    assert layout[0] == tile and (layout[1] > 1) == split, layout
    x, wg, wu, _ = ff_case(*shape)
    m, k, f = shape
    act = act_of(*shape)
    g, u = torch.empty(m, f, device="cuda", dtype=BF), torch.empty(m, f, device="cuda", dtype=BF)
    h = rrm.gated_ff(x, wg, wu, act, save=(g, u))
    ff_forward_close(x, wg, wu, act, h, g, u)
    assert torch.equal(rrm.gated_ff(x, wg, wu, act), h)
    # not-a-numbers and infinities stay in their row and feature, also in the last ones
    x[m - 1, k - 1], x[1, k // 2], wg[f - 1, k - 1], wu[f // 2, 0] = math.nan, math.inf, math.nan, math.inf
    spoilt = rrm.gated_ff(x, wg, wu, "none")
    x[m - 1, k - 1], x[1, k // 2], wg[f - 1, k - 1], wu[f // 2, 0] = 0, 0, 0, 0
    clean = rrm.gated_ff(x, wg, wu, "none")
    assert not torch.isfinite(spoilt[[1, m - 1]]).any() and not torch.isfinite(spoilt[:, f // 2]).any()
    for t in (spoilt, clean):
        t[[1, m - 1]] = 0
        t[:, [f // 2, f - 1]] = 0
    # (elsewhere the zeros put in their places count for nothing: those rows and features were not the others')
    assert torch.equal(spoilt, clean)


@gpu
@pytest.mark.parametrize("tile,split,shape", [(*q, s) for q, v in FF_DX.items() for s in v])
def test_ff_input_gradient_of_every_tile(tile, split, shape):
    layout = ff_layout(*shape, 1)
    assert layout[0] == tile and (layout[1] > 1) == split, layout
    x, wg, wu, dh = ff_case(*shape)
    g, u = ff_saved(x, wg, wu)
    dx = torch.full_like(x, 7.0)
    ff_gradients(x, wg, wu, g, u, dh, act_of(*shape), dx, None, None)
    ff_backward_close(x, wg, wu, dh, g, u, act_of(*shape), dx=dx)


@gpu
@pytest.mark.parametrize("tile,split,shape", [(*q, s) for q, v in FF_DW.items() for s in v])
def test_ff_weights_gradients_of_every_tile(tile, split, shape):
    layout = ff_layout(*shape, 2)
    assert layout[2] == tile and (layout[3] > 1) == split, layout
    x, wg, wu, dh = ff_case(*shape)
    g, u = ff_saved(x, wg, wu)
    dw = torch.full_like(wg, 7.0), torch.full_like(wu, 7.0)
    ff_gradients(x, wg, wu, g, u, dh, act_of(*shape), None, *dw)
    ff_backward_close(x, wg, wu, dh, g, u, act_of(*shape), dw=dw)


@gpu
@pytest.mark.parametrize("form", [*FF_BOTH, *FF_APART], ids=str)
def test_ff_gradients_together_and_apart(form):
    shape = FF_BOTH[form] if form in FF_BOTH else FF_APART[form]
    layout = ff_layout(*shape, 3)
    if form in FF_BOTH:
        assert layout[4] == 1 and (layout[0], layout[1] > 1, layout[3] > 1) == form, layout
    else:
        assert layout[4] == 0 and (layout[0], layout[2]) == form, layout
    x, wg, wu, dh = ff_case(*shape)
    g, u = ff_saved(x, wg, wu)
    act = act_of(*shape)
    got = rrm.gated_ff_backward(dh, x, wg, wu, g, u, act)
    ff_backward_close(x, wg, wu, dh, g, u, act, got[0], got[1:])
    assert all(torch.equal(a, b) for a, b in zip(got, rrm.gated_ff_backward(dh, x, wg, wu, g, u, act)))


# -- the norm's forms --------------------------------------------------------------------------------------------------------------------

def norm_layout(n, positions, c, groups, x_elem, backward):
    d = ops.NormDesc(n, positions, c, groups, x_elem, 0, 0, 1e-5, positions * c, c, positions * c, c, positions * c, c)
    layout = (ctypes.c_int * 2)()
    assert rrm.lib().rrm_aux_norm_layout(ctypes.byref(d), backward, layout) == 0
    return layout[0], layout[1]


# n, positions, c, groups: forms (the size of workgroup and its channels; -1: in slices) of fp32 forward and backward, of bf16 forward and backward
NORM_FORMS = {
    # each size of workgroup; runs of channels as narrow as they get, and widened where there are workgroups enough
    (5000, 1, 9, 3): ((0, 9), (0, 9), (0, 9), (0, 9)), (3000, 1, 64, 4): ((0, 64), (0, 64), (0, 64), (0, 64)),
    (1024, 7, 105, 7): ((0, 120), (0, 120), (0, 105), (0, 105)), (1100, 30, 24, 3): ((0, 32), (0, 32), (0, 24), (0, 24)),
    (600, 10, 64, 8): ((0, 32), (0, 32), (0, 32), (0, 32)), (520, 63, 250, 25): ((1, 40), (1, 40), (1, 80), (1, 80)),
    (64, 784, 128, 32): ((2, 16), (2, 16), (2, 32), (2, 32)), (129, 1001, 13, 13): ((2, 9), (2, 9), (2, 12), (2, 12)),
    (8, 196, 512, 8): ((2, 64), (2, 64), (2, 64), (2, 64)), (300, 4000, 8, 1): ((3, 8), (3, 8), (2, 8), (2, 8)),
    (64, 3136, 64, 32): ((3, 16), (3, 8), (3, 16), (3, 16)), (140, 2000, 40, 5): ((3, 16), (3, 16), (3, 32), (3, 32)),
    (130, 3000, 40, 8): ((3, 15), (3, 5), (3, 30), (3, 15)), (256, 3000, 35, 5): ((3, 14), (3, 7), (3, 28), (3, 14)),
    (130, 900, 17, 1): ((3, 17), (3, 17), (2, 17), (2, 17)), (300, 1, 8192, 1): ((-1, 1), (-1, 1), (3, 8192), (3, 8192)),
    # slices: long samples, few workgroups, groups wider than a workgroup
    (1, 22650, 36, 6): ((-1, 354), (-1, 354), (-1, 177), (-1, 177)), (1, 60000, 16, 2): ((-1, 235), (-1, 235), (-1, 118), (-1, 118)),
    (1, 70000, 3, 1): ((-1, 274), (-1, 274), (-1, 274), (-1, 274)), (2, 3000, 1030, 10): ((-1, 250), (-1, 250), (-1, 500), (-1, 500)),
    (1, 40, 9000, 3): ((-1, 10), (-1, 10), (-1, 10), (-1, 10)),
}


@gpu
@pytest.mark.parametrize("types", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")], ids="-".join)
@pytest.mark.parametrize("shape", NORM_FORMS, ids=str)
def test_norm_of_every_form(shape, types):
    """Element by element, with gradients in which the group's two means count as much as dz itself: dy has a mean and a part along xh."""
    n, positions, c, groups = shape
    e = types[0] == "bf16"
    assert (norm_layout(*shape, int(e), 0), norm_layout(*shape, int(e), 1)) == NORM_FORMS[shape][2 * e:2 * e + 2]
    cg, act = c // groups, ("silu", "none", "gelu", "relu")[(positions + groups) % 4]
    gn = torch.Generator(device="cuda").manual_seed(n + c)

    def normal(*s, shift=0.0, scale=1.0):
        return torch.empty(s, device="cuda").normal_(shift, scale, generator=gn)

    def grouped(t):
        return t.view(n, positions, groups, cg)

    def mean(t):
        return grouped(t).mean((1, 3), keepdim=True).expand(n, positions, groups, cg).reshape(n, positions, c)

    x = (normal(n, positions, c, scale=1.5) + normal(n, 1, c)).to(DT[types[0]])
    gamma, beta = normal(c, shift=1.0, scale=0.2), normal(c, scale=0.3)
    # the definition, its eps such that a group of few values has no r above 30
    eps = 1e-3
    v = x.double()
    mu = mean(v)
    r = 1 / torch.sqrt(mean((v - mu) ** 2) + eps)
    xh = (v - mu) * r
    z = (xh * gamma.double() + beta.double()).requires_grad_()
    y64 = act64(act, z)
    slope = torch.autograd.grad(y64.sum(), z)[0]
    y64, z = y64.detach(), z.detach()
    # what xh and z may be off by: sums in trees, the mean's own rounding times r
    top = grouped(v).abs().amax((1, 3), keepdim=True).expand(n, positions, groups, cg).reshape(n, positions, c)
    e_xh = SUM * (r * top + xh.abs())
    e_z = gamma.double().abs() * e_xh + 4 * U * (z.abs() + beta.double().abs())
    stats = torch.empty(n, groups, 2, device="cuda")
    y = rrm.group_norm_act(x, groups, gamma, beta, act, eps=eps, out_dtype=DT[types[1]], stats=stats)

    def whole(slack, want, got):
        return slack + (V if got.dtype is BF else U) * (want.abs() + slack)

    close(y, y64, whole(1.2 * e_z + GATE * (1 + z.abs()), y64, y), "y")
    dy = (0.5 + 0.7 * xh + normal(n, positions, c)).to(DT[types[1]])
    if act == "relu":  # where the sign of z may fall either way no gradient comes in
        dy[z.abs() <= 4 * e_z] = 0
    d = dy.double()
    dz = d * slope
    e_dz = d.abs() * (1.2 * e_z + GATE)
    ga = gamma.double()
    p, q = mean(ga * dz), mean(ga * dz * xh)
    e_p = mean(ga.abs() * e_dz) + SUM * mean((ga * dz).abs())
    e_q = mean(ga.abs() * (e_dz * xh.abs() + dz.abs() * e_xh)) + SUM * mean((ga * dz * xh).abs())
    want = r * (ga * dz - p - xh * q)
    off = r * (ga.abs() * e_dz + e_p + xh.abs() * e_q + q.abs() * e_xh + 8 * U * ((ga * dz).abs() + p.abs() + (xh * q).abs())) + SUM * want.abs()
    dx, dgamma, dbeta = rrm.group_norm_act_backward(dy, x, stats, gamma, beta, act)
    close(dx, want, whole(off, want, dx), "dx")
    if act != "relu" and n * positions * c > 1000 and cg * positions > 8:
        # (the bound is one that a gradient without either mean does not keep)
        assert ((r * p).abs() > whole(off, want, dx)).any() and ((r * xh * q).abs() > whole(off, want, dx)).any()
    close(dbeta, dz.sum((0, 1)), (e_dz + SUM * dz.abs()).sum((0, 1)), "dbeta")
    close(dgamma, (dz * xh).sum((0, 1)), (e_dz * xh.abs() + dz.abs() * e_xh + SUM * (dz * xh).abs()).sum((0, 1)), "dgamma")
    again = rrm.group_norm_act_backward(dy, x, stats, gamma, beta, act)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))


@gpu
@pytest.mark.parametrize("shape", [(1, 9000, 12, 3), (2, 400, 40, 4)])
def test_gradients_in_slices_and_in_large_workgroups_against_differences(shape):
    """The derivative along random directions against the difference quotient of the definition in 64 bits."""
    n, positions, c, groups = shape
    assert n == 2 or norm_layout(*shape, 0, 1)[0] == -1
    g = gen(n)
    args = [torch.randn(n, positions, c, generator=g), 1 + 0.1 * torch.randn(c, generator=g), torch.randn(c, generator=g)]
    dy = 0.5 + torch.randn(n, positions, c, generator=g)
    stats = torch.empty(n, groups, 2, device="cuda")
    dev = [a.cuda() for a in args]
    rrm.group_norm_act(dev[0], groups, dev[1], dev[2], "silu", stats=stats)
    grads = rrm.group_norm_act_backward(dy.cuda(), dev[0], stats, dev[1], dev[2], "silu")

    def loss(v):
        return float((norm64(v[0], groups, v[1], v[2], "silu")[0] * dy.double()).sum())

    step = 1e-5
    for k in range(3):
        d = torch.randn(args[k].shape, generator=g).double()
        lo, hi = [a.double() for a in args], [a.double() for a in args]
        lo[k], hi[k] = lo[k] - step * d, hi[k] + step * d
        quotient = (loss(hi) - loss(lo)) / (2 * step)
        got = float((grads[k].cpu().double() * d).sum())
        # step^2 of the third derivatives (of 36000 values, some units each), 1e-16 / step of the loss (some thousands), roundings of the gradient
        assert abs(got - quotient) <= 1e-6 * float(grads[k].cpu().double().norm() * d.norm()) + 1e-6, (k, got, quotient)


# -- the scan's long blocks ----------------------------------------------------------------------------------------------------------------

def scan_layout(n, t, c, elem, backward):
    d = ops.ScanDesc(n, t, c, elem, t * c, c, t * c, c, t * c, c, t * c, c, t * c, c)
    layout = (ctypes.c_int * 2)()
    assert rrm.lib().rrm_aux_scan_layout(ctypes.byref(d), backward, layout) == 0
    return layout[0], layout[1]


@gpu
@pytest.mark.parametrize("dtype,t", [("f32", 16384), ("f32", 16700), ("f32", 24577), ("bf16", 16700)])
@pytest.mark.parametrize("c", [3, 5, 70])
def test_long_scans_that_end_at_borders(dtype, t, c):
    """Videos that end with a block of frames (128, 256), a group of 32 blocks (4096, 8192), one beside them, or at once; x and f out of a joint tensor at
    odd addresses, frames before videos, not-a-numbers behind the ends; the same bits in every call."""
    ends = [t, 8192, 8193, 256, 0, 16384, 4095, 1]
    n = len(ends)
    blocks = 256 if dtype == "f32" else 128
    assert scan_layout(n, t, c, int(dtype == "bf16"), 0) == (2, blocks) and scan_layout(n, t, c, int(dtype == "bf16"), 1) == (2, 128)
    g = torch.Generator(device="cuda").manual_seed(t + c)
    joint = torch.empty(t, n, 2 * c + 3, device="cuda").normal_(generator=g)
    joint[..., 1 + c:1 + 2 * c] += 4 * torch.rand(c, device="cuda", generator=g)
    joint = joint.to(DT[dtype]).transpose(0, 1)
    x, f = joint[..., 1:1 + c], joint[..., 1 + c:1 + 2 * c]
    h0, dh = (torch.empty(n, c, device="cuda").normal_(generator=g) for _ in range(2))
    dy = torch.empty(n, t, c, device="cuda").normal_(generator=g).to(DT[dtype])
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    live = (torch.arange(t, device="cuda") < lengths.view(n, 1))[..., None]
    a = torch.where(live, torch.sigmoid(f.double()), 1.0)
    o = torch.where(live, torch.sigmoid(-f.double()), 0.0)
    x64, d64 = x.double(), torch.where(live, dy.double(), 0.0)
    for i, end in enumerate(ends):
        x[i, end:], f[i, end:], dy[i, end:] = math.nan, math.inf, math.nan
    hs, grads = torch.empty(n, t + 1, c, device="cuda", dtype=torch.float64), torch.empty_like(d64)
    hs[:, 0] = h0.double()
    b = o * x64
    for k in range(t):
        torch.addcmul(b[:, k], a[:, k], hs[:, k], out=hs[:, k + 1])
    carry = dh.double()
    for k in range(t - 1, -1, -1):
        torch.add(carry, d64[:, k], out=grads[:, k])
        carry = grads[:, k] * a[:, k]
    marks = rrm.gated_scan_marks(x)
    out = torch.full((n, t, c + 2), 7.0, device="cuda", dtype=DT[dtype])
    y, last = rrm.gated_scan(x, f, h0, lengths=lengths, out=out[..., 1:1 + c], marks=marks)
    got = rrm.gated_scan_backward(dy, x, f, marks, lengths=lengths, dh_last=dh)
    assert (out[..., 0] == 7).all() and (out[..., 1 + c] == 7).all()
    half = V if dtype == "bf16" else U
    # as in test_scan_of_many_frames
    slack = 5 * (SUM + 2 * U * 64 + GATE) * 2
    want = torch.where(live, hs[:, 1:], 0.0)
    close(y, want, slack + half * (want.abs() + slack), "y")
    close(last, hs[:, t], slack, "h_last")
    close(marks, hs[:, 0:t:64], slack, "marks")
    gs = slack * max(1.0, float(grads.abs().max()) / 5)
    for have, want, s, what in ((got[0], o * grads, gs, "dx"), (got[1], grads * (hs[:, :-1] - x64) * a * o, gs * 10, "df"), (got[2], carry, gs, "dh0")):
        close(have, want, s + half * (want.abs() + s), what)
    assert not y[~live.expand_as(y)].any() and not got[0][~live.expand_as(y)].any() and not got[1][~live.expand_as(y)].any()
    for _ in range(2):
        marks2 = rrm.gated_scan_marks(x)
        y2, last2 = rrm.gated_scan(x, f, h0, lengths=lengths, marks=marks2)
        assert torch.equal(y2, y) and torch.equal(last2, last) and torch.equal(marks2, marks)
        assert all(torch.equal(p, q) for p, q in zip(got, rrm.gated_scan_backward(dy, x, f, marks, lengths=lengths, dh_last=dh)))
