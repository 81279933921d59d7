"""Performance cases of the operators that stand between and behind the linear layers of a video network.

Three operators, each forward and backward:
  norm   group norm with an activation, channels last: what turns a convolution's stored projection into the next layer's input
  scan   a gated linear recurrence over the frames' features, h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(f_t),
         with a state that a live video carries from frame to frame
  ff     a gated feed-forward block, act(x Wg^T) * (x Wu^T), the head on those features

Fields of a case
  kind    "norm", "scan" or "ff"
  train   whether the pass is a training step's (forward and backward, gradients returned) or the forward alone
  norm    n maps of h x w positions and c channels in `groups` groups; x and y: the types of the input and of the result
  scan    n videos of t frames with c features; x: their type; ragged: the videos have lengths of their own (one of them zero,
          where there are several) and what stands behind a video's end is not a number
  ff      m rows of k features, f hidden features; bf16
  act     "none", "relu", "silu" or "gelu"
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _norm(name, n, h, w, c, groups, x, y, act, train):
    return dict(name=name, kind="norm", n=n, h=h, w=w, c=c, groups=groups, x=x, y=y, act=act, train=train)


def _scan(name, n, t, c, x, ragged, train):
    return dict(name=name, kind="scan", n=n, t=t, c=c, x=x, ragged=ragged, train=train)


def _ff(name, m, k, f, act, train):
    return dict(name=name, kind="ff", m=m, k=k, f=f, act=act, train=train)


def listed():
    return [
        # the last stage of a ResNet-shaped network on one live video: latency
        _norm("norm_live", 1, 7, 7, 512, 32, "f32", "bf16", "silu", False),
        # its first stage over many streams: the projection in 32 bits becomes the next layer's input in 16
        _norm("norm_streams", 64, 56, 56, 64, 32, "f32", "bf16", "silu", False),
        # its second stage in training, 16 bits in and out
        _norm("norm_train", 64, 28, 28, 128, 32, "bf16", "bf16", "silu", True),
        # an odd map, channels off the powers of two, 32 bits throughout, training
        _norm("norm_odd_train", 9, 35, 29, 105, 7, "f32", "f32", "gelu", True),
        # one frame of one live video: the state takes one step
        _scan("scan_live", 1, 1, 4096, "bf16", False, False),
        # clips of many streams at once: throughput
        _scan("scan_streams", 64, 256, 4096, "bf16", False, False),
        # one long video with few features: the time axis is all there is to divide
        _scan("scan_long", 1, 65536, 512, "f32", False, False),
        # training on long videos of different lengths, features off the powers of two
        _scan("scan_ragged_train", 4, 8192, 1000, "bf16", True, True),
        # the head on one frame of one live video: the weights are read for one row
        _ff("ff_live", 1, 4096, 4096, "silu", False),
        # the head on one frame of many streams
        _ff("ff_streams", 64, 4096, 9216, "silu", False),
        # training on 32 frames of 512 streams (the largest case)
        _ff("ff_train", 16384, 4096, 4096, "silu", True),
        # training with rows that no vector load divides
        _ff("ff_odd_train", 333, 1001, 2050, "gelu", True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi, steps):
    """log-uniform, in whole multiples of one of `steps`"""
    v, step = _log(rng, lo, hi), rng.choice(steps)
    return int(min(hi, max(step, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(("norm", "scan", "ff"))
    train = rng.random() < 0.5
    if kind == "norm":
        c = _size(rng, 16, 512, (32, 16, 8, 1))
        groups = rng.choice([g for g in range(1, 65) if c % g == 0])
        h, w = _size(rng, 7, 56, (7, 1)), _size(rng, 7, 56, (7, 1))
        n = max(1, min(_size(rng, 1, 64, (1,)), (64 * 56 * 56 * 64) // (h * w * c)))
        x, y = rng.choice((("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")))
        case = _norm("", n, h, w, c, groups, x, y, rng.choice(("none", "silu", "gelu") if train else ("none", "relu", "silu", "gelu")), train)
    elif kind == "scan":
        n, c = _size(rng, 1, 64, (1,)), _size(rng, 16, 4096, (64, 8, 1))
        t = max(1, min(_size(rng, 1, 65536, (1,)), (64 * 256 * 4096) // (n * c)))
        case = _scan("", n, t, c, rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.5, train)
    else:
        case = _ff("", _size(rng, 1, 4096, (64, 1)), _size(rng, 64, 4096, (64, 8, 1)), _size(rng, 64, 9216, (64, 8, 1)),
                   rng.choice(("silu", "gelu")), train)
    del case["name"]
    return case


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype="f32", scale=1.0, shift=0.0):
        t = torch.empty(shape, device="cuda", dtype=torch.float32).normal_(shift, scale, generator=g)
        return t.to(TYPES[dtype])

    s = {"case": case}
    if case["kind"] == "norm":
        shape = (case["n"], case["h"], case["w"], case["c"])
        # a projection of post-ReLU inputs: channels with means of their own
        s["x"] = (normal(*shape, scale=1.5) + normal(case["c"])).to(TYPES[case["x"]])
        s["gamma"], s["beta"] = normal(case["c"], scale=0.2, shift=1.0), normal(case["c"], scale=0.3)
        if case["train"]:
            s["dy"] = normal(*shape, dtype=case["y"])
    elif case["kind"] == "scan":
        n, t, c = case["n"], case["t"], case["c"]
        s["x"] = normal(n, t, c, dtype=case["x"])
        # gates that remember between a frame or two and some hundred frames
        s["f"] = (normal(n, t, c) + 4.0 * torch.rand((c,), device="cuda", generator=g)).to(TYPES[case["x"]])
        s["h0"] = normal(n, c)
        s["lengths"] = None
        if case["ragged"]:
            lengths = torch.randint(0, t + 1, (n,), device="cuda", generator=g, dtype=torch.int32)
            if n > 1:
                lengths[0], lengths[n - 1] = t, 0
            s["lengths"] = lengths
            gone = torch.arange(t, device="cuda").view(1, t, 1) >= lengths.view(n, 1, 1)
            s["x"].masked_fill_(gone, math.nan)
            s["f"].masked_fill_(gone, math.nan)
        if case["train"]:
            s["dy"], s["dh_last"] = normal(n, t, c, dtype=case["x"]), normal(n, c)
    else:
        m, k, f = case["m"], case["k"], case["f"]
        s["x"] = normal(m, k, dtype="bf16")
        s["wg"], s["wu"] = normal(f, k, dtype="bf16", scale=k ** -0.5), normal(f, k, dtype="bf16", scale=k ** -0.5)
        if case["train"]:
            s["dh"] = normal(m, f, dtype="bf16")
    return s


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end -----------------------------------------


def _act(act, z):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(act, z):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _plain_norm(s):
    case = s["case"]
    n, c, groups = case["n"], case["c"], case["groups"]
    x = s["x"].float().view(n, -1, groups, c // groups)
    mean = x.mean((1, 3), keepdim=True)
    x = x - mean
    rstd = 1 / torch.sqrt((x * x).mean((1, 3), keepdim=True) + EPS)
    xhat = (x * rstd).view(n, -1, c)
    z = xhat * s["gamma"] + s["beta"]
    y = _act(case["act"], z).view(s["x"].shape).to(TYPES[case["y"]])
    if not case["train"]:
        return {"y": y}
    dz = s["dy"].float().view(n, -1, c) * _act_slope(case["act"], z)
    dgamma, dbeta = (dz * xhat).sum((0, 1)), dz.sum((0, 1))
    p, q = (dz * s["gamma"]).view(n, -1, groups, c // groups), xhat.view(n, -1, groups, c // groups)
    dx = rstd * (p - p.mean((1, 3), keepdim=True) - q * (p * q).mean((1, 3), keepdim=True))
    return {"y": y, "dx": dx.view(s["x"].shape).to(TYPES[case["x"]]), "dgamma": dgamma, "dbeta": dbeta}


def _recur(a, b):
    """h_t = a_t h_{t-1} + b_t from h = 0, along dimension 1: pairs of neighbours, of pairs, of fours, .. are joined"""
    step, t = 1, a.shape[1]
    while step < t:
        b = torch.cat((b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]), 1)
        a = torch.cat((a[:, :step], a[:, step:] * a[:, :-step]), 1)
        step *= 2
    return b


def _plain_scan(s):
    case = s["case"]
    kind = TYPES[case["x"]]
    x, a, h0 = s["x"].float(), 1 / (1 + torch.exp(-s["f"].float())), s["h0"]
    here = torch.ones((1, 1, 1), device=x.device, dtype=torch.bool)
    if s["lengths"] is not None:
        here = torch.arange(case["t"], device=x.device).view(1, -1, 1) < s["lengths"].view(-1, 1, 1)
        x, a = torch.where(here, x, 0.0), torch.where(here, a, 1.0)
    b = (1 - a) * x
    first = torch.cat((b[:, :1] + a[:, :1] * h0[:, None], b[:, 1:]), 1)
    h = _recur(a, first)
    out = {"y": torch.where(here, h, 0.0).to(kind), "h_last": h[:, -1].clone()}
    if not case["train"]:
        return out
    dy = torch.where(here, s["dy"].float(), 0.0)
    dy = torch.cat((dy[:, :-1], dy[:, -1:] + s["dh_last"][:, None]), 1)
    after = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
    g = _recur(after.flip(1), dy.flip(1)).flip(1)
    before = torch.cat((h0[:, None], h[:, :-1]), 1)
    out["dx"] = ((1 - a) * g).to(kind)
    out["df"] = (g * (before - x) * a * (1 - a)).to(kind)
    out["dh0"] = a[:, 0] * g[:, 0]
    return out


def _plain_ff(s):
    case = s["case"]
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    p = _act(case["act"], g)
    h = (p * u).bfloat16()
    if not case["train"]:
        return {"h": h}
    dh = s["dh"].float()
    dg, du = dh * u * _act_slope(case["act"], g), dh * p
    return {"h": h, "dx": (dg @ wg + du @ wu).bfloat16(), "dwg": (dg.t() @ x).bfloat16(), "dwu": (du.t() @ x).bfloat16()}


# ---- the same through the package's entry points -------------------------------------------------------------------------


def _own_norm(s):
    import paper_1802_09723_amd as rrm
    case = s["case"]
    kind = TYPES[case["y"]]
    if not case["train"]:
        return {"y": rrm.group_norm_act(s["x"], case["groups"], s["gamma"], s["beta"], case["act"], EPS, out_dtype=kind)}
    stats = torch.empty((case["n"], case["groups"], 2), device="cuda")
    y = rrm.group_norm_act(s["x"], case["groups"], s["gamma"], s["beta"], case["act"], EPS, out_dtype=kind, stats=stats)
    dx, dgamma, dbeta = rrm.group_norm_act_backward(s["dy"], s["x"], stats, s["gamma"], s["beta"], case["act"])
    return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_scan(s):
    import paper_1802_09723_amd as rrm
    case = s["case"]
    if not case["train"]:
        y, h_last = rrm.gated_scan(s["x"], s["f"], s["h0"], lengths=s["lengths"])
        return {"y": y, "h_last": h_last}
    marks = rrm.gated_scan_marks(s["x"])
    y, h_last = rrm.gated_scan(s["x"], s["f"], s["h0"], lengths=s["lengths"], marks=marks)
    dx, df, dh0 = rrm.gated_scan_backward(s["dy"], s["x"], s["f"], marks, lengths=s["lengths"], dh_last=s["dh_last"])
    return {"y": y, "h_last": h_last, "dx": dx, "df": df, "dh0": dh0}


def _own_ff(s):
    import paper_1802_09723_amd as rrm
    case = s["case"]
    if not case["train"]:
        return {"h": rrm.gated_ff(s["x"], s["wg"], s["wu"], case["act"])}
    g = torch.empty((case["m"], case["f"]), device="cuda", dtype=torch.bfloat16)
    u = torch.empty_like(g)
    h = rrm.gated_ff(s["x"], s["wg"], s["wu"], case["act"], save=(g, u))
    dx, dwg, dwu = rrm.gated_ff_backward(s["dh"], s["x"], s["wg"], s["wu"], g, u, case["act"])
    return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "scan": _own_scan, "ff": _own_ff}[kind](state)
    return {"norm": _plain_norm, "scan": _plain_scan, "ff": _plain_ff}[kind](state)


def work(case):
    """What a pass has to read, write and compute; a training pass reads its inputs for the forward and, apart from that, for the
    backward pass, as its two calls do.  Flops are those of the products alone where there are products."""
    train = case["train"]
    if case["kind"] == "norm":
        e = case["n"] * case["h"] * case["w"] * case["c"]
        x, y = BYTES[case["x"]], BYTES[case["y"]]
        # forward: x in, y out, some ten operations a value; backward: x and dy in, dx out, some thirty
        return {"bytes": e * (x + y) + (e * (2 * x + y) if train else 0) + 16 * case["c"], "flops": e * (40 if train else 10)}
    if case["kind"] == "scan":
        e, b = case["n"] * case["t"] * case["c"], BYTES[case["x"]]
        # forward: x and f in, y out; backward: x, f and dy in, dx and df out; the states beside them
        return {"bytes": e * b * (8 if train else 3) + 8 * case["n"] * case["c"] * (2 if train else 1), "flops": e * (30 if train else 10)}
    m, k, f = case["m"], case["k"], case["f"]
    fwd = 2 * (m * k + 2 * f * k + m * f)
    # backward: dh, the two projections, x and the weights in, dx and the weights' gradients out
    return {"bytes": fwd + (2 * (2 * m * f) + 2 * (3 * m * f + 2 * m * k + 4 * f * k) if train else 0), "flops": (12 if train else 4) * m * k * f}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------


def _act64(act, z):
    if act == "relu":
        return torch.relu(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z


def _exact_norm(s, case):
    leaves = [s[k].double().requires_grad_(case["train"]) for k in ("x", "gamma", "beta")]
    x, gamma, beta = leaves
    per = case["c"] // case["groups"]
    parts = []
    for i in range(case["groups"]):
        one = x[..., i * per:(i + 1) * per]
        var, mean = torch.var_mean(one, dim=(1, 2, 3), keepdim=True, unbiased=False)
        parts.append((one - mean) / torch.sqrt(var + EPS))
    y = _act64(case["act"], torch.cat(parts, -1) * gamma + beta)
    if not case["train"]:
        return {"y": y}
    dx, dgamma, dbeta = torch.autograd.grad(y, leaves, s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _exact_scan(s, case):
    n, t, c = case["n"], case["t"], case["c"]
    h = s["h0"].double()
    x, a = s["x"].double(), torch.sigmoid(s["f"].double())
    ends = [t] * n if s["lengths"] is None else s["lengths"].tolist()
    for i, e in enumerate(ends):
        x[i, e:], a[i, e:] = 0, 1
    every = torch.empty((n, t + 1, c), device="cuda", dtype=torch.float64)
    every[:, 0] = h
    b = (1 - a) * x
    for j in range(t):
        torch.addcmul(b[:, j], a[:, j], every[:, j], out=every[:, j + 1])
    y = every[:, 1:].clone()
    for i, e in enumerate(ends):
        y[i, e:] = 0
    out = {"y": y, "h_last": every[:, t].clone()}
    if not case["train"]:
        return out
    dy = s["dy"].double()
    for i, e in enumerate(ends):
        dy[i, e:] = 0
    carry, grads = s["dh_last"].double(), torch.empty_like(dy)
    for j in range(t - 1, -1, -1):
        torch.add(carry, dy[:, j], out=grads[:, j])
        carry = grads[:, j] * a[:, j]
    out["dx"] = grads * (1 - a)
    out["df"] = grads * (every[:, :-1] - x) * a * (1 - a)
    out["dh0"] = carry
    return out


def _exact_ff(s, case):
    leaves = [s[k].double().requires_grad_(case["train"]) for k in ("x", "wg", "wu")]
    x, wg, wu = leaves
    h = _act64(case["act"], torch.nn.functional.linear(x, wg)) * torch.nn.functional.linear(x, wu)
    if not case["train"]:
        return {"h": h}
    dx, dwg, dwu = torch.autograd.grad(h, leaves, s["dh"].double())
    return {"h": h.detach(), "dx": dx, "dwg": dwg, "dwu": dwu}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "scan": _exact_scan, "ff": _exact_ff}[case["kind"]](s, case)
