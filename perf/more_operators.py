"""Performance cases of the operators of a residual block over the frames' features, and of training it.

  mix    linear attention over a video's frames with a decay for each head: S_t = lambda S_{t-1} + k_t^T v_t, o_t = scale q_t S_t; whole clips,
         one frame of live videos with the state that they carry, and the gradients
  res    what stands between two blocks: the norm behind the one, its gate, the residual scale and sum, and the norm before the next,
         r = x + s sigmoid(z) (rms(b) p), u = rms(r) w; and the gradients
  orth   a weight matrix's update made orthogonal by Newton-Schulz products, X <- a X + (b A + c A^2) X with A = X X^T

Fields of a case
  kind    "mix", "res" or "orth"
  train   (mix, res) whether the pass is a training step's (forward and backward, gradients returned) or the forward alone
  mix     n videos of t frames, h heads with keys of dk and values of dv features; x: the type of q, k, v and o; ragged: the videos have lengths
          of their own (one of them zero, where there are several) and what stands behind a video's end is not a number
  res     m rows of c features; x: the type of the residual stream, b: of the block's output, of its gate and of the next block's input;
          gate, scale, post: whether there is a gate, a residual scale, a norm behind the block
  orth    n matrices of rows x cols; x: their type (the result is bf16)
"""
import math

import torch

own = False

EPS = 1e-6
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
ORTH_EPS = 1e-7
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _mix(name, n, t, h, dk, dv, x, ragged, train):
    return dict(name=name, kind="mix", n=n, t=t, h=h, dk=dk, dv=dv, x=x, ragged=ragged, train=train)


def _res(name, m, c, x, b, gate, scale, post, train):
    return dict(name=name, kind="res", m=m, c=c, x=x, b=b, gate=gate, scale=scale, post=post, train=train)


def _orth(name, n, rows, cols, x):
    return dict(name=name, kind="orth", n=n, rows=rows, cols=cols, x=x)


def listed():
    return [
        # one frame of one live video: the states of its heads take one step; latency
        _mix("mix_live", 1, 1, 16, 64, 64, "bf16", False, False),
        # one frame of many live videos: the states are the traffic
        _mix("mix_streams_live", 64, 1, 16, 128, 128, "bf16", False, False),
        # clips of many streams at once: throughput
        _mix("mix_clips", 64, 256, 32, 128, 128, "bf16", False, False),
        # one long video with few heads: the time axis is all there is to divide
        _mix("mix_long", 1, 65536, 8, 128, 128, "bf16", False, False),
        # training on long videos of different lengths, keys and values of sizes of their own
        _mix("mix_ragged_train", 4, 8192, 12, 80, 136, "bf16", True, True),
        # training in 32 bits, nothing divides
        _mix("mix_odd_train", 3, 777, 5, 45, 67, "f32", True, True),
        # between two blocks, one frame of one live video: latency
        _res("res_live", 1, 4096, "f32", "bf16", True, True, True, False),
        # between two blocks on 32 frames of 512 streams: throughput
        _res("res_streams", 16384, 4096, "bf16", "bf16", True, True, True, False),
        # the same in training, the residual stream in 32 bits
        _res("res_train", 16384, 4096, "f32", "bf16", True, True, True, True),
        # training with rows that no vector load divides, no gate
        _res("res_odd_train", 3333, 1001, "f32", "f32", False, True, True, True),
        # the update of a small head's weights: latency
        _orth("orth_small", 1, 128, 512, "f32"),
        # the updates of a feed-forward block's two weights (the largest case)
        _orth("orth_head", 2, 4096, 4096, "bf16"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi, steps):
    """log-uniform, in whole multiples of one of `steps`"""
    v, step = _log(rng, lo, hi), rng.choice(steps)
    return int(min(hi, max(step, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(("mix", "mix", "res", "orth"))
    train = rng.random() < 0.5
    if kind == "mix":
        h = _size(rng, 1, 32, (4, 1))
        dk, dv = _size(rng, 16, 256, (64, 16, 1)), _size(rng, 16, 256, (64, 16, 1))
        n = _size(rng, 1, 64, (1,))
        live = rng.random() < 0.25
        t = 1 if live else max(1, min(_size(rng, 2, 65536, (1,)), (64 * 256 * 32 * 128) // (n * h * max(dk, dv))))
        case = _mix("", n, t, h, dk, dv, rng.choice(("bf16", "bf16", "f32")), not live and rng.random() < 0.5, not live and train)
    elif kind == "res":
        c = _size(rng, 16, 8192, (64, 8, 1))
        m = max(1, min(_size(rng, 1, 65536, (1,)), (16384 * 4096) // c))
        x, b = rng.choice((("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")))
        case = _res("", m, c, x, b, rng.random() < 0.6, rng.random() < 0.6, rng.random() < 0.7, train)
    else:
        rows, cols = _size(rng, 16, 4096, (64, 8, 1)), _size(rng, 16, 4096, (64, 8, 1))
        n = max(1, min(_size(rng, 1, 16, (1,)), (2 * 4096 * 4096) // (rows * cols)))
        case = _orth("", n, rows, cols, rng.choice(("bf16", "f32")))
    del case["name"]
    return case


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype="f32", scale=1.0, shift=0.0):
        t = torch.empty(shape, device="cuda", dtype=torch.float32).normal_(shift, scale, generator=g)
        return t.to(TYPES[dtype])

    s = {"case": case}
    if case["kind"] == "mix":
        n, t, h, dk, dv, x = (case[k] for k in ("n", "t", "h", "dk", "dv", "x"))
        s["q"], s["k"], s["v"] = normal(n, t, h, dk, dtype=x), normal(n, t, h, dk, dtype=x), normal(n, t, h, dv, dtype=x)
        # heads that remember between 8 and some 500 frames
        s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(3.0, 9.0, h, dtype=torch.float64))).float().cuda()
        s["s0"] = normal(n, h, dk, dv, scale=3.0)
        s["lengths"] = None
        if case["ragged"]:
            lengths = torch.randint(0, t + 1, (n,), device="cuda", generator=g, dtype=torch.int32)
            if n > 1:
                lengths[0], lengths[n - 1] = t, 0
            s["lengths"] = lengths
            gone = torch.arange(t, device="cuda").view(1, t, 1, 1) >= lengths.view(n, 1, 1, 1)
            for name in ("q", "k", "v"):
                s[name].masked_fill_(gone, math.nan)
        if case["train"]:
            s["do"], s["ds_last"] = normal(n, t, h, dv, dtype=x), normal(n, h, dk, dv)
            if case["ragged"]:
                s["do"].masked_fill_(gone, math.nan)
    elif case["kind"] == "res":
        m, c = case["m"], case["c"]
        # a residual stream that has grown over some blocks, with channels of means of their own
        s["x"] = (normal(m, c, scale=2.0) + normal(c)).to(TYPES[case["x"]])
        s["b"] = normal(m, c, dtype=case["b"], scale=0.7)
        s["gate"] = normal(m, c, dtype=case["b"]) if case["gate"] else None
        s["scale"] = normal(c, scale=0.1, shift=0.5) if case["scale"] else None
        s["post"] = normal(c, scale=0.2, shift=1.0) if case["post"] else None
        s["pre"] = normal(c, scale=0.2, shift=1.0)
        if case["train"]:
            s["dr"], s["du"] = normal(m, c, dtype=case["x"]), normal(m, c, dtype=case["b"])
    else:
        n, rows, cols = case["n"], case["rows"], case["cols"]
        # an update as training makes it: a few directions that many samples agree on, noise about them, rows and columns of their own scales
        few = min(8, rows, cols)
        u = normal(n, rows, cols) * torch.exp(normal(n, rows, 1, scale=0.5)) * torch.exp(normal(n, 1, cols, scale=0.5))
        u += 2.0 * torch.matmul(normal(n, rows, few), normal(n, few, cols))
        s["g"] = (u * 1e-3).to(TYPES[case["x"]])
    return s


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end -----------------------------------------


def _powers(log_decay, exponents):
    """lambda^e for every head and exponent, the product of exponent and logarithm in 64 bits: [h, ..]"""
    e = torch.as_tensor(exponents, device=log_decay.device, dtype=torch.float64)
    return torch.exp(log_decay.double().view(-1, *([1] * e.dim())) * e).float()


CHUNK = 64


def _attend(q, k, v, log_decay, s0, backwards=False):
    """sums over j <= i of lambda^(i-j) (q_i . k_j) v_j, and the state behind the last frame, in chunks of the time axis; q, k, v [n, t, h, d] in
    32 bits, t whole chunks.  The state before the first frame comes in with lambda^(i+1); `backwards`: with lambda^i, and the last one takes a
    step more (the gradient of a state is what the state before it is multiplied by)."""
    n, t, h, dk = q.shape
    dv, c = v.shape[-1], t // CHUNK
    late = 0 if backwards else 1
    q, k, v = (a.view(n, c, CHUNK, h, -1).permute(0, 3, 1, 2, 4).contiguous() for a in (q, k, v))  # [n, h, c, CHUNK, d]
    ar = torch.arange(CHUNK, device=q.device)
    apart = ar.view(-1, 1) - ar
    mask = torch.where(apart >= 0, _powers(log_decay, apart.clamp(min=0)), 0.0).view(h, 1, CHUNK, CHUNK)
    # what each chunk adds to the state, and the state before each chunk: one product over the chunks
    weighted = v * _powers(log_decay, CHUNK - late - ar).view(h, 1, CHUNK, 1)
    adds = torch.matmul(k.transpose(-1, -2), weighted)  # [n, h, c, dk, dv]
    ac = torch.arange(c + 1, device=q.device)
    between = ac.view(-1, 1) - 1 - ac[:c]
    carry = torch.where(between >= 0, _powers(log_decay, CHUNK * between.clamp(min=0)), 0.0)  # [h, c + 1, c]
    states = torch.matmul(carry, adds.view(n, h, c, dk * dv)) + _powers(log_decay, CHUNK * ac).view(h, c + 1, 1) * s0.reshape(n, h, 1, dk * dv)
    states = states.view(n, h, c + 1, dk, dv)
    o = torch.matmul(q, states[:, :, :c]) * _powers(log_decay, ar + late).view(h, 1, CHUNK, 1)
    o += torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * mask, v)
    return o.permute(0, 2, 3, 1, 4).reshape(n, t, h, dv), states[:, :, c].clone()


def _plain_mix(s):
    case = s["case"]
    kind, n, t, h = TYPES[case["x"]], case["n"], case["t"], case["h"]
    scale, ld = case["dk"] ** -0.5, s["log_decay"]
    s0 = s["s0"]
    names = ("q", "k", "v", "do") if case["train"] else ("q", "k", "v")
    if t == 1:
        q, k, v = (s[a][:, 0].float() for a in names)
        state = _powers(ld, 1).view(h, 1, 1) * s0 + k[..., :, None] * v[..., None, :]
        return {"o": (scale * (q[..., None] * state).sum(-2)).to(kind)[:, None], "s_last": state}
    whole = -(-t // CHUNK) * CHUNK
    lengths = torch.full((n,), t, device="cuda") if s["lengths"] is None else s["lengths"]
    here = torch.arange(whole, device="cuda").view(1, whole, 1, 1) < lengths.view(n, 1, 1, 1)
    # videos are moved to end with the last chunk: what lies before them, and so decays nothing but zeros, is the padding
    at = torch.arange(whole, device="cuda").view(1, whole) - (whole - lengths.view(n, 1))
    rows, inside = at.clamp(min=0), (at >= 0).view(n, whole, 1, 1)
    vid = torch.arange(n, device="cuda").view(n, 1)

    def behind(a):
        return torch.where(inside, a[vid, rows.clamp(max=t - 1)].float(), 0.0)

    def before(a):
        shift = (torch.arange(t, device="cuda").view(1, t) + (whole - lengths.view(n, 1))).clamp(max=whole - 1)
        return torch.where(here[:, :t], a[vid, shift], 0.0)

    # (the state before a video would decay over the padding: it is added by itself)
    data = [behind(s[a]) for a in names]
    q, k, v = data[:3]
    zero = torch.zeros_like(s0)
    o, s_last = _attend(q, k, v, ld, zero)
    since = _powers(ld, (at + 1).clamp(min=0)).permute(1, 2, 0)[..., None]  # [n, whole, h, 1]
    full = _powers(ld, lengths).permute(1, 0)[..., None, None]              # [n, h, 1, 1]

    def through(a, state):  # a [n, whole, h, i] times state [n, h, i, j]
        return torch.matmul(a.permute(0, 2, 1, 3).contiguous(), state).permute(0, 2, 1, 3)

    o = scale * (o + since * through(q, s0))
    s_last = s_last + full * s0
    out = {"o": before(o).to(kind), "s_last": s_last}
    if not case["train"]:
        return out
    do, ds_last = data[3], s["ds_last"]
    turned = s0.transpose(-1, -2).contiguous()
    dq, _ = _attend(do, v, k, ld, torch.zeros_like(turned))
    out["dq"] = before(scale * (dq + since * through(do, turned))).to(kind)
    # (turned in time the padding lies behind a video, and only the gradient of the state before it is taken from its own sum)
    fq, fk, fv, fdo = (a.flip(1) for a in (q, k, v, do))
    inv = ds_last.transpose(-1, -2).contiguous()
    dk, _ = _attend(fv, fdo, fq * scale, ld, inv, backwards=True)
    dv, _ = _attend(fk, fq * scale, fdo, ld, ds_last, backwards=True)
    out["dk"], out["dv"] = before(dk.flip(1)).to(kind), before(dv.flip(1)).to(kind)
    weighted = torch.where(inside, since, 0.0) * do * scale
    out["ds0"] = torch.matmul(q.permute(0, 2, 3, 1).contiguous(), weighted.permute(0, 2, 1, 3).contiguous()) + full * ds_last
    return out


def _plain_res(s):
    case = s["case"]
    kx, kb = TYPES[case["x"]], TYPES[case["b"]]
    x, b, pre = s["x"].float(), s["b"].float(), s["pre"]
    rb = 1 / torch.sqrt((b * b).mean(-1, keepdim=True) + EPS) if case["post"] else 1.0
    bh = b * rb
    p = bh * s["post"] if case["post"] else b
    sg = 1 / (1 + torch.exp(-s["gate"].float())) if case["gate"] else 1.0
    sc = s["scale"] if case["scale"] else 1.0
    r = x + sc * sg * p
    rr = 1 / torch.sqrt((r * r).mean(-1, keepdim=True) + EPS)
    rh = r * rr
    out = {"r": r.to(kx), "u": (rh * pre).to(kb)}
    if not case["train"]:
        return out
    dr, du = s["dr"].float(), s["du"].float()
    w = du * pre
    dr = dr + rr * (w - rh * (w * rh).mean(-1, keepdim=True))
    out["dx"], out["dpre"] = dr.to(kx), (du * rh).sum(0)
    if case["gate"]:
        out["dgate"] = (dr * sc * p * sg * (1 - sg)).to(kb)
    if case["scale"]:
        out["dscale"] = (dr * sg * p).sum(0)
    dp = dr * sc * sg
    if case["post"]:
        out["dpost"] = (dp * bh).sum(0)
        dp = dp * s["post"]
        dp = rb * (dp - bh * (dp * bh).mean(-1, keepdim=True))
    out["db"] = dp.to(kb)
    return out


def _plain_orth(s):
    a, b, c = COEFFICIENTS
    x = s["g"].float()
    x = x / (torch.sqrt((x * x).sum((-1, -2), keepdim=True)) + ORTH_EPS)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2).contiguous()
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(-1, -2))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    if tall:
        x = x.transpose(-1, -2)
    return {"x": x.bfloat16().contiguous()}


# ---- the same through the package's entry points -------------------------------------------------------------------------


def _own_mix(s):
    import paper_1802_09723_amd as rrm
    case = s["case"]
    scale = case["dk"] ** -0.5
    o, s_last = rrm.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], scale, s0=s["s0"], lengths=s["lengths"])
    out = {"o": o, "s_last": s_last}
    if case["train"]:
        out["dq"], out["dk"], out["dv"], out["ds0"] = rrm.decay_attention_backward(
            s["do"], s["q"], s["k"], s["v"], s["log_decay"], scale, s0=s["s0"], lengths=s["lengths"], ds_last=s["ds_last"])
    return out


def _own_res(s):
    import paper_1802_09723_amd as rrm
    case = s["case"]
    stats = torch.empty((case["m"], 2), device="cuda") if case["train"] else None
    r, u = rrm.residual_norm(s["x"], s["b"], s["gate"], s["scale"], s["post"], s["pre"], EPS, stats=stats)
    out = {"r": r, "u": u}
    if case["train"]:
        grads = rrm.residual_norm_backward(s["dr"], s["du"], s["x"], s["b"], stats, s["gate"], s["scale"], s["post"], s["pre"])
        out.update((k, v) for k, v in zip(("dx", "db", "dgate", "dscale", "dpost", "dpre"), grads) if v is not None)
    return out


def _own_orth(s):
    import paper_1802_09723_amd as rrm
    return {"x": rrm.orthogonalize(s["g"], STEPS, COEFFICIENTS, ORTH_EPS)}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"mix": _own_mix, "res": _own_res, "orth": _own_orth}[kind](state)
    return {"mix": _plain_mix, "res": _plain_res, "orth": _plain_orth}[kind](state)


def work(case):
    """What a pass has to read, write and compute; a training pass reads its inputs for the forward and, apart from that, for the
    backward pass, as its two calls do."""
    if case["kind"] == "mix":
        dk, dv, e, b = case["dk"], case["dv"], case["n"] * case["t"] * case["h"], BYTES[case["x"]]
        state = 4 * case["n"] * case["h"] * dk * dv
        # forward: q, k, v in, o out, a state in and one out, the update and the reading of a state a frame; backward: q, k, v, do in, three
        # gradients out, three states, five such products
        fwd, back = e * b * 2 * (dk + dv) + 2 * state, e * b * (4 * dk + 3 * dv) + 3 * state
        return {"bytes": fwd + (back if case["train"] else 0), "flops": e * dk * dv * (14 if case["train"] else 4)}
    if case["kind"] == "res":
        e, x, b, gate = case["m"] * case["c"], BYTES[case["x"]], BYTES[case["b"]], int(case["gate"])
        # forward: x, b and the gate in, r and u out; backward: x, b, the gate, dr and du in, dx, db and the gate's gradient out
        fwd, back = e * (2 * x + (2 + gate) * b), e * (3 * x + (3 + 2 * gate) * b)
        return {"bytes": fwd + (back if case["train"] else 0) + 16 * case["c"], "flops": e * (50 if case["train"] else 15)}
    few, many = sorted((case["rows"], case["cols"]))
    # of the two symmetric products half is enough
    return {"bytes": case["n"] * few * many * (BYTES[case["x"]] + 2), "flops": case["n"] * STEPS * (few * few * many + few ** 3 + 2 * few * few * many)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------


def _exact_mix(s, case):
    n, t, h, dk, dv = (case[k] for k in ("n", "t", "h", "dk", "dv"))
    scale, lam = dk ** -0.5, torch.exp(s["log_decay"].double()).view(1, h, 1, 1)
    ends = [t] * n if s["lengths"] is None else s["lengths"].tolist()
    state = s["s0"].double().clone()
    out = {"o": torch.zeros((n, t, h, dv), device="cuda", dtype=torch.float64)}
    if case["train"]:
        for name, d in (("dq", dk), ("dk", dk), ("dv", dv)):
            out[name] = torch.zeros((n, t, h, d), device="cuda", dtype=torch.float64)
        grad = s["ds_last"].double().clone()
    # the recurrence itself, frame by frame; videos that have ended stand still
    order = sorted(range(n), key=lambda i: -ends[i])
    pick = torch.tensor(order, device="cuda")
    state = state[pick]
    q, k, v = (s[a].double()[pick] for a in ("q", "k", "v"))
    o = out["o"][pick]
    live = n
    if case["train"]:
        do, dq, gk, gv, grad = s["do"].double()[pick], out["dq"][pick], out["dk"][pick], out["dv"][pick], grad[pick]
    for j in range(max(ends)):
        while ends[order[live - 1]] <= j:
            live -= 1
        st = state[:live]
        st.mul_(lam).addcmul_(k[:live, j, :, :, None], v[:live, j, :, None, :])
        o[:live, j] = scale * torch.matmul(q[:live, j, :, None, :], st)[:, :, 0]
        if case["train"]:
            dq[:live, j] = scale * torch.matmul(st, do[:live, j, :, :, None])[..., 0]
    back = torch.argsort(pick)
    got = {"o": o[back], "s_last": state[back]}
    if not case["train"]:
        return got
    live = 0
    for j in range(max(ends) - 1, -1, -1):
        while live < n and ends[order[live]] > j:
            live += 1
        gr = grad[:live]
        gr.addcmul_(q[:live, j, :, :, None], do[:live, j, :, None, :], value=scale)
        gk[:live, j] = torch.matmul(gr, v[:live, j, :, :, None])[..., 0]
        gv[:live, j] = torch.matmul(k[:live, j, :, None, :], gr)[:, :, 0]
        gr.mul_(lam)
    got.update(dq=dq[back], dk=gk[back], dv=gv[back], ds0=grad[back])
    return got


def _exact_res(s, case):
    names = ["x", "b"] + [k for k in ("gate", "scale", "post") if case[k]] + ["pre"]
    leaves = {k: s[k].double().requires_grad_(case["train"]) for k in names}
    b = leaves["b"]
    if case["post"]:
        b = b * torch.rsqrt(b.square().mean(-1, keepdim=True) + EPS) * leaves["post"]
    if case["gate"]:
        b = b * torch.sigmoid(leaves["gate"])
    if case["scale"]:
        b = b * leaves["scale"]
    r = leaves["x"] + b
    u = r * torch.rsqrt(r.square().mean(-1, keepdim=True) + EPS) * leaves["pre"]
    out = {"r": r.detach(), "u": u.detach()}
    if case["train"]:
        grads = dict(zip(names, torch.autograd.grad((r, u), list(leaves.values()), (s["dr"].double(), s["du"].double()))))
        out["dx"], out["dpre"] = grads["x"], grads["pre"]
        for k in ("gate", "scale", "post"):
            if case[k]:
                out["d" + k] = grads[k]
        out["db"] = grads["b"]
    return out


def _exact_orth(s, case):
    a, b, c = COEFFICIENTS
    done = []
    for g in s["g"]:
        x = g.double()
        x = x / (torch.linalg.vector_norm(x) + ORTH_EPS)
        eye = torch.eye(min(x.shape), device="cuda", dtype=torch.float64)
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                gram = x @ x.t().contiguous()
                x = (a * eye + gram @ (b * eye + c * gram)) @ x
            else:
                gram = x.t().contiguous() @ x
                x = x @ (a * eye + gram @ (b * eye + c * gram))
        done.append(x)
    return {"x": torch.stack(done)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"mix": _exact_mix, "res": _exact_res, "orth": _exact_orth}[case["kind"]](s, case)
