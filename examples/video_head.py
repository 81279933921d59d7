"""A small video network end to end: convolutions advanced by their differences, and the operators between and behind them.

    frame -> conv (delta step) -> group norm + SiLU -> conv (delta step) -> group norm + SiLU -> mean over positions
          -> gated recurrence over the frames -> gated feed-forward block -> fully-connected layer -> logits

`Net.serve` takes one frame of n live videos (the layers keep their snapshots, the recurrence its state); `train_head` fits the second norm's
parameters, the gates, the feed-forward block and the last layer on clips whose projections the convolutions have made, with every gradient
from the package's backward passes (the plain matrix products around them are torch's).

    python examples/video_head.py        # a live loop and some training steps on synthetic clips
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1802_09723_amd as rrm  # noqa: E402


def bits(t) -> np.ndarray:
    """bfloat16 patterns of a float tensor, as rrm.Layer takes weights"""
    return t.to(torch.bfloat16).cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def shape(kind, **kw):
    v = dict(kind=kind, n=1, h=1, w=1, c_in=1, c_out=1, kh=1, kw=1, stride=1, pad=0, groups=1)
    v.update(kw)
    return rrm.Shape(*v.values())


class Net:
    """Sizes: n videos of side x side frames with c0 channels; c1 and c2 channels behind the convolutions, f hidden features, k classes."""

    def __init__(self, n=4, side=16, c0=16, c1=32, c2=64, f=128, k=10, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*s, scale):
            return torch.randn(*s, generator=g) * scale

        self.n, self.k = n, k
        self.w1, self.w2 = rand(c1, 3, 3, c0, scale=(9 * c0) ** -0.5), rand(c2, 3, 3, c1, scale=(9 * c1) ** -0.5)
        self.conv1 = rrm.Layer(shape(rrm.CONV, n=n, h=side, w=side, c_in=c0, c_out=c1, kh=3, kw=3, pad=1), rrm.BF16, bits(self.w1))
        self.conv2 = rrm.Layer(shape(rrm.CONV, n=n, h=side, w=side, c_in=c1, c_out=c2, kh=3, kw=3, stride=2, pad=1), rrm.BF16, bits(self.w2))
        self.norm1 = [torch.ones(c1, device="cuda"), torch.zeros(c1, device="cuda")]
        self.norm2 = [torch.ones(c2, device="cuda"), torch.zeros(c2, device="cuda")]
        self.gate = rand(c2, c2, scale=c2 ** -0.5).bfloat16().cuda()  # the gates' logits: features times this
        self.wg, self.wu = rand(f, c2, scale=c2 ** -0.5).bfloat16().cuda(), rand(f, c2, scale=c2 ** -0.5).bfloat16().cuda()
        self.out = rand(k, f, scale=f ** -0.5).bfloat16().cuda()
        self.state = torch.zeros(n, c2, device="cuda")
        self._head_layers()

    def _head_layers(self):
        c2, f = self.gate.shape[1], self.out.shape[1]
        self.gate_layer = rrm.Layer(shape(rrm.FC, n=self.n, c_in=c2, c_out=c2), rrm.BF16, bits(self.gate))
        self.out_layer = rrm.Layer(shape(rrm.FC, n=self.n, c_in=f, c_out=self.k), rrm.BF16, bits(self.out))

    def projections(self, frame):
        """The second convolution's stored projection for this frame, in place (no copy); ``frame`` [n, side, side, c0] bfloat16."""
        self.conv1.step(frame)
        self.conv2.step(rrm.group_norm_act_of(self.conv1, 8, *self.norm1, act="silu"))

    def serve(self, frame):
        """Logits, float32 [n, k], of one frame of the live videos."""
        self.projections(frame)
        a = rrm.group_norm_act_of(self.conv2, 8, *self.norm2, act="silu")
        feat = a.float().mean((1, 2)).bfloat16()
        gates = torch.empty(feat.shape, device="cuda")
        self.gate_layer.dense(feat, gates)
        y, _ = rrm.gated_scan(feat[:, None], gates.bfloat16()[:, None], self.state, h_last=self.state)
        h = rrm.gated_ff(y[:, 0], self.wg, self.wu, "silu")
        logits = torch.empty(self.n, self.k, device="cuda")
        self.out_layer.dense(h, logits)
        return logits

    def reset(self):
        """New videos: forget the frames."""
        self.conv1.reset()
        self.conv2.reset()
        self.state.zero_()


def train_head(net: Net, clip, labels, lengths, steps=100, rate=0.15):
    """SGD on the clip of projections [n, t, ho, wo, c2] (float32): cross-entropy of every frame before a video's end against
    ``labels`` [n].  Returns the losses."""
    n, t, ho, wo, c2 = clip.shape
    x = clip.view(n * t, ho, wo, c2)
    k, f = net.out.shape
    live = (torch.arange(t, device="cuda") < lengths.view(n, 1)).float()
    weight = live / live.sum()
    master = [p.float() for p in (net.gate, net.wg, net.wu, net.out)]
    losses = []
    for _ in range(steps):
        gate, wg, wu, out = (m.bfloat16() for m in master)
        # forward
        stats = torch.empty(n * t, 8, 2, device="cuda")
        a = rrm.group_norm_act(x, 8, *net.norm2, act="silu", out_dtype=torch.bfloat16, stats=stats)
        feat = a.float().mean((1, 2)).bfloat16().view(n, t, c2)
        gates = (feat.view(n * t, c2) @ gate.t()).view(n, t, c2)
        marks = rrm.gated_scan_marks(feat)
        y, _ = rrm.gated_scan(feat, gates, lengths=lengths, marks=marks)
        g, u = torch.empty(n * t, f, device="cuda", dtype=torch.bfloat16), torch.empty(n * t, f, device="cuda", dtype=torch.bfloat16)
        h = rrm.gated_ff(y.view(n * t, c2), wg, wu, "silu", save=(g, u))
        logits = (h @ out.t()).float().view(n, t, k)
        logp = torch.log_softmax(logits, -1)
        losses.append(float(-(logp.gather(-1, labels.view(n, 1, 1).expand(n, t, 1))[..., 0] * weight).sum()))
        # backward
        dl = (logp.exp() - torch.nn.functional.one_hot(labels, k).view(n, 1, k)) * weight[..., None]
        dl = dl.view(n * t, k).bfloat16()
        dout = dl.t().float() @ h.float()
        dy, dwg, dwu = rrm.gated_ff_backward(dl @ out, y.view(n * t, c2), wg, wu, g, u, "silu")
        dfeat, dgates, _ = rrm.gated_scan_backward(dy.view(n, t, c2), feat, gates, marks, lengths=lengths)
        dgate = dgates.view(n * t, c2).t().float() @ feat.view(n * t, c2).float()
        dfeat = dfeat.view(n * t, c2).float() + dgates.view(n * t, c2).float() @ gate.float()
        da = (dfeat / (ho * wo)).bfloat16().view(n * t, 1, 1, c2).expand(n * t, ho, wo, c2).contiguous()
        _, dgamma, dbeta = rrm.group_norm_act_backward(da, x, stats, *net.norm2, act="silu")
        for p, d in zip(master + net.norm2, (dgate, dwg, dwu, dout, dgamma, dbeta)):
            p -= rate * d.float()
    net.gate, net.wg, net.wu, net.out = (m.bfloat16() for m in master)
    net._head_layers()
    return losses


def synthetic_clip(net: Net, t: int, side=16, c0=16, seed=1):
    """Frames [t] of [n, side, side, c0]: a static background of its own colours in every video, with a patch that moves."""
    g = torch.Generator().manual_seed(seed)
    tint = 3 * torch.rand(net.n, 1, 1, c0, generator=g)  # a video has colours of its own
    back = torch.randn(net.n, side, side, c0, generator=g).clamp(min=0) * tint
    patch = 2 * torch.randn(net.n, 5, 5, c0, generator=g).clamp(min=0)
    frames = []
    for i in range(t):
        fr = back.clone()
        at = i % (side - 5)
        fr[:, at:at + 5, at:at + 5] = patch
        frames.append(fr.bfloat16().cuda())
    return frames


def main():
    torch.cuda.set_device(0)
    net = Net()
    t = 24
    frames = synthetic_clip(net, t)
    # the clip's projections, once through the convolutions
    clip = []
    for fr in frames:
        net.projections(fr)
        clip.append(net.conv2.y_snapshot())
    clip = torch.stack(clip, 1)
    labels = torch.arange(net.n, device="cuda") % net.k
    lengths = torch.tensor([t, t - 5, t, 7], dtype=torch.int32, device="cuda")
    losses = train_head(net, clip, labels, lengths)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps")
    net.reset()
    for fr in frames:
        logits = net.serve(fr)
    torch.cuda.synchronize()
    print("classes of the live videos behind the last frame:", logits.argmax(-1).tolist(), "wanted", labels.tolist())
    return losses, logits, labels


if __name__ == "__main__":
    main()
