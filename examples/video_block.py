"""Residual blocks over the features of a video's frames: served frame by frame from a carried state, trained on clips of different lengths.

    features -> norm -> q, k, v -> linear attention over the frames -> product with Wo
             -> (norm behind, gate, residual scale and sum, norm before) -> gated feed-forward block -> product with Wd
             -> (norm behind, gate, residual scale and sum, norm before) -> the next block, or the features that leave

`Block.clip` is the forward pass over whole clips, `Block.gradients` its backward pass, `Block.frame` one frame of live videos; `update` takes a step of the
weight matrices along their gradients made orthogonal.  The plain matrix products around the operators are torch's.

    python examples/video_block.py        # some training steps on synthetic clips, then the same videos live
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1802_09723_amd as rrm  # noqa: E402

MATRICES = ("wq", "wk", "wv", "wo", "wz", "wg", "wu", "wd")
EPS = 1e-6


class Block:
    """c features, h heads of d keys and d values, f hidden features.  Matrices lie [out][in], bfloat16; vectors are float32."""

    def __init__(self, c=128, h=4, d=32, f=256, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*s):
            return (torch.randn(*s, generator=g) * s[-1] ** -0.5).bfloat16().cuda()

        self.h, self.d = h, d
        self.wq, self.wk, self.wv, self.wo = rand(h * d, c), rand(h * d, c), rand(h * d, c), rand(c, h * d)
        self.wz = rand(c, c)  # the first sum's gate
        self.wg, self.wu, self.wd = rand(f, c), rand(f, c), rand(c, f)
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2.0, 6.0, h))).cuda()
        self.before = torch.ones(c, device="cuda")                       # weights of the norm before the block,
        self.post1, self.pre1, self.scale1 = (torch.ones(c, device="cuda") for _ in range(3))  # of the first sum
        self.post2, self.pre2, self.scale2 = (torch.ones(c, device="cuda") for _ in range(3))  # and of the second

    def _mix(self, u, s0=None, lengths=None, s_last=None):
        n, t, c = u.shape
        q, k, v = ((u @ w.t()).view(n, t, self.h, self.d) for w in (self.wq, self.wk, self.wv))
        o, s_last = rrm.decay_attention(q, k, v, self.log_decay, s0=s0, lengths=lengths, s_last=s_last)
        return q, k, v, o, s_last

    def _feed(self, u, save=None):
        m = u.view(-1, u.shape[-1])
        return rrm.gated_ff(m, self.wg, self.wu, "silu", save=save)

    def state(self, n):
        return torch.zeros(n, self.h, self.d, self.d, device="cuda")

    def frame(self, x, state):
        """One frame x [n, c] (float32) of n live videos: the features that leave (bfloat16); ``state`` is advanced in place."""
        x = x[:, None]
        _, u = rrm.residual_norm(x, pre=self.before, u_dtype=torch.bfloat16)
        _, _, _, o, _ = self._mix(u, state, s_last=state)
        r, u1 = rrm.residual_norm(x, o.flatten(2) @ self.wo.t(), u @ self.wz.t(), self.scale1, self.post1, self.pre1)
        h = self._feed(u1).view(*u1.shape[:2], -1)
        _, y = rrm.residual_norm(r, h @ self.wd.t(), None, self.scale2, self.post2, self.pre2, out=r)
        return y[:, 0]

    def clip(self, x, lengths=None):
        """Clips x [n, t, c] (float32): the features that leave, bfloat16, and what the backward pass reads."""
        n, t, c = x.shape
        stats = [torch.empty(n, t, 2, device="cuda") for _ in range(3)]
        _, u = rrm.residual_norm(x, pre=self.before, u_dtype=torch.bfloat16, stats=stats[0])
        q, k, v, o, _ = self._mix(u, lengths=lengths)
        b, z = o.flatten(2) @ self.wo.t(), u @ self.wz.t()
        r, u1 = rrm.residual_norm(x, b, z, self.scale1, self.post1, self.pre1, stats=stats[1])
        f = self.wg.shape[0]
        g, up = (torch.empty(n * t, f, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        h = self._feed(u1, (g, up)).view(n, t, f)
        b2 = h @ self.wd.t()
        _, y = rrm.residual_norm(r, b2, None, self.scale2, self.post2, self.pre2, stats=stats[2])
        return y, (x, lengths, stats, u, q, k, v, o, b, z, r, u1, g, up, h, b2)

    def gradients(self, dy, kept):
        """Of the clips and of every weight, from the gradient ``dy`` (bfloat16) of the features that leave."""
        x, lengths, stats, u, q, k, v, o, b, z, r, u1, g, up, h, b2 = kept
        n, t, c = x.shape

        def weight(d, a):  # of a product a w^T with the gradient d
            return d.reshape(n * t, -1).t().float() @ a.reshape(n * t, -1).float()

        out = {}
        dr, db2, _, out["scale2"], out["post2"], out["pre2"] = rrm.residual_norm_backward(None, dy, r, b2, stats[2], None, self.scale2, self.post2, self.pre2)
        out["wd"] = weight(db2, h)
        du1, out["wg"], out["wu"] = rrm.gated_ff_backward((db2 @ self.wd).view(n * t, -1), u1.view(n * t, c), self.wg, self.wu, g, up, "silu")
        dx, db, dz, out["scale1"], out["post1"], out["pre1"] = rrm.residual_norm_backward(dr, du1.view(n, t, c), x, b, stats[1], z, self.scale1, self.post1, self.pre1)
        out["wo"], out["wz"] = weight(db, o), weight(dz, u)
        do = (db @ self.wo).view(n, t, self.h, self.d)
        grads = rrm.decay_attention_backward(do, q, k, v, self.log_decay, lengths=lengths)[:3]
        du = dz.float() @ self.wz.float()
        for name, d in zip(("wq", "wk", "wv"), grads):
            out[name] = weight(d, u)
            du += d.reshape(n, t, -1).float() @ getattr(self, name).float()
        out["x"], _, _, _, _, out["before"] = rrm.residual_norm_backward(dx, du.bfloat16(), x, None, stats[0], pre=self.before)
        return out


def update(block: Block, grads, momenta, rate=0.02, hold=0.9):
    """Matrices take a step along their momenta made orthogonal, of a size that goes by their shape; vectors one along their gradients."""
    for name, g in grads.items():
        if name == "x":
            continue
        p = getattr(block, name)
        if name not in MATRICES:
            p -= rate * g
            continue
        m = momenta.setdefault(name, torch.zeros(p.shape, device="cuda"))
        m.mul_(hold).add_(g)
        step = rrm.orthogonalize(m)
        p.copy_((p.float() - rate * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * step.float()).bfloat16())


def main():
    torch.cuda.set_device(0)
    block, n, t, c = Block(), 4, 96, 128
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, t, c, generator=g).cuda()
    target = torch.randn(n, 1, c, generator=g).cuda()  # features that a video's frames are to agree on
    lengths = torch.tensor([t, t - 9, 40, 1], dtype=torch.int32, device="cuda")
    live = (torch.arange(t, device="cuda") < lengths.view(n, 1)).float()[..., None]
    momenta, losses = {}, []
    for _ in range(20):
        y, kept = block.clip(x, lengths)
        d = (y.float() - target) * live / live.sum()
        losses.append(float((d * (y.float() - target)).sum()))
        update(block, block.gradients(d.bfloat16(), kept), momenta)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps")
    y, _ = block.clip(x)
    state = block.state(n)
    last = [block.frame(x[:, j].contiguous(), state) for j in range(t)][-1]
    off = float((last.float() - y[:, -1].float()).norm() / y[:, -1].float().norm())
    print(f"the last live frame is {off:.4f} of its norm off the clip's")
    return losses, off


if __name__ == "__main__":
    main()
