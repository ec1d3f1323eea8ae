"""Train a small net of feed-forward blocks on the GPU, then search its input box for a violation.

The blocks run on ``paper_2011_13824_amd.blocks``: each adds its input to the residual stream,
norms it, and keeps what its backward pass needs in 8 bits.  Training fits a synthetic function
with Adam; the search is projected gradient descent on a margin of the trained net over an l_inf
box, and ends with an upper bound on the margin's minimum there: the least value it has met (a
point with a negative margin violates the property margin >= 0).  The points it tries are values of
the net's type inside the box.

    python examples/train_and_attack.py [--steps 60] [--width 256] [--hidden 704] [--rows 2048]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2011_13824_amd import blocks  # noqa: E402


class Net:
    """x -> h += block(norm(h)) for every block -> outputs h W_out^T."""

    def __init__(self, width, hidden, depth, outputs, dtype, gate="silu", seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape):
            w = torch.randn(*shape, generator=gen, device="cuda") * shape[1] ** -0.5
            return w.to(dtype)

        self.params = {"out": normal(outputs, width)}
        for i in range(depth):
            self.params[f"norm{i}"] = torch.ones(width, dtype=dtype, device="cuda")
            self.params[f"Wg{i}"] = normal(hidden, width)
            self.params[f"Wu{i}"] = normal(hidden, width)
            self.params[f"Wd{i}"] = normal(width, hidden)
        self.norms = [blocks.Norm(self.params[f"norm{i}"]) for i in range(depth)]
        self.ffns = [blocks.FeedForward(self.params[f"Wg{i}"], self.params[f"Wu{i}"],
                                        self.params[f"Wd{i}"], gate) for i in range(depth)]

    def forward(self, x, keep):
        """(outputs in 32 bits, the tape of the backward pass)"""
        h, out, tape = x, None, []
        for norm, ffn in zip(self.norms, self.ffns):
            n = norm.forward(h, out, want8=keep)  # adds the last block's output to the stream
            if keep:
                out, kept = ffn.forward(n.y, keep=8, x8=n.y8)
                tape.append((n.sum, n.rstd, kept))
            else:
                out = ffn.forward(n.y)
            h = n.sum
        last = h + out
        return last.float() @ self.params["out"].float().t(), (last, tape)

    def backward(self, dy, tape, weights=True):
        """Gradients of the parameters (none without ``weights``), and that of x."""
        last, steps = tape
        grads = {}
        if weights:
            grads["out"] = dy.t() @ last.float()
        dh = (dy @ self.params["out"].float()).to(last.dtype)  # of the stream after the last block
        for i in reversed(range(len(steps))):
            h, rstd, kept = steps[i]
            if weights:
                g = self.ffns[i].backward(dh, kept)
                grads.update({k[1:] + str(i): g[k] for k in ("dWg", "dWu", "dWd")})
            else:
                g = self.ffns[i].backward(dh, kept, want=("dx",))
            dh, dw = self.norms[i].backward(g["dx"], h, rstd, dsum=dh, want_dw=weights)
            if weights:
                grads[f"norm{i}"] = dw
        return grads, dh


def train(net, steps, rows, width, outputs, dtype, lr=2e-3):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    teacher = torch.randn(width, outputs, generator=gen, device="cuda") * width ** -0.5
    master = {k: p.float() for k, p in net.params.items()}
    m = {k: torch.zeros_like(p) for k, p in master.items()}
    v = {k: torch.zeros_like(p) for k, p in master.items()}
    losses = []
    for t in range(1, steps + 1):
        x = torch.randn(rows, width, generator=gen, device="cuda").to(dtype)
        y, tape = net.forward(x, keep=True)
        err = y - torch.sin(2 * (x.float() @ teacher))
        losses.append(err.square().mean())
        grads, _ = net.backward(2 * err / err.numel(), tape)
        for k, g in grads.items():
            g = g.float()
            m[k].mul_(0.9).add_(g, alpha=0.1)
            v[k].mul_(0.999).addcmul_(g, g, value=0.001)
            rate = lr * (1 - 0.999 ** t) ** 0.5 / (1 - 0.9 ** t)
            master[k].addcdiv_(m[k], v[k].sqrt().add_(1e-8), value=-rate)
            net.params[k].copy_(master[k])
    return [float(x) for x in losses]


def box(x0, eps, dtype):
    """(lowest, highest) values of `dtype` with |v - x0| <= eps in every place, in 64 bits."""
    ends = []
    for sign in (-1, 1):
        end = x0.double() + sign * eps
        v = end.to(dtype).double()
        # one past the end by rounding: the next value inwards is at most two units of v away
        unit = v.abs().clamp(min=torch.finfo(dtype).tiny) * torch.finfo(dtype).eps
        for part in (0.25, 0.5, 1.0):
            v = torch.where(sign * (v - end) > 0, (v - sign * part * unit).to(dtype).double(), v)
        ends.append(v)
    lo, hi = ends
    if (lo > hi).any():
        raise ValueError(f"{dtype} has no value within {eps} of x0 in some places")
    return lo, hi


def attack(net, x0, eps, c, steps=20, starts=64):
    """The least c . f(x) met over ||x - x0||_inf <= eps, from `starts` random points."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    dtype = net.params["out"].dtype
    lo, hi = box(x0, eps, dtype)
    x = x0 + eps * (2 * torch.rand(starts, x0.numel(), generator=gen, device="cuda") - 1)
    least = float("inf")
    for t in range(steps + 1):
        at = torch.clamp(x.to(dtype).double(), lo, hi).to(dtype)  # clamp rounds nothing
        y, tape = net.forward(at, keep=t < steps)
        least = min(least, float((y @ c).min()))
        if t < steps:
            _, dx = net.backward(c.expand(starts, -1).contiguous(), tape, weights=False)
            x = torch.clamp(x - eps / 4 * dx.float().sign(), x0 - eps, x0 + eps)
    return least


def run(steps=60, width=256, hidden=704, depth=2, rows=2048, outputs=4, eps=0.05,
        dtype=torch.bfloat16):
    net = Net(width, hidden, depth, outputs, dtype)
    losses = train(net, steps, rows, width, outputs, dtype)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x0 = torch.randn(width, generator=gen, device="cuda")
    y0 = net.forward(x0[None].to(dtype), keep=False)[0][0]
    best = int(y0.argmax())
    second = int(y0.masked_fill(torch.arange(outputs, device="cuda") == best, -1e30).argmax())
    c = torch.zeros(outputs, device="cuda")
    c[best], c[second] = 1.0, -1.0
    margin, least = float(y0 @ c), attack(net, x0, eps, c)
    return losses, margin, least


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 60), ("width", 256), ("hidden", 704), ("depth", 2),
                        ("rows", 2048)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--eps", type=float, default=0.05)
    losses, margin, least = run(**vars(ap.parse_args()))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    print(f"margin at x0 {margin:.4f}, least found in the box {least:.4f}"
          + (": violated" if least < 0 else ""))


if __name__ == "__main__":
    main()
