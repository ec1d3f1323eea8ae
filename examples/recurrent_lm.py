"""Train a small recurrent language model on the GPU, then let it go on with a text.

Every layer mixes the rows of a sequence (norm, projection, short convolution, selective scan) and
then each row by itself (norm, feed-forward block); the table of the embedding is the last layer's
weight too.  All of it but the projections runs on ``paper_2011_13824_amd.blocks``.  Training packs
texts of any length behind each other; answering reads a prompt once, keeps every sequence's states
in a cache and takes one token of all sequences at a time.

The texts are synthetic: a few words, repeated.

    python examples/recurrent_lm.py [--steps 80] [--width 128] [--rows 2048]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2011_13824_amd import blocks  # noqa: E402

TAPS, STATES = 4, 16


class Net:
    """tokens -> log probabilities of the tokens that follow."""

    def __init__(self, vocab, width, depth, dtype, rank=8, seed=0, keep=8):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        inner, hidden = 2 * width, 2 * width
        self.width, self.inner, self.rank, self.keep = width, inner, rank, keep

        def normal(*shape):
            return (torch.randn(*shape, generator=gen, device="cuda") * shape[-1] ** -0.5).to(dtype)

        ones = torch.ones(width, dtype=dtype, device="cuda")
        p = self.params = {"table": normal(vocab, width), "norm": ones.clone()}
        self.layers = []
        for i in range(depth):
            p[f"norm1_{i}"], p[f"norm2_{i}"] = ones.clone(), ones.clone()
            p[f"in_{i}"], p[f"out_{i}"] = normal(2 * inner, width), normal(width, inner)
            p[f"x_{i}"], p[f"dt_{i}"] = normal(rank + 2 * STATES, inner), normal(inner, rank)
            p[f"w_{i}"], p[f"b_{i}"] = normal(TAPS, inner), torch.zeros_like(ones).repeat(2)
            # the scan's own parameters are in 32 bits: A = -exp(log_A)
            p[f"log_A_{i}"] = torch.log(torch.arange(1.0, STATES + 1, device="cuda")).repeat(inner, 1)
            p[f"D_{i}"] = torch.ones(inner, device="cuda")
            step = torch.exp(torch.rand(inner, generator=gen, device="cuda") * 4.6) * 1e-3
            p[f"bias_{i}"] = step + torch.log(-torch.expm1(-step))  # log(1 + e^bias) = step
            p[f"Wg_{i}"], p[f"Wu_{i}"] = normal(hidden, width), normal(hidden, width)
            p[f"Wd_{i}"] = normal(width, hidden)
            self.layers.append((blocks.Norm(p[f"norm1_{i}"]),
                                blocks.CausalConv(p[f"w_{i}"], p[f"b_{i}"]),
                                blocks.Norm(p[f"norm2_{i}"]),
                                blocks.FeedForward(p[f"Wg_{i}"], p[f"Wu_{i}"], p[f"Wd_{i}"])))
        self.embed = blocks.Embedding(p["table"], width ** 0.5)
        self.norm, self.logprobs = blocks.Norm(p["norm"]), blocks.LogProbs(top=3)

    def scan(self, i):
        p = self.params
        return blocks.SelectiveScan(-torch.exp(p[f"log_A_{i}"]), p[f"D_{i}"], p[f"bias_{i}"])

    def cache(self, slots):
        """The states of `slots` sequences."""
        dtype = self.params["table"].dtype
        return [(torch.zeros(slots, TAPS - 1, self.inner, dtype=dtype, device="cuda"),
                 torch.zeros(slots, self.inner, STATES, device="cuda")) for _ in self.layers]

    def mix(self, i, y, seq, states, single, tape):
        """A layer's first half behind its norm."""
        p, r = self.params, self.rank
        conv, scan = self.layers[i][1], self.scan(i)
        xz = y @ p[f"in_{i}"].t()
        x, z = xz[:, :self.inner], xz[:, self.inner:]
        if states is None:
            c = conv.forward(x, seq)
        elif single:
            c = conv.step(x, states[i][0], seq, state_out=states[i][0])
        else:
            c = conv.forward(x, seq, states[i][0], state_out=states[i][0])
        q = c @ p[f"x_{i}"].t()
        dt = q[:, :r] @ p[f"dt_{i}"].t()
        args = (c, dt, q[:, r:r + STATES], q[:, r + STATES:], z)
        if tape is not None:
            s, kept = scan.forward(*args, seq, keep=True)
            tape.update(x=x, c=c, q=q, s=s, kept=kept, scan=scan)
        elif single:
            s = scan.step(*args, states[i][1], seq, state_out=states[i][1])
        elif states is not None:
            s = scan.forward(*args, seq, states[i][1], state_out=states[i][1])
        else:
            s = scan.forward(*args, seq)
        return s @ p[f"out_{i}"].t()

    def logits(self, tokens, seq=None, states=None, single=False, tape=None):
        """Rows of logits; ``tape``, a list, receives what the backward pass needs."""
        h, out = self.embed.forward(tokens), None
        for i, (norm1, _, norm2, ffn) in enumerate(self.layers):
            kept = {} if tape is not None else None
            n1 = norm1.forward(h, out)
            mixed = self.mix(i, n1.y, seq, states, single, kept)
            n2 = norm2.forward(n1.sum, mixed, want8=tape is not None and self.keep == 8)
            if tape is not None:
                out, k = ffn.forward(n2.y, keep=self.keep, x8=n2.y8)
                tape.append(dict(kept, n1=n1, n2=n2, ffn=k))
            else:
                out = ffn.forward(n2.y)
            h = n2.sum
        n = self.norm.forward(h, out)
        if tape is not None:
            tape.append(n)
        return n.y @ self.params["table"].t()

    def backward(self, tokens, seq, dlogits, tape):
        """Gradients of the parameters."""
        p, r, grads = self.params, self.rank, {}
        n = tape.pop()
        dtable = dlogits.t() @ n.y
        dh, grads["norm"] = self.norm.backward(dlogits @ p["table"], n.sum, n.rstd)
        for i in reversed(range(len(self.layers))):
            norm1, conv, norm2, ffn = self.layers[i]
            t = tape[i]
            g = ffn.backward(dh, t["ffn"])
            grads.update({f"{k[1:]}_{i}": g[k] for k in ("dWg", "dWu", "dWd")})
            dh, grads[f"norm2_{i}"] = norm2.backward(g["dx"], t["n2"].sum, t["n2"].rstd, dsum=dh)
            grads[f"out_{i}"] = dh.t() @ t["s"]
            g = t["scan"].backward(dh @ p[f"out_{i}"], t["kept"])
            grads[f"log_A_{i}"] = g["dA"] * t["scan"].A
            grads[f"D_{i}"], grads[f"bias_{i}"] = g["dD"], g["dbias"]
            grads[f"dt_{i}"] = g["ddt"].t() @ t["q"][:, :r]
            dq = torch.cat([g["ddt"] @ p[f"dt_{i}"], g["dB"], g["dC"]], 1)
            grads[f"x_{i}"] = dq.t() @ t["c"]
            c = conv.backward(g["du"] + dq @ p[f"x_{i}"], t["x"], seq)
            grads[f"w_{i}"], grads[f"b_{i}"] = c["dw"], c["dbias"]
            dxz = torch.cat([c["dx"], g["dz"]], 1)
            grads[f"in_{i}"] = dxz.t() @ t["n1"].y
            dh, grads[f"norm1_{i}"] = norm1.backward(dxz @ p[f"in_{i}"], t["n1"].sum, t["n1"].rstd,
                                                     dsum=dh)
        grads["table"] = self.embed.backward(tokens, dh, base=dtable, out=dtable)
        return grads

    def loss(self, tokens, targets, seq):
        """(mean of -log p over the targets that are not padding, gradients)"""
        tape = []
        logits = self.logits(tokens, seq, tape=tape)
        f = self.logprobs.forward(logits, targets)
        count = (targets >= 0).sum()
        weight = (-1 / count.float()).expand(len(targets)).contiguous()
        dlogits = self.logprobs.backward(logits, targets, f.lse, dlogp=weight, out=logits)
        return -f.logp.sum() / count, self.backward(tokens, seq, dlogits, tape)

    def answer(self, prompts, count):
        """The most likely `count` tokens behind each prompt (lists of tokens), one by one."""
        slots = torch.arange(len(prompts), dtype=torch.int32, device="cuda")
        states = self.cache(len(prompts))
        seq = blocks.sequences([len(p) for p in prompts])
        tokens = torch.tensor([t for p in prompts for t in p], device="cuda")
        ends = torch.tensor([len(p) for p in prompts], device="cuda").cumsum(0) - 1
        logits = self.logits(tokens, seq, states)[ends]
        out = []
        for _ in range(count):
            out.append(self.logprobs.forward(logits).top_tokens[:, 0].contiguous())
            logits = self.logits(out[-1], slots, states, single=True)
        return torch.stack(out, 1)


def texts(gen, rows, vocab):
    """(tokens, targets, seq): sequences of words of 3 tokens; a word's tokens follow each other."""
    lengths, left = [], rows - rows // 50
    while left > 0:
        lengths.append(min(left, int(torch.randint(5, 200, (1,), generator=gen))))
        left -= lengths[-1]
    words = torch.randint(0, vocab // 3, (rows,), generator=gen)
    tokens = torch.cat([3 * words[:n // 3 + 1, None] + torch.arange(3) for n in lengths]).flatten()
    at, first = [], 0
    for n in lengths:
        at.append(torch.arange(first, first + n))
        first += 3 * (n // 3 + 1)
    tokens = torch.nn.functional.pad(tokens[torch.cat(at)], (0, rows - sum(lengths)), value=-1)
    seq = blocks.sequences(lengths, rows)
    tokens = tokens.cuda()
    targets = torch.full_like(tokens, -1)
    follows = seq[1:] == seq[:-1]  # the last token of a sequence has none behind it
    targets[:-1][follows] = tokens[1:][follows]
    targets[seq < 0] = -1
    return tokens, targets, seq


def train(net, steps, rows, vocab, lr=3e-3):
    gen = torch.Generator()
    gen.manual_seed(1)
    master = {k: p.float() for k, p in net.params.items()}
    m = {k: torch.zeros_like(p) for k, p in master.items()}
    v = {k: torch.zeros_like(p) for k, p in master.items()}
    losses = []
    for t in range(1, steps + 1):
        loss, grads = net.loss(*texts(gen, rows, vocab))
        losses.append(loss)
        for k, g in grads.items():
            g = g.float()
            m[k].mul_(0.9).add_(g, alpha=0.1)
            v[k].mul_(0.99).addcmul_(g, g, value=0.01)
            rate = lr * (1 - 0.99 ** t) ** 0.5 / (1 - 0.9 ** t)
            master[k].addcdiv_(m[k], v[k].sqrt().add_(1e-8), value=-rate)
            net.params[k].copy_(master[k])
    return [float(x) for x in losses]


def run(steps=80, width=128, depth=2, rows=2048, vocab=96, dtype=torch.bfloat16):
    net = Net(vocab, width, depth, dtype)
    losses = train(net, steps, rows, vocab)
    return losses, net.answer([[0, 1, 2, 9, 10], [30], [5, 12]], 8).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 80), ("width", 128), ("depth", 2), ("rows", 2048), ("vocab", 96)):
        ap.add_argument("--" + name, type=int, default=value)
    losses, answers = run(**vars(ap.parse_args()))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    for a in answers:
        print("goes on with", a)


if __name__ == "__main__":
    main()
