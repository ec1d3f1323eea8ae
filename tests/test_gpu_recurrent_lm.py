"""The operators together, as examples/recurrent_lm.py runs them: gradients of the whole net against
64 bits, and an answer token by token against the text read at once.

In 32 bits every step of the net is off by at most some 300 roundings (the longest sum that is not
itself a gradient's has 300 terms), 2e-5 of what it works on; about 20 such steps lie between a
parameter and the loss, which leaves 1e-3 of a gradient's norm as a bound with room for what a norm
or a gate magnifies."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "recurrent_lm.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("recurrent_lm", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(net, p, tokens, runs):
    """The net's function by its definition, a sequence after the other, for autograd."""
    def norm(h, w):
        return h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-5) * w

    def silu(x):
        return x / (1 + torch.exp(-x))

    r, N, taps = net.rank, 16, 4
    rows = []
    for a, n in runs:
        h = p["table"][tokens[a:a + n]] * net.width ** 0.5
        for i in range(len(net.layers)):
            xz = norm(h, p[f"norm1_{i}"]) @ p[f"in_{i}"].T
            x, z = xz[:, :net.inner], xz[:, net.inner:]
            x = torch.nn.functional.pad(x, (0, 0, taps - 1, 0))
            c = silu(sum(p[f"w_{i}"][k] * x[k:k + n] for k in range(taps)) + p[f"b_{i}"])
            q = c @ p[f"x_{i}"].T
            delta = torch.log1p(torch.exp(q[:, :r] @ p[f"dt_{i}"].T + p[f"bias_{i}"]))
            A = -torch.exp(p[f"log_A_{i}"])
            s, ys = torch.zeros_like(A), []
            for t in range(n):
                s = torch.exp(delta[t][:, None] * A) * s \
                    + (delta[t] * c[t])[:, None] * q[t, r:r + N]
                ys.append(s @ q[t, r + N:])
            y = (torch.stack(ys) + p[f"D_{i}"] * c) * silu(z)
            h = h + y @ p[f"out_{i}"].T
            y = norm(h, p[f"norm2_{i}"])
            h = h + (silu(y @ p[f"Wg_{i}"].T) * (y @ p[f"Wu_{i}"].T)) @ p[f"Wd_{i}"].T
        rows.append(norm(h, p["norm"]) @ p["table"].T)
    return rows


def test_gradients_of_the_net(ex):
    from paper_2011_13824_amd import blocks
    vocab, lengths, rows = 33, [1, 70, 20], 97
    net = ex.Net(vocab, 24, 2, torch.float32, rank=3, seed=4, keep=0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    seq = blocks.sequences(lengths, rows)
    tokens[seq < 0], targets[seq < 0], targets[3] = -1, -1, -1
    loss, grads = net.loss(tokens, targets, seq)
    p = {k: v.double().requires_grad_() for k, v in net.params.items()}
    runs = [(0, 1), (1, 70), (71, 20)]
    logits = torch.cat(plain_logits(net, p, tokens, runs))
    named = (targets[:91] >= 0).nonzero()[:, 0]
    log_p = torch.log_softmax(logits, 1)[named, targets[named]]
    want = -log_p.sum() / len(named)
    with torch.no_grad():
        assert abs(float(loss) - float(want)) <= 1e-4 * float(want)
    for (k, _), g in zip(p.items(), torch.autograd.grad(want, list(p.values()))):
        off = (grads[k].double().reshape(g.shape) - g).norm()
        assert float(off) <= 1e-3 * float(g.norm()) + 1e-9, k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32],
                         ids=lambda t: str(t)[6:])
def test_it_trains_and_answers(ex, dtype):
    losses, answers = ex.run(steps=6, width=64, rows=700, vocab=30, dtype=dtype)
    assert all(x == x and x < 100 for x in losses)
    assert len(answers) == 3 and all(0 <= t < 30 for a in answers for t in a)


def test_token_by_token_is_the_text_at_once(ex):
    """Logits behind a prompt and single tokens, for three sequences in a cache of five slots."""
    net = ex.Net(40, 48, 2, torch.float32, seed=2)
    gen = torch.Generator()
    gen.manual_seed(3)
    whole = [torch.randint(0, 40, (n,), generator=gen).tolist() for n in (30, 7, 19)]
    split = [25, 2, 14]
    slots = [4, 0, 2]
    from paper_2011_13824_amd import blocks
    states = net.cache(5)
    prompts = [w[:s] for w, s in zip(whole, split)]
    net.logits(torch.tensor(sum(prompts, []), device="cuda"), blocks.sequences(split, slots=slots),
               states)
    seq = torch.tensor(slots, dtype=torch.int32, device="cuda")
    p = {k: v.double() for k, v in net.params.items()}
    runs, first = [], 0
    for w in whole:
        runs.append((first, len(w)))
        first += len(w)
    want = plain_logits(net, p, torch.tensor(sum(whole, []), device="cuda"), runs)
    for t in range(5):
        tokens = torch.tensor([w[s + t] for w, s in zip(whole, split)], device="cuda")
        got = net.logits(tokens, seq, states, single=True)
        for i, s in enumerate(split):
            row = want[i][s + t]
            assert (got[i].double() - row).norm() <= 1e-3 * row.norm(), (t, i)
