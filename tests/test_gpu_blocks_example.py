"""The blocks' operators together, as examples/train_and_attack.py runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "train_and_attack.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("train_and_attack", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(net, x, dtype=torch.float64):
    """The net's function in 64 bits."""
    p = {k: w.to(dtype) for k, w in net.params.items()}
    h = x
    for i in range(len(net.ffns)):
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-5) * p[f"norm{i}"]
        g = y @ p[f"Wg{i}"].T
        h = h + ((g * torch.sigmoid(g)) * (y @ p[f"Wu{i}"].T)) @ p[f"Wd{i}"].T
    return h @ p["out"].T


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32],
                         ids=lambda t: str(t)[6:])
def test_training_lowers_the_loss_and_the_search_the_margin(ex, dtype):
    losses, margin, least = ex.run(steps=40, width=96, hidden=200, rows=512, dtype=dtype)
    # the targets' mean square is about 1/2: a net that learned nothing stays above it
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5])
    assert least <= margin + 0.05 * abs(margin)


def test_gradient_of_the_net_by_differences(ex):
    """In 32 bits, but through activations kept in 8: a gradient through them is off by their
    steps, at most 1/127 of a group's largest value each."""
    net = ex.Net(64, 136, 2, 3, torch.float32, seed=5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    x = torch.randn(40, 64, generator=gen, device="cuda")
    dy = torch.randn(40, 3, generator=gen, device="cuda")
    y, tape = net.forward(x, keep=True)
    assert (y.double() - plain(net, x.double())).abs().max() < 1e-4
    grads, dx = net.backward(dy, tape)
    v = torch.randn(40, 64, generator=gen, device="cuda", dtype=torch.float64)
    s = 1e-6
    num = ((plain(net, x.double() + s * v) - plain(net, x.double() - s * v)) * dy.double()).sum()
    num = float(num) / (2 * s)
    got = float((dx.double() * v).sum())
    assert abs(num - got) <= 0.02 * float((dx.double() * v).norm()) * 40 ** 0.5
    for name in ("Wg0", "Wd1", "norm1", "out"):
        w = net.params[name]
        u = torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
        keep = w.clone()
        ends = []
        for sign in (1, -1):
            net.params[name] = keep.double() + sign * s * u
            ends.append(float((plain(net, x.double()) * dy.double()).sum()))
        net.params[name] = keep
        g = grads[name].double().reshape(w.shape)
        num = (ends[0] - ends[1]) / (2 * s)
        assert abs(num - float((g * u).sum())) <= 0.05 * float((g * u).norm()) * 5, name
