"""examples/train_and_attack.py: its search descends, and its gradients are those of what was kept."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "train_and_attack.py")
E = 2.0 ** -24


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("train_and_attack", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32],
                         ids=lambda t: str(t)[6:])
def test_search_descends_from_its_starts(ex, dtype):
    """With a linear margin of slope s a step reaches eps |s|_1, about 0.8 sqrt(96) = 7.8 eps |s|_2,
    and the best of 64 random points 2.4 standard deviations of 0.58 eps |s|_2: a fifth of it.  A
    search without slopes, or with their signs turned, gains nothing over its starts."""
    width, outputs, eps = 96, 4, 0.05
    net = ex.Net(width, 200, 2, outputs, dtype)
    ex.train(net, 30, 512, width, outputs, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for _ in range(3):
        x0 = torch.randn(width, generator=g, device="cuda")
        c = torch.zeros(outputs, device="cuda")
        y0 = net.forward(x0[None].to(dtype), keep=False)[0][0]
        c[y0.argmax()], c[y0.argmin()] = 1.0, -1.0
        margin = float(y0 @ c)
        starts, found = ex.attack(net, x0, eps, c, steps=0), ex.attack(net, x0, eps, c)
        assert starts < margin
        assert margin - found > 2 * (margin - starts)


def test_search_stays_in_the_box(ex):
    """Every point that is evaluated, as the net reads it."""
    dtype, width, eps = torch.bfloat16, 64, 0.05
    net = ex.Net(width, 136, 1, 2, dtype)
    x0 = 3 * torch.randn(width, generator=torch.Generator().manual_seed(1)).cuda()
    seen, forward = [], net.forward
    net.forward = lambda x, keep: (seen.append(x.clone()), forward(x, keep))[1]
    ex.attack(net, x0, eps, torch.tensor([1.0, -1.0], device="cuda"))
    assert len(seen) == 21
    for x in seen:
        assert x.dtype == dtype
        assert ((x.double() - x0.double()).abs() <= eps).all()


def test_gradients_of_what_was_kept(ex):
    """The net's gradients in 32 bits against the chain in 64 bits through the values kept in 8."""
    rows, width, hidden, outputs = 40, 64, 136, 3
    net = ex.Net(width, hidden, 2, outputs, torch.float32, seed=5)
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x = torch.randn(rows, width, generator=g, device="cuda")
    dy = torch.randn(rows, outputs, generator=g, device="cuda")
    _, tape = net.forward(x, keep=True)
    grads, dx = net.backward(dy, tape)
    last, steps = tape
    p = {k: w.double() for k, w in net.params.items()}
    want = {"out": dy.double().T @ last.double()}
    dh = dy.double() @ p["out"]
    for i in reversed(range(2)):
        h, rstd, kept = steps[i]
        vx, vg, vu = (t.values().double() for t in (kept.x, kept.g, kept.u))
        s = torch.sigmoid(vg)
        da = dh @ p[f"Wd{i}"]
        dg, du = da * vu * s * (1 + vg * (1 - s)), da * vg * s
        want[f"Wg{i}"], want[f"Wu{i}"] = dg.T @ vx, du.T @ vx
        want[f"Wd{i}"] = dh.T @ (vg * s * vu)
        dn = dg @ p[f"Wg{i}"] + du @ p[f"Wu{i}"]
        r, xhat = rstd.double()[:, None], h.double() * rstd.double()[:, None]
        want[f"norm{i}"] = (dn * xhat).sum(0)
        t = dn * p[f"norm{i}"]
        dh = dh + r * (t - xhat * (t * xhat).mean(1, keepdim=True))
    want["x"], grads["x"] = dh, dx
    assert set(grads) == set(want)
    # some 10 sums of at most 136 terms in a row, each off by (terms + 8) e of its magnitudes, which
    # are taken for 30 times the results (rows of both signs cancel to a fraction of theirs)
    for name, w in want.items():
        off = (grads[name].double().reshape(w.shape) - w).norm()
        assert off <= 10 * (136 + 8) * E * 30 * w.norm(), (name, float(off / w.norm()))
