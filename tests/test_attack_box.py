"""The points that examples/train_and_attack.py searches lie in the box (no GPU)."""
import importlib.util
import os

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "train_and_attack.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("train_and_attack", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def neighbour(v, dtype, up):
    """The next value of dtype, by its bits."""
    ints = {torch.bfloat16: torch.int16, torch.float16: torch.int16, torch.float32: torch.int32}
    bits = v.to(dtype).view(ints[dtype]).to(torch.int64)
    least = -(1 << (15 if dtype != torch.float32 else 31))
    order = torch.where(bits < 0, least - bits, bits) + (1 if up else -1)  # monotone in the value
    return torch.where(order < 0, least - order, order).to(ints[dtype]).view(dtype).double()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32],
                         ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("eps", [0.05, 0.3, 1e-2, 2.0])
def test_box_holds_the_values_inside_and_no_others(ex, dtype, eps):
    g = torch.Generator().manual_seed(3)
    x0 = torch.randn(20000, generator=g)
    x0[:64] = torch.cat([torch.linspace(-eps, eps, 32), torch.tensor([0.0, 1.0, -1.0, 2.0] * 8)])
    x0[64:128] *= 1e-3
    x0 = x0.clamp(-1.2, 1.2)
    lo, hi = ex.box(x0, eps, dtype)
    for v in (lo, hi):
        assert torch.equal(v.to(dtype).double(), v)
        assert ((v - x0.double()).abs() <= eps).all()
    # the next values outwards are outside
    assert ((neighbour(hi, dtype, True) - x0.double()) > eps).all()
    assert ((x0.double() - neighbour(lo, dtype, False)) > eps).all()


def test_box_without_a_value_is_refused(ex):
    with pytest.raises(ValueError, match="no value"):
        ex.box(torch.tensor([1.003]), 1e-3, torch.bfloat16)
