"""The 8-bit operators and the draws run together, as the example does: its
rounds, and one step's gradients against autograd in binary64."""
import importlib.util
import os

import pytest
import torch

from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("online_selection", os.path.join(ROOT, "examples", "online_selection.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_rounds():
    lines = []
    regrets = example().run("tiny", rounds=4, say=lines.append)
    assert len(regrets) == len(lines) == 4 and all(0.0 <= r <= 1.0 for r in regrets)
    assert regrets[-1] <= regrets[0]


def test_step_follows_the_gradient():
    """Weight updates against autograd in binary64 on unquantised values.  Every
    operand of a gradient has been rounded to 3 (E4M3) or 2 (E5M2) digits two or
    three times on its way: 2^-4 and 2^-3 at most for one element of random
    sign, some 7 % of the norm together; 20 % is asked, and a cosine of 0.98."""
    ex = example()
    g = torch.Generator(device="cuda").manual_seed(5)
    net = ex.Net(96, g, "cuda")
    x = torch.randn(700, 96, generator=g, device="cuda")
    target = torch.randn(700, generator=g, device="cuda")
    W = [w.double().clone().requires_grad_() for w in net.W]
    b = [v.double().clone().requires_grad_() for v in net.b]
    h = x.double()
    for i in (0, 1):
        h = torch.nn.functional.gelu(h @ W[i].t() + b[i])
    y = (h @ W[2].t() + b[2])[:, 0]
    ((y - target.double()) ** 2).sum().mul(0.5 / 700).backward()
    y = y.detach()
    got, inputs = net.forward(hwsel.hwsel_fp8_quantise(x))
    assert float((got.double() - y).norm() / y.norm()) < 0.1
    before = [t.clone() for t in net.W + net.b]
    net.step(inputs, ((got - target) / 700).detach(), 1.0)
    for was, now, want in zip(before, net.W + net.b, W + b):
        step, grad = (was - now).double().flatten(), want.grad.flatten()
        assert float((step - grad).norm()) <= 0.2 * float(grad.norm())
        assert float(step @ grad) >= 0.98 * float(step.norm() * grad.norm())
