"""The example with a norm and with its table in 8 bits: it runs from training to words, and its
gradients are those of the formulas."""
import importlib.util
import os

import numpy as np
import pytest

from conftest import ROOT
from oracle import layers as ref

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    path = os.path.join(ROOT, "examples", "language_model.py")
    spec = importlib.util.spec_from_file_location("language_model_layers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("normed,eight_bits", [(True, False), (False, True), (True, True)])
def test_runs(example, normed, eight_bits):
    r = example.main(steps=20, sequences=16, length=6, normed=normed, eight_bits=eight_bits)
    words = r["words"]
    assert tuple(words.shape) == (16, example.CONTEXT + 6)
    assert int(words.min()) >= example.SPECIAL and int(words.max()) < example.VOCABULARY
    assert 0 < r["chance"] <= 1 and np.isfinite(r["last"])


@pytest.mark.parametrize("use_h", [False, True])
def test_norm_gradients(example, use_h):
    """Through autograd, against the formulas in 64 bits: the tolerances of the operators' own tests
    (chains of 38 additions over 64 columns), and one more addition for the two uses of h."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)

    def draw(*shape):
        return torch.randn(shape, device="cuda", generator=g)
    x, r, w = (t.requires_grad_() for t in (draw(9, 64), draw(9, 64), draw(64)))
    a, b = draw(9, 64), draw(9, 64)
    y, h = example.Norm.apply(x, r, w, 1e-5)
    loss = (y * a).sum() + ((h * b).sum() if use_h else 0.0)
    loss.backward()
    num = [t.detach().double().cpu().numpy() for t in (x, r, w, a, b)]
    dx, dw, size, size_w = ref.norm_grad(num[3], num[0] + num[1], num[2], 1e-5,
                                         num[4] if use_h else None)
    # (h is rounded once before its gradient is taken: 4 eps of each term)
    slack = size * (2 * 38 + 21) * EPS
    for got in (x.grad, r.grad):
        assert (np.abs(got.double().cpu().numpy() - dx) <= slack).all()
    assert (np.abs(w.grad.double().cpu().numpy() - dw) <= size_w * (80 + 38 + 15) * EPS).all()


def test_model_gradients_against_differences(example):
    """The whole normed model's loss by its gain and inner weights, in float: a step of 2^-6 of
    a unit leaves its third differences (under 1e-3 of the gradient's own size here) and the
    loss's rounding, 64 words' 2^-22, over twice the step."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    model = example.Model(g, normed=True)
    rows = torch.randn(32 * example.CONTEXT, example.WIDTH, device="cuda", generator=g)
    target = torch.randint(0, example.VOCABULARY, (32,), device="cuda", generator=g)

    def loss():
        return torch.nn.functional.cross_entropy(model.logits(rows).double(), target)
    loss().backward()
    step = 2.0 ** -6
    for p in (model.gain, model.outer):
        direction = torch.randn(p.shape, device="cuda", generator=g)
        direction /= direction.norm()
        with torch.no_grad():
            p += step * direction
            up = float(loss())
            p -= 2 * step * direction
            down = float(loss())
            p += step * direction
        want = (up - down) / (2 * step)
        got = float((p.grad * direction).sum())
        assert abs(got - want) < 2e-3 * float(p.grad.norm()) + 1e-4, (got, want)
