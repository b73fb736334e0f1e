"""The training-step operators and the optimizer together, as the example uses
them: its gradients against torch's own automatic differentiation of the same
model in fp32, and a short run whose loss falls.

Tolerance of the gradients: activations pass through bf16 (2^-9 a rounding, a
handful in a row) and the kept copies through 8 bits (e4m3: up to 2^-4 an
element, about 2.6% in the mean square; int8: about 1%), and these errors are
independent from token to token; 8% of a gradient's norm allowed."""

import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import tiny_lm
    finally:
        sys.path.pop(0)
    return tiny_lm


def reference(m, model, x, y):
    p = [t.float().requires_grad_() for t in model.params()]

    def norm(h, g):
        return h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + 1e-6) * g

    h = p[0][x]
    for b in range(m.BLOCKS):
        g, up, down = p[1 + 3 * b: 4 + 3 * b]
        h = h + torch.nn.functional.gelu(norm(h, g) @ up.t(), approximate="tanh") @ down.t()
    z = norm(h, p[-2]) @ p[-1].t()
    loss = torch.nn.functional.cross_entropy(z, y, ignore_index=-1)
    return loss, torch.autograd.grad(loss, p)


def test_gradients_match_automatic_differentiation(example):
    model = example.TinyLM()
    x, y = example.tokens(123)
    loss, grads = model.loss_and_grads(x, y)
    want_loss, want = reference(example, model, x, y)
    assert abs(float(loss) - float(want_loss)) <= 1e-2 * float(want_loss)
    for i, (g, w) in enumerate(zip(grads, want)):
        assert g.shape == w.shape
        rel = float((g.float() - w).norm() / w.norm())
        assert rel <= 8e-2, (i, rel)


def test_loss_falls(example):
    losses = example.train(40, log=lambda *a: None)
    assert losses[-1] < 0.75 * losses[0], losses
