"""The 8-bit layers, the queries' and keys' operators and the head together, as
the attention example uses them: its gradients against torch's own automatic
differentiation of the same model, whose linear layers round what the example
rounds to 8 bits, in fp32 otherwise.

Tolerance of the gradients.  The example's values pass through bf16, some 40
roundings of 2^-9 one after another from the embedding through the loss and
back: about 1% in the mean square.  A value that is off by a relative 0.2% to 1%
falls on another 8-bit code with a chance of its error over the codes' spacing
(6 to 12%), and is then off by that spacing: the root of 0.01 / 0.09 times 9%,
up to 3% in the mean square for each of the layers' 8 forward and 8 backward
roundings, which add up as independent errors to 12% at most.  A short run's
losses are finite."""

import math
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
        import tiny_attention_lm
    finally:
        sys.path.pop(0)
    return tiny_attention_lm


def reference(m, model, x, y):
    from paper_2605_19811_gb300 import training as T
    kept = lambda t: T.checkpoint8(t.contiguous(), "e4m3").unpack(torch.float32)  # noqa: E731

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            x8, w8 = kept(x.detach()), T.weight8(w.detach()).unpack(torch.float32)
            ctx.save_for_backward(x8, w8)
            return x8 @ w8.t()

        @staticmethod
        def backward(ctx, dy):
            x8, w8 = ctx.saved_tensors
            return kept(dy) @ w8, dy.t() @ x8

    p = [t.float().requires_grad_() for t in model.params()]
    norm = lambda h, g: h * torch.rsqrt(h.square().mean(dim=-1, keepdim=True) + 1e-6) * g  # noqa: E731
    c, s = model.table[model.positions][:, None].unbind(-1)

    def turn(t):
        a, b = t.chunk(2, dim=-1)
        return torch.cat((a * c - b * s, b * c + a * s), dim=-1)

    h = p[0][x]
    for b in range(m.BLOCKS):
        n1, qkv, qg, kg, out, n2, up, down = p[1 + 8 * b:9 + 8 * b]
        t = Layer.apply(norm(h, n1), qkv).unflatten(1, (-1, m.DIM))
        q, k, v = t.split([m.HEADS, m.KEYS, m.KEYS], dim=1)
        q, k, v = (u.unflatten(0, (m.BATCH, m.LENGTH)).transpose(1, 2) for u in (turn(norm(q, qg)), turn(norm(k, kg)), v))
        o = torch.nn.functional.scaled_dot_product_attention(q, *(u.repeat_interleave(m.HEADS // m.KEYS, dim=1) for u in (k, v)), is_causal=True)
        h = h + Layer.apply(o.transpose(1, 2).reshape(m.TOKENS, -1), out)
        h = h + Layer.apply(torch.nn.functional.silu(Layer.apply(norm(h, n2), up)), down)
    z = norm(h, p[-2]) @ p[-1].t()
    loss = torch.nn.functional.cross_entropy(z, y, ignore_index=-1)
    return loss, torch.autograd.grad(loss, p)


def test_gradients_match_automatic_differentiation(example):
    model = example.TinyAttentionLM()
    x, y = example.tokens(123)
    loss, grads = model.loss_and_grads(x, y)
    want_loss, want = reference(example, model, x, y)
    assert abs(float(loss) - float(want_loss.detach())) <= 2e-2 * float(want_loss.detach())
    assert len(grads) == len(want) == len(model.params())
    for i, (g, w) in enumerate(zip(grads, want)):
        assert g.shape == w.shape
        rel = float((g.float() - w).norm() / w.norm())
        assert rel <= 0.12, (i, rel)


def test_a_run(example):
    losses = example.train(12, log=lambda *a: None)
    assert len(losses) == 12 and all(math.isfinite(v) for v in losses)


def test_a_step_in_a_graph(example):
    """The whole forward and backward pass captured once and replayed gives the eager call's bits."""
    model = example.TinyAttentionLM()
    x, y = example.tokens(5)
    model.loss_and_grads(x, y)
    other, other_y = example.tokens(6)
    want = model.loss_and_grads(other, other_y)[1]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, got = model.loss_and_grads(x, y)
    x.copy_(other)
    y.copy_(other_y)
    graph.replay()
    torch.cuda.synchronize()
    # (the embedding's index_add_ has no fixed order, and what it adds is compared instead)
    for g, w in list(zip(got, want))[1:]:
        assert torch.equal(g, w)
