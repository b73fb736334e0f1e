"""A small language model trained with the optimizer and the training-step
operators: what makes the gradients that ``lm_step`` takes.

Two residual blocks of RMS norm and MLP over random-walk tokens.  The forward
pass keeps activations in 8 bits (the norms' outputs and the MLPs' hidden
values), the loss and its gradient come from one call over the logits, weight
gradients from the 8-bit checkpoints, norm gradients from the residual stream;
the matrices then take the Muon or Lion step, the norm gains the Lion step.

    python examples/tiny_lm.py [steps]
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_19811_gb300 import lionmuon as L  # noqa: E402
from paper_2605_19811_gb300 import training as T  # noqa: E402

VOCAB, WIDTH, HIDDEN, BLOCKS, TOKENS = 509, 256, 1024, 2, 4096


def tokens(step: int):
    """Inputs and targets: a walk over the vocabulary whose next token is one of
    four, three of them rare; an eighth of the positions carries no target."""
    g = torch.Generator(device="cuda").manual_seed(step)
    x = torch.randint(0, VOCAB, (TOKENS,), device="cuda", generator=g)
    hop = torch.randint(0, 16, (TOKENS,), device="cuda", generator=g).clamp(max=3)
    y = (3 * x + 7 * hop + 1) % VOCAB
    y[torch.rand(TOKENS, device="cuda", generator=g) < 1 / 8] = -1
    return x, y


class TinyLM:
    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(0)
        mat = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[-1] ** -0.5).bfloat16()  # noqa: E731
        self.embed = (torch.randn(VOCAB, WIDTH, device="cuda", generator=g)).bfloat16()
        self.blocks = [(torch.ones(WIDTH, device="cuda", dtype=torch.bfloat16), mat(HIDDEN, WIDTH), mat(WIDTH, HIDDEN)) for _ in range(BLOCKS)]
        self.gain = torch.ones(WIDTH, device="cuda", dtype=torch.bfloat16)
        self.head = mat(VOCAB, WIDTH)

    def params(self):
        return [self.embed, *(p for b in self.blocks for p in b), self.gain, self.head]

    def loss_and_grads(self, x, y):
        """Mean -log p of the targets, and the gradients in params() order."""
        h, r, kept = self.embed[x], None, []
        for gain, up, down in self.blocks:
            n = T.rmsnorm(h, gain, residual=r, checkpoint="e4m3")
            u = n.y @ up.t()
            a = torch.nn.functional.gelu(u, approximate="tanh")
            kept.append((n, u, T.checkpoint8(a, "i8")))
            h, r = n.h, a @ down.t()
        last = T.rmsnorm(h, self.gain, residual=r, checkpoint="e4m3")
        count = (y >= 0).sum().clamp(min=1)
        weight = (-1.0 / count).expand(len(y)).contiguous()
        out = T.token_logprob(last.y @ self.head.t(), y, g_logp=weight)
        loss = -out.logp.sum() / count

        dhead = T.linear_wgrad8(out.dlogits, last.checkpoint)
        dh, dgain = T.rmsnorm_grad(out.dlogits @ self.head, last.h, last.rstd, self.gain)
        grads = [dgain, dhead]
        for (gain, up, down), (n, u, a8) in zip(reversed(self.blocks), reversed(kept)):
            ddown = T.linear_wgrad8(dh, a8)                     # dh is the gradient of the block's output as well
            t = torch.tanh(0.7978845608 * (u.float() + 0.044715 * u.float() ** 3))
            slope = 0.5 * (1 + t) + 0.5 * u.float() * (1 - t * t) * 0.7978845608 * (1 + 0.134145 * u.float() ** 2)
            du = ((dh @ down).float() * slope).bfloat16()
            dup = T.linear_wgrad8(du, n.checkpoint)
            dh, dg = T.rmsnorm_grad(du @ up, n.h, n.rstd, gain, dh=dh)
            grads = [dg, dup, ddown] + grads
        dembed = torch.zeros(VOCAB, WIDTH, device="cuda").index_add_(0, x, dh.float())
        return loss, [dembed.bfloat16()] + grads


def train(steps: int = 60, log=print):
    """Losses of the first and the last steps."""
    model = TinyLM()
    opt = L.LionMuon(model.params(), period=2, eta_muon=2e-2, eta_lion=2e-3, weight_decay=0.01)
    losses = []
    for step in range(steps):
        loss, grads = model.loss_and_grads(*tokens(step))
        opt.step(grads, step)
        losses.append(loss)                                     # read at the end: no step waits for the device
    losses = [float(v) for v in losses]
    if opt.status() != 0:
        raise RuntimeError("device status flags set")
    opt.close()
    for step in range(0, steps, 10):
        log(f"step {step:4d}  loss {losses[step]:.4f}")
    log(f"step {steps - 1:4d}  loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
