"""A small language model with attention, trained with the optimizer and the
training-step operators: every linear layer's forward product and input gradient
in 8 bits, its weight gradient from the 8-bit activations, queries and keys
normed and turned in one pass, the loss from the last hidden states without
logits.  (The attention itself, which the library leaves to its user, is written
out in torch.)

    python examples/tiny_attention_lm.py [steps]
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_19811_gb300 import lionmuon as L  # noqa: E402
from paper_2605_19811_gb300 import training as T  # noqa: E402

VOCAB, WIDTH, HIDDEN, BLOCKS, BATCH, LENGTH = 509, 256, 1024, 2, 16, 256
HEADS, KEYS, DIM = 8, 4, 64
TOKENS, QKV = BATCH * LENGTH, (HEADS + 2 * KEYS) * DIM


def tokens(step: int):
    """Inputs and targets: the next token is the one before the last plus a rare
    hop, so that attention has something to find."""
    g = torch.Generator(device="cuda").manual_seed(step)
    x = torch.randint(0, VOCAB, (BATCH, LENGTH + 1), device="cuda", generator=g)
    hop = (torch.rand(BATCH, LENGTH + 1, device="cuda", generator=g) < 0.1).long()
    for t in range(2, LENGTH + 1):
        x[:, t] = (x[:, t - 2] + hop[:, t]) % VOCAB
    return x[:, :-1].reshape(-1), x[:, 1:].reshape(-1).contiguous()


class Linear:
    """y = x W^T in 8 bits: W is packed once a step, x comes as a checkpoint."""

    def __init__(self, w):
        self.w = w

    def forward(self, x: T.Checkpoint8):
        self.kept, self.w8 = x, T.weight8(self.w)
        return T.linear8(x, self.w8)

    def backward(self, dy):
        return T.linear8_grad(T.checkpoint8(dy, "e4m3"), self.w8), T.linear_wgrad8(dy, self.kept)


def attend(q, k, v):
    """Causal attention of (batch, heads, length, dim) in fp32, and its probabilities."""
    k, v = (t.repeat_interleave(HEADS // KEYS, dim=1) for t in (k, v))
    s = (q @ k.transpose(2, 3)) * DIM ** -0.5
    s = s.masked_fill(torch.ones(LENGTH, LENGTH, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
    p = (s - s.amax(dim=-1, keepdim=True)).exp()
    p = p / p.sum(dim=-1, keepdim=True)
    return p @ v, p


def attend_grad(do, q, k, v, p):
    k2, v2 = (t.repeat_interleave(HEADS // KEYS, dim=1) for t in (k, v))
    dp = do @ v2.transpose(2, 3)
    ds = p * (dp - (dp * p).sum(dim=-1, keepdim=True)) * DIM ** -0.5
    fold = lambda t: t.unflatten(1, (KEYS, HEADS // KEYS)).sum(dim=2)  # noqa: E731
    return ds @ k2, fold(ds.transpose(2, 3) @ q), fold(p.transpose(2, 3) @ do)


def split(t):
    """(tokens, heads, dim) to (batch, heads, length, dim) in fp32, and back."""
    return t.view(BATCH, LENGTH, -1, DIM).transpose(1, 2).float()


def join(t):
    return t.transpose(1, 2).reshape(TOKENS, -1, DIM).bfloat16()


class TinyAttentionLM:
    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(0)
        mat = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[-1] ** -0.5).bfloat16()  # noqa: E731
        one = lambda n: torch.ones(n, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        self.embed = torch.randn(VOCAB, WIDTH, device="cuda", generator=g).bfloat16()
        self.blocks = [dict(n1=one(WIDTH), qkv=Linear(mat(QKV, WIDTH)), q=one(DIM), k=one(DIM), out=Linear(mat(WIDTH, HEADS * DIM)),
                            n2=one(WIDTH), up=Linear(mat(HIDDEN, WIDTH)), down=Linear(mat(WIDTH, HIDDEN))) for _ in range(BLOCKS)]
        self.gain = one(WIDTH)
        self.head = mat(VOCAB, WIDTH)
        self.positions = torch.arange(LENGTH, device="cuda").repeat(BATCH)
        self.table = T.rotary_table(LENGTH, T.rotary_frequencies(DIM))

    def params(self):
        return [self.embed, *(p.w if isinstance(p, Linear) else p for b in self.blocks for p in b.values()), self.gain, self.head]

    def loss_and_grads(self, x, y):
        """Mean -log p of the targets, and the gradients in params() order."""
        h, r, kept = self.embed[x], None, []
        for b in self.blocks:
            n1 = T.rmsnorm(h, b["n1"], residual=r, checkpoint="e4m3", y=False)
            qkv = b["qkv"].forward(n1.checkpoint)
            q, k, v = (t.unflatten(1, (-1, DIM)) for t in qkv.split([HEADS * DIM, KEYS * DIM, KEYS * DIM], dim=1))
            turned = T.qk_rotary(q, k, self.positions, self.table, b["q"], b["k"])
            qs, ks, vs = split(turned.q), split(turned.k), split(v)
            o, p = attend(qs, ks, vs)
            a = b["out"].forward(T.checkpoint8(join(o).flatten(1), "e4m3"))
            n2 = T.rmsnorm(n1.h, b["n2"], residual=a, checkpoint="e4m3", y=False)
            u = b["up"].forward(n2.checkpoint)
            act = torch.nn.functional.silu(u.float())
            kept.append((n1, q, k, qs, ks, vs, p, n2, u))
            h, r = n2.h, b["down"].forward(T.checkpoint8(act.bfloat16(), "e4m3"))
        last = T.rmsnorm(h, self.gain, residual=r)
        count = (y >= 0).sum().clamp(min=1)
        out = T.linear_logprob(last.y, self.head, y, g_logp=(-1.0 / count).expand(TOKENS).contiguous())
        loss = -out.logp.sum() / count

        dh, dgain = T.rmsnorm_grad(out.dh, last.h, last.rstd, self.gain)
        grads = [dgain, out.dweight]
        for b, (n1, q, k, qs, ks, vs, p, n2, u) in zip(reversed(self.blocks), reversed(kept)):
            da, ddown = b["down"].backward(dh)                  # dh is the gradient of the block's output as well
            s = torch.sigmoid(u.float())
            du = (da.float() * s * (1 + u.float() * (1 - s))).bfloat16()
            dn, dup = b["up"].backward(du)
            dh, dn2 = T.rmsnorm_grad(dn, n2.h, n2.rstd, b["n2"], dh=dh)
            do, dout = b["out"].backward(dh)
            dqs, dks, dvs = attend_grad(split(do.unflatten(1, (-1, DIM))), qs, ks, vs, p)
            dqkv = torch.empty(TOKENS, QKV, device="cuda", dtype=torch.bfloat16)
            dq, dk, dv = (t.unflatten(1, (-1, DIM)) for t in dqkv.split([HEADS * DIM, KEYS * DIM, KEYS * DIM], dim=1))
            turned = T.qk_rotary_grad(join(dqs), join(dks), self.positions, self.table, q, k, b["q"], b["k"], dq_out=dq, dk_out=dk)
            dv.copy_(join(dvs))
            dn, dwqkv = b["qkv"].backward(dqkv)
            dh, dn1 = T.rmsnorm_grad(dn, n1.h, n1.rstd, b["n1"], dh=dh)
            grads = [dn1, dwqkv, turned.dq_weight, turned.dk_weight, dout, dn2, dup, ddown] + grads
        dembed = torch.zeros(VOCAB, WIDTH, device="cuda").index_add_(0, x, dh.float())
        return loss, [dembed.bfloat16()] + grads


def train(steps: int = 60, log=print):
    """The losses of all steps."""
    model = TinyAttentionLM()
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
