"""Log probabilities whose logits lie far from zero, on the GPU: log p, the
entropy and the gradient depend on differences of logits alone, so their errors
do not grow with the logits' size (the logits are fp32 numbers, exact in the
64-bit reference).

Tolerances, u = 2^-24.  With d = (z - max) log2 e and S = sum 2^d, log p is
ln 2 (d - log2 S): d, log2 S, their difference and the product are rounded
once, at most u (3 |log p| + log V) in all, and the two constants' product is off
from 1 by less than u.  S is off by its exponentials' 2^-22 and as much for its
additions (some hundred a thread, independent over 256 threads):
    log p    2^-21 + u (4 |log p| + log V)
The entropy log S - T / S adds T's error, the same relative to terms that sum
to at most H + 1:
    entropy  2^-20 (2 + H)
A gradient p (..) is off by log p's error relatively, its exponential, and half
a unit."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.training_testutil import f64, logprob_gradient

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(rows, vocab, shift, seed=0):
    """Rows around shift, each at its own distance; some tokens of each lifted so
    that they carry about half of the probability."""
    g = torch.Generator().manual_seed(vocab + seed)
    z = torch.randn(rows, vocab, generator=g) + shift * (1 + 0.25 * torch.rand(rows, 1, generator=g))
    y = torch.randint(0, vocab, (rows,), generator=g)
    z[torch.arange(rows), y] += float(np.log(vocab)) + 1.0
    w = [torch.randn(rows, generator=g).cuda() for _ in range(3)]
    return z.cuda(), y.cuda(), w


def exact(z):
    """log p, entropy and lse of every row in 64 bits."""
    d = f64(z) - f64(z).max(axis=1, keepdims=True)
    ls = np.log(np.exp(d).sum(axis=1, keepdims=True))
    lp = d - ls
    return lp, -(np.exp(lp) * lp).sum(axis=1), (f64(z).max(axis=1, keepdims=True) + ls)[:, 0]


SHIFTS = [0.0, 20.0, -100.0, 100.0, 1000.0, -3000.0, 20000.0]
SIZES = [(64, 49152), (300, 3001), (2, 131072)]


@pytest.mark.parametrize("shift", SHIFTS)
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_log_p_entropy_and_gradient_do_not_depend_on_the_size_of_logits(rows, vocab, shift):
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(rows, vocab, shift)
    lp, ent, lse = exact(z)
    r, t = np.arange(rows), y.cpu().numpy()
    tol = lambda q: 2.0 ** -21 + U * (4 * np.abs(q) + np.log(vocab))  # noqa: E731
    o = T.token_logprob(z, y, top_k=4, g_logp=w[0], g_entropy=w[1], g_lse=w[2])
    worst = {"log p": (np.abs(f64(o.logp) - lp[r, t]) / tol(lp[r, t])).max(),
             "entropy": (np.abs(f64(o.entropy) - ent) / (2.0 ** -20 * (2 + ent))).max()}
    best = np.take_along_axis(lp, o.top_index.cpu().numpy(), axis=1)
    worst["alternatives"] = (np.abs(f64(o.top_logp) - best) / tol(best)).max()
    want = logprob_gradient(f64(z), t, lse, ent, *(f64(x) for x in w))
    gl, gh, gz = (np.abs(f64(x))[:, None] for x in w)
    size = gz + gl + gh * (np.abs(lp) + ent[:, None] + 1)
    worst["gradient"] = (np.abs(f64(o.dlogits) - want) /
                         ((2.0 ** -20 + 2 * tol(lp)) * np.exp(lp) * size + 2 * U * np.abs(want) + 1e-37)).max()
    assert max(worst.values()) <= 1.0, worst


@pytest.mark.parametrize("shift", SHIFTS)
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_lse_is_rounded_once(rows, vocab, shift):
    """lse = max + log S: log S off as above, and half a unit of lse."""
    from paper_2605_19811_gb300 import training as T
    z, y, _ = make(rows, vocab, shift, seed=1)
    _, _, lse = exact(z)
    got = f64(T.token_logprob(z, y).lse)
    worst = (np.abs(got - lse) / (U * np.abs(lse) + 2.0 ** -21 + 2 * U * np.log(vocab))).max()
    assert worst <= 1.0, worst
