"""Log probabilities of rows that are masked with large finite values, on the
GPU: such a value has p = 0 beside ordinary logits, as -inf has, so everything
but its own log p is what -inf in its place gives.

Tolerances as in tests/test_gpu_logprob.py, in the size of the logits that are
not masked."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_logprob import DT, check_forward, check_gradient
from tests.training_testutil import f64

pytestmark = pytest.mark.gpu

# ordinary masks, powers of two, and values at which a rounded product z log2 e is off by 100 and more
MASKS = [-1e4, -1e9, -2.5e9, -1694498816.0, -2147483648.0, -3405774848.0, -1e10, -13086228480.0, -1e12, -1e30, -1e38, -3e38]


def make(rows, vocab, dtype, mask, spread):
    """Every row but the last masked; only a few logits of the first and about a
    third of the others' are not."""
    g = torch.Generator().manual_seed(vocab)
    z = 3 * torch.randn(rows, vocab, generator=g)
    hide = torch.rand(rows, vocab, generator=g) < 0.7
    hide[0] = True
    hide[0, torch.randperm(vocab, generator=g)[:4]] = False
    hide[-1] = False
    fill = torch.full_like(z, mask)
    if spread:
        fill *= 1 + torch.rand(rows, vocab, generator=g)          # masks added to logits, or scaled
        fill = fill.clamp(min=float(torch.finfo(DT[dtype]).min))
    hide, z, fill = hide.cuda(), z.to(DT[dtype]).cuda(), fill.to(DT[dtype]).cuda()
    masked, gone = torch.where(hide, fill, z), torch.where(hide, float("-inf"), z)
    y = gone.float().argmax(dim=1)
    return masked, gone, y, [torch.randn(rows, generator=g).cuda() for _ in range(3)]


@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("rows,vocab", [(3, 50304), (5, 1003), (153, 20100)])
def test_finite_masks(rows, vocab, mask, dtype, spread):
    from paper_2605_19811_gb300 import training as T
    z, gone, y, w = make(rows, vocab, dtype, mask, spread)
    check_forward(gone, y, T.token_logprob(z, y, top_k=4), 4)
    o = T.token_logprob(z, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2])
    check_forward(gone, y, o, 0)
    check_gradient(gone, y, o.dlogits, w, dtype)
    check_gradient(gone, y, T.token_logprob_grad(z, y, o.lse, o.entropy, w[0], w[1], w[2]), w, dtype)
    # a plain cross entropy: its gradient has no use for the entropy
    check_gradient(gone, y, T.token_logprob(z, y, g_logp=w[0]).dlogits, (w[0], None, None), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS)
def test_a_masked_target(mask, dtype):
    """log p of a masked token is its logit's distance from lse."""
    from paper_2605_19811_gb300 import training as T
    z, gone, _, w = make(4, 5000, dtype, mask, False)
    y = torch.tensor([int(torch.isinf(row).float().argmax()) for row in gone], device="cuda")
    o = T.token_logprob(z, y, g_logp=w[0])
    want = f64(z)[np.arange(4), y.cpu().numpy()] - f64(T.token_logprob(gone, y).lse)
    assert np.all(np.abs(f64(o.logp) - want) <= 2.0 ** -18 + 2.0 ** -22 * np.abs(want))
    check_gradient(gone, y, o.dlogits, (w[0], None, None), dtype)
