"""Non-finite gradients in the weight gradient, on the GPU: an infinite dY gives
what dY^T X is, an infinity with the sign of its product (NaN where X is zero
or infinities of both signs meet), the same for dY in bf16 and in fp32."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dydt", [torch.bfloat16, torch.float32])
def test_infinite_gradients(dydt, to):
    from paper_2605_19811_gb300 import training as T
    tokens, out, cols = 700, 300, 150
    g = torch.Generator().manual_seed(9)
    x = torch.randn(tokens, cols, generator=g)
    x[5, 17] = 0.0
    ck = T.checkpoint8(x.cuda(), "i8")
    dy = torch.randn(tokens, out, generator=g)
    inf = float("inf")
    dy[5, 11], dy[600, 12], dy[6, 13] = inf, -inf, float("nan")
    dy[7, 14], dy[650, 14] = inf, -inf
    dy[8, 15] = torch.finfo(dydt).max
    w = T.linear_wgrad8(dy.to(dydt).cuda(), ck, dtype=to).cpu()
    q = ck.unpack(torch.float32).cpu()
    for row, token, sign in ((11, 5, 1.0), (12, 600, -1.0)):
        want = sign * torch.sign(q[token]) * inf                     # NaN where q is 0
        assert torch.equal(w[row].float().nan_to_num(7.0, inf, -inf), want.nan_to_num(7.0, inf, -inf))
    assert bool(w[13].isnan().all())
    meet = torch.sign(q[7]) * inf - torch.sign(q[650]) * inf
    assert torch.equal(w[14].float().nan_to_num(7.0, inf, -inf), meet.nan_to_num(7.0, inf, -inf))
    rest = [r for r in range(out) if r not in (11, 12, 13, 14, 15)]
    assert bool(torch.isfinite(w[rest]).all())
