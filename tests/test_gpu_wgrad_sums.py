"""The weight gradient's sum over tokens, on the GPU: held in 32 bits whatever
its length and the type of dW.

Operands of one sign, so that errors of one sign show.  The tensor cores drop
up to a unit of the last place (2^-23) at each addition of 16 tokens; a sum of
512 tokens has 32 of them and grows along the way, so at most 16 units are lost
on average over it: 2^-19.  Those sums are added in fp32, half a unit an
addition: fewer than 2048 additions are off by at most 2^-13 together, and
without a preferred sign.  A bf16 result is off by at most 2^-8 more, half a
unit, and that without a preferred sign too (channels have scales of their own,
so that results fall anywhere between two bf16 numbers): the mean over n
elements by 2^-8 / sqrt(3 n) in the mean square, five times that allowed.  None
of it grows with the tokens."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def relative(tokens, out, cols, dydt, to, kind):
    """(dW - dY^T X) / dY^T X against 64 bits."""
    from paper_2605_19811_gb300 import training as T
    g = torch.Generator(device="cuda").manual_seed(tokens)
    own = lambda n: torch.exp(torch.rand(n, device="cuda", generator=g))  # noqa: E731
    dy = ((torch.rand(tokens, out, device="cuda", generator=g) + 0.5) * own(out)).to(dydt)
    ck = T.checkpoint8((torch.rand(tokens, cols, device="cuda", generator=g) + 0.5) * own(cols), kind)
    w = T.linear_wgrad8(dy, ck, dtype=to)
    want = torch.zeros(out, cols, device="cuda", dtype=torch.float64)
    x = ck.unpack(torch.float32)
    for at in range(0, tokens, 1 << 15):
        want += dy[at:at + (1 << 15)].double().t() @ x[at:at + (1 << 15)].double()
    return (w.double() - want) / want


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("dydt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,out,cols", [(16384, 768, 2304), (16385, 300, 70), (300001, 40, 24), (300000, 512, 256)])
def test_bf16_results_of_long_sums(tokens, out, cols, dydt, kind):
    rel = relative(tokens, out, cols, dydt, torch.bfloat16, kind)
    assert float(rel.abs().max()) <= 2.0 ** -8 + 2.0 ** -13 + 2.0 ** -18
    assert abs(float(rel.mean())) <= 2.0 ** -18 + 5 * 2.0 ** -8 / (3 * out * cols) ** 0.5


def test_a_long_sum_that_one_pair_takes_whole():
    """A whole wave of tiles, so that no other pair takes a part of a tile's tokens."""
    rel = relative(100000, 9728, 512, torch.bfloat16, torch.bfloat16, "i8")
    assert float(rel.abs().max()) <= 2.0 ** -8 + 2.0 ** -13 + 2.0 ** -18
    assert abs(float(rel.mean())) <= 2.0 ** -18 + 5 * 2.0 ** -8 / (3 * 9728 * 512) ** 0.5


@pytest.mark.parametrize("dydt", [torch.bfloat16, torch.float32])
def test_fp32_results_of_long_sums(dydt):
    rel = relative(300001, 40, 24, dydt, torch.float32, "i8")
    assert float(rel.abs().max()) <= 2.0 ** -13 + 2.0 ** -18


@pytest.mark.parametrize("dydt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,out,cols", [(513, 20000, 1300), (1100, 5120, 4096)])
def test_bf16_results_of_many_tiles(tokens, out, cols, dydt):
    """Several tiles a pair, a whole wave of them and more, each with a sum that is cut."""
    rel = relative(tokens, out, cols, dydt, torch.bfloat16, "e4m3")
    assert float(rel.abs().max()) <= 2.0 ** -8 + 2.0 ** -13 + 2.0 ** -18
