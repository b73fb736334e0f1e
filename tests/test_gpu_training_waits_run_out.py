"""A limit of 1 ns on the weight gradient's waits is felt: some wait gives up
and leaves NaN, in the wait test's own sizes, and the next call is right."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("to", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,out,cols", [(2048, 512, 768), (300, 4096, 4096)])
def test_some_wait_gives_up(tokens, out, cols, to, monkeypatch):
    from paper_2605_19811_gb300 import training as T
    dy = torch.randn(tokens, out, device="cuda", dtype=torch.bfloat16)
    ck = T.checkpoint8(torch.randn(tokens, cols, device="cuda"), "i8")
    right = T.linear_wgrad8(dy, ck, dtype=to)
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    w = T.linear_wgrad8(dy, ck, dtype=to)
    torch.cuda.synchronize()
    assert bool(w.isnan().any())
    assert bool((w.isnan() | (w == right)).all())
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    assert torch.equal(T.linear_wgrad8(dy, ck, dtype=to), right)
