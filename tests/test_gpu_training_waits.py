"""The weight gradient's bounded waits: under a limit that every wait passes at
once (1 ns) the call ends, the context stays usable, and what was not computed
is NaN, never a wrong number; without the limit the same call is right."""

import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("to", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,out,cols", [(2048, 512, 768), (300, 4096, 4096)])
def test_wgrad_wait_that_gives_up(tokens, out, cols, to, monkeypatch):
    from paper_2605_19811_gb300 import training as T
    dy = torch.randn(tokens, out, device="cuda", dtype=torch.bfloat16)
    ck = T.checkpoint8(torch.randn(tokens, cols, device="cuda"), "i8")
    right = T.linear_wgrad8(dy, ck, dtype=to)
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    w = T.linear_wgrad8(dy, ck, dtype=to)
    torch.cuda.synchronize()
    assert bool((w.isnan() | (w == right)).all())
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    assert torch.equal(T.linear_wgrad8(dy, ck, dtype=to), right)
