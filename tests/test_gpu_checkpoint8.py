"""8-bit checkpoints and the weight gradient taken from them, on the GPU.

Packing and unpacking are compared bit for bit with the format's definition
(every step of it is exact or a single rounding).  The weight gradient's
tolerance, element by element, is a count of roundings times the sum of the
products' magnitudes A = |dY|^T |X|: a product of a bf16 piece of dY and a
bf16 value of X is exact in fp32; the tensor cores may lose a unit of the last
place (2^-23) at each addition of 16 tokens' products, and fp32 results sum at
most 512 tokens in one accumulator before its value is added to the others:
    fp32: (32 + T / 512 + 8) 2^-23 A          (three pieces a value for fp32 dY: 3 (..))
    bf16: (T / 16 + 8) 2^-23 A + 2^-8 |dW|"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.training_testutil import Held, checkpoint_values, code_values, f64, pack_reference

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def compare_pack(x, ck):
    vals, scales = pack_reference(f64(x), ck.format)
    np.testing.assert_array_equal(ck.scales.cpu().numpy().astype(np.float64).T[:ck.rows], scales)
    got = code_values(ck.codes.cpu().numpy()[:, :ck.cols].copy(), ck.format)
    np.testing.assert_array_equal(got, vals)


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 127), (2, 128), (5, 129), (4, 1000), (3, 4096), (700, 1283), (2, 20000)])
def test_pack_and_unpack(rows, cols, dtype, kind):
    from paper_2605_19811_gb300 import training as T
    g = torch.Generator().manual_seed(rows * cols)
    for pad, offset in ((0, 0), (3, 1), (8, 8)):
        x = Held(rows, cols, DT[dtype], pad, offset, torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, cols, generator=g)))
        ck = T.checkpoint8(x.t, kind)
        compare_pack(x.t, ck)
        want = checkpoint_values(ck)
        np.testing.assert_array_equal(f64(ck.unpack(torch.float32)), want)
        np.testing.assert_array_equal(f64(ck.unpack(torch.bfloat16)), want)      # exact in bf16
        out = Held(rows, cols, DT[dtype], pad + 1, offset)
        ck.unpack(out=out.t)
        np.testing.assert_array_equal(f64(out.t), want)
        assert out.untouched() and x.untouched()


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_pack_edges(kind):
    """Zeros, limits and their neighbours, ties, tiny and huge magnitudes, NaN and infinities."""
    from paper_2605_19811_gb300 import training as T
    limit = {"i8": 127.0, "e4m3": 448.0}[kind]
    x = torch.zeros(16, 256)
    x[1, :128] = limit
    x[2, 0] = float(np.nextafter(np.float32(limit), np.float32(1e9)))
    x[3, 0] = float(np.nextafter(np.float32(limit), np.float32(0)))
    x[4, :128] = torch.arange(128) + 0.5                      # ties
    x[4, 5] = 0.75 * limit
    x[5, :128] = -x[4, :128]
    x[6] = 1e-40                                              # subnormal
    x[7, 0], x[7, 1] = 1.0, 1e-30
    x[8] = torch.finfo(torch.float32).max
    x[9] = float(torch.finfo(torch.bfloat16).max)
    x[9, 3] = -1.0
    x[10, 3] = float("nan")
    x[11, 200] = float("-inf")
    x[12] = torch.linspace(-3, 3, 256)
    x[13] = 2.0 ** -120
    x[14, :128], x[14, 128:] = 1e-3, 1e3
    x[15] = 2.0 ** 127
    x = x.cuda()
    ck = T.checkpoint8(x, kind)
    compare_pack(x, ck)
    u = ck.unpack(torch.float32).cpu()
    assert bool(u[10, :128].isnan().all()) and bool((u[10, 128:] == 0).all())
    assert bool(u[11, 128:].isnan().all()) and bool((u[11, :128] == 0).all())
    fine = [r for r in range(16) if r not in (10, 11)]
    assert bool(torch.isfinite(u[fine]).all())
    np.testing.assert_array_equal(f64(u[fine]), checkpoint_values(ck)[fine])


def exact_wgrad(dy, ck, old=None):
    a, x = torch.from_numpy(f64(dy)).cuda(), torch.from_numpy(checkpoint_values(ck)).cuda()
    return f64(a.t() @ x) + (0.0 if old is None else f64(old)), f64(a.abs().t() @ x.abs()) + (0.0 if old is None else np.abs(f64(old)))


def check_wgrad(got, dy, ck, old=None):
    want, size = exact_wgrad(dy, ck, old)
    tokens = dy.shape[0]
    pieces = 3 if dy.dtype == torch.float32 else 1
    if got.dtype == torch.float32:
        tol = pieces * (32 + tokens / 512 + 8) * 2.0 ** -23 * size
    else:
        tol = pieces * (tokens / 16 + 8) * 2.0 ** -23 * size + 2.0 ** -8 * np.abs(want)
    worst = (np.abs(f64(got) - want) / (tol + 1e-37)).max()
    assert worst <= 1.0, worst


WGRAD = [(1, 1, 1), (1, 768, 96), (2, 16, 33), (15, 130, 129), (64, 128, 128), (65, 256, 256), (200, 257, 300), (1000, 513, 64),
         (1024, 768, 768), (4100, 640, 1000), (3000, 96, 2304), (700, 4096, 1280), (9000, 130, 70)]


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("dydt,to", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,out,cols", WGRAD)
def test_wgrad(tokens, out, cols, dydt, to, kind):
    from paper_2605_19811_gb300 import training as T
    g = torch.Generator().manual_seed(tokens + out + cols)
    for pad, offset, accumulate in ((0, 0, False), (5, 1, True), (8, 8, False)):
        dy = Held(tokens, out, DT[dydt], pad, offset, torch.randn(tokens, out, generator=g) * torch.exp(torch.randn(tokens, 1, generator=g)))
        ck = T.checkpoint8((torch.randn(tokens, cols, generator=g) * torch.exp(torch.randn(tokens, cols, generator=g))).cuda(), kind)
        w = Held(out, cols, DT[to], pad, offset, torch.randn(out, cols, generator=g))
        old = w.t.clone() if accumulate else None
        T.linear_wgrad8(dy.t, ck, out=w.t, accumulate=accumulate)
        check_wgrad(w.t, dy.t, ck, old)
        assert w.untouched() and dy.untouched()


def test_wgrad_wide_pitches_and_scales_of_another_pitch():
    """A checkpoint inside larger buffers: pitches beyond the extent, bytes and
    scales around it that are no numbers."""
    from paper_2605_19811_gb300 import training as T
    tokens, cols, out = 300, 200, 140
    base = T.checkpoint8(torch.randn(tokens, cols, device="cuda"), "e4m3")
    codes = torch.full((tokens + 2, 320), 0x7F, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, tokens + 9), float("nan"), device="cuda")
    codes[:tokens, :cols] = base.codes[:, :cols]
    scales[:, :tokens] = base.scales
    ck = T.Checkpoint8(codes[:tokens], scales, cols, "e4m3")
    dy = torch.randn(tokens, out, device="cuda", dtype=torch.bfloat16)
    a, b = T.linear_wgrad8(dy, base, dtype=torch.float32), T.linear_wgrad8(dy, ck, dtype=torch.float32)
    assert torch.equal(a, b)
    assert torch.equal(base.unpack(), ck.unpack())
    rstd = torch.ones(tokens, device="cuda")
    g = torch.randn(tokens, cols, device="cuda")
    for p, q in zip(T.rmsnorm_grad(g, base, rstd), T.rmsnorm_grad(g, ck, rstd)):
        assert torch.equal(p, q)


def test_wgrad_nonfinite_stays_where_it_belongs():
    """A NaN group reaches its 128 columns and a non-finite dy its row of dW; the rest is untouched."""
    from paper_2605_19811_gb300 import training as T
    tokens, cols, out = 130, 400, 300
    x = torch.randn(tokens, cols, device="cuda")
    x[70, 130] = float("inf")
    dy = torch.randn(tokens, out, device="cuda", dtype=torch.bfloat16)
    ck = T.checkpoint8(x, "i8")
    w = T.linear_wgrad8(dy, ck, dtype=torch.float32).cpu()
    assert bool(w[:, 128:256].isnan().all()) and bool(torch.isfinite(w[:, :128]).all()) and bool(torch.isfinite(w[:, 256:]).all())
    ck = T.checkpoint8(torch.randn(tokens, cols, device="cuda"), "i8")
    dy[5, 11] = float("nan")
    w = T.linear_wgrad8(dy, ck, dtype=torch.float32).cpu()
    assert bool(w[11].isnan().all()) and bool(torch.isfinite(w[:11]).all()) and bool(torch.isfinite(w[12:]).all())
    dy32 = torch.randn(tokens, out, device="cuda")
    dy32[5, 11] = float("inf")
    w = T.linear_wgrad8(dy32, ck, dtype=torch.float32).cpu()
    assert not bool(torch.isfinite(w[11]).any()) and bool(torch.isfinite(w[:11]).all()) and bool(torch.isfinite(w[12:]).all())


def test_wgrad_no_tokens():
    from paper_2605_19811_gb300 import training as T
    ck = T.Checkpoint8.empty(0, 96, "i8")
    dy = torch.empty(0, 40, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(40, 96, device="cuda")
    T.linear_wgrad8(dy, ck, out=w, accumulate=True)
    assert bool((w == 1).all())
    T.linear_wgrad8(dy, ck, out=w)
    assert bool((w == 0).all())


@pytest.mark.parametrize("to", ["bf16", "f32"])
def test_wgrad_same_bits_twice_on_another_stream_and_in_a_graph(to):
    from paper_2605_19811_gb300 import training as T
    dy = torch.randn(6000, 700, device="cuda", dtype=torch.bfloat16)
    ck = T.checkpoint8(torch.randn(6000, 520, device="cuda"), "e4m3")
    a = T.linear_wgrad8(dy, ck, dtype=DT[to])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = T.linear_wgrad8(dy, ck, dtype=DT[to], stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = T.linear_wgrad8(dy, ck, dtype=DT[to])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_wgrad_gradient_against_differences():
    """dW is linear in dY: the loss sum(dY * (X W^T)) changes by <dW, V> for a
    change V of W, exactly; both sides in 64 bits but for dW's own roundings."""
    from paper_2605_19811_gb300 import training as T
    dy = torch.randn(300, 60, device="cuda")
    ck = T.checkpoint8(torch.randn(300, 90, device="cuda"), "i8")
    w = T.linear_wgrad8(dy, ck, dtype=torch.float32)
    x = checkpoint_values(ck)
    g = np.random.default_rng(0)
    W, V = g.standard_normal((60, 90)), g.standard_normal((60, 90))
    loss = lambda m: float((f64(dy) * (x @ m.T)).sum())  # noqa: E731
    _, size = exact_wgrad(dy, ck)
    assert abs((loss(W + V) - loss(W - V)) / 2 - float((f64(w) * V).sum())) <= 3 * 48 * 2.0 ** -23 * float((size * np.abs(V)).sum())
