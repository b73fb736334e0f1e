"""8-bit weights and the linear layer's products with them.

Codes and scales are compared bit by bit with the definition in 64 bits.  A
product of two codes is exact.  The tensor cores drop up to 2^-23 of what they
have at each addition of 32 products, at most 64 additions in a row, then fp32
additions (2^-24) of such sums; nothing they have is above S = sum |x w|: together
at most S (2^-17 + k / 512 2^-24).  Of a sum of one sign they have half on
average, so that half as much is dropped.  The result is rounded once, 2^-8 (bf16) or 2^-24
(fp32) of itself."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from training_testutil import Held, LEAST, LIMIT, code_values, f64, nearest_code  # noqa: E402

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def T():
    from paper_2605_19811_gb300 import training
    return training


def pack_reference(w):
    """(codes' values, scales) of a 64-bit matrix, a 128 x 128 block at a time."""
    rows, cols = w.shape
    scales = np.empty((-(-rows // 128), -(-cols // 128)))
    vals = np.empty_like(w)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = np.s_[128 * i:128 * i + 128, 128 * j:128 * j + 128]
            part = w[at]
            if not np.isfinite(part).all():
                scales[i, j], vals[at] = np.nan, 0.0
                continue
            m, e = np.frexp(np.abs(part).max() / LIMIT["e4m3"])
            s = max(np.ldexp(1.0, e - (m == 0.5)) if m > 0 else 0.0, LEAST["e4m3"])
            q = nearest_code(part / s, "e4m3")
            if s == 2.0 ** 120:
                q = np.clip(q, -240, 240)
            scales[i, j], vals[at] = s, q
    return vals, scales


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 130, 0, 0), (129, 7, 0, 0), (128, 128, 0, 0), (256, 384, 8, 8),
                                                  (300, 517, 3, 1), (127, 1283, 0, 3), (1000, 257, 16, 0)])
def test_pack_and_back(T, rows, cols, pad, offset, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    w = torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(3 * torch.randn(rows, cols, device="cuda", generator=g))
    held = Held(rows, cols, dtype, pad, offset, w)
    out = T.Weight8.empty(rows + 1, cols + 20)
    out.codes.fill_(0x55)
    out.scales.fill_(3.0)
    k = T.Weight8(out.codes[:rows], out.scales[:-(-rows // 128)], cols)
    assert T.weight8(held.t, out=k) is k
    vals, scales = pack_reference(f64(held.t))
    assert np.array_equal(code_values(k.codes.cpu().numpy()[:, :cols].copy(), "e4m3"), vals)
    assert np.array_equal(k.scales.cpu().numpy()[:, :scales.shape[1]], scales)
    assert bool((out.codes[rows:] == 0x55).all()) and bool((out.codes[:rows, -(-cols // 16) * 16:] == 0x55).all())
    assert bool((out.scales[:, scales.shape[1]:] == 3).all()) and bool((out.scales[scales.shape[0]:] == 3).all())
    want = vals * np.repeat(np.repeat(scales, 128, 0), 128, 1)[:rows, :cols]
    for to in (torch.bfloat16, torch.float32):
        back = Held(rows, cols, to, pad, offset)
        k.unpack(to, out=back.t)
        assert np.array_equal(f64(back.t), want) and back.untouched()


def test_pack_of_extremes(T):
    w = torch.zeros(384, 256, device="cuda")
    w[5, 7] = float("nan")
    w[130, 3] = float("inf")
    w[200, 200] = 3e38
    w[201, 200] = -3e38
    w[300, 10] = 1e-45
    w[300, 200] = 2.0 ** -110
    k = T.weight8(w)
    vals, scales = pack_reference(f64(w))
    assert np.array_equal(code_values(k.codes.cpu().numpy(), "e4m3"), vals)
    assert np.array_equal(k.scales.cpu().numpy(), scales, equal_nan=True)
    back = k.unpack(torch.float32)
    assert bool(back[:128, :128].isnan().all()) and bool(back[128:256, :128].isnan().all()) and bool(back[:, 128:].isfinite().all())


def layer(T, rows, cols, out, grad, seed, spread=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, out if grad else cols, device="cuda", generator=g) * torch.exp(spread * torch.randn(rows, 1, device="cuda", generator=g))
    w = torch.randn(out, cols, device="cuda", generator=g) * torch.exp(spread * torch.randn(1, cols, device="cuda", generator=g))
    w *= torch.exp2(torch.randint(-6, 6, (-(-out // 128), -(-cols // 128)), device="cuda", generator=g).float()).repeat_interleave(128, 0)[:out].repeat_interleave(128, 1)[:, :cols]
    return T.checkpoint8(x, "e4m3"), T.weight8(w)


def product(x, w, grad):
    """y and sum |x w| in 64 bits."""
    a, b = x.unpack(torch.float32).double(), w.unpack(torch.float32).double()
    b = b if grad else b.t()
    return a @ b, a.abs() @ b.abs()


SIZES = [(1, 1, 1), (1, 64, 7), (1, 4096, 2304), (3, 129, 130), (8, 1024, 300), (16, 512, 4097), (17, 517, 128), (31, 16, 1000), (33, 2049, 640),
         (64, 96, 256), (65, 300, 511), (127, 128, 128), (128, 1024, 512), (129, 640, 257), (256, 256, 256), (257, 1283, 517), (1000, 4096, 768), (2049, 64, 130),
         (5, 300, 10000), (32, 1030, 19999), (33, 1030, 9999)]


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows,cols,out", SIZES)
def test_products(T, rows, cols, out, grad, to):
    x, w = layer(T, rows, cols, out, grad, rows + cols + out)
    want, most = product(x, w, grad)
    n = cols if grad else out
    y = Held(rows, n, to, pad=rows % 3 * 4, offset=rows % 5)
    (T.linear8_grad if grad else T.linear8)(x, w, out=y.t)
    bound = most * (2.0 ** -17 + (out if grad else cols) / 512 * 2.0 ** -24) + HALF[to] * want.abs()
    off = (y.t.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    assert y.untouched()
    again = (T.linear8_grad if grad else T.linear8)(x, w, dtype=to)
    assert torch.equal(again, y.t)


@pytest.mark.parametrize("grad", [False, True])
def test_long_sums_of_one_sign(T, grad):
    """20000 products of one sign: what is dropped does not grow with the sum."""
    g = torch.Generator(device="cuda").manual_seed(3)
    k, n, rows = 20000, 300, 130
    x = T.checkpoint8(torch.rand(rows, k, device="cuda", generator=g) + 0.5, "e4m3")
    w = T.weight8(torch.rand(*((k, n) if grad else (n, k)), device="cuda", generator=g) + 0.5)
    want, _ = product(x, w, grad)
    y = (T.linear8_grad if grad else T.linear8)(x, w, dtype=torch.float32)
    assert float(((y.double() - want) / want).abs().max()) <= 2.0 ** -18 + 40 * 2.0 ** -24


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("grad", [False, True])
def test_wide_scales_and_nan(T, rows, grad):
    """Groups 2^40 apart, a NaN group in one token and one block of the weights."""
    cols, out = 384, 390
    k = out if grad else cols
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, k, device="cuda", generator=g)
    x[:, :128] *= 2.0 ** 40
    x[0, 128:256] *= 2.0 ** -60
    w = torch.randn(out, cols, device="cuda", generator=g)
    (w[:128] if grad else w[:, :128]).mul_(2.0 ** -40)
    cx, cw = T.checkpoint8(x, "e4m3"), T.weight8(w)
    want, most = product(cx, cw, grad)
    f = T.linear8_grad if grad else T.linear8
    y = f(cx, cw, dtype=torch.float32)
    assert bool(((y.double() - want).abs() <= most * 2.0 ** -16.9).all())
    x[rows - 1, 300] = float("nan")
    cx = T.checkpoint8(x, "e4m3")
    z = f(cx, cw, dtype=torch.float32)
    assert bool(z[rows - 1].isnan().all()) and torch.equal(z[:rows - 1], y[:rows - 1])
    w[140, 150] = float("inf")
    cw = T.weight8(w)
    z = f(cx, cw, dtype=torch.float32)
    assert bool(z[:rows - 1, 128:256].isnan().all())
    assert torch.equal(z[:rows - 1, :128], y[:rows - 1, :128]) and torch.equal(z[:rows - 1, 256:], y[:rows - 1, 256:])
    assert y.shape == z.shape == (rows, cols if grad else out)


def test_views_empty_and_refused(T):
    x, w = layer(T, 40, 256, 384, False, 1)
    one = T.Checkpoint8(x.codes[3:4], x.scales[:, 3:4], 256, "e4m3")
    assert float((T.linear8(one, w, dtype=torch.float32) - T.linear8(x, w, dtype=torch.float32)[3:4]).abs().max()) <= \
        2.0 ** -16 * float(product(one, w, False)[1].max())
    part = T.Weight8(w.codes[128:], w.scales[1:], 256)        # rows of the weights from the second block on
    off = (T.linear8(x, part, dtype=torch.float32).double() - product(x, w, False)[0][:, 128:]).abs()
    assert bool((off <= 2.0 ** -16.9 * product(x, w, False)[1][:, 128:]).all())
    none = T.Checkpoint8(x.codes[:0], x.scales[:, :0], 256, "e4m3")
    assert T.linear8(none, w).shape == (0, 384)
    empty = T.Weight8.empty(384, 0)
    assert bool((T.linear8(T.Checkpoint8.empty(5, 0, "e4m3"), empty) == 0).all())
    with pytest.raises(RuntimeError):
        T.linear8(T.checkpoint8(torch.randn(4, 256, device="cuda"), "i8"), w)
    with pytest.raises(RuntimeError):
        T.linear8(x, part, out=torch.empty(40, 384, device="cuda"))
    with pytest.raises(RuntimeError):
        T.linear8_grad(x, w)


def test_results_beyond_31_bits(T):
    """2.2 G elements of y: the last tokens' are those of a call with them alone."""
    tokens, cols, out = 270001, 128, 8192
    g = torch.Generator(device="cuda").manual_seed(9)
    x = T.checkpoint8(torch.randn(tokens, cols, device="cuda", generator=g), "e4m3")
    w = T.weight8(torch.randn(out, cols, device="cuda", generator=g))
    y = T.linear8(x, w)
    for at in (0, 135000, tokens - 500):
        part = T.Checkpoint8(x.codes[at:at + 500], x.scales[:, at:at + 500], cols, "e4m3")
        want, most = product(part, w, False)
        assert bool(((y[at:at + 500].double() - want).abs() <= most * 2.0 ** -17 + 2.0 ** -8 * want.abs()).all())


def test_streams_and_graphs(T):
    x, w = layer(T, 300, 512, 640, False, 2)
    x1, _ = layer(T, 1, 512, 640, False, 3)
    want, want1 = T.linear8(x, w), T.linear8(x1, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = T.linear8(x, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g, c in zip(graphs, (x, x1)):
        with torch.cuda.graph(g):
            outs.append(T.linear8(c, w))
    for o in outs:
        o.zero_()
    for _ in range(3):
        graphs[1].replay()
        graphs[0].replay()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want1)


@pytest.mark.parametrize("rows,cols,out", [(1, 2048, 512), (300, 4096, 4096), (2048, 768, 512)])
def test_waits_that_run_out_leave_nan(T, rows, cols, out, monkeypatch):
    x, w = layer(T, rows, cols, out, False, 4)
    right = T.linear8(x, w)
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    y = T.linear8(x, w)
    torch.cuda.synchronize()
    assert bool((y.isnan() | (y == right)).all())
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    assert torch.equal(T.linear8(x, w), right)


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows,cols,out", [(2048, 4096, 4864), (2048, 4096, 4865), (2750, 4001, 4100), (33, 40001, 5100), (5001, 1029, 9999)])
def test_products_of_more_work(T, rows, cols, out, grad, to):
    """From 2433 tiles of 256 x 256 x 256 on, the scales are laid out before the product."""
    test_products(T, rows, cols, out, grad, to)


def test_more_work_wide_scales_nan_and_waits(T, monkeypatch):
    rows, cols, out = 3000, 4000, 4100
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x[:, :128] *= 2.0 ** 40
    x[2999, 3840:3968] = float("nan")
    w = torch.randn(out, cols, device="cuda", generator=g)
    w[:, :128] *= 2.0 ** -40
    w[4097, 3999] = float("inf")
    cx, cw = T.checkpoint8(x, "e4m3"), T.weight8(w)
    y = T.linear8(cx, cw, dtype=torch.float32)
    want, most = product(cx, cw, False)
    assert torch.equal(y.isnan(), want.isnan()) and bool(y[:2999, :4096].isfinite().all())
    fine = ~want.isnan()
    bound = most * (2.0 ** -17 + cols / 512 * 2.0 ** -24) + HALF[torch.float32] * want.abs()
    assert bool(((y.double() - want).abs() <= bound)[fine].all())
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    z = T.linear8(cx, cw, dtype=torch.float32)
    torch.cuda.synchronize()
    assert bool((z.isnan() | (z == y)).all())
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    assert torch.equal(T.linear8(cx, cw, dtype=torch.float32).nan_to_num(), y.nan_to_num())


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows,cols,out", [(1, 1100, 700), (40, 1100, 700), (2050, 4100, 5000)])
def test_scales_that_are_no_powers_of_two(T, rows, cols, out, grad):
    """The products multiply by powers of two: with any other scale what it counts for is
    NaN, and nothing else is; a scale of 0 counts as 2^-127."""
    x, w = layer(T, rows, cols, out, grad, 7)
    f = T.linear8_grad if grad else T.linear8
    y = f(x, w, dtype=torch.float32)
    n, k = (cols, out) if grad else (out, cols)
    block = -(-n // 128) // 2                                  # of y's columns
    where = (lambda g: (g, block)) if grad else (lambda g: (block, g))
    inside = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    inside[:, 128 * block:128 * block + 128] = True
    for bad in (1.5, -1.0, -2.0 ** -60, 2.0 ** -128, float("inf"), float("-inf"), 1.0 + 2.0 ** -23):
        for g in (0, 3, -(-k // 128) - 1):
            s = w.scales.clone()
            s[where(g)] = bad
            z = f(x, T.Weight8(w.codes, s, cols), dtype=torch.float32)
            assert torch.equal(z.isnan(), inside) and torch.equal(z[~inside], y[~inside]), (bad, g)
            s = x.scales.clone()
            s[g, rows // 2] = bad
            z = f(T.Checkpoint8(x.codes, s, k, "e4m3"), w, dtype=torch.float32)
            here = torch.arange(rows, device="cuda") == rows // 2
            assert bool(z[here].isnan().all()) and torch.equal(z[~here], y[~here]), (bad, g)
    # a group of zeros with scale 0, as another packing may leave it
    codes, s = x.codes.clone(), x.scales.clone()
    codes[rows // 2, 128:256] = 0
    want = f(T.Checkpoint8(codes, s, k, "e4m3"), w, dtype=torch.float32)
    s[1, rows // 2] = 0.0
    assert torch.equal(f(T.Checkpoint8(codes, s, k, "e4m3"), w, dtype=torch.float32), want)


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows,k,n", [(1, 300, 517), (2, 300, 29), (40, 130, 4), (300, 1024, 260), (257, 640, 5), (128, 128, 127), (3000, 4096, 5001), (5000, 128, 1254)])
def test_results_beside_other_columns(T, rows, k, n, grad, to):
    """Rows that end between 16-byte boundaries, of a pitch that is a multiple of 16 bytes:
    what lies behind them stays as it was."""
    x, w = layer(T, rows, n if grad else k, k if grad else n, grad, rows + n)
    want, most = product(x, w, grad)
    for more in (0, 64):
        y = Held(rows, n, to, pad=-n % 8 + more)
        (T.linear8_grad if grad else T.linear8)(x, w, out=y.t)
        assert y.untouched()
        bound = most * (2.0 ** -17 + k / 512 * 2.0 ** -24) + HALF[to] * want.abs()
        assert bool(((y.t.double() - want).abs() <= bound).all())
