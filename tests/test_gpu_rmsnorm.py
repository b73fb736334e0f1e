"""RMS norm with the residual's addition and an 8-bit output, and its
gradient, on the GPU against their formulas in 64 bits.

Tolerances, with u = 2^-24 and C channels: a thread adds at most max(C / 128,
32) squares before sums are joined pairwise, so sums are off by at most
k = max(C / 128, 32) + 16 units u of the sum of magnitudes; rstd by half of
that relatively, plus a few roundings.  A result carries half a unit of its
own type (2^-9 of a bf16 value; 2^-8 allowed where it is rounded after a sum).
An 8-bit value is off by half a step of its code plus the error of y."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.training_testutil import Held, checkpoint_values, f64

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}
U = 2.0 ** -24
SIZES = [(1, 1), (2, 3), (1, 128), (3, 130), (5, 768), (4, 1280), (2, 1283), (3, 4096), (2, 8200), (1, 16384), (2, 33000),
         (700, 96), (1300, 256), (6, 500), (9, 1000), (7, 1200), (5, 2047), (3, 3001), (2, 6000), (2, 9999)]


def terms(cols):
    return (max(cols / 128, 32) + 16) * U


def make(rows, cols, dtype, pad, offset, seed, wdtype=None):
    g = torch.Generator().manual_seed(seed)
    x = Held(rows, cols, DT[dtype], pad, offset, torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)))
    r = Held(rows, cols, DT[dtype], pad + 1, offset, torch.randn(rows, cols, generator=g))
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to(DT[wdtype or dtype]).cuda()
    return x, r, w


def check_kept(ck, y, err):
    """Codes within half a step of y, under the least scale that holds it
    (one step either way where the largest magnitude is within err of the limit)."""
    from tests.training_testutil import GROUP, LIMIT, pack_reference
    assert ck.rows == y.shape[0] and ck.cols == y.shape[1]
    s = ck.scales.cpu().numpy().astype(np.float64).T
    lo, hi = (pack_reference(y * (1 + f * err), ck.format)[1] for f in (-2, 2))
    assert np.all((s >= lo) & (s <= hi))
    full = np.repeat(s, GROUP, axis=1)[:, :ck.cols]
    step = full / 2 if ck.format == "i8" else np.maximum(np.abs(y) * 2.0 ** -4, full * 2.0 ** -10)
    assert np.all(np.abs(checkpoint_values(ck) - y) <= step * (1 + 8 * err) + 2 * err * np.abs(y))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype):
    from paper_2605_19811_gb300 import training as T
    for pad, offset, fmt, wd, res in ((0, 0, "e4m3", dtype, True), (3, 1, "i8", "f32", False), (8, 8, None, "bf16", True),
                                      (5, 0, "i8", "bf16", True)):
        x, r, w = make(rows, cols, dtype, pad, offset, seed=cols, wdtype=wd)
        o = T.rmsnorm(x.t, w, residual=r.t if res else None, eps=1e-5, checkpoint=fmt)
        h = f64(x.t) + (f64(r.t) if res else 0.0)
        rstd = 1 / np.sqrt((h * h).mean(axis=1) + 1e-5)
        y = h * rstd[:, None] * f64(w)
        err = terms(cols) + 6 * U
        assert np.all(np.abs(f64(o.rstd) - rstd) <= err * rstd)
        assert np.all(np.abs(f64(o.y) - y) <= (2 * err + ROUND[dtype]) * np.abs(y) + 1e-37)
        if res:
            assert np.all(np.abs(f64(o.h) - h) <= ROUND[dtype] * np.abs(h))
        else:
            assert o.h is x.t
        if fmt:
            check_kept(o.checkpoint, y, 2 * err)
        else:
            assert o.checkpoint is None
        assert x.untouched() and r.untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_gradient(rows, cols, dtype):
    from paper_2605_19811_gb300 import training as T
    for pad, offset, fmt, wd, past in ((0, 0, None, dtype, True), (3, 1, "i8", "f32", False), (8, 8, "e4m3", "bf16", True),
                                       (1, 0, None, "bf16", False)):
        x, r, w = make(rows, cols, dtype, pad, offset, seed=cols + 1, wdtype=wd)
        dy, dh = r, Held(rows, cols, DT[dtype], pad, offset, torch.randn(rows, cols))
        source = x.t if fmt is None else T.checkpoint8(x.t, fmt)
        h = f64(x.t) if fmt is None else checkpoint_values(source)
        rstd = torch.from_numpy(1 / np.sqrt((h * h).mean(axis=1) + 1e-5)).float().cuda()
        out = Held(rows, cols, DT[dtype], pad + 2, offset)
        dx, dw = T.rmsnorm_grad(dy.t, source, rstd, w, dh=dh.t if past else None, dx=out.t)
        rs, g, ww = f64(rstd)[:, None], f64(dy.t), f64(w)
        xh = h * rs
        mean = (ww * g * xh).mean(axis=1, keepdims=True)
        absmean = np.abs(ww * g * xh).mean(axis=1, keepdims=True)
        want = rs * (ww * g - xh * mean) + (f64(dh.t) if past else 0.0)
        size = rs * (np.abs(ww * g) + np.abs(xh) * absmean) + (np.abs(f64(dh.t)) if past else 0.0)
        tol = (terms(cols) + 8 * U) * size + ROUND[dtype] * np.abs(want) + 1e-37
        assert np.all(np.abs(f64(dx) - want) <= tol)
        wantw, absw = (g * xh).sum(axis=0), np.abs(g * xh).sum(axis=0)
        tolw = (rows + 16) * U * absw + ROUND[wd] * np.abs(wantw) + 1e-37   # at worst one row after another
        assert dw.dtype == w.dtype and np.all(np.abs(f64(dw) - wantw) <= tolw)
        assert out.untouched() and dy.untouched() and x.untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_weight_and_in_place(dtype):
    from paper_2605_19811_gb300 import training as T
    x, r, w = make(33, 1280, dtype, 0, 0, seed=2)
    a = T.rmsnorm(x.t, None, residual=r.t)
    b = T.rmsnorm(x.t, torch.ones(1280, dtype=DT[dtype], device="cuda"), residual=r.t)
    assert torch.equal(a.y, b.y) and torch.equal(a.h, b.h) and torch.equal(a.rstd, b.rstd)
    dx, dw = T.rmsnorm_grad(r.t, a.h, a.rstd, w, dh=x.t)
    for over in ("dy", "dh"):
        dy, dh = r.t.clone(), x.t.clone()
        dx2, dw2 = T.rmsnorm_grad(dy, a.h, a.rstd, w, dh=dh, dx=dy if over == "dy" else dh)
        assert dx2 is (dy if over == "dy" else dh)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    only, none = T.rmsnorm_grad(r.t, a.h, a.rstd, w, dh=x.t, dweight=False)
    assert none is None and torch.equal(only, dx)
    assert T.rmsnorm_grad(r.t, a.h, a.rstd, None)[1].dtype == torch.float32


@pytest.mark.parametrize("over", ["x", "residual"])
def test_h_over_an_input(over):
    """The C call's h may be x or residual itself."""
    import ctypes
    from paper_2605_19811_gb300 import lionmuon as L
    from paper_2605_19811_gb300 import training as T
    for cols in (96, 1283, 4096, 33000):
        x, r, w = make(7, cols, "bf16", 0, 0, seed=3)
        a = T.rmsnorm(x.t, w, residual=r.t)
        xs, rs = x.t.clone(), r.t.clone()
        y = torch.empty_like(xs)
        mats = [T._matrix(t, "m") for t in (xs, rs, xs if over == "x" else rs, y)]
        lib = L.load_library()
        st = lib.lm_rmsnorm(ctypes.byref(mats[0]), ctypes.byref(mats[1]), ctypes.byref(T._vector(w, "w")), 1e-6,
                            ctypes.byref(mats[2]), ctypes.byref(mats[3]), None, None, L._stream_handle(None))
        assert st == 0
        assert torch.equal(xs if over == "x" else rs, a.h) and torch.equal(y, a.y)


def test_zero_rows_nonfinite_rows_and_huge_values():
    from paper_2605_19811_gb300 import training as T
    x = torch.randn(5, 300, device="cuda")
    x[1] = 0.0
    x[2, 7] = float("nan")
    x[3, 8] = float("inf")
    x[4] *= 1e18
    o = T.rmsnorm(x, torch.ones(300, device="cuda"), eps=1e-6, checkpoint="e4m3")
    y = o.y.cpu()
    assert torch.equal(y[1], torch.zeros(300)) and abs(float(o.rstd[1]) - 1e3) < 1e-2
    assert bool(y[2].isnan().all()) and bool(torch.isfinite(y[0]).all()) and bool(torch.isfinite(y[4]).all())
    assert bool(y[3, 8].isnan()) and float(y[3, 0]) == 0.0            # inf * (1 / inf), and x / inf
    k = o.checkpoint.unpack(torch.float32).cpu()
    assert bool(k[2].isnan().all())
    assert bool(k[3, :128].isnan().all()) and bool((k[3, 128:] == 0).all())
    assert bool((k[1] == 0).all()) and bool(torch.isfinite(k[4]).all())


def test_gradient_against_differences():
    """Central differences of the forward call in fp32, h = 2^-6 along v: the
    cut-off is h^2 / 6 times a third derivative of order 10 |v|^3, the forward's
    rounding 2^-21 sqrt(C) / h of the loss: 5e-3 of the loss's scale allowed."""
    from paper_2605_19811_gb300 import training as T
    g = torch.Generator().manual_seed(0)
    x, w, c = torch.randn(4, 200, generator=g).cuda(), torch.randn(200, generator=g).cuda(), torch.randn(4, 200, generator=g).cuda()
    o = T.rmsnorm(x, w)
    dx, dw = T.rmsnorm_grad(c, x, o.rstd, w)

    def loss(a, b):
        return (T.rmsnorm(a.contiguous(), b.contiguous()).y.double() * c.double()).sum()

    h = 2.0 ** -6
    for _ in range(4):
        v, u = torch.randn(4, 200, generator=g).cuda() / 8, torch.randn(200, generator=g).cuda() / 8
        d = float((loss(x + h * v, w) - loss(x - h * v, w)) / (2 * h))
        assert abs(d - float((dx * v).sum())) <= 5e-3 * float((c * v).norm() + 1)
        d = float((loss(x, w + h * u) - loss(x, w - h * u)) / (2 * h))
        assert abs(d - float((dw * u).sum())) <= 5e-3 * float((c.norm() * u.norm()) + 1)


def test_same_bits_twice_and_on_another_stream():
    from paper_2605_19811_gb300 import training as T
    x, r, w = make(5000, 1280, "bf16", 0, 0, seed=6)
    a = T.rmsnorm(x.t, w, residual=r.t, checkpoint="i8")
    ga = T.rmsnorm_grad(r.t, a.h, a.rstd, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = T.rmsnorm(x.t, w, residual=r.t, checkpoint="i8", stream=side)
    gb = T.rmsnorm_grad(r.t, b.h, b.rstd, w, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*a[:3], *ga), (*b[:3], *gb)))
    assert torch.equal(a.checkpoint.codes, b.checkpoint.codes) and torch.equal(a.checkpoint.scales, b.checkpoint.scales)


def test_graph_capture_and_no_rows():
    from paper_2605_19811_gb300 import training as T
    x, r, w = make(65, 768, "bf16", 0, 0, seed=7)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = T.rmsnorm(x.t, w, residual=r.t, checkpoint="e4m3")
        dx, dw = T.rmsnorm_grad(r.t, o.checkpoint, o.rstd, w)
    x.t.copy_(torch.randn(65, 768))
    graph.replay()
    torch.cuda.synchronize()
    q = T.rmsnorm(x.t, w, residual=r.t, checkpoint="e4m3")
    dx2, dw2 = T.rmsnorm_grad(r.t, q.checkpoint, q.rstd, w)
    assert torch.equal(o.y, q.y) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    e = torch.empty(0, 64, device="cuda")
    o = T.rmsnorm(e, torch.ones(64, device="cuda"), checkpoint="i8")
    assert o.y.shape == (0, 64)
    dx, dw = T.rmsnorm_grad(e, e, o.rstd, torch.ones(64, device="cuda"))
    assert torch.equal(dw, torch.zeros(64, device="cuda"))            # a sum over no rows
