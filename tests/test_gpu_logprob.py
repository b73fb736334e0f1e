"""Token log probabilities, entropy, top alternatives and their gradient on
the GPU against their definition in 64 bits (tests/training_testutil.py).

Tolerances.  With u = 2^-24: the argument z - m of an exponential is off by at
most u |z - m| (one rounding) and the scaling to base 2 by as much again, the
exponential itself by 2 ulp; a term e^d weighs |d| e^d <= 1/e, so a sum of
exponentials is off by at most about 8 u relative, and by 8 u more for its own
roundings (threads add pairwise beyond a few hundred terms; 24 u allowed).
lse = m + log S adds a rounding of its size:       |err| <= 2^-19 + 2^-22 max|z|
entropy = log S - T / S, each part at most H + 1:  |err| <= 2^-18 (1 + H)
p = exp(z - lse) carries lse's error relatively, and the argument's:
rel <= 2^-18 + 2^-22 (|lp| + max|z|), and a gradient term p (..) as much, plus
half a unit of its own type."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.training_testutil import Held, f64, log_probabilities, logprob_gradient, logprob_reference

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_UNIT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}


def make(rows, vocab, dtype, pad=0, offset=0, seed=0, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    z = Held(rows, vocab, DT[dtype], pad, offset, scale * torch.randn(rows, vocab, generator=g))
    y = torch.randint(0, vocab, (rows,), generator=g)
    w = [torch.randn(rows, generator=g).cuda() for _ in range(3)]
    return z, y.cuda(), w


def check_forward(z, y, o, top_k):
    zz, yy = f64(z), y.cpu().numpy()
    lse, ent, logp, top = logprob_reference(zz, yy, top_k)
    fin = np.where(np.isfinite(zz), np.abs(zz), 0.0).max(axis=1)
    tol = 2.0 ** -19 + 2.0 ** -22 * fin
    for got, want, t in ((f64(o.lse), lse, tol), (f64(o.entropy), ent, 2.0 ** -18 * (1 + np.abs(ent))),
                         (f64(o.logp), logp, 2 * tol)):
        same = np.isfinite(want)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        np.testing.assert_array_equal(got[~same & ~np.isnan(want)], want[~same & ~np.isnan(want)])
        assert np.all(np.abs(got - want)[same] <= t[same]), np.abs(got - want)[same].max()
    if top_k:
        np.testing.assert_array_equal(o.top_index.cpu().numpy(), top)
        got = f64(o.top_logp)
        for r in range(len(yy)):
            for k in range(top_k):
                if np.isnan(lse[r]):
                    assert np.isnan(got[r, k])
                elif top[r, k] < 0:
                    assert got[r, k] == -np.inf
                else:
                    assert abs(got[r, k] - log_probabilities(zz[r])[top[r, k]]) <= 2 * tol[r]


def check_gradient(z, y, d, w, dtype):
    zz, yy = f64(z), y.cpu().numpy()
    lse, ent, _, _ = logprob_reference(zz, yy)
    gl, gh, gz = (np.zeros(len(yy)) if x is None else f64(x) for x in w)
    want, got = logprob_gradient(zz, yy, lse, ent, gl, gh, gz), f64(d)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    fin = np.where(np.isfinite(zz), np.abs(zz), 0.0).max(axis=1, keepdims=True)
    lp, p = np.zeros_like(zz), np.zeros_like(zz)
    for r in np.flatnonzero(np.isfinite(lse)):
        q = log_probabilities(zz[r])
        lp[r], p[r] = np.where(np.isfinite(q), q, 0.0), np.exp(q)
    rel = 2.0 ** -18 + 2.0 ** -22 * (np.abs(lp) + fin)
    size = np.abs(gz)[:, None] + np.abs(gl)[:, None] + np.abs(gh)[:, None] * (np.abs(lp) + np.abs(ent)[:, None] + 1)
    tol = rel * p * size + HALF_UNIT[dtype] * np.abs(want) + 1e-37
    ok = ~np.isnan(want)
    worst = (np.abs(got - want)[ok] / tol[ok]).max() if ok.any() else 0.0
    assert worst <= 1.0, worst


SIZES = [(1, 1), (1, 2), (3, 7), (2, 31), (5, 128), (4, 257), (3, 1000), (2, 1024), (7, 4099), (1, 50304), (3, 50257),
         (2, 131071), (1, 262144), (600, 515)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_forward_and_both_gradients(rows, vocab, dtype):
    from paper_2605_19811_gb300 import training as T
    for pad, offset in ((0, 0), (5, 1), (8, 8)):
        z, y, w = make(rows, vocab, dtype, pad, offset, seed=rows + vocab)
        k = min(vocab, 5)
        check_forward(z.t, y, T.token_logprob(z.t, y, top_k=k), k)
        d = Held(rows, vocab, DT[dtype], pad + 3, offset)
        o = T.token_logprob(z.t, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2], dlogits=d.t)
        check_forward(z.t, y, o, 0)
        check_gradient(z.t, y, d.t, w, dtype)
        assert d.untouched() and z.untouched()
        d2 = Held(rows, vocab, DT[dtype], pad, offset)
        T.token_logprob_grad(z.t, y, o.lse, o.entropy, w[0], w[1], w[2], dlogits=d2.t)
        check_gradient(z.t, y, d2.t, w, dtype)
        assert d2.untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(609, 16400), (1000, 8200), (700, 36000), (620, 70001)])
def test_many_long_rows(rows, vocab, dtype):
    """Enough rows for every SM several times over, pitches that shift the
    rows' alignment, masked and missing rows among them; in place as well."""
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(rows, vocab, dtype, pad=3, offset=1, seed=rows)
    z.t[5] = float("-inf")
    z.t[170, 100:] = float("-inf")
    z.t[171, 7] = float("nan")
    z.t[300] = torch.finfo(DT[dtype]).min
    z.t[rows - 1, ::3] = float("-inf")
    y[11], y[200] = -100, vocab
    o = T.token_logprob(z.t, y, top_k=3)
    check_forward(z.t, y, o, 3)
    d = Held(rows, vocab, DT[dtype], 3, 1)
    q = T.token_logprob(z.t, y, top_k=3, g_logp=w[0], g_entropy=w[1], g_lse=w[2], dlogits=d.t)
    check_forward(z.t, y, q, 3)                 # (another kernel may have summed in another order)
    check_gradient(z.t, y, d.t, w, dtype)
    assert d.untouched() and z.untouched()
    d2 = Held(rows, vocab, DT[dtype], 2, 0)     # vectors that do not line up with the logits'
    T.token_logprob(z.t, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2], dlogits=d2.t)
    assert torch.equal(d.t.nan_to_num(9.0), d2.t.nan_to_num(9.0)) and d2.untouched()
    T.token_logprob(z.t, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2], dlogits=z.t)
    assert torch.equal(d.t.nan_to_num(9.0), z.t.nan_to_num(9.0)) and z.untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [65, 1504, 50304])
def test_masks_infinities_and_missing_targets(vocab, dtype):
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(12, vocab, dtype, seed=vocab)
    t, low = z.t, torch.finfo(DT[dtype]).min
    t[0, 3:] = float("-inf")                   # three tokens left
    t[1] = float("-inf")                       # nothing left
    t[2] = low                                 # everything at the type's lowest value
    t[3, 1:] = low                             # one token above it
    t[4, 5] = float("nan")
    t[5, 7] = float("inf")
    t[6, ::2] = float("-inf")
    y[6] = 2                                   # a masked target
    y[7] = -100                                # no target
    y[8] = vocab                               # beyond the vocabulary
    t[9] = 0.0                                 # all equal: ties go to the lowest index
    t[10] = torch.finfo(DT[dtype]).max         # the largest finite value
    t[11, 0], t[11, 1] = torch.finfo(DT[dtype]).max, low
    y[1], y[0] = 0, 1
    before = t.clone()
    k = min(32, vocab)
    o = T.token_logprob(t, y, top_k=k)
    check_forward(t, y, o, k)
    assert f64(o.logp)[7] == 0.0
    d = T.token_logprob(t, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2]).dlogits
    check_gradient(t, y, d, w, dtype)
    check_gradient(t, y, T.token_logprob_grad(t, y, o.lse, o.entropy, w[0], w[1], w[2]), w, dtype)
    assert torch.equal(t.nan_to_num(1.0), before.nan_to_num(1.0))
    # in place, over the logits themselves
    g = t.clone()
    T.token_logprob(g, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2], dlogits=g)
    assert torch.equal(g.nan_to_num(3.0), d.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_at_the_lowest_value_is_uniform(dtype):
    """Every logit at the type's lowest value: p = 1 / V, although lse cannot
    hold log V beside it."""
    from paper_2605_19811_gb300 import training as T
    v = 4096
    z = torch.full((2, v), torch.finfo(DT[dtype]).min, dtype=DT[dtype], device="cuda")
    y, one, zero = torch.tensor([3, -1], device="cuda"), torch.ones(2, device="cuda"), torch.zeros(2, device="cuda")
    o = T.token_logprob(z, y, g_logp=one, g_entropy=zero, g_lse=one)
    want = torch.zeros(2, v)
    want[0, 3], want[1] = 1.0, 1.0 / v
    for d in (o.dlogits, T.token_logprob_grad(z, y, o.lse, o.entropy, one, zero, one)):
        assert float((d.float().cpu() - want).abs().max()) <= 2.0 ** -18 / v
    assert abs(float(o.logp[0]) + np.log(v)) <= 2.0 ** -18 and abs(float(o.entropy[1]) - np.log(v)) <= 2.0 ** -16


@pytest.mark.parametrize("order", ["rising", "falling", "one stride", "ties", "two values"])
@pytest.mark.parametrize("top_k", [1, 7, 32])
@pytest.mark.parametrize("rows,vocab", [(2, 50304), (400, 20000), (3, 33), (700, 20000)])
def test_alternatives_in_hard_orders(rows, vocab, top_k, order):
    """Arrangements that crowd the largest logits: sorted rows, all of them at
    one stride, many ties."""
    from paper_2605_19811_gb300 import training as T
    i = torch.arange(vocab, dtype=torch.float32)
    base = {"rising": i / 64, "falling": -i / 64, "one stride": torch.where(i % 4096 < 8, 5.0 + i / 8192, -i / vocab),
            "ties": torch.floor(i / 7) % 3, "two values": (i % 5 == 0).float()}[order]
    z = base[None].repeat(rows, 1).to(torch.bfloat16).cuda()
    o = T.token_logprob(z, None, top_k=top_k)
    want = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :top_k]
    assert torch.equal(o.top_index, want)
    assert o.logp is None


def test_weights_left_out_and_entropy_only():
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(9, 777, "f32", seed=5)
    for keep in ((0,), (1,), (2,), (0, 2)):
        ws = [w[i] if i in keep else None for i in range(3)]
        o = T.token_logprob(z.t, y, g_logp=ws[0], g_entropy=ws[1], g_lse=ws[2])
        check_gradient(z.t, y, o.dlogits, ws, "f32")
    # no targets at all: entropy's gradient alone
    o = T.token_logprob(z.t, None, g_entropy=w[1])
    check_gradient(z.t, torch.full_like(y, -1), o.dlogits, (None, w[1], None), "f32")


def test_gradient_against_differences():
    """d/dt L(z + t v) at t = 0 by central differences of the forward call, h =
    2^-5: the cut-off is h^2 / 6 |L'''| <= 2e-4 |v|^3-sized terms of order one,
    the forward's rounding 2 * 2^-19 / (2 h) = 6e-5 a row; 4e-3 allowed."""
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(6, 40, "f32", seed=8, scale=1.0)
    o = T.token_logprob(z.t, y, g_logp=w[0], g_entropy=w[1], g_lse=w[2])

    def loss(x):
        q = T.token_logprob(x.contiguous(), y)
        return f64(q.logp) * f64(w[0]) + f64(q.entropy) * f64(w[1]) + f64(q.lse) * f64(w[2])

    g = torch.Generator().manual_seed(1)
    for _ in range(8):
        v = torch.randn(6, 40, generator=g).cuda() / 4
        h = 2.0 ** -5
        diff = (loss(z.t + h * v) - loss(z.t - h * v)) / (2 * h)
        assert np.all(np.abs(diff - f64((o.dlogits * v).sum(dim=1))) <= 4e-3)


def test_same_bits_twice_and_on_another_stream():
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(37, 50257, "bf16", seed=3)
    a = T.token_logprob(z.t, y, top_k=8, g_logp=w[0], g_entropy=w[1], g_lse=w[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = T.token_logprob(z.t, y, top_k=8, g_logp=w[0], g_entropy=w[1], g_lse=w[2], stream=side)
    torch.cuda.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_graph_capture():
    from paper_2605_19811_gb300 import training as T
    z, y, w = make(5, 3001, "bf16", seed=4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = T.token_logprob(z.t, y, top_k=3, g_logp=w[0])
    z.t.copy_(torch.randn(5, 3001))
    graph.replay()
    torch.cuda.synchronize()
    check_forward(z.t, y, o, 3)
    check_gradient(z.t, y, o.dlogits, (w[0], None, None), "bf16")


def test_no_rows():
    from paper_2605_19811_gb300 import training as T
    z = torch.empty(0, 100, device="cuda")
    y = torch.empty(0, dtype=torch.int64, device="cuda")
    o = T.token_logprob(z, y, top_k=2)
    assert o.lse.shape == (0,) and o.top_index.shape == (0, 2)
