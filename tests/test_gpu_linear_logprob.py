"""Log probabilities and gradients from hidden states, against 64 bits.

Errors that the tolerances count.  A logit z = sum h w of bf16 factors: the
products are exact; the tensor cores add 16 at a time and drop up to 2^-23 of
what they have at each addition, at most 32 additions in a row, then one fp32
addition (2^-24) for each 512 of the width; nothing they have is above
S = sum |h w|, so
  |dz| <= E = S (2^-18 + width / 512 2^-24)
lse moves by at most E; its sum of V terms, each 2^-22 off by the exponential
unit and 2^-23 |d| by its argument (|d| e^d < 1), is added in fp32 in chains of
fewer than 256: 2^-16 in all, and its own rounding 2^-23 |lse|.  log p likewise,
from z_y - max, with E twice.  The entropy moves by sum p |log p + H| E <=
2 ln V E, and its rounding errors are as those of lse, times the 1 + ln V that
its terms add up to.
dz = p (a - g_H (log p + H)) + g_logp: p is off by E + 2^-18 of itself (the
exponential and lse); a call that computes lse and the gradients together keeps
logits in steps of 2^-10, 2^-11 more; then dz is rounded to bf16, 2^-8.  A product's sum of them adds
2^-18 of the magnitudes it adds up, and its result is rounded to its type, 2^-8
(bf16) of itself."""

import math

import pytest

torch = pytest.importorskip("torch")

from training_testutil import Held  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


@pytest.fixture(scope="module")
def T():
    from paper_2605_19811_gb300 import training
    return training


def inputs(rows, vocab, width, seed, pad=0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = 2.0 * width ** -0.5 * torch.randn(vocab, width, device="cuda", generator=g)
    y = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    h = torch.randn(rows, width, device="cuda", generator=g) + 2.0 * torch.rand(rows, 1, device="cuda", generator=g) * w[y]
    y[torch.rand(rows, device="cuda", generator=g) < 0.2] = -1
    hh, ww = Held(rows, width, torch.bfloat16, pad, offset, h), Held(vocab, width, torch.bfloat16, pad, offset, w)
    gl = torch.randn(rows, device="cuda", generator=g) / rows
    gh = 0.1 * torch.randn(rows, device="cuda", generator=g) / rows
    gz = 0.1 * torch.randn(rows, device="cuda", generator=g) / rows
    return hh, ww, y, gl, gh, gz


def reference(h, w, y, gl=None, gh=None, gz=None):
    """lse, H, log p with bounds, and (with weights) dh and dW with bounds, a part of the rows at a time."""
    w = w.double()
    v, c = w.shape
    parts, dw, dwb = [], torch.zeros_like(w), torch.zeros_like(w)
    for at in range(0, h.shape[0], 8192):
        x, t = h[at:at + 8192].double(), y[at:at + 8192]
        z = x @ w.t()
        e = (x.abs() @ w.abs().t()).amax(dim=1, keepdim=True) * (2.0 ** -18 + c / 512 * 2.0 ** -24)
        lse = torch.logsumexp(z, dim=1, keepdim=True)
        lp = z - lse
        p = lp.exp()
        ent = -(p * lp).sum(dim=1, keepdim=True)
        has = (t >= 0)[:, None]
        logp = torch.where(has, lp.gather(1, t.clamp(min=0)[:, None]), 0.0)
        r = {"lse": lse, "lse_b": e + 2.0 ** -16 + 2.0 ** -23 * lse.abs(),
             "entropy": ent, "entropy_b": 2 * (1 + math.log(v)) * e + (1 + math.log(v)) * 2.0 ** -16,
             "logp": logp, "logp_b": torch.where(has, 2 * e + 2.0 ** -16 + 2.0 ** -22 * logp.abs(), 0.0)}
        if gl is not None:
            a, b, k = (q[at:at + 8192, None].double() for q in (gl, gh, gz))
            a = torch.where(has, a, 0.0)
            d = p * ((k - a) - b * (lp + ent))
            db = (e + 2.0 ** -18 + 2.0 ** -11) * p * ((k - a).abs() + b.abs() * ((lp + ent).abs() + 1 + 2 * math.log(v)))
            d.scatter_add_(1, t.clamp(min=0)[:, None], a)
            db += (U + 2.0 ** -18) * (d.abs() + db)
            r["dh"] = d @ w
            r["dh_b"] = db @ w.abs() + U * r["dh"].abs() + 1e-38
            dw += d.t() @ x
            dwb += db.t() @ x.abs()
        parts.append(r)
    out = {k: torch.cat([q[k] for q in parts]).squeeze(1) if k[:2] != "dh" else torch.cat([q[k] for q in parts]) for k in parts[0]}
    if gl is not None:
        out["dweight"], out["dweight_b"] = dw, dwb
    return out


def near(got, ref, name, more=0.0):
    off = (got.double() - ref[name]).abs()
    bound = ref[name + "_b"] + more * ref[name].abs()
    assert bool((off <= bound).all()), (name, float((off / bound).max()))


SIZES = [(1, 1, 1, 0, 0), (1, 7, 8, 0, 0), (1, 1000, 64, 0, 0), (2, 129, 65, 3, 1), (31, 257, 63, 0, 0), (256, 256, 512, 0, 0),
         (257, 255, 513, 8, 0), (255, 5003, 200, 0, 0), (300, 128, 1283, 5, 3), (1000, 1000, 768, 0, 8), (3, 50257, 128, 0, 0),
         (513, 2049, 1024, 0, 0), (40, 20000, 1100, 8, 8), (32, 5000, 96, 0, 0), (33, 5000, 96, 8, 0)]


@pytest.mark.parametrize("rows,vocab,width,pad,offset", SIZES)
def test_against_64_bits(T, rows, vocab, width, pad, offset):
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, rows + vocab + width, pad, offset)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    o = T.linear_logprob(h.t, w.t, y)
    assert o.dh is None and o.dweight is None
    for k in ("lse", "entropy", "logp"):
        near(getattr(o, k), ref, k)
    dh, dw = Held(rows, width, torch.bfloat16, pad, offset), Held(vocab, width, torch.bfloat16, pad, offset)
    o2 = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=dh.t, dweight=dw.t)
    for k in ("lse", "entropy", "logp"):
        assert torch.equal(getattr(o, k), getattr(o2, k)), k
    near(dh.t, ref, "dh")
    near(dw.t, ref, "dweight", U)
    assert dh.untouched() and dw.untouched() and h.untouched() and w.untouched()
    # twice the same bits; afterwards, from lse and entropy
    o3 = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    assert torch.equal(o3.dh, dh.t) and torch.equal(o3.dweight, dw.t)
    o4 = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=dh.t, dweight=dw.t)
    assert o4[0] is dh.t and o4[1] is dw.t
    near(dh.t, ref, "dh")
    near(dw.t, ref, "dweight", U)
    assert dh.untouched() and dw.untouched()
    dh2, dw2 = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz)
    assert torch.equal(dh2, dh.t) and torch.equal(dw2, dw.t)


@pytest.mark.parametrize("rows,vocab,width", [(131073, 5003, 40), (2500, 270001, 24)])
def test_several_pieces_of_the_tokens(T, rows, vocab, width):
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 5)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    for k in ("lse", "entropy", "logp", "dh"):
        near(getattr(o, k), ref, k)
    near(o.dweight, ref, "dweight", U)
    assert torch.equal(T.linear_logprob(h.t, w.t, y, gl, gh, gz).dh, o.dh)
    dw = torch.ones_like(w.t, dtype=torch.float32)
    T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=False, dweight=dw, accumulate=True)
    ref["dweight"] = ref["dweight"] + 1.0
    near(dw, ref, "dweight", 2.0 ** -22)       # four pieces' additions and the first value's
    ref["dweight"] = ref["dweight"] - 1.0
    _, dw = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=False, dweight=torch.empty_like(w.t, dtype=torch.float32))
    near(dw, ref, "dweight", 2.0 ** -22)
    # added to a bf16 sum
    before = (torch.randn(w.t.shape, device="cuda") * o.dweight.float().std()).bfloat16()
    added = before.clone()
    again = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dweight=added, accumulate=True)
    near(again[0], ref, "dh")
    ref["dweight"] = ref["dweight"] + before.double()
    near(added, ref, "dweight", U)


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
def test_one_gradient_alone_and_added(T, to):
    h, w, y, gl, gh, gz = inputs(300, 777, 130, 1)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=False)
    assert o.dh is None
    near(o.dweight, ref, "dweight", U)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dweight=False)
    assert o.dweight is None
    near(o.dh, ref, "dh")
    before = torch.randn(777, 130, device="cuda").to(to) / 300
    dw = before.clone()
    T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=False, dweight=dw, accumulate=True)
    ref["dweight"] = ref["dweight"] + before.double()
    near(dw, ref, "dweight", U if to == torch.bfloat16 else 2.0 ** -24)


def test_weights_left_out(T):
    h, w, y, gl, gh, gz = inputs(70, 300, 96, 2)
    zero = torch.zeros_like(gl)
    for a, b, k in ((gl, None, None), (None, gh, None), (None, None, gz), (gl, None, gz)):
        o = T.linear_logprob(h.t, w.t, y, a, b, k)
        full = T.linear_logprob(h.t, w.t, y, *(zero if q is None else q for q in (a, b, k)))
        assert torch.equal(o.dh, full.dh) and torch.equal(o.dweight, full.dweight)
    o = T.linear_logprob(h.t, w.t, None, None, gh, None)
    assert o.logp is None and bool(o.dh.isfinite().all())


def test_targets_beyond_the_vocabulary(T):
    h, w, y, gl, gh, gz = inputs(64, 300, 96, 3)
    y[5] = 300
    y[6] = 1 << 40
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    bad = torch.zeros(64, dtype=torch.bool, device="cuda")
    bad[5] = bad[6] = True
    assert torch.equal(o.logp.isnan(), bad) and not bool(o.lse.isnan().any())
    assert torch.equal(o.dh.isnan().all(dim=1), bad) and torch.equal(o.dh.isnan().any(dim=1), bad)
    assert bool(o.dweight.isnan().all())
    o = T.linear_logprob(h.t, w.t, y, None, gh, gz)
    assert bool(o.dh.isfinite().all()) and bool(o.dweight.isfinite().all())


def test_infinite_and_nan_logits(T):
    """Logits of -inf are masked, rows of -inf only have lse = -inf and no
    gradient, rows with NaN or +inf are NaN."""
    rows, vocab, width = 40, 700, 64
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 4)
    h.t.abs_().clamp_(min=0.01)
    masked = torch.arange(vocab, device="cuda") % 3 == 0
    w.t[masked, 7] = float("-inf")
    y.clamp_(min=1)
    y[y % 3 == 0] += 1
    y[9] = 3                                                  # a masked target
    ref = reference(h.t, w.t[~masked], torch.zeros_like(y))   # statistics of the others
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=False)
    near(o.lse, ref, "lse")
    near(o.entropy, ref, "entropy")
    assert float(o.logp[9]) == float("-inf")
    assert bool(o.logp[torch.arange(rows, device="cuda") != 9].isfinite().all())
    plain = T.token_logprob(h.t.float() @ w.t.float().t(), y, g_logp=gl, g_entropy=gh, g_lse=gz)
    rows9 = torch.arange(rows, device="cuda") != 9
    only = masked & ~torch.isin(torch.arange(vocab, device="cuda"), y)
    assert bool((o.dweight[only] == 0).all())
    want = plain.dlogits.double().t() @ h.t.double()
    assert float((o.dweight.double() - want).norm() / want.norm()) < 2.0 ** -7
    del rows9
    # every logit of every row -inf
    w.t[:, 7] = float("-inf")
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=False)
    assert bool((o.lse == float("-inf")).all()) and bool((o.entropy == 0).all()) and bool((o.logp == float("-inf")).all())
    assert bool((o.dweight == 0).all())
    y2 = torch.full_like(y, -1)
    assert bool((T.linear_logprob(h.t, w.t, y2).logp == 0).all())
    # +inf in one token's logit, NaN in one row
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 4)
    clean = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    h.t[3, 5] = float("nan")
    h.t[8] = 0.0
    h.t[8, 0] = float("inf")                                  # logits of +inf and -inf
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[3] = bad[8] = True
    for k in ("lse", "entropy"):
        assert torch.equal(getattr(o, k).isnan(), bad)
        assert torch.equal(getattr(o, k)[~bad], getattr(clean, k)[~bad])
    assert torch.equal(o.dh.isnan().all(dim=1), bad) and torch.equal(o.dh[~bad], clean.dh[~bad])


def test_large_logits(T):
    """Logits around +-20000, whose differences alone matter."""
    rows, vocab, width = 33, 900, 128
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 6)
    for shift in (20000.0, -20000.0):
        h.t[:, 0] = 128.0
        w.t[:, 0] = shift / 128.0
        ref = reference(h.t, w.t, y, gl, gh, gz)
        o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
        for k in ("lse", "entropy", "logp", "dh"):
            near(getattr(o, k), ref, k)


def test_no_rows_and_leading_dimensions(T):
    h, w, y, gl, gh, gz = inputs(24, 100, 48, 7)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    b = T.linear_logprob(h.t.view(2, 12, 48), w.t, y.view(2, 12), gl, gh, gz)
    assert b.lse.shape == (2, 12) and b.dh.shape == (2, 12, 48)
    assert torch.equal(b.dh.view(24, 48), o.dh) and torch.equal(b.lse.view(24), o.lse)
    z = T.linear_logprob(h.t[:0], w.t, y[:0], gl[:0])
    assert z.lse.shape == (0,) and bool((z.dweight == 0).all())
    kept = torch.ones_like(w.t)
    T.linear_logprob(h.t[:0], w.t, y[:0], gl[:0], dweight=kept, accumulate=True)
    assert bool((kept == 1).all())


def test_streams_and_graphs(T):
    """On another stream, and two captured calls replayed with new inputs between eager ones."""
    h, w, y, gl, gh, gz = inputs(200, 1500, 200, 8)
    want = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(o.dh, want.dh) and torch.equal(o.dweight, want.dweight)
    hs, graphs, outs = [h.t.clone(), h.t.clone()], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for k in range(2):
        with torch.cuda.graph(graphs[k]):
            outs.append(T.linear_logprob(hs[k], w.t, y, gl, gh, gz))
    other = (2 * h.t.float()).bfloat16()
    hs[1].copy_(other)
    graphs[0].replay()
    graphs[1].replay()
    eager = T.linear_logprob(other, w.t, y, gl, gh, gz)
    torch.cuda.synchronize()
    assert torch.equal(outs[0].dh, want.dh) and torch.equal(outs[0].dweight, want.dweight)
    assert torch.equal(outs[1].dh, eager.dh) and torch.equal(outs[1].dweight, eager.dweight)


def test_gradient_against_differences(T):
    """The loss in 64 bits along a direction of h and of W, by central differences
    (off by the third derivative, step^2), against the gradients' inner products:
    each gradient's error is at most its bound, added up in the 1-norm."""
    h, w, y, gl, gh, gz = inputs(60, 400, 72, 9)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    g = torch.Generator(device="cuda").manual_seed(1)
    dh, dw = (torch.randn(t.shape, device="cuda", generator=g).double() for t in (h.t, w.t))

    def loss(x, m):
        lp = torch.log_softmax(x @ m.t(), dim=1)
        p = lp.exp()
        logp = torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None]).squeeze(1), 0.0)
        return (gl * logp - gh * (p * lp).sum(dim=1) + gz * torch.logsumexp(x @ m.t(), dim=1)).sum()

    e = 1e-5
    x, m = h.t.double(), w.t.double()
    for d, got, name, f in ((dh, o.dh, "dh", lambda s: loss(x + s * dh, m)), (dw, o.dweight, "dweight", lambda s: loss(x, m + s * dw))):
        slope = float((f(e) - f(-e)) / (2 * e))
        bound = float(((ref[name + "_b"] + U * ref[name].abs()) * d.abs()).sum()) + 1e-8
        assert abs(float((got.double() * d).sum()) - slope) <= bound


@pytest.mark.parametrize("rows,vocab,width", [(300, 2000, 768), (1000, 4000, 64)])
def test_waits_that_run_out_leave_nan(T, rows, vocab, width, monkeypatch):
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 10)
    right = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    torch.cuda.synchronize()
    for k in ("lse", "dh", "dweight"):
        got, want = getattr(o, k), getattr(right, k)
        assert bool((got.isnan() | (got == want)).all()), k
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    again = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    assert torch.equal(again.dh, right.dh) and torch.equal(again.dweight, right.dweight)


@pytest.mark.parametrize("later", [False, True])
@pytest.mark.parametrize("g", [-1.0, -1.02, -1 / 3, -0.9, 1.7, -1e-30])
def test_the_targets_gradients_are_rounded_finely(T, g, later):
    """Tokens that count alike have their weight scaled to 127/64 of a power of two
    before dz is rounded.  |z| <= 1 over 300 tokens: p <= e^2 / 300 < 2^-5, so that the
    targets' dz are at least 1.92 there and rounded by 2^-8 / 1.92; p is off by
    2^-11 + 2^-17 of itself; 1 - p, the scale, its inverse and the products by 2^-19
    at most.  (A rounding without the scale is up to 2^-8 off.)"""
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.rand(300, 64, device="cuda", generator=gen) / 4 - 1 / 8).bfloat16()
    h = (torch.rand(40, 64, device="cuda", generator=gen) / 4 - 1 / 8).bfloat16()
    y = torch.arange(0, 280, 7, device="cuda")
    weight = torch.full((40,), g, device="cuda")
    p = torch.softmax(h.double() @ w.double().t(), dim=1)
    # one token's at a time, the others without a target: dW's row is that token's alone but for their zeros
    for i in (0, 17, 39):
        t = torch.full_like(y, -1)
        t[i] = y[i]
        dw = torch.empty(300, 64, device="cuda")
        if later:
            o = T.linear_logprob(h, w, t)
            T.linear_logprob_grad(h, w, t, o.lse, o.entropy, weight, dh=False, dweight=dw)
        else:
            T.linear_logprob(h, w, t, weight, dh=False, dweight=dw)
        want = float(weight[0]) * (1 - p[i, y[i]]) * h[i].double()
        assert bool(((dw[y[i]].double() - want).abs() <= (2.0 ** -8 / 1.92 + 2.0 ** -15) * want.abs()).all())


def test_scale_with_weights_that_are_none(T):
    """Zero, infinite, NaN and the smallest weights among the first tokens: no scale, the rest as ever."""
    h, w, y, gl, gh, gz = inputs(70, 300, 96, 4)
    ref = reference(h.t, w.t, y, torch.zeros_like(gl), gh, gz)
    o = T.linear_logprob(h.t, w.t, y, torch.zeros_like(gl), gh, gz)
    near(o.dh, ref, "dh")
    near(o.dweight, ref, "dweight", U)
    y[:] = 5
    for bad in (float("inf"), float("nan")):
        for f in (0, 1):
            g = gl.clone()
            g[3] = bad
            a = T.linear_logprob(h.t, w.t, y, g, gh, gz)
            dh = a.dh if f == 0 else T.linear_logprob_grad(h.t, w.t, y, a.lse, a.entropy, g, gh, gz)[0]
            ref = reference(h.t, w.t, y, gl, gh, gz)
            rest = torch.arange(70, device="cuda") != 3
            off = (dh.double() - ref["dh"]).abs()
            assert bool((off <= ref["dh_b"])[rest].all()) and bool(dh[3].isnan().all())


def later_reference(h, w, y, gl, gh, gz):
    """dh, dW and their bounds for lse and entropy of an earlier call: both the logits and
    that lse are off by E, lse by its sum and rounding too (2^-16 + 2^-23 |lse|), the
    exponential by 2^-18, so that p is off by their sum of itself; H of the earlier
    call by at most 1 + ln V times that.  The rest as above."""
    x, m = h.double(), w.double()
    v, c = m.shape
    z = x @ m.t()
    e = (x.abs() @ m.abs().t()).amax(dim=1, keepdim=True) * (2.0 ** -18 + c / 512 * 2.0 ** -24)
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    lp = z - lse
    p = lp.exp()
    ent = -(p * lp).sum(dim=1, keepdim=True)
    a, b, k = (q[:, None].double() for q in (gl, gh, gz))
    a = torch.where((y >= 0)[:, None], a, 0.0)
    d = p * ((k - a) - b * (lp + ent))
    db = (2 * e + 2.0 ** -16 + 2.0 ** -23 * lse.abs() + 2.0 ** -18) * p * ((k - a).abs() + b.abs() * ((lp + ent).abs() + 1 + 2 * math.log(v)))
    d.scatter_add_(1, y.clamp(min=0)[:, None], a)
    db += (U + 2.0 ** -18) * (d.abs() + db)
    dh, dw = d @ m, d.t() @ x
    return {"dh": dh, "dh_b": db @ m.abs() + U * dh.abs() + 1e-38, "dweight": dw, "dweight_b": db.t() @ x.abs()}


@pytest.mark.parametrize("shift", [-20000.0, -100.0, 100.0, 20000.0])
@pytest.mark.parametrize("rows,vocab,width", [(33, 900, 128), (300, 64, 128), (70, 50257, 64), (5, 129, 128)])
def test_large_logits_and_weights_known_later(T, rows, vocab, width, shift):
    """All logits of a token far below or above 0: what lies between the vocabulary and
    the next multiple of 64 has logits of 0 in the products and counts for nothing, also
    where a token has no weights at all."""
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 6)
    h.t[:, 0] = 128.0
    w.t[:, 0] = shift / 128.0
    for g in (gl, gh, gz):
        g[2::5] = 0.0
    o = T.linear_logprob(h.t, w.t, y)
    dw = torch.empty(vocab, width, device="cuda")
    dh, _ = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dweight=dw)
    ref = later_reference(h.t, w.t, y, gl, gh, gz)
    near(dh, ref, "dh")
    near(dw, ref, "dweight", 2.0 ** -23)
    assert bool((dh[2::5] == 0).all())


def test_masked_and_non_finite_logits_and_weights_known_later(T):
    """From lse and entropy of an earlier call: logits of -inf have no gradient, nor has a row
    of them; a row with NaN or +inf is NaN, and no other is."""
    rows, vocab, width = 40, 700, 64
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 4)
    h.t.abs_().clamp_(min=0.01)
    masked = torch.arange(vocab, device="cuda") % 3 == 0
    w.t[masked, 7] = float("-inf")
    y.clamp_(min=1)
    y[y % 3 == 0] -= 1
    o = T.linear_logprob(h.t, w.t, y)
    dw = torch.empty(vocab, width, device="cuda")
    T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=False, dweight=dw)
    assert bool((dw[masked] == 0).all())
    index = torch.cumsum((~masked).long(), 0) - 1              # of the words that are left
    ref = later_reference(h.t, w.t[~masked], index[y], gl, gh, gz)
    near(dw[~masked], ref, "dweight", 2.0 ** -23)
    w.t[:, 7] = float("-inf")
    o = T.linear_logprob(h.t, w.t, y)
    T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=False, dweight=dw)
    assert bool((o.lse == float("-inf")).all()) and bool((dw == 0).all())
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 4)
    clean = T.linear_logprob(h.t, w.t, y)
    want, _ = T.linear_logprob_grad(h.t, w.t, y, clean.lse, clean.entropy, gl, gh, gz, dweight=False)
    h.t[3, 5] = float("nan")
    h.t[8] = 0.0
    h.t[8, 0] = float("inf")
    o = T.linear_logprob(h.t, w.t, y)
    dh, _ = T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dweight=False)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[3] = bad[8] = True
    assert torch.equal(dh.isnan().all(dim=1), bad) and torch.equal(dh[~bad], want[~bad])


FEW = [(1, 50304, 768, 0, 0), (7, 5003, 1283, 5, 3), (32, 20000, 4096, 8, 8), (31, 513, 2049, 0, 0), (2, 1000, 8192, 0, 0), (17, 50257, 1280, 5, 0),
       (1, 100000, 130, 0, 0)]


@pytest.mark.parametrize("rows,vocab,width,pad,offset", FEW)
def test_few_tokens_of_wide_models(T, rows, vocab, width, pad, offset):
    """At most 32 tokens without gradients: sums are cut every 128 products (8 additions of
    the tensor cores, 2^-20 of S) and width / 128 such sums are added in fp32, which is
    below the E above up to a width of 8192: 2^-20 + width / 128 2^-24 <= 2^-18 + width /
    512 2^-24.  The same bits from call to call, and from a captured one."""
    h, w, y, _, _, _ = inputs(rows, vocab, width, rows + vocab + width, pad, offset)
    ref = reference(h.t, w.t, y)
    o = T.linear_logprob(h.t, w.t, y)
    for k in ("lse", "entropy", "logp"):
        near(getattr(o, k), ref, k)
    assert h.untouched() and w.untouched()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = T.linear_logprob(h.t, w.t, y)
    for _ in range(2):
        graph.replay()
        again = T.linear_logprob(h.t, w.t, y)
        for k in ("lse", "entropy", "logp"):
            assert torch.equal(getattr(c, k), getattr(o, k)) and torch.equal(getattr(again, k), getattr(o, k)), k
    # the gradients' call cuts its sums elsewhere
    if rows * vocab <= 1 << 20:
        o2 = T.linear_logprob(h.t, w.t, y, g_lse=torch.ones(rows, device="cuda") / rows, dweight=False)
        for k in ("lse", "entropy", "logp"):
            near(getattr(o2, k), ref, k)


def test_few_tokens_waits_that_run_out_leave_nan(T, monkeypatch):
    h, w, y, _, _, _ = inputs(5, 60000, 2048, 11)
    right = T.linear_logprob(h.t, w.t, y)
    torch.cuda.synchronize()
    monkeypatch.setenv("LM_WAIT_LIMIT_NS", "1")
    o = T.linear_logprob(h.t, w.t, y)
    torch.cuda.synchronize()
    for k in ("lse", "entropy"):
        got, want = getattr(o, k), getattr(right, k)
        assert bool((got.isnan() | (got == want)).all()), k
    monkeypatch.delenv("LM_WAIT_LIMIT_NS")
    assert torch.equal(T.linear_logprob(h.t, w.t, y).lse, right.lse)


@pytest.mark.parametrize("rows,vocab,width", [(16384, 50304, 768), (4096, 50257, 1024)])
def test_large_steps_repeat_their_bits(T, rows, vocab, width):
    """Several pieces, teams and split sums: every output of a whole step is the same, call after call."""
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 12)
    first = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
    for _ in range(8):
        o = T.linear_logprob(h.t, w.t, y, gl, gh, gz)
        assert all(torch.equal(a, b) for a, b in zip(o, first))
    later = T.linear_logprob_grad(h.t, w.t, y, first.lse, first.entropy, gl, gh, gz)
    for _ in range(4):
        o = T.linear_logprob_grad(h.t, w.t, y, first.lse, first.entropy, gl, gh, gz)
        assert all(torch.equal(a, b) for a, b in zip(o, later))


@pytest.mark.parametrize("shift", [-4096.0, -512.0, 0.0, 512.0, 4096.0])
@pytest.mark.parametrize("rows,vocab", [(64, 900), (40, 20000)])
def test_gradients_of_tokens_that_are_almost_certain(T, rows, vocab, shift):
    """1 - p of 1e-6 to 1e-2, all logits far from 0: in the one call lse's rounding at its own
    size (2^-24 |lse|, 2^-12 here) does not reach dz.  1 - p is the others' sum, off by 2 E +
    2^-18 of itself, and by what numbers near 1 lose: the sum's additions (32 of a
    chain in a tile, fewer than 96 after it), 2^-24 each, the logarithm and the
    exponential, 2^-22 each.  The others' p are off by 2 E + 2^-11 + 2^-18 of
    themselves; then dz is rounded, and the products' sums, as above."""
    width = 64
    g = torch.Generator(device="cuda").manual_seed(vocab)
    w = torch.randn(vocab, width, device="cuda", generator=g)
    h = torch.randn(rows, width, device="cuda", generator=g) / 8
    y = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    h += torch.linspace(12, 24, rows, device="cuda")[:, None] * w[y] / w[y].square().sum(dim=1, keepdim=True)
    h[:, 0] = 128.0
    w[:, 0] = shift / 128.0
    h, w = h.bfloat16(), w.bfloat16()
    gl = torch.full((rows,), -1.0 / rows, device="cuda")
    o = T.linear_logprob(h, w, y, gl, dweight=False)
    x, m = h.double(), w.double()
    z = x @ m.t()
    e = (x.abs() @ m.abs().t()).amax(dim=1, keepdim=True) * (2.0 ** -18 + 2.0 ** -27)
    p = torch.softmax(z, dim=1)
    at = y[:, None]
    others = p.scatter(1, at, 0.0)
    rest = others.sum(dim=1, keepdim=True)                     # 1 - p of the target
    assert float(rest.min()) < 1e-4
    d = others.scatter(1, at, -rest) / rows
    db = ((2 * e + 2.0 ** -11 + 2.0 ** -18) * others).scatter(1, at, (2 * e + 2.0 ** -18) * rest + 128 * 2.0 ** -24 + 2.0 ** -21) / rows
    db = db + (U + 2.0 ** -18) * (d.abs() + db)
    want = d @ m
    off, bound = (o.dh.double() - want).abs(), db @ m.abs() + U * want.abs() + 1e-38
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("to", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,width", [(1, 575, 5), (5, 1, 29), (2, 129, 29), (129, 2003, 437), (40, 3000, 4), (300, 700, 255), (1344, 183, 1181), (2043, 134, 5), (600, 3000, 260)])
def test_gradients_beside_other_columns(T, rows, vocab, width, to):
    """Rows that end between 16-byte boundaries, of a pitch that is a multiple of 16 bytes:
    what lies behind them stays as it was, written or added to."""
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, rows + vocab + width)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    dh, dw = Held(rows, width, torch.bfloat16, -width % 8), Held(vocab, width, to, -width % 8 + 8)
    o = T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=dh.t, dweight=dw.t)
    assert dh.untouched() and dw.untouched()
    near(dh.t, ref, "dh")
    near(dw.t, ref, "dweight", U)
    first = dw.t.clone()
    T.linear_logprob_grad(h.t, w.t, y, o.lse, o.entropy, gl, gh, gz, dh=dh.t, dweight=dw.t, accumulate=True)
    assert dh.untouched() and dw.untouched()
    near(dh.t, ref, "dh")
    ref["dweight"] = ref["dweight"] + first.double()
    near(dw.t, ref, "dweight", U)


def test_several_pieces_beside_other_columns(T):
    """The same where dW's sums go on from piece to piece."""
    rows, vocab, width = 2500, 270001, 21
    h, w, y, gl, gh, gz = inputs(rows, vocab, width, 5)
    ref = reference(h.t, w.t, y, gl, gh, gz)
    for to in (torch.bfloat16, torch.float32):
        dh, dw = Held(rows, width, torch.bfloat16, 3), Held(vocab, width, to, 3)
        T.linear_logprob(h.t, w.t, y, gl, gh, gz, dh=dh.t, dweight=dw.t)
        assert dh.untouched() and dw.untouched()
        near(dh.t, ref, "dh")
        near(dw.t, ref, "dweight", U)
