"""Queries and keys: norm, gain and rotation in one pass, and the gradient,
against 64 bits.

Errors that the tolerances count.  rstd: a sum of dim squares in chains of at
most 40 additions, a division and a square root, fewer than 64 roundings of
2^-24.  A result is rotated from two channels of a few products each, fewer
than 16 roundings of what they add up to in magnitude: together 2^-17 of it,
then rounded to its type, 2^-8 (bf16) or 2^-24 (fp32) of itself.  The mean of the
gradient is such a sum of magnitudes itself.  dweight adds n = tokens x heads
terms: a group's own share one after another (at least 4864 groups, or 16 heads
each), then the block's 2048 / dim groups (or 8 warps), then at most 912 blocks
in eight chains: fewer than n / 4864 + 16 + 2048 / dim + 130 roundings of what
they add up to."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E = 2.0 ** -17
EPS = 1e-5


@pytest.fixture(scope="module")
def T():
    from paper_2605_19811_gb300 import training
    return training


def turn(x, cs, n, interleaved, back=False):
    """The first n channels turned by (cos, sin), tokens x 1 x n / 2 each; and what magnitudes are added up."""
    c, s = cs
    s = -s if back else s
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if interleaved else (x[..., :n // 2], x[..., n // 2:n])
    u, v = a * c - b * s, b * c + a * s
    mu, mv = a.abs() * c.abs() + b.abs() * s.abs(), b.abs() * c.abs() + a.abs() * s.abs()
    join = lambda p, q: torch.stack((p, q), dim=-1).flatten(-2) if interleaved else torch.cat((p, q), dim=-1)  # noqa: E731
    return torch.cat((join(u, v), x[..., n:]), dim=-1), torch.cat((join(mu, mv), x[..., n:].abs()), dim=-1)


def forward(x, w, cs, n, interleaved, norm):
    x = x.double()
    if norm:
        x = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * (1.0 if w is None else w.double())
    return turn(x, cs, n, interleaved)


def gradient(dy, x, w, cs, n, interleaved, norm):
    """dx, dweight and what magnitudes each adds up."""
    d, md = turn(dy.double(), cs, n, interleaved, back=True)
    if not norm:
        return d, md, None, None
    x = x.double()
    w = 1.0 if w is None else w.double()
    rstd = (x.square().mean(dim=-1, keepdim=True) + EPS) ** -0.5
    xh = x * rstd
    dx = rstd * (w * d - xh * (w * d * xh).mean(dim=-1, keepdim=True))
    aw = w if isinstance(w, float) else w.abs()
    m = rstd * (aw * md + xh.abs() * (aw * md * xh.abs()).mean(dim=-1, keepdim=True))
    return dx, m, (d * xh).sum(dim=(0, 1)), (md * xh.abs()).sum(dim=(0, 1))


class Case:
    """q and k as views of one buffer: packed (a QKV product), apart (heads first), or off 16-byte boundaries."""

    def __init__(self, tokens, hq, hk, dim, turned, interleaved, norm, dtype, lay, seed=0, gains=True):
        g = torch.Generator(device="cuda").manual_seed(seed + tokens + dim)
        r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.n, self.inter, self.norm, self.dtype = turned, interleaved, norm, dtype
        self.views = lambda buf: self.cut(buf, tokens, hq, hk, dim, lay)
        self.size = (hq + 2 * hk) * dim * tokens + 64 + tokens * 3
        self.buf = (r(self.size) * 2).to(dtype)
        self.q, self.k = self.views(self.buf)
        self.dbuf = r(self.size).to(dtype)
        self.dq, self.dk = self.views(self.dbuf)
        w = (lambda: (1 + 0.3 * r(dim)).to(dtype)) if norm and gains else (lambda: None)
        self.qw, self.kw = w(), w()
        self.rows = 5000
        self.pos = torch.randint(0, self.rows, (tokens,), device="cuda", generator=g)
        f = 100.0 ** (-torch.arange(0, turned, 2, device="cuda", dtype=torch.float64) / max(turned, 1))
        a = torch.arange(self.rows, device="cuda", dtype=torch.float64)[:, None] * f
        self.table = torch.stack((a.cos(), a.sin()), dim=-1).float() if turned else None

    @staticmethod
    def cut(buf, tokens, hq, hk, dim, lay):
        if lay == "apart":
            q = buf[:tokens * hq * dim].view(hq, tokens, dim).transpose(0, 1)
            return q, buf[tokens * hq * dim:tokens * (hq + hk) * dim].view(hk, tokens, dim).transpose(0, 1)
        first, pitch = (3, (hq + 2 * hk) * dim + 3) if lay == "odd" else (0, (hq + 2 * hk) * dim)
        whole = torch.as_strided(buf, (tokens, (hq + 2 * hk) * dim), (pitch, 1), first)
        return whole[:, :hq * dim].unflatten(1, (hq, dim)), whole[:, hq * dim:(hq + hk) * dim].unflatten(1, (hk, dim))

    def cs(self):
        if not self.n:
            return torch.zeros(1, device="cuda", dtype=torch.float64), torch.zeros(1, device="cuda", dtype=torch.float64)
        t = self.table.double()[self.pos][:, None]
        return t[..., 0], t[..., 1]

    def args(self):
        return dict(norm=self.norm, eps=EPS, interleaved=self.inter)

    def pairs(self):
        return ((self.q, self.dq, self.qw), (self.k, self.dk, self.kw))


def near(got, want, most, dtype, e=E):
    off = (got.double() - want).abs()
    bound = e * most + HALF[dtype] * want.abs() + 1e-38
    assert bool((off <= bound).all()), float((off / bound).max())


CASES = [(1, 32, 8, 128, 128, False, True, "packed"), (1, 1, 1, 2, 2, False, True, "packed"), (7, 3, 1, 64, 64, False, True, "packed"),
         (130, 12, 12, 64, 64, True, True, "packed"), (33, 5, 2, 80, 32, False, True, "packed"), (33, 4, 4, 80, 40, False, True, "packed"),
         (20, 4, 2, 96, 96, True, True, "apart"), (300, 8, 2, 128, 64, False, True, "apart"), (65, 2, 2, 50, 24, True, True, "packed"),
         (17, 3, 3, 50, 50, False, False, "odd"), (19, 4, 1, 128, 128, False, True, "odd"), (9, 2, 1, 256, 256, False, True, "packed"),
         (40, 6, 3, 192, 192, True, False, "packed"), (12, 2, 2, 1024, 1024, False, True, "packed"), (5, 2, 1, 513, 2, False, True, "packed"),
         (21, 3, 2, 128, 0, False, True, "packed"), (4, 2, 2, 1, 0, False, True, "packed"), (2000, 10, 5, 128, 128, False, True, "packed"),
         (50, 4, 4, 48, 16, False, True, "packed"), (50, 4, 4, 8, 8, False, True, "packed"), (50, 4, 4, 16, 16, True, False, "packed"),
         (28, 3, 1, 320, 64, False, True, "packed"), (28, 3, 1, 576, 576, True, True, "apart")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,hq,hk,dim,turned,interleaved,norm,lay", CASES)
def test_against_64_bits(T, tokens, hq, hk, dim, turned, interleaved, norm, lay, dtype):
    c = Case(tokens, hq, hk, dim, turned, interleaved, norm, dtype, lay)
    cs, kept = c.cs(), c.buf.clone()
    out = torch.full_like(c.buf, 77.0)
    qo, ko = c.views(out)
    T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args(), q_out=qo, k_out=ko)
    for (x, _, w), got in zip(c.pairs(), (qo, ko)):
        near(got, *forward(x, w, cs, c.n, c.inter, c.norm), dtype)
    mark = torch.zeros_like(out, dtype=torch.bool)
    for v in c.views(mark):
        v.fill_(True)
    assert bool((out[~mark] == 77).all()) and torch.equal(c.buf, kept)
    o = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args())
    assert o.q.is_contiguous() and torch.equal(o.q, qo) and torch.equal(o.k, ko)
    # the gradient
    dout = torch.full_like(c.buf, 77.0)
    dqo, dko = c.views(dout)
    r = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args(), dq_out=dqo, dk_out=dko)
    for (x, d, w), got, dw in zip(c.pairs(), (dqo, dko), (r.dq_weight, r.dk_weight)):
        dx, m, dwant, dm = gradient(d, x, w, cs, c.n, c.inter, c.norm)
        near(got, dx, m, dtype)
        if norm:
            near(dw, dwant, dm, dtype, E + (x[..., 0].numel() / 4864 + 146 + 2048 / dim) * 2.0 ** -24)
        else:
            assert dw is None
    assert bool((dout[~mark] == 77).all())
    r2 = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    assert torch.equal(r2.dq, dqo) and torch.equal(r2.dk, dko)
    if norm:
        assert torch.equal(r2.dq_weight, r.dq_weight) and torch.equal(r2.dk_weight, r.dk_weight)
    # in place
    T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args(), q_out=c.q, k_out=c.k)
    assert torch.equal(c.q, qo) and torch.equal(c.k, ko)
    c.buf.copy_(kept)
    T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args(), dq_out=c.dq, dk_out=c.dk)
    assert torch.equal(c.dq, dqo) and torch.equal(c.dk, dko)


def test_queries_alone_no_gain_no_dweight(T):
    c = Case(40, 4, 4, 64, 64, False, True, torch.float32, "packed", gains=False)
    o = T.qk_rotary(c.q, None, c.pos, c.table, **c.args())
    assert o.k is None
    near(o.q, *forward(c.q, None, c.cs(), 64, False, True), torch.float32)
    r = T.qk_rotary_grad(c.dq, None, c.pos, c.table, c.q, **c.args())
    assert r.dk is None and r.dk_weight is None and r.dq_weight.dtype == torch.float32
    n = T.qk_rotary_grad(c.dq, None, c.pos, c.table, c.q, **c.args(), dweight=False)
    assert n.dq_weight is None and torch.equal(n.dq, r.dq)
    # fp32 gains of bf16 heads
    b = Case(40, 4, 4, 64, 64, False, True, torch.bfloat16, "packed")
    full = T.qk_rotary(b.q, b.k, b.pos, b.table, b.qw.float(), b.kw, **b.args())
    assert torch.equal(full.q, T.qk_rotary(b.q, b.k, b.pos, b.table, b.qw, b.kw, **b.args()).q)
    assert T.qk_rotary_grad(b.dq, b.dk, b.pos, b.table, b.q, b.k, b.qw.float(), b.kw, **b.args()).dq_weight.dtype == torch.float32


def test_positions_outside_the_table(T):
    c = Case(10, 2, 1, 64, 32, False, True, torch.float32, "packed")
    want = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args())
    wantg = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    for k, bad in ((2, -1), (5, c.rows), (7, 1 << 62), (8, -(1 << 62))):
        c.pos[k] = bad
    ok = torch.ones(10, dtype=torch.bool, device="cuda")
    ok[[2, 5, 7, 8]] = False
    o = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args())
    assert bool(o.q[~ok][..., :32].isnan().all()) and torch.equal(o.q[..., 32:], want.q[..., 32:]) and torch.equal(o.q[ok], want.q[ok])
    r = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    assert bool(r.dk[~ok].isnan().all()) and torch.equal(r.dk[ok], wantg.dk[ok])


def test_rows_of_zeros_infinity_and_nan(T):
    c = Case(6, 2, 2, 128, 128, False, True, torch.bfloat16, "packed")
    c.q[1, 0] = 0.0
    c.q[2, 1, 5] = float("nan")
    c.k[3, 0, 7] = float("inf")
    o = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args())
    assert bool((o.q[1, 0] == 0).all()) and bool(o.q[2, 1].isnan().all())
    assert int(o.k[3, 0].isnan().sum()) == 2 and int(o.q.isnan().any(dim=-1).sum()) == 1      # inf * 0 in its pair, zeros elsewhere
    assert bool((o.k[3, 0][~o.k[3, 0].isnan()] == 0).all())


def test_offsets_beyond_31_bits(T):
    """2.6 G elements: the last tokens' results, forward and gradient, are those of a call with them alone."""
    tokens, heads, dim = 500001, 40, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.empty(tokens, heads, dim, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    pos = torch.arange(tokens, device="cuda") % 1000
    table = T.rotary_table(1000, T.rotary_frequencies(dim))
    w = torch.rand(dim, device="cuda", generator=g)
    o = T.qk_rotary(q, None, pos, table, w)
    r = T.qk_rotary_grad(q, None, pos, table, q, None, w)
    for at in (0, tokens - 300):
        e = slice(at, at + 300)
        assert torch.equal(o.q[e], T.qk_rotary(q[e], None, pos[e], table, w).q)
        assert torch.equal(r.dq[e], T.qk_rotary_grad(q[e], None, pos[e], table, q[e], None, w).dq)


def test_no_tokens(T):
    c = Case(3, 2, 2, 64, 64, False, True, torch.float32, "packed")
    o = T.qk_rotary(c.q[:0], c.k[:0], c.pos[:0], c.table, c.qw, c.kw, **c.args())
    assert o.q.shape == (0, 2, 64)
    r = T.qk_rotary_grad(c.dq[:0], c.dk[:0], c.pos[:0], c.table, c.q[:0], c.k[:0], c.qw, c.kw, **c.args())
    assert bool((r.dq_weight == 0).all()) and bool((r.dk_weight == 0).all())


def test_leading_dimensions_streams_and_graphs(T):
    c = Case(64, 4, 2, 128, 128, False, True, torch.bfloat16, "packed")
    want = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args())
    b = T.qk_rotary(c.q.unflatten(0, (4, 16)), c.k.unflatten(0, (4, 16)), c.pos.view(4, 16), c.table, c.qw, c.kw, **c.args())
    assert b.q.shape == (4, 16, 4, 128) and torch.equal(b.q.flatten(0, 1), want.q)
    grad = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args(), stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(o.k, want.k)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    with torch.cuda.graph(graphs[0]):
        outs.append(T.qk_rotary(c.q, c.k, c.pos, c.table, c.qw, c.kw, **c.args()))
    with torch.cuda.graph(graphs[1]):
        outs.append(T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args()))
    for g in graphs + graphs:
        g.replay()
    assert torch.equal(outs[0].q, want.q) and torch.equal(outs[1].dq, grad.dq) and torch.equal(outs[1].dq_weight, grad.dq_weight)


def test_gradient_against_differences(T):
    """Along a direction of q and of its gain, the forward definition in 64 bits by central differences."""
    c = Case(30, 3, 2, 80, 32, True, True, torch.float32, "packed")
    r = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    g = torch.Generator(device="cuda").manual_seed(1)
    dx, dw = torch.randn(c.q.shape, device="cuda", generator=g).double(), torch.randn(80, device="cuda", generator=g).double()
    f = lambda s, t: float((forward(c.q.double() + s * dx, c.qw.double() + t * dw, c.cs(), 32, True, True)[0] * c.dq.double()).sum())  # noqa: E731
    e = 1e-6
    for slope, got in (((f(e, 0) - f(-e, 0)) / (2 * e), (r.dq.double() * dx).sum()), ((f(0, e) - f(0, -e)) / (2 * e), (r.dq_weight.double() * dw).sum())):
        assert abs(float(got) - slope) <= 1e-5 * (1 + abs(slope)) + 1e-3 * 2.0 ** -10 * c.dq.numel()


@pytest.mark.parametrize("dims,factor,original", [(64, 1.0, 0), (128, 8.0, 0), (128, 8.0, 8192)])
def test_tables(T, dims, factor, original):
    """The table's angles in 64 bits at far positions, and which frequencies a longer context divides."""
    f = T.rotary_frequencies(dims, 10000.0, factor, original)
    plain = T.rotary_frequencies(dims, 10000.0)
    turns = 8192 * plain / (2 * 3.141592653589793)
    if not original:
        assert torch.allclose(f * factor, plain, rtol=1e-15)
    else:
        assert torch.equal(f[turns >= 4], plain[turns >= 4]) and torch.allclose(f[turns <= 1] * factor, plain[turns <= 1], rtol=1e-15)
        between = (turns > 1) & (turns < 4)
        assert bool((f[between] < plain[between]).all()) and bool((f[between] * factor > plain[between]).all())
    t = T.rotary_table(200000, f, amplitude=1.5)
    at = torch.tensor([0, 1, 777, 131071, 199999])
    a = at.double()[:, None] * f
    want = 1.5 * torch.stack((a.cos(), a.sin()), dim=-1)
    # the two machines' 64-bit cosines of angles up to 2^18 agree to 2^-33
    assert t.shape == (200000, dims // 2, 2) and float((t.cpu()[at].double() - want).abs().max()) <= 1.5 * (2.0 ** -24 + 2.0 ** -33)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,hq,hk,dim,turned,interleaved,norm,lay", [case for case in CASES if case[6]])
def test_gradient_over_an_input(T, tokens, hq, hk, dim, turned, interleaved, norm, lay, dtype):
    """Over dy, or over the forward call's queries and keys: the same bits."""
    c = Case(tokens, hq, hk, dim, turned, interleaved, norm, dtype, lay)
    want = T.qk_rotary_grad(c.dq, c.dk, c.pos, c.table, c.q, c.k, c.qw, c.kw, **c.args())
    for over in ("x", "dy"):
        d = Case(tokens, hq, hk, dim, turned, interleaved, norm, dtype, lay)
        to = (d.q, d.k) if over == "x" else (d.dq, d.dk)
        got = T.qk_rotary_grad(d.dq, d.dk, d.pos, d.table, d.q, d.k, d.qw, d.kw, **d.args(), dq_out=to[0], dk_out=to[1])
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def longest_chain(tokens, hq, hk, dim, fp32):
    """Of the roundings that one term of each dweight goes through: eight channels a lane,
    in one wave of 304 blocks (fp32: 152), which the two parts share by their steps of four
    heads; a group of lanes adds up its items' heads, a block its groups, the join
    the blocks in eight chains."""
    lanes = 1
    while 8 * lanes < dim:
        lanes *= 2
    groups, most = 256 // lanes, 152 if fp32 else 304
    size = min(max(1, tokens * (hq + hk) // (152 * 32 * (32 // lanes))), 16)
    parts = []
    for n in (hq, hk):
        a = -(-n // -(-n // size)) if n else 0
        a = -(-a // 4) * 4 if a > 4 else a
        parts.append((a, -(-n // a) if n else 0))
    steps = [items * -(-a // 4) for a, items in parts]
    out = []
    for (a, items), mine in zip(parts, steps):
        if not items:
            continue
        blocks = min(-(-tokens * items // groups), max(1, most * mine // sum(steps)))
        out.append(a * -(-tokens * items // (blocks * groups)) + groups + -(-blocks // 8) + 8)
    return out


MANY = [(8193, 20, 5, 80, 32, True, "packed"), (8193, 20, 5, 256, 256, False, "packed"), (9001, 9, 9, 128, 64, False, "packed"),
        (4097, 33, 3, 64, 64, True, "apart"), (20011, 13, 0, 48, 48, False, "packed"), (8193, 17, 7, 50, 50, False, "packed"), (8193, 11, 6, 80, 80, False, "odd")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,hq,hk,dim,turned,interleaved,lay", MANY)
def test_many_heads_an_item(T, tokens, hq, hk, dim, turned, interleaved, lay, dtype):
    """Items of 8 to 16 heads, several steps each, and numbers of heads that they do not
    divide; heads of other sizes and alignments one after another.  Both gains' gradients
    of up to 260000 heads."""
    c = Case(tokens, hq, hk, dim, turned, interleaved, True, dtype, lay)
    cs = c.cs()
    k, dk, kw = (c.k, c.dk, c.kw) if hk else (None, None, None)
    o = T.qk_rotary(c.q, k, c.pos, c.table, c.qw, kw, **c.args())
    r = T.qk_rotary_grad(c.dq, dk, c.pos, c.table, c.q, k, c.qw, kw, **c.args())
    eight = dim % 8 == 0 and lay != "odd"
    # a warp's own terms, 8 warps, and 304 blocks in eight chains, or as above
    chains = longest_chain(tokens, hq, hk, dim, dtype == torch.float32) if eight else \
        [-(-tokens * n // (8 * 304)) + 8 + 38 + 8 for n in (hq, hk)]
    for (x, d, w), got, dx, dw, chain in zip(c.pairs()[:2 if hk else 1], (o.q, o.k), (r.dq, r.dk), (r.dq_weight, r.dk_weight), chains):
        near(got, *forward(x, w, cs, c.n, interleaved, True), dtype)
        want, m, dwant, dm = gradient(d, x, w, cs, c.n, interleaved, True)
        near(dx, want, m, dtype)
        near(dw, dwant, dm, dtype, E + chain * 2.0 ** -24)
        del want, m
    r2 = T.qk_rotary_grad(c.dq, dk, c.pos, c.table, c.q, k, c.qw, kw, **c.args())
    assert all(torch.equal(a, b) for a, b in zip(r, r2) if a is not None)
