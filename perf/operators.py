"""Cases that measure the training-step operators next to the optimizer: token
log probabilities with entropy, top alternatives and gradient; RMS norm with
the residual's addition, an 8-bit output and gradient; 8-bit activation
checkpoints and the weight gradient of a linear layer taken from them.

Every operator has a plain form (elementary torch operations in 32 bits,
rounded once at the end), which runs where ``own`` is false, and the
framework's calls, which run where it is true.  ``exact`` gives the operator's
definition in 64 bits.

An 8-bit checkpoint of a rows x cols matrix is: codes, one byte an element
(int8 or e4m3), row pitch a multiple of 16; scales, float32, one row for each
group of 128 channels and one column for each token.  A scale is the least
power of two s with max|x| <= limit * s over its group (limit 127 or 448), a
code is x / s rounded to nearest even, and the value it stands for is code * s.
"""

import math

import torch

own = False

GROUP = 128
LIMIT = {"i8": 127.0, "e4m3": 448.0}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6

# The largest listed sizes; a drawn case costs no more.
MOST_LOGITS = 16384 * 50304
MOST_NORM = 16384 * 1280
MOST_PACK = 32768 * 5120
MOST_WGRAD = 16384 * 4096 * 14336


def listed():
    return [
        # One decoded token: its log probability, entropy and the 8 best alternatives.  Latency.
        {"name": "logprob_one_token", "op": "logprob", "rows": 1, "vocab": 50304, "pad": 0, "dtype": "bf16", "top": 8},
        # Scoring a batch of sampled sequences over an unpadded vocabulary, fp32 logits, odd rows and pitch.
        {"name": "logprob_scoring", "op": "logprob", "rows": 2049, "vocab": 50257, "pad": 0, "dtype": "f32", "top": 5},
        # Cross entropy with an entropy bonus and a squared-lse term over 16 sequences of 1024: loss and gradient in one call.
        {"name": "logprob_loss", "op": "logprob_loss", "rows": 16384, "vocab": 50304, "pad": 0, "dtype": "bf16", "top": 0},
        # The gradient alone, for weights that are known only after the forward pass (policy gradients).
        {"name": "logprob_grad", "op": "logprob_grad", "rows": 8192, "vocab": 50257, "pad": 47, "dtype": "bf16", "top": 0},
        # One decoded token's norm with an 8-bit output for an 8-bit product.  Latency.
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 4096, "pad": 0, "dtype": "bf16", "format": "e4m3", "residual": True},
        # A block's pre-norm over 16 sequences of 1024, its output kept in 8 bits for the weight gradient.
        {"name": "norm_forward", "op": "norm", "rows": 16384, "cols": 1280, "pad": 0, "dtype": "bf16", "format": "e4m3", "residual": True},
        # The same norm's gradient from the stored residual stream.
        {"name": "norm_grad", "op": "norm_grad", "rows": 16384, "cols": 1280, "pad": 0, "dtype": "bf16", "format": "none", "residual": True},
        # A norm's gradient whose input was kept in 8 bits; fp32 activations, odd rows and channels, padded rows.
        {"name": "norm_grad_kept", "op": "norm_grad", "rows": 8191, "cols": 1283, "pad": 5, "dtype": "f32", "format": "i8", "residual": False},
        # The MLP's hidden activations kept in 8 bits, and read back.
        {"name": "checkpoint_hidden", "op": "checkpoint", "rows": 32768, "cols": 5120, "pad": 0, "dtype": "bf16", "format": "i8"},
        # The QKV weight gradient of the 768-wide model: few output tiles, a long sum over tokens.
        {"name": "wgrad_qkv", "op": "wgrad", "rows": 16384, "cols": 768, "out": 2304, "pad": 0, "dtype": "bf16", "format": "e4m3", "to": "bf16"},
        # An odd layer in fp32: ragged in every direction.
        {"name": "wgrad_odd", "op": "wgrad", "rows": 1021, "cols": 1283, "out": 517, "pad": 0, "dtype": "f32", "format": "i8", "to": "f32"},
        # The 4096 x 14336 MLP matrices of the large set, fp32 weight gradients.
        {"name": "wgrad_mlp", "op": "wgrad", "rows": 16384, "cols": 4096, "out": 14336, "pad": 0, "dtype": "bf16", "format": "i8", "to": "f32"},
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], even over its logarithm; one in three is rounded to a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 1 / 3 and high >= 64:
        v = -(-v // 64) * 64
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["logprob", "logprob_loss", "logprob_grad", "norm", "norm", "norm_grad", "norm_grad", "checkpoint", "wgrad", "wgrad", "wgrad"])
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"]), "pad": rng.choice([0, 0, 1, 8, 13])}
    size = 2 if case["dtype"] == "f32" else 1
    if op.startswith("logprob"):
        case["vocab"] = _spread(rng, 1000, 160000)
        case["rows"] = _spread(rng, 1, max(1, min(16384, MOST_LOGITS // (size * (case["vocab"] + 13)))))
        case["top"] = rng.choice([0, 1, 4, 8, 20]) if op == "logprob" else 0
        return case
    if op == "wgrad":
        case["cols"] = _spread(rng, 64, 8192)
        case["out"] = _spread(rng, 64, 16384)
        case["rows"] = _spread(rng, 1, max(1, min(32768, MOST_WGRAD // (3 * size * case["cols"] * case["out"]))))
        case["format"] = rng.choice(["i8", "e4m3"])
        case["to"] = rng.choice(["bf16", "f32"])
        return case
    most = MOST_PACK if op == "checkpoint" else MOST_NORM
    case["cols"] = _spread(rng, 64, 16384)
    case["rows"] = _spread(rng, 1, max(1, min(32768, most // (size * (case["cols"] + 13)))))
    case["format"] = rng.choice(["i8", "e4m3"] if op == "checkpoint" else ["none", "i8", "e4m3"])
    if op != "checkpoint":
        case["residual"] = rng.random() < 0.5
    return case


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    rows = case["rows"]
    if case["op"].startswith("logprob"):
        n = rows * case["vocab"]
        if case["op"] == "logprob":
            return {"bytes": n * e + rows * (8 + 12 + 12 * case["top"]), "flops": 7 * n}
        if case["op"] == "logprob_loss":
            return {"bytes": 2 * n * e + rows * (8 + 12 + 12), "flops": 13 * n}
        return {"bytes": 2 * n * e + rows * (8 + 12 + 8), "flops": 7 * n}
    cols = case["cols"]
    n, groups = rows * cols, -(-cols // GROUP)
    kept = 0 if case["format"] == "none" else n + 4 * rows * groups  # codes and scales
    if case["op"] == "norm":
        # the kept copy is written, read back and given as 16-bit values
        return {"bytes": n * e * (4 if case["residual"] else 2) + 4 * cols + 4 * rows + (2 * kept + 2 * n if kept else 0), "flops": 6 * n + (4 * n if kept else 0)}
    if case["op"] == "norm_grad":
        return {"bytes": n * e * (3 if case["residual"] else 2) + (kept or n * e) + 8 * cols + 4 * rows, "flops": 11 * n}
    if case["op"] == "checkpoint":
        return {"bytes": 2 * n * e + 2 * kept, "flops": 4 * n}
    return {"bytes": rows * case["out"] * e + kept + cols * case["out"] * (4 if case["to"] == "f32" else 2), "flops": 2 * n * case["out"]}


def _activations(g, rows, cols):
    """A residual stream: normal tokens of unequal size, with a few channels far larger than the rest."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=g))
    big = torch.rand(cols, device="cuda", generator=g) < 0.004
    return x * torch.where(big, 20.0, 1.0)


def _padded(x, pad, dtype):
    """x in the given type, as a view of a tensor with `pad` more columns."""
    whole = torch.zeros(x.shape[0], x.shape[1] + pad, device="cuda", dtype=dtype)
    whole[:, : x.shape[1]] = x
    return whole[:, : x.shape[1]]


def _grouped(x):
    """rows x groups x 128, zeros past the last channel."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    return torch.nn.functional.pad(x, (0, groups * GROUP - cols)).reshape(rows, groups, GROUP)


def _scales(x, kind):
    """The least power of two s with max|x| <= limit * s for each group: rows x groups."""
    lead, limit_lead, shift = x.abs().amax(dim=2), LIMIT[kind], (7 if kind == "i8" else 9)
    m, e = torch.frexp(lead)
    e = e - shift + (m > limit_lead / 2.0**shift).to(e.dtype)
    return torch.ldexp(torch.ones_like(lead), e)


def _codes(x, s, kind):
    q = x / s[:, :, None]
    return torch.round(q).to(torch.int8) if kind == "i8" else q.to(torch.float8_e4m3fn)


def _keep(x, kind):
    """The codes (rows x pitch bytes) and scales (groups x rows) of x."""
    rows, cols = x.shape
    g = _grouped(x.float())
    s = _scales(g, kind)
    q = _codes(g, s, kind).view(torch.uint8).reshape(rows, -1)[:, :cols]
    codes = torch.zeros(rows, -(-cols // 16) * 16, device="cuda", dtype=torch.uint8)
    codes[:, :cols] = q
    return codes, s.t().contiguous()


def _kept_values(codes, scales, cols, kind, dtype=torch.float32):
    """The values that codes and scales stand for."""
    q = codes[:, :cols].contiguous().view(torch.int8 if kind == "i8" else torch.float8_e4m3fn).to(dtype)
    return q * scales.to(dtype).t().repeat_interleave(GROUP, dim=1)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, dtype, pad = case["rows"], DTYPES[case["dtype"]], case["pad"]
    s = {"case": case}
    if case["op"].startswith("logprob"):
        v = case["vocab"]
        # half of the tokens are predicted well, a tenth carry no target, a padded vocabulary's last entries are masked
        z = 2.5 * torch.randn(rows, v, device="cuda", generator=g)
        s["targets"] = torch.randint(0, v, (rows,), device="cuda", generator=g)
        lift = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.5, 12.0, 2.0)
        z.scatter_add_(1, s["targets"][:, None], lift[:, None])
        if v % 64 == 0:
            z[:, v - 47 :] = float("-inf")
            s["targets"] %= v - 47
        s["logits"] = _padded(z, pad, dtype)
        del z
        if rows > 1:
            s["targets"][torch.rand(rows, device="cuda", generator=g) < 0.1] = -100
        if case["op"] != "logprob":
            s["g_logp"] = -torch.rand(rows, device="cuda", generator=g) / rows
            s["g_entropy"] = -0.01 * torch.ones(rows, device="cuda") / rows
            s["g_lse"] = 0.002 * torch.randn(rows, device="cuda", generator=g) / rows
            s["dlogits"] = _padded(torch.zeros(rows, v, device="cuda", dtype=dtype), pad, dtype)
        if case["op"] == "logprob_grad":
            d = torch.log_softmax(s["logits"].double(), dim=1)
            s["lse"] = (s["logits"][:, :1].double() - d[:, :1]).squeeze(1).float()
            s["entropy"] = -(d.exp() * torch.where(torch.isinf(d), 0.0, d)).sum(dim=1).float()
        return s
    cols = case["cols"]
    if case["op"] == "wgrad":
        dy = 1e-3 * torch.randn(rows, case["out"], device="cuda", generator=g)
        dy *= torch.exp(0.7 * torch.randn(rows, 1, device="cuda", generator=g))
        s["dy"] = _padded(dy, pad, dtype)
        s["codes"], s["scales"] = _keep(_activations(g, rows, cols), case["format"])
        return s
    x = _activations(g, rows, cols)
    s["x"] = _padded(x, pad, dtype)
    if case["op"] == "checkpoint":
        return s
    s["weight"] = (1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(dtype)
    if case["op"] == "norm":
        if case["residual"]:
            s["residual"] = _padded(torch.randn(rows, cols, device="cuda", generator=g), pad, dtype)
        return s
    s["dy"] = _padded(1e-3 * torch.randn(rows, cols, device="cuda", generator=g), pad, dtype)
    if case["residual"]:
        s["dh"] = _padded(1e-3 * torch.randn(rows, cols, device="cuda", generator=g), pad, dtype)
    s["rstd"] = torch.rsqrt(s["x"].double().square().mean(dim=1) + EPS).float()
    if case["format"] != "none":
        s["codes"], s["scales"] = _keep(s["x"], case["format"])
        del s["x"]
    return s


def _top(z, lse, k):
    """The k largest of each row, ties to the lowest index; what is masked is no alternative."""
    v, i = torch.sort(z, dim=1, descending=True, stable=True)
    v, i = v[:, :k], i[:, :k]
    return v - lse[:, None], torch.where(torch.isinf(v), -1, i)


def _plain_gradient(z, t, lse, entropy, s, dtype):
    lp = z - lse[:, None]
    p = lp.exp()
    has = t >= 0
    gl = torch.where(has, s["g_logp"].to(z.dtype), 0.0)
    d = (s["g_lse"].to(z.dtype) - gl)[:, None] - s["g_entropy"].to(z.dtype)[:, None] * (torch.where(torch.isinf(lp), 0.0, lp) + entropy[:, None])
    d = d * p
    d.scatter_add_(1, t.clamp(min=0)[:, None], gl[:, None])
    return d.to(dtype)


def _plain_logprob(s, case):
    z, t = s["logits"].float(), s["targets"]
    if case["op"] == "logprob_grad":
        return {"dlogits": _plain_gradient(z, t, s["lse"], s["entropy"], s, s["logits"].dtype)}
    m = z.amax(dim=1)
    d = z - m[:, None]
    e = d.exp()
    total = e.sum(dim=1)
    lse = m + total.log()
    entropy = total.log() - (e * torch.where(torch.isinf(d), 0.0, d)).sum(dim=1) / total
    logp = torch.where(t >= 0, d.gather(1, t.clamp(min=0)[:, None]).squeeze(1) - total.log(), 0.0)
    r = {"logp": logp, "entropy": entropy, "lse": lse}
    if case["op"] == "logprob_loss":
        r["dlogits"] = _plain_gradient(z, t, lse, entropy, s, s["logits"].dtype)
    if case["top"]:
        r["top_logp"], r["top_index"] = _top(z, lse, case["top"])
    return r


def _plain_norm(s, case):
    x = s["x"].float()
    h = x + s["residual"].float() if case["residual"] else x
    rstd = torch.rsqrt(h.square().mean(dim=1) + EPS)
    y = h * rstd[:, None] * s["weight"].float()
    r = {"y": y.to(s["x"].dtype), "rstd": rstd}
    if case["residual"]:
        r["h"] = h.to(s["x"].dtype)
    if case["format"] != "none":
        codes, scales = _keep(y, case["format"])
        r["kept"] = _kept_values(codes, scales, case["cols"], case["format"]).to(torch.bfloat16)
    return r


def _plain_norm_grad(s, case):
    h = s["x"].float() if case["format"] == "none" else _kept_values(s["codes"], s["scales"], case["cols"], case["format"])
    dy = s["dy"].float()
    xh = h * s["rstd"][:, None]
    wdy = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (wdy - xh * (wdy * xh).mean(dim=1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * xh).sum(dim=0).to(s["weight"].dtype)}


def _plain(s, case):
    if case["op"].startswith("logprob"):
        return _plain_logprob(s, case)
    if case["op"] == "norm":
        return _plain_norm(s, case)
    if case["op"] == "norm_grad":
        return _plain_norm_grad(s, case)
    if case["op"] == "checkpoint":
        codes, scales = _keep(s["x"], case["format"])
        return {"kept": _kept_values(codes, scales, case["cols"], case["format"]).to(s["x"].dtype)}
    x = _kept_values(s["codes"], s["scales"], case["cols"], case["format"])
    return {"dweight": torch.matmul(s["dy"].float().t(), x).to(DTYPES[case["to"]])}


def run(s):
    case = s["case"]
    if not own:
        return _plain(s, case)
    from paper_2605_19811_gb300 import training as T

    if case["op"] == "logprob_grad":
        d = T.token_logprob_grad(s["logits"], s["targets"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"], s["g_lse"], dlogits=s["dlogits"])
        return {"dlogits": d}
    if case["op"].startswith("logprob"):
        loss = {k: s[k] for k in ("g_logp", "g_entropy", "g_lse", "dlogits")} if case["op"] == "logprob_loss" else {}
        o = T.token_logprob(s["logits"], s["targets"], top_k=case["top"], **loss)
        r = {"logp": o.logp, "entropy": o.entropy, "lse": o.lse}
        if loss:
            r["dlogits"] = o.dlogits
        if case["top"]:
            r["top_logp"], r["top_index"] = o.top_logp, o.top_index
        return r
    fmt = None if case["format"] == "none" else case["format"]
    if case["op"] == "norm":
        o = T.rmsnorm(s["x"], s["weight"], residual=s.get("residual"), eps=EPS, checkpoint=fmt)
        r = {"y": o.y, "rstd": o.rstd}
        if case["residual"]:
            r["h"] = o.h
        if fmt:
            r["kept"] = o.checkpoint.unpack(torch.bfloat16)
        return r
    if case["op"] == "checkpoint":
        return {"kept": T.checkpoint8(s["x"], fmt).unpack(s["x"].dtype)}
    kept = T.Checkpoint8(s["codes"], s["scales"], case["cols"], fmt) if fmt else None
    if case["op"] == "norm_grad":
        dx, dw = T.rmsnorm_grad(s["dy"], kept if fmt else s["x"], s["rstd"], s["weight"], dh=s.get("dh"))
        return {"dx": dx, "dweight": dw}
    return {"dweight": T.linear_wgrad8(s["dy"], kept, dtype=DTYPES[case["to"]])}


# --- the definitions in 64 bits, on their own ---


def _exact_values(codes, scales, cols, kind):
    """Values of a checkpoint from its bytes: e4m3 as sign, 4 bits of exponent (bias 7) and 3 of fraction."""
    b = codes[:, :cols].to(torch.int64)
    if kind == "i8":
        v = torch.where(b > 127, b - 256, b).double()
    else:
        e, f = (b >> 3) & 15, (b & 7).double()
        v = torch.where(e == 0, f / 8 * 2.0**-6, (1 + f / 8) * torch.pow(2.0, (e - 7).double()))
        v = torch.where(b > 127, -v, v)
    group = torch.arange(cols, device=codes.device) // GROUP
    return v * scales.double()[group].t()


def _exact_logprob(s, case):
    parts = []
    for at in range(0, case["rows"], 2048):  # a part of the rows at a time, for the memory's sake
        z, t = s["logits"][at : at + 2048].double(), s["targets"][at : at + 2048]
        lp = torch.log_softmax(z, dim=1)
        p = lp.exp()
        plogp = torch.xlogy(p, p)
        one = torch.zeros_like(z)
        one[torch.arange(len(t), device=z.device)[t >= 0], t[t >= 0]] = 1.0
        r = {"logp": torch.where(one > 0, lp, 0.0).sum(dim=1), "entropy": -plogp.sum(dim=1), "lse": torch.logsumexp(z, dim=1)}
        if case["op"] != "logprob":
            gl, gh, gz = (s[k][at : at + 2048, None].double() for k in ("g_logp", "g_entropy", "g_lse"))
            h = r["entropy"][:, None]
            r["dlogits"] = gl * (one - p * (t >= 0)[:, None]) - gh * (plogp + p * h) + gz * p
        if case["top"]:
            r["top_logp"] = lp.topk(case["top"], dim=1).values
        parts.append(r)
    r = {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    if case["op"] == "logprob_grad":
        return {"dlogits": r["dlogits"]}
    if case["top"]:
        r["top_index"] = None
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("logprob"):
        return _exact_logprob(s, case)
    if case["op"] == "checkpoint":
        return {"kept": s["x"].double()}  # what is kept is to stand for these
    kind = case["format"]
    if case["op"] == "wgrad":
        return {"dweight": s["dy"].double().t() @ _exact_values(s["codes"], s["scales"], case["cols"], kind)}
    if case["op"] == "norm":
        h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        rstd = (h.square().sum(dim=1) / case["cols"] + EPS) ** -0.5
        y = torch.einsum("tc,t,c->tc", h, rstd, s["weight"].double())
        r = {"y": y, "rstd": rstd}
        if case["residual"]:
            r["h"] = h
        if kind != "none":
            r["kept"] = y
        return r
    h = s["x"].double() if kind == "none" else _exact_values(s["codes"], s["scales"], case["cols"], kind)
    # y_c = w_c h_c rstd: the gradient by rstd goes back through the mean square, d rstd / d h_c = -rstd^3 h_c / cols
    dy, w, rstd = s["dy"].double(), s["weight"].double(), s["rstd"].double()[:, None]
    through = (dy * w * h).sum(dim=1, keepdim=True)
    dx = dy * w * rstd - through * rstd**3 * h / case["cols"]
    if case["residual"]:
        dx = dx + s["dh"].double()
    return {"dx": dx, "dweight": torch.einsum("tc,tc,t->c", dy, h, rstd[:, 0])}
