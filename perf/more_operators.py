"""Cases that measure the operators around the 8-bit linear layer, the model's
head and the attention's inputs: log probabilities and their loss's gradients
from the last hidden states and the head's matrix, without logits; 8-bit linear
layers (weights with one scale for each block of 128 x 128, forward product and
input gradient); the norm of queries and keys for each head with the rotation
by position in the same pass, and its gradient.

Every operator has a plain form (elementary torch operations in 32 bits,
rounded once at the end), which runs where ``own`` is false, and the
framework's calls, which run where it is true.  ``exact`` gives the operator's
definition in 64 bits.

8-bit activations are e4m3 codes, one byte an element (row pitch a multiple of
16), with one float32 scale for each token's group of 128 channels, stored
group by group.  8-bit weights are e4m3 codes with one scale for each block of
128 x 128.  A scale is the least power of two s with max|x| <= 448 s over its
group or block, a code is x / s rounded to nearest even and stands for code * s.
"""

import math

import torch

own = False

BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6

# The largest listed sizes; a drawn case costs no more.
MOST_LOGITS = 16384 * 50304
MOST_HEAD = 4096 * 4096 * 50257
MOST_LINEAR = 16384 * 4096 * 14336
MOST_HEADS = 16384 * 40 * 128


def listed():
    return [
        # One sampled token scored from its hidden state, the 768-wide model's head.  Latency: the head's matrix read once.
        {"name": "head_one_token", "op": "head", "rows": 1, "width": 768, "vocab": 50304, "pad": 0},
        # Scoring a batch of sequences with the 1280-wide model: odd rows, an unpadded vocabulary, an odd pitch.
        {"name": "head_scoring", "op": "head", "rows": 2049, "width": 1280, "vocab": 50257, "pad": 5},
        # A training step's loss over 16 sequences of 1024 (cross entropy, entropy bonus, squared-lse term) with both gradients, 768 wide.
        {"name": "head_loss", "op": "head_loss", "rows": 16384, "width": 768, "vocab": 50304, "pad": 0},
        # The same for a 4096-wide model over an unpadded vocabulary.
        {"name": "head_loss_wide", "op": "head_loss", "rows": 4096, "width": 4096, "vocab": 50257, "pad": 0},
        # One decoded token through the large set's MLP matrix, its weights kept in 8 bits.  Latency: the codes read once.
        {"name": "linear_one_token", "op": "linear", "rows": 1, "in": 4096, "out": 14336, "pack": False, "to": "bf16", "dtype": "bf16", "pad": 0},
        # The same matrix in a training step: this step's weights made 8 bits, then the forward product over 16 sequences of 1024.
        {"name": "linear_mlp", "op": "linear", "rows": 16384, "in": 4096, "out": 14336, "pack": True, "to": "bf16", "dtype": "bf16", "pad": 0},
        # The input gradient of the 1280-wide model's MLP matrix, whose 8-bit weights are there from the forward pass.
        {"name": "linear_grad_mlp", "op": "linear_grad", "rows": 16384, "in": 1280, "out": 5120, "pack": False, "to": "bf16", "dtype": "bf16", "pad": 0},
        # An odd layer: ragged in every direction, fp32 weights and result.
        {"name": "linear_grad_odd", "op": "linear_grad", "rows": 1021, "in": 1283, "out": 517, "pack": True, "to": "f32", "dtype": "f32", "pad": 3},
        # One decoded token's queries and keys: 32 heads of 128 with 8 key heads.  Latency.
        {"name": "heads_one_token", "op": "heads", "rows": 1, "q": 32, "k": 8, "dim": 128, "turned": 128, "interleaved": False, "norm": True, "dtype": "bf16"},
        # A block's queries and keys over 16 sequences of 1024, views of one QKV product.
        {"name": "heads_forward", "op": "heads", "rows": 16384, "q": 32, "k": 8, "dim": 128, "turned": 128, "interleaved": False, "norm": True, "dtype": "bf16"},
        # Their gradient.
        {"name": "heads_grad", "op": "heads_grad", "rows": 16384, "q": 32, "k": 8, "dim": 128, "turned": 128, "interleaved": False, "norm": True, "dtype": "bf16"},
        # Heads of 80 of which 32 channels turn, in neighbouring pairs, fp32, odd rows: the gradient.
        {"name": "heads_grad_odd", "op": "heads_grad", "rows": 4097, "q": 20, "k": 20, "dim": 80, "turned": 32, "interleaved": True, "norm": True, "dtype": "f32"},
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], even over its logarithm; one in three is rounded to a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 1 / 3 and high >= 64:
        v = -(-v // 64) * 64
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["head", "head_loss", "head_loss", "linear", "linear", "linear_grad", "linear_grad", "heads", "heads_grad"])
    case = {"op": op}
    if op.startswith("head") and not op.startswith("heads"):
        case["width"] = _spread(rng, 64, 8192)
        case["vocab"] = _spread(rng, 1000, 160000)
        most = min(16384, MOST_LOGITS // case["vocab"], MOST_HEAD // (case["vocab"] * case["width"]))
        case["rows"] = _spread(rng, 1, max(1, most))
        case["pad"] = rng.choice([0, 0, 8, 5])
        return case
    if op.startswith("linear"):
        case["in"] = _spread(rng, 64, 8192)
        case["out"] = _spread(rng, 64, 16384)
        case["rows"] = _spread(rng, 1, max(1, min(32768, MOST_LINEAR // (case["in"] * case["out"]))))
        case["pack"] = rng.random() < 0.5
        case["to"] = rng.choice(["bf16", "bf16", "f32"])
        case["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        case["pad"] = rng.choice([0, 0, 8, 3])
        return case
    case["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    case["dim"] = rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256, 50])
    case["turned"] = rng.choice([case["dim"], case["dim"], case["dim"] // 4 * 2])
    case["interleaved"] = rng.random() < 0.4
    case["norm"] = rng.random() < 0.7
    case["k"] = rng.choice([1, 2, 4, 5, 8, 12])
    case["q"] = case["k"] * rng.choice([1, 1, 2, 4, 5])
    size = 2 if case["dtype"] == "f32" else 1
    case["rows"] = _spread(rng, 1, max(1, min(65536, MOST_HEADS // (size * (case["q"] + case["k"]) * case["dim"]))))
    return case


def work(case):
    rows = case["rows"]
    if case["op"] in ("head", "head_loss"):
        v, d = case["vocab"], case["width"]
        passes = 1 if case["op"] == "head" else 2  # with the gradients each matrix is written once too
        return {"bytes": 2 * passes * (rows * d + v * d) + rows * (8 + 12 + (12 if passes == 2 else 0)), "flops": (2 if passes == 1 else 6) * rows * v * d}
    if case["op"].startswith("linear"):
        a, b = (case["in"], case["out"]) if case["op"] == "linear" else (case["out"], case["in"])
        blocks = -(-case["in"] // BLOCK) * -(-case["out"] // BLOCK)
        weights, e = case["in"] * case["out"] + 4 * blocks, 4 if case["dtype"] == "f32" else 2
        n = rows * a + 4 * rows * -(-a // BLOCK) + weights + rows * b * (4 if case["to"] == "f32" else 2)
        if case["pack"]:  # the weights are read, kept, and given as 16-bit values
            n += case["in"] * case["out"] * (e + 2) + weights
        return {"bytes": n, "flops": 2 * rows * case["in"] * case["out"]}
    e = 4 if case["dtype"] == "f32" else 2
    n = rows * (case["q"] + case["k"]) * case["dim"]
    per = rows * (8 + 4 * case["turned"])
    if case["op"] == "heads":
        return {"bytes": 2 * n * e + per, "flops": 7 * n}
    return {"bytes": (3 if case["norm"] else 2) * n * e + per, "flops": 14 * n}


def _padded(x, pad, dtype):
    """x in the given type, as a view of a tensor with `pad` more columns."""
    whole = torch.zeros(x.shape[0], x.shape[1] + pad, device="cuda", dtype=dtype)
    whole[:, : x.shape[1]] = x
    return whole[:, : x.shape[1]]


def _activations(g, rows, cols):
    """A residual stream after its norm: normal tokens, with a few channels far larger than the rest."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x *= torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))
    big = torch.rand(cols, device="cuda", generator=g) < 0.004
    return x * torch.where(big, 20.0, 1.0)


def _least_power(lead):
    """The least power of two s with lead <= 448 s, at least 2^-117."""
    m, e = torch.frexp(lead)
    e = torch.clamp(e - 9 + (m > 0.875).to(e.dtype), min=-117)
    return ((e + 127) << 23).view(torch.float32)  # 2^e


def _keep(x):
    """The codes (rows x pitch bytes) and scales (groups x rows) of activations x."""
    rows, cols = x.shape
    groups = -(-cols // BLOCK)
    g = torch.nn.functional.pad(x.float(), (0, groups * BLOCK - cols)).reshape(rows, groups, BLOCK)
    s = _least_power(g.abs().amax(dim=2))
    q = (g / s[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, -1)[:, :cols]
    codes = torch.zeros(rows, -(-cols // 16) * 16, device="cuda", dtype=torch.uint8)
    codes[:, :cols] = q
    return codes, s.t().contiguous()


def _keep_weights(w):
    """The codes (out x pitch bytes) and scales (blocks of rows x blocks of columns) of weights w."""
    out, cols = w.shape
    bo, bc = -(-out // BLOCK), -(-cols // BLOCK)
    g = torch.nn.functional.pad(w.float(), (0, bc * BLOCK - cols, 0, bo * BLOCK - out)).reshape(bo, BLOCK, bc, BLOCK)
    s = _least_power(g.abs().amax(dim=(1, 3)))
    q = (g / s[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(bo * BLOCK, bc * BLOCK)
    codes = torch.zeros(out, -(-cols // 16) * 16, device="cuda", dtype=torch.uint8)
    codes[:, :cols] = q[:out, :cols]
    return codes, s


def _kept(codes, scales, cols):
    """The values that codes and scales of activations stand for."""
    q = codes[:, :cols].contiguous().view(torch.float8_e4m3fn).float()
    return q * scales.t().repeat_interleave(BLOCK, dim=1)[:, :cols]


def _kept_weights(codes, scales, cols):
    q = codes[:, :cols].contiguous().view(torch.float8_e4m3fn).float()
    return q * scales.repeat_interleave(BLOCK, dim=0)[: codes.shape[0]].repeat_interleave(BLOCK, dim=1)[:, :cols]


def _table(positions, turned):
    """Cosines and sines of position times frequency, in 64 bits, rounded once: positions x turned / 2 x 2."""
    f = 10000.0 ** (-torch.arange(0, turned, 2, device="cuda", dtype=torch.float64) / turned)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), dim=2).float().contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = case["rows"]
    s = {"case": case}
    if case["op"] in ("head", "head_loss"):
        # half of the tokens are predicted well, a tenth carry no target
        v, d = case["vocab"], case["width"]
        w = 2.0 * d**-0.5 * torch.randn(v, d, device="cuda", generator=g)
        s["targets"] = torch.randint(0, v, (rows,), device="cuda", generator=g)
        lift = torch.where(torch.rand(rows, 1, device="cuda", generator=g) < 0.5, 2.5, 0.4)
        h = torch.randn(rows, d, device="cuda", generator=g) + lift * w[s["targets"]]
        s["h"], s["weight"] = _padded(h, case["pad"], torch.bfloat16), _padded(w, case["pad"], torch.bfloat16)
        if rows > 1:
            s["targets"][torch.rand(rows, device="cuda", generator=g) < 0.1] = -100
        if case["op"] == "head_loss":
            s["g_logp"] = -(0.5 + torch.rand(rows, device="cuda", generator=g)) / rows
            s["g_entropy"] = -0.01 * torch.ones(rows, device="cuda") / rows
            s["g_lse"] = 0.002 * torch.randn(rows, device="cuda", generator=g) / rows
        return s
    if case["op"].startswith("linear"):
        out, cols = case["out"], case["in"]
        if case["op"] == "linear":
            x = _activations(g, rows, cols)
        else:
            x = 1e-3 * torch.randn(rows, out, device="cuda", generator=g) * torch.exp(0.7 * torch.randn(rows, 1, device="cuda", generator=g))
        s["codes"], s["scales"] = _keep(x)
        w = _padded(0.02 * torch.randn(out, cols, device="cuda", generator=g) * torch.exp(0.5 * torch.randn(out, 1, device="cuda", generator=g)), case["pad"], DTYPES[case["dtype"]])
        if case["pack"]:
            s["weight"] = w
        else:
            s["wcodes"], s["wscales"] = _keep_weights(w)
        return s
    dtype, dim, q, k = DTYPES[case["dtype"]], case["dim"], case["q"], case["k"]
    # sequences of 1024 one behind the other, the first beginning far into a long context
    first = 30000 if rows > 1 else 100000
    s["positions"] = torch.arange(rows, device="cuda") % 1024 + first
    s["table"] = _table(first + 1024, case["turned"])
    qkv = (torch.randn(rows, (q + 2 * k) * dim, device="cuda", generator=g) * torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))).to(dtype)
    s["q"], s["k"] = qkv[:, : q * dim].view(rows, q, dim), qkv[:, q * dim : (q + k) * dim].view(rows, k, dim)
    if case["norm"]:
        s["qw"], s["kw"] = ((1.0 + 0.2 * torch.randn(dim, device="cuda", generator=g)).to(dtype) for _ in range(2))
    if case["op"] == "heads_grad":
        s["dq"], s["dk"] = ((1e-3 * torch.randn(rows, n, dim, device="cuda", generator=g)).to(dtype) for n in (q, k))
    return s


def _plain_head(s, case):
    h, w, t = s["h"].float(), s["weight"].float(), s["targets"]
    z = torch.matmul(h, w.t())
    m = z.amax(dim=1)
    d = z - m[:, None]
    del z
    e = d.exp()
    total = e.sum(dim=1)
    lse = m + total.log()
    entropy = total.log() - (e * d).sum(dim=1) / total
    logp = torch.where(t >= 0, d.gather(1, t.clamp(min=0)[:, None]).squeeze(1) - total.log(), 0.0)
    r = {"logp": logp, "entropy": entropy, "lse": lse}
    if case["op"] == "head_loss":
        gl = torch.where(t >= 0, s["g_logp"], 0.0)
        d -= (total.log() - entropy)[:, None]  # log p + entropy
        e /= total[:, None]
        d = ((s["g_lse"] - gl)[:, None] - s["g_entropy"][:, None] * d) * e
        d.scatter_add_(1, t.clamp(min=0)[:, None], gl[:, None])
        r["dh"] = torch.matmul(d, w).to(torch.bfloat16)
        r["dweight"] = torch.matmul(d.t(), h).to(torch.bfloat16)
    return r


def _plain_linear(s, case):
    r = {}
    codes, scales = (s["wcodes"], s["wscales"]) if not case["pack"] else _keep_weights(s["weight"])
    w = _kept_weights(codes, scales, case["in"])
    if case["pack"]:
        r["weight"] = w.to(torch.bfloat16)
    x = _kept(s["codes"], s["scales"], case["in"] if case["op"] == "linear" else case["out"])
    r["y"] = torch.matmul(x, w.t() if case["op"] == "linear" else w).to(DTYPES[case["to"]])
    return r


def _pairs(x, case):
    """The two channels of each pair that turns, and the channels that do not."""
    n = case["turned"]
    if case["interleaved"]:
        return x[..., 0:n:2], x[..., 1:n:2], x[..., n:]
    return x[..., : n // 2], x[..., n // 2 : n], x[..., n:]


def _whole(a, b, rest, case):
    if case["interleaved"]:
        return torch.cat((torch.stack((a, b), dim=-1).flatten(-2), rest), dim=-1)
    return torch.cat((a, b, rest), dim=-1)


def _plain_heads(x, w, s, case):
    y = x.float()
    if case["norm"]:
        y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + EPS) * w.float()
    t = s["table"][s["positions"]][:, None]
    a, b, rest = _pairs(y, case)
    return _whole(a * t[..., 0] - b * t[..., 1], b * t[..., 0] + a * t[..., 1], rest, case).to(x.dtype)


def _plain_heads_grad(dy, x, w, s, case):
    t = s["table"][s["positions"]][:, None]
    a, b, rest = _pairs(dy.float(), case)
    d = _whole(a * t[..., 0] + b * t[..., 1], b * t[..., 0] - a * t[..., 1], rest, case)
    if not case["norm"]:
        return d.to(x.dtype), None
    x = x.float()
    rstd = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
    xh, wd = x * rstd, d * w.float()
    dx = rstd * (wd - xh * (wd * xh).mean(dim=-1, keepdim=True))
    return dx.to(dy.dtype), (d * xh).sum(dim=(0, 1)).to(w.dtype)


def _plain(s, case):
    if case["op"] in ("head", "head_loss"):
        return _plain_head(s, case)
    if case["op"].startswith("linear"):
        return _plain_linear(s, case)
    if case["op"] == "heads":
        return {"q": _plain_heads(s["q"], s.get("qw"), s, case), "k": _plain_heads(s["k"], s.get("kw"), s, case)}
    (dq, dqw), (dk, dkw) = _plain_heads_grad(s["dq"], s["q"], s.get("qw"), s, case), _plain_heads_grad(s["dk"], s["k"], s.get("kw"), s, case)
    return {"dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw}


def run(s):
    case = s["case"]
    if not own:
        return _plain(s, case)
    from paper_2605_19811_gb300 import training as T

    if case["op"] in ("head", "head_loss"):
        loss = {k: s[k] for k in ("g_logp", "g_entropy", "g_lse")} if case["op"] == "head_loss" else {}
        o = T.linear_logprob(s["h"], s["weight"], s["targets"], **loss)
        r = {"logp": o.logp, "entropy": o.entropy, "lse": o.lse}
        if loss:
            r["dh"], r["dweight"] = o.dh, o.dweight
        return r
    if case["op"].startswith("linear"):
        r = {}
        if case["pack"]:
            w = T.weight8(s["weight"])
            r["weight"] = w.unpack(torch.bfloat16)
        else:
            w = T.Weight8(s["wcodes"], s["wscales"], case["in"])
        x = T.Checkpoint8(s["codes"], s["scales"], case["in"] if case["op"] == "linear" else case["out"], "e4m3")
        r["y"] = (T.linear8 if case["op"] == "linear" else T.linear8_grad)(x, w, dtype=DTYPES[case["to"]])
        return r
    how = {"norm": case["norm"], "eps": EPS, "interleaved": case["interleaved"]}
    if case["op"] == "heads":
        o = T.qk_rotary(s["q"], s["k"], s["positions"], s["table"], s.get("qw"), s.get("kw"), **how)
        return {"q": o.q, "k": o.k}
    o = T.qk_rotary_grad(s["dq"], s["dk"], s["positions"], s["table"], s["q"], s["k"], s.get("qw"), s.get("kw"), **how)
    return {"dq": o.dq, "dk": o.dk, "dqw": o.dq_weight, "dkw": o.dk_weight}


# --- the definitions in 64 bits, on their own ---


def _exact_head(s, case):
    w, parts, dweight = s["weight"].double(), [], 0.0
    for at in range(0, case["rows"], 2048):  # a part of the rows at a time, for the memory's sake
        h, t = s["h"][at : at + 2048].double(), s["targets"][at : at + 2048]
        z = h @ w.t()
        lp = torch.log_softmax(z, dim=1)
        p = lp.exp()
        plogp = torch.xlogy(p, p)
        one = torch.zeros_like(z)
        one[torch.arange(len(t), device=z.device)[t >= 0], t[t >= 0]] = 1.0
        r = {"logp": torch.where(one > 0, lp, 0.0).sum(dim=1), "entropy": -plogp.sum(dim=1), "lse": torch.logsumexp(z, dim=1)}
        if case["op"] == "head_loss":
            gl, gh, gz = (s[k][at : at + 2048, None].double() for k in ("g_logp", "g_entropy", "g_lse"))
            d = gl * (one - p * (t >= 0)[:, None]) - gh * (plogp + p * r["entropy"][:, None]) + gz * p
            r["dh"] = d @ w
            dweight = dweight + d.t() @ h
        parts.append(r)
    r = {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    if case["op"] == "head_loss":
        r["dweight"] = dweight
    return r


def _power(e):
    """2^e in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_codes(codes, cols):
    """e4m3 bytes as sign, 4 bits of exponent (bias 7) and 3 of fraction."""
    b = codes[:, :cols].to(torch.int64)
    e, f = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, f / 8 * 2.0**-6, (1 + f / 8) * _power(e - 7))
    return torch.where(b > 127, -v, v)


def _exact_weights(w):
    """What is kept of weights: each 128 x 128 block in steps of its scale, four significant bits, ties to even."""
    w = w.double()
    kept = torch.empty_like(w)
    for r in range(0, w.shape[0], BLOCK):
        rows = w[r : r + BLOCK]
        lead = torch.nn.functional.pad(rows.abs().amax(dim=0), (0, -w.shape[1] % BLOCK)).reshape(-1, BLOCK).amax(dim=1)
        s = _power(torch.ceil(torch.log2(lead / 448.0)))
        s = torch.where(s * 224.0 >= lead, s / 2, torch.where(s * 448.0 < lead, s * 2, s))  # the logarithm's rounding
        s = s.repeat_interleave(BLOCK)[: w.shape[1]]
        q = rows / s
        step = _power(torch.clamp(torch.frexp(q)[1] - 1, min=-6) - 3)
        kept[r : r + BLOCK] = torch.round(q / step) * step * s
    return kept


def _exact_linear(s, case):
    x = _exact_codes(s["codes"], case["in"] if case["op"] == "linear" else case["out"])
    x = x * s["scales"].double()[torch.arange(x.shape[1], device=x.device) // BLOCK].t()
    if case["pack"]:
        w = _exact_weights(s["weight"])
    else:
        w = _exact_codes(s["wcodes"], case["in"])
        rows, cols = (torch.arange(n, device=w.device) // BLOCK for n in w.shape)
        w = w * s["wscales"].double()[rows][:, cols]
    r = {"y": torch.einsum("ti,oi->to" if case["op"] == "linear" else "to,oi->ti", x, w)}
    if case["pack"]:
        r["weight"] = w
    return r


def _turn(s, case):
    """The rotation of each token as matrices: turned / 2 complex numbers."""
    t = s["table"].double()[s["positions"]]
    return torch.complex(t[..., 0], t[..., 1])[:, None]


def _as_complex(x, case):
    n = case["turned"]
    if case["interleaved"]:
        return torch.view_as_complex(x[..., :n].unflatten(-1, (n // 2, 2)).contiguous())
    return torch.view_as_complex(x[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2).contiguous())


def _from_complex(z, x, case):
    pairs = torch.view_as_real(z)
    if not case["interleaved"]:
        pairs = pairs.transpose(-1, -2)
    return torch.cat((pairs.flatten(-2), x[..., case["turned"] :]), dim=-1)


def _exact_heads(s, case):
    r = {}
    for name in ("q", "k"):
        x = s[name].double()
        if case["norm"]:
            x = x / torch.sqrt(x.square().sum(dim=-1, keepdim=True) / case["dim"] + EPS) * s[name + "w"].double()
        if case["op"] == "heads":
            r[name] = _from_complex(_as_complex(x, case) * _turn(s, case), x, case)
            continue
        d = s["d" + name].double()
        d = _from_complex(_as_complex(d, case) * _turn(s, case).conj(), d, case)
        r["d" + name + "w"] = None
        if case["norm"]:
            # y_c = w_c x_c rstd: the gradient by rstd goes back through the mean square, d rstd / d x_c = -rstd^3 x_c / dim
            x, w = s[name].double(), s[name + "w"].double()
            rstd = (x.square().sum(dim=-1, keepdim=True) / case["dim"] + EPS) ** -0.5
            r["d" + name + "w"] = torch.einsum("thc,thc,th->c", d, x, rstd[..., 0])
            through = (d * w * x).sum(dim=-1, keepdim=True)
            d = d * w * rstd - through * rstd**3 * x / case["dim"]
        r["d" + name] = d
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("head", "head_loss"):
        return _exact_head(s, case)
    if case["op"].startswith("linear"):
        return _exact_linear(s, case)
    return _exact_heads(s, case)
