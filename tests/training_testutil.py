"""Shared helpers of the training-step operator tests: matrices inside larger
buffers whose other elements are watched, and plain 64-bit forms of the
operators, written from their definitions with numpy."""

import numpy as np

GROUP = 128
LIMIT = {"i8": 127.0, "e4m3": 448.0}
LEAST = {"i8": 2.0 ** -126, "e4m3": 2.0 ** -117}


class Held:
    """A rows x cols CUDA matrix inside a larger buffer: row pitch cols + pad,
    the first element `offset` elements into the buffer.  Every other element
    holds a marker; untouched() says whether they still do."""

    MARK = 77.0

    def __init__(self, rows, cols, dtype, pad=0, offset=0, values=None):
        import torch
        self.ld = cols + pad
        self.buf = torch.full((offset + max(rows, 1) * self.ld + 16,), self.MARK, dtype=dtype, device="cuda")
        self.t = torch.as_strided(self.buf, (rows, cols), (self.ld, 1), offset)
        if values is not None:
            self.t.copy_(values)

    def untouched(self):
        import torch
        outside = torch.ones_like(self.buf, dtype=torch.bool)
        torch.as_strided(outside, self.t.shape, (self.ld, 1), self.t.storage_offset()).fill_(False)
        return bool((self.buf[outside] == self.MARK).all())


def f64(t):
    return t.detach().double().cpu().numpy()


def e4m3_value(b):
    """Values of e4m3 bytes: sign, 4 bits of exponent (bias 7), 3 of fraction."""
    b = b.astype(np.int64)
    e, f = (b >> 3) & 15, (b & 7) / 8.0
    v = np.where(e == 0, f * 2.0 ** -6, (1 + f) * 2.0 ** (e - 7.0))
    return np.where(b & 128, -v, v)


def code_values(codes, kind):
    return codes.view(np.int8).astype(np.float64) if kind == "i8" else e4m3_value(codes)


def checkpoint_values(ck):
    """What a Checkpoint8 stands for, in 64 bits."""
    q = code_values(ck.codes.cpu().numpy()[:, :ck.cols].copy(), ck.format)
    s = ck.scales.cpu().numpy().astype(np.float64)[:, :ck.rows]
    return q * np.repeat(s.T, GROUP, axis=1)[:, :ck.cols]


_E4M3 = np.sort(np.unique(np.abs(e4m3_value(np.array([b for b in range(128) if b != 127])))))


def nearest_code(q, kind):
    """q rounded to the format's numbers, ties to the even code."""
    if kind == "i8":
        return np.rint(q)
    a = np.abs(q)
    hi = np.clip(np.searchsorted(_E4M3, a), 0, len(_E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _E4M3[lo], _E4M3[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)   # code order is value order
    return np.copysign(_E4M3[pick], q)


def pack_reference(x, kind):
    """(codes' values, scales as rows x groups) of a 64-bit matrix."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    scales = np.empty((rows, groups))
    vals = np.empty_like(x)
    for g in range(groups):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        bad = ~np.isfinite(part).all(axis=1)
        most = np.where(bad, 0.0, np.abs(np.where(np.isfinite(part), part, 0.0)).max(axis=1))
        m, e = np.frexp(most / LIMIT[kind])
        s = np.where(most > 0, np.ldexp(1.0, e - (m == 0.5)), 0.0)   # least power of two >= most / limit
        s = np.maximum(s, LEAST[kind])
        q = nearest_code(np.where(np.isfinite(part), part, 0.0) / s[:, None], kind)
        top, cap = (2.0 ** 122, 63) if kind == "i8" else (2.0 ** 120, 240)   # the next code would stand for 2^128
        q = np.where((s == top)[:, None], np.clip(q, -cap, cap), q)
        vals[:, g * GROUP:(g + 1) * GROUP] = np.where(bad[:, None], 0.0, q)
        scales[:, g] = np.where(bad, np.nan, s)
    return vals, scales


def logprob_reference(z, y, top_k=0):
    """lse, entropy, logp, top indices of 64-bit logits (see lm_token_logprob_args)."""
    n, v = z.shape
    lse, ent, logp = np.empty(n), np.empty(n), np.zeros(n)
    top = -np.ones((n, top_k), dtype=np.int64)
    for r in range(n):
        row = z[r]
        if np.isnan(row).any() or np.isposinf(row).any():
            lse[r] = ent[r] = logp[r] = np.nan
            continue
        m = row.max()
        if m == -np.inf:
            lse[r], ent[r] = -np.inf, 0.0
        else:
            e = np.exp(row - m)
            lse[r] = m + np.log(e.sum())
            lp = (row - m) - np.log(e.sum())      # kept apart from m, beside which it may vanish
            p = np.exp(lp)
            ent[r] = -np.sum(p[p > 0] * lp[p > 0])
        if y[r] >= v:
            logp[r] = np.nan
        elif y[r] >= 0:
            logp[r] = lp[y[r]] if m > -np.inf else -np.inf
        order = np.argsort(-row, kind="stable")[:top_k]
        order = order[row[order] > -np.inf]
        top[r, :len(order)] = order
    return lse, ent, logp, top


def log_probabilities(row):
    """(z - max) - log sum exp(z - max) of a row with a finite maximum."""
    d = row - row.max()
    return d - np.log(np.exp(d).sum())


def logprob_gradient(z, y, lse, ent, gl, gh, gz):
    n, v = z.shape
    g = np.zeros((n, v))
    for r in range(n):
        if np.isnan(lse[r]) or y[r] >= v:
            g[r] = np.nan
            continue
        if lse[r] == -np.inf:
            continue
        lp = log_probabilities(z[r])
        p = np.exp(lp)
        wl = gl[r] if y[r] >= 0 else 0.0
        g[r] = np.where(p > 0, p * (gz[r] - wl - gh[r] * (np.where(p > 0, lp, 0.0) + ent[r])), 0.0)
        if y[r] >= 0:
            g[r, y[r]] += wl
    return g
