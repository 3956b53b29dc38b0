"""Plain 64-bit forms of the 8-bit MoE block's operators and seeded inputs for them (torch, double)."""
from __future__ import annotations

import numpy as np
import torch

HIT, LORE, EXACT = 0, 1, 2


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def norm_ref(x, resid, w, eps):
    """-> s, y, q (as doubles), q_scale; a row that is not finite has q 0 and q_scale NaN."""
    s = x.double() + (0 if resid is None else resid.double())
    a = s if w is None else s * w.double()
    ms = (s * s).mean(1, keepdim=True)
    rstd = torch.where(ms == 0, 0, 1 / torch.sqrt(ms + eps))
    top = a.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(127 * a / top), 0)
    scale = (top * rstd / 127)[:, 0]
    bad = ~torch.isfinite(a).all(1)
    q[bad], scale[bad] = 0, torch.nan
    return s, a * rstd, q, scale


def route_ref(z, K, sigmoid=False, groups=1, keep=1, top=1, balance=None, renorm=False, scale=1.0):
    """Experts and weights of each token from its logits z (NumPy, double): one token and one rule at a time."""
    T, N = z.shape
    idx, w = np.zeros((T, K), np.int64), np.zeros((T, K))
    for t in range(T):
        masked = np.isneginf(z[t])
        s = np.zeros(N)
        if sigmoid:
            s[~masked] = 1 / (1 + np.exp(-z[t][~masked]))
        elif not masked.all():
            e = np.exp(z[t] - z[t].max())
            s = e / e.sum()
        c = s + (0 if balance is None else balance.astype(np.float64))
        c[masked] = -np.inf
        per = N // groups
        live = []
        values = []
        for g in range(groups):
            best = sorted(c[g * per:(g + 1) * per], reverse=True)[:top]
            values.append(sum(v for v in best if v != -np.inf) if best[0] != -np.inf else -np.inf)
        for g in sorted(range(groups), key=lambda g: (-values[g], g))[:keep]:
            live += list(range(g * per, (g + 1) * per))
        idx[t] = sorted(live, key=lambda e: (-c[e], e))[:K]
        w[t] = s[idx[t]]
        if renorm:
            w[t] = w[t] / w[t].sum() if w[t].sum() > 0 else 0
        w[t] = w[t] * float(np.float32(scale))
    return idx, w


def buckets_ref(idx, cls, N):
    key = (cls.astype(np.int64) * N + idx).reshape(-1)
    perm = np.argsort(key, kind="stable")
    inv = np.empty_like(perm)
    inv[perm] = np.arange(perm.size)
    off = np.zeros((3, N + 1), np.int64)
    ends = np.cumsum(np.bincount(key, minlength=3 * N)).reshape(3, N)
    off[:, 1:] = ends
    off[:, 0] = np.concatenate([[0], ends[:2, -1]])
    return perm, inv, off


def blob(a):
    """Rows of weights (fp32) as an 8-bit blob, by a generator of its own: codes, then a scale per row."""
    scale = a.abs().amax(1) / 127
    codes = torch.round(a / torch.where(scale > 0, scale, 1)[:, None]).clamp(-127, 127).to(torch.int8)
    return torch.cat([codes.reshape(-1).view(torch.uint8), scale.float().view(torch.uint8)])


def unblob(b, rows, k):
    n = rows * k
    return b[:n].view(torch.int8).view(rows, k).double(), b[n:].clone().view(torch.float32).double()


U = 2.0 ** -24  # half a step of fp32, relative


def swiglu_i8_ref(xq, xs, w13, w2, d, I):
    """Rows of 8-bit activations through one expert: y and how far fp32 arithmetic may be from it.

    With g and u from exact int32 sums, fp32 rounds 4 times before each (the sum, the scales' product,
    the product: 3 U; counted 4), silu(g) = g / (1 + e^-g) takes a hardware exponential whose argument
    is rounded (|g| U on e^-g and 2 U of its own), a sum and a division: h is off by at most
    (4 (1 + |g|) + |g| + 6 + 4 + 1) U relative, under (16 + 5 |g|) U.  The row's scale has the error of
    its largest h and a division.  A code whose exact quotient is nearer to a half than 127 times the
    errors of h and the scale may be the neighbour's: that moves y_j by at most sh s2_j |W2_jk|.  The
    rest of y is a sum of exact integers and four roundings, and the scale's error."""
    a, s = unblob(w13, 2 * I, d)
    acc = xq.double() @ a.t()
    gu = acc * xs.double()[:, None] * s
    g, u = gu[:, :I], gu[:, I:]
    h = g / (1 + torch.exp(-g)) * u
    err = (16 + 5 * g.abs()) * U
    top = h.abs().amax(1, keepdim=True)
    eh = err.amax(1, keepdim=True)
    t = torch.where(top > 0, 127 * h / top, 0)
    q = torch.round(t)
    border = (((t - torch.floor(t)) - 0.5).abs() <= t.abs() * (err + eh + 4 * U)).double()
    b, s2 = unblob(w2, d, I)
    y = (q @ b.t()) * (top / 127) * s2
    tol = (border @ b.abs().t()) * (top / 127) * s2 * (1 + eh) + y.abs() * (eh + 8 * U)
    return y, tol


def swiglu_i8_tiny_ref(xq, xs, w13, w2, d, I):
    """The same for rows whose h may lie below the smallest normal fp32, and max |h| of each row.

    There h and the row's scale are rounded to whole steps of 2^-149, half a step each: that is what a code's
    quotient t = 127 h / top may be off by, over top / 127 (h's share) and times t / 127 (top's), and y by half
    a step over the scale."""
    half = 2.0 ** -150
    a, s = unblob(w13, 2 * I, d)
    gu = (xq.double() @ a.t()) * xs.double()[:, None] * s
    g, u = gu[:, :I], gu[:, I:]
    h = g / (1 + torch.exp(-g)) * u
    err = (16 + 5 * g.abs()) * U
    top = h.abs().amax(1, keepdim=True)
    eh = err.amax(1, keepdim=True)
    t = 127 * h / top
    q = torch.round(t)
    off = t.abs() * (err + eh + 4 * U) + (127 + t.abs()) * half / top
    border = (((t - torch.floor(t)) - 0.5).abs() <= off).double()
    b, s2 = unblob(w2, d, I)
    step = 127 * half / top  # of the scale, relative
    y = (q @ b.t()) * (top / 127) * s2
    return y, (border @ b.abs().t()) * (top / 127) * s2 * (1 + eh + step) + y.abs() * (eh + 8 * U + step), top[:, 0]


def lore_ref(x, A, B):
    return x.double() @ A.double().t() @ B.double().t()


# Calls (T, d, N, K, I, Is, C) of the 8-bit experts and the tile shape that takes each: small contractions and
# many features, so that a call is long enough for its shape and quick to check.
SHAPE_CALLS = [
    ((120, 48, 10, 1, 272, 144, 6), 0), ((400, 64, 64, 2, 128, 320, 64), 1), ((1000, 80, 36, 2, 528, 272, 30), 2),
    ((2300, 64, 64, 4, 1296, 400, 64), 3), ((4200, 64, 32, 4, 1040, 400, 32), 3)]
# Calls whose shared block's down contraction is split, with the parts, and one just too short for it.
SPLIT_CALLS = [
    ((1, 64, 4, 1, 16, 8192, 1), 4), ((70, 208, 4, 2, 32, 4112, 2), 2), ((3, 4096, 8, 2, 48, 16400, 8), 8),
    ((500, 128, 4, 1, 64, 6160, 0), 3), ((1, 64, 4, 1, 16, 4080, 1), 1)]

# Calls (T, d, N, K, fp32) of the scored routing that run in tiles with the whole workspace: the blocks of 16 tokens
# split the contraction in so many parts and share the experts in so many chunks of so many.
SCORED_TILES = [
    ((120, 2048, 256, 8, False), (8, 4, 64)), ((250, 2048, 256, 8, False), (4, 4, 64)),   # one launch
    ((250, 1024, 100, 6, True), (8, 1, 100)), ((150, 512, 160, 4, False), (4, 2, 96)),
    ((300, 2048, 191, 3, False), (6, 2, 96)), ((300, 2048, 130, 3, False), (8, 1, 130)),  # an uneven chunk, one refused
    ((257, 1040, 192, 64, True), (5, 3, 64)), ((1000, 4096, 256, 8, False), (1, 4, 64)),  # chunks alone
    ((2000, 2048, 128, 8, False), (1, 2, 64))]
