"""The 8-bit layer's operators in 64 bits (CPU tensors), written from their definitions: what the tests compare with."""
import math

import torch


def two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def block_exponent(v):
    """Per block of 32: the smallest e >= -126 with max |v| <= 448 * 2^e (finite values)"""
    top = v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32).abs().amax(-1)
    m, k = torch.frexp(top.clamp_min(2.0 ** -140))              # top = m * 2^k, 1/2 <= m < 1; 448 = 0.875 * 2^9
    return (k - 9 + (m > 0.875).to(k.dtype)).clamp_min(-126)


def to_e4m3(t):
    """Nearest e4m3 value, ties to even, of |t| <= 448"""
    k = torch.frexp(t.abs().clamp_min(2.0 ** -6)).exponent - 1
    step = two_to(k - 3)
    return torch.round(t / step) * step


def mx(v, e=None):
    """(values of the 8-bit format that v [.., n] becomes, exponents of its blocks)"""
    e = block_exponent(v) if e is None else e
    scale = two_to(e).repeat_interleave(32, -1)
    return to_e4m3((v / scale).clamp(-448.0, 448.0)) * scale, e


def values(pair):
    """64-bit values of a (float8_e4m3fn, float8_e8m0fnu) pair, on the CPU"""
    q, s = (t.cpu() for t in pair)
    return q.double() * s.double().repeat_interleave(32, -1)


def norm(x, y, weight, eps):
    u = x.double() + (0.0 if y is None else y.double())
    n = u / torch.sqrt(u.square().mean(-1, keepdim=True) + eps)
    return u, n if weight is None else n * weight.double()


def logits(x, Wr):
    """fp32 logits in the defined order: element h is in partial sum (h / 8) mod 64, ascending h; the partials fold pairwise"""
    T, H = x.shape
    n = -(-H // 512)
    pad = lambda a: torch.nn.functional.pad(a.float(), (0, 512 * n - H)).reshape(a.shape[0], n, 64, 8)
    xp, wp = pad(x), pad(Wr)
    acc = torch.zeros((T, Wr.shape[0], 64))
    for c in range(n):
        for i in range(8):
            acc = acc + xp[:, None, c, :, i] * wp[None, :, c, :, i]      # (products of bf16 are exact)
    while acc.shape[-1] > 1:
        acc = acc[..., 0::2] + acc[..., 1::2]
    return acc[..., 0]


def route(x, Wr, balance, K, score, groups, top_groups, best, renorm, scale):
    """ids, weights, token by token with Python's own comparisons; NaN counts as less than everything"""
    l = logits(x, Wr).double()
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, -1)
    s32 = s.float()
    c = s32 if balance is None else s32 + balance.float()
    ids, w = [], []
    order = lambda v: (0, 0.0) if math.isnan(v) else (1, v)
    size = Wr.shape[0] // groups
    for t in range(x.shape[0]):
        row = c[t].tolist()
        value = []
        for g in range(groups):
            top = sorted(row[g * size:(g + 1) * size], key=order, reverse=True)[:best]
            value.append(torch.tensor(top, dtype=torch.float32).sum().item())
        kept = sorted(range(groups), key=lambda g: order(value[g]), reverse=True)[:top_groups]      # (stable: the lower id first)
        chosen = sorted((e for e in range(len(row)) if e // size in kept), key=lambda e: order(row[e]), reverse=True)[:K]
        ids.append(chosen)
        wt = s[t, chosen]
        w.append((wt / (wt.sum() + 1e-20) if renorm else wt) * scale)
    return torch.tensor(ids, dtype=torch.int32).reshape(-1, K), torch.stack(w) if w else torch.empty(0, K)


def experts(x, rows, counts, Wg, Wu, Wd):
    """Yp in 64 bits (no rounding on the way) and how far a right evaluation may be from it, element by element.

    Gate and up: the matrix instruction adds eight 8-bit products at a time and cuts each below 2^-13 of the largest of them:
    at most 8 * 2^-13 of that one per eight.  Its fp32 sums: at most two roundings per 128 products and eight to join the
    parts.  SiLU's slope is at most 1.1, the fast exponential and quotient are off by 2^-20, and the hidden value is rounded
    to bf16 (2^-8 at most).  Then the sum over the hidden row, four roundings per 128, and the output's own rounding."""
    Y, tol, at = [], [], 0
    chain = lambda n, per: (per * n / 128 + 8.0) * 2.0 ** -24
    largest = lambda v: v.abs().reshape(*v.shape[:-1], v.shape[-1] // 8, 8).amax(-1)
    for e, n in enumerate(counts):
        if n == 0:
            continue
        r = x[rows[at:at + n]]
        g, u = r @ Wg[e].T, r @ Wu[e].T
        dg, du = (2.0 ** -10 * (largest(r) @ largest(w[e]).T) + chain(r.shape[1], 2.0) * (r.abs() @ w[e].abs().T) for w in (Wg, Wu))
        sg = g * torch.sigmoid(g)
        h = sg * u
        dh = 1.1 * dg * (u.abs() + du) + sg.abs() * du + (2.0 ** -8 + 2.0 ** -20) * h.abs()
        y = h @ Wd[e].T
        wd = Wd[e].abs().T
        Y.append(y)
        tol.append((dh + chain(h.shape[1], 4.0) * h.abs()) @ wd * (1 + 2.0 ** -7) + 2.0 ** -8 * y.abs() + 1e-30)
        at += n
    return torch.cat(Y), torch.cat(tol)
