"""Plain statements, in 64 bits, of token scores and of Newton-Schulz products, with
bounds of what the library's arithmetic may be off them by. Test infrastructure only.

Scores. A log-probability is off by LOGP + 2u |lp| as in token_ref (sums of exponentials are off by
8e-6 of themselves at most, 3e-6 by the exponentials and 5e-6 by the additions). The
entropy is log S - log 2 T / S, T the sum of e_v 2^e_v with exponents e_v <= 0, each term off as
S's are: both sums by 8e-6 of themselves, their quotient by 1.6e-5 |T / S|; log 2 |T / S| is the entropy
less log S, |log S| <= H + 1 (S >= 1/2). ENTROPY = 1e-5 + 2e-5 (H + 1) covers it. The gradient
s (g_v - p_v (G + h (lp_v + H))) is off by p_v's P of its second term, by h p_v times what lp_v and
H are off by, and at a given token by g (1 - p) of token_ref: 2 LOGP + 4u of g; terms below the
smallest float may be 0. The rounding to its type comes on top.

Products. The library's own roundings are made here in 64 bits (`rounded`): X as two halves, its
products' factors as one half or two, the diagonals of A and B apart. Its result is as far from the
exact one as that is, within a factor of 2 (the roundings fall in other places), plus what sums
in 32 bits add: as far as the plain products in float32 are (`in_float32`), within the same factor.
"""
import numpy as np
import torch

from token_ref import LOGP, P, ROUND, U, log_softmax  # noqa: F401

QUINTIC = (3.4445, -4.7750, 2.0315)


def scores(x, y, top, scale):
    """(logp, entropy, top_logp, top_index) of rows x (numpy, exact values of their type); y: (n, given)."""
    lp = log_softmax(x, scale)
    n = len(x)
    counts = (y >= 0).any(1) if y.shape[1] else np.ones(n, bool)
    logp = np.where(y >= 0, np.take_along_axis(lp, np.maximum(y, 0), 1), 0.0) if y.shape[1] else np.zeros((n, 0))
    with np.errstate(invalid="ignore"):
        h = -np.where(np.exp(lp) > 0, np.exp(lp) * lp, 0.0).sum(1)
    order = np.argsort(-x.astype(np.float64), 1, kind="stable")[:, :top]
    best = np.take_along_axis(lp, order, 1)
    return (logp, np.where(counts, h, 0.0), np.where(counts[:, None], best, 0.0), np.where(counts[:, None], order, -1))


def entropy_bound(h):
    return 1e-5 + 2e-5 * (np.abs(h) + 1)


def gradient(x, y, g, h, scale):
    """d/dx of sum g logp + sum h H."""
    lp = log_softmax(x, scale)
    p = np.exp(lp)
    fin = np.where(p > 0, lp, 0.0)
    ent = -(p * fin).sum(1, keepdims=True)
    counts = (y >= 0).any(1) if y.shape[1] else np.ones(len(x), bool)
    gg = np.where(y >= 0, g, 0.0)
    hh = np.where(counts, h, 0.0)[:, None]
    d = -p * (gg.sum(1, keepdims=True) + hh * (fin + ent))
    for j in range(y.shape[1]):
        d[np.arange(len(x)), np.maximum(y[:, j], 0)] += gg[:, j]
    d[np.isneginf(x.astype(np.float64)).all(1)] = 0.0
    return d * scale


def gradient_bound(x, y, g, h, scale, kind):
    lp = log_softmax(x, scale)
    p = np.exp(lp)
    fin = np.where(p > 0, lp, 0.0)
    ent = -(p * fin).sum(1, keepdims=True)
    gg = np.where(y >= 0, np.abs(g), 0.0)
    G, hh = gg.sum(1, keepdims=True), np.abs(h)[:, None]
    off = p * (P * (G + hh * (np.abs(fin + ent))) + hh * (LOGP + 2 * U * np.abs(fin) + entropy_bound(ent)) + 8 * U * G)
    off = off + 2.0 ** -126 * (G + 300 * hh)
    at = np.zeros_like(p)
    for j in range(y.shape[1]):
        at[np.arange(len(x)), np.maximum(y[:, j], 0)] += gg[:, j]
    off = (off + at * (2 * LOGP + 8 * U)) * scale
    rel, low = ROUND[kind]
    return off + rel * (np.abs(gradient(x, y, g, h, scale)) + off) + low


# -- Newton-Schulz products (torch, float64) -----------------------------------------
def _two(x, scale=2.0 ** 10):
    """x as the sum of two halves."""
    hi = (x * scale).to(torch.float16).to(x.dtype) / scale
    return hi + ((x - hi) * scale * 2.0 ** 11).to(torch.float16).to(x.dtype) / scale / 2.0 ** 11


def _one(x, scale=2.0 ** 10):
    return (x * scale).to(torch.float16).to(x.dtype) / scale


def _coefficients(c, steps):
    return [tuple(c)] * steps if not hasattr(c[0], "__len__") else [tuple(v) for v in c]


def products(g, steps=5, coefficients=QUINTIC, dtype=torch.float64):
    """X of each matrix (K, m, n) after `steps`, by the formula."""
    x = g.to(dtype)
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    size = g.double().square().sum((1, 2), keepdim=True).sqrt().to(dtype)
    x = torch.where(size > 0, x / size, torch.zeros_like(x))
    for a, b, c in _coefficients(coefficients, steps):
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.transpose(1, 2) if tall else x


def in_float32(g, steps=5, coefficients=QUINTIC):
    return products(g, steps, coefficients, torch.float32).double()


def rounded(g, steps=5, coefficients=QUINTIC, fine=False):
    """The same with the library's roundings of X and of the products' factors."""
    q = _two if fine else _one
    x = g.double()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    size = x.square().sum((1, 2), keepdim=True).sqrt()
    x = _two(torch.where(size > 0, x / size, torch.zeros_like(x)))
    for a, b, c in _coefficients(coefficients, steps):
        X = q(x)
        A = X @ X.transpose(1, 2)
        d = torch.diagonal(A, dim1=1, dim2=2)
        off = q(A - torch.diag_embed(d))
        S = off @ off + (d[:, :, None] + d[:, None, :]) * off + torch.diag_embed(d * d)
        B = b * (off + torch.diag_embed(d)) + c * S
        e = torch.diagonal(B, dim1=1, dim2=2)
        x = _two((a + e)[:, :, None] * x + q(B - torch.diag_embed(e)) @ X)
    return x.transpose(1, 2) if tall else x
